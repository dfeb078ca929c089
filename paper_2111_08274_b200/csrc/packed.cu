// Launches of the kernels in packed.cuh.
#include "packed.cuh"

#include <stddef.h>
#include <string.h>

#include <type_traits>

namespace hadfl {
namespace {

template <bool V>
using Flag = std::integral_constant<bool, V>;
template <typename T>
struct Type {
  using type = T;
};

template <typename F>
void with_flag(bool v, F &&f) {
  if (v)
    f(Flag<true>{});
  else
    f(Flag<false>{});
}
template <typename F>
void with_storage(bool bf16, F &&f) {
  if (bf16)
    f(Type<__nv_bfloat16>{});
  else
    f(Type<float>{});
}

unsigned column_blocks(int64_t columns) {
  return (unsigned)((columns + (int64_t)kThreads * kPackedE - 1) / ((int64_t)kThreads * kPackedE));
}

}  // namespace

void launch_pack(const PackedShape &s, const PackedRows &rows, const void *base, float *residual, bool stochastic,
                 uint64_t round, const PhiloxKeys &keys, uint8_t *messages) {
  PackParams q;
  q.rows = rows;
  q.rows_per_block = rows.n;
  q.round_lo = (uint32_t)round;
  q.tag = kTagPack | ((uint32_t)(round >> 32) & 0xFFFFFFu);
  q.n_params = s.n_params;
  q.stride = s.stride;
  q.scales_at = packed_scales_at(s.n_params);
  q.message_bytes = packed_bytes(s.n_params);
  q.code_columns = q.scales_at * 2;
  q.scale_columns = (q.message_bytes - q.scales_at) * kPackedBlock;
  const dim3 grid(column_blocks(q.scale_columns), (unsigned)((rows.n + q.rows_per_block - 1) / q.rows_per_block));
  with_storage(s.bf16, [&](auto wt) {
    using WT = typename decltype(wt)::type;
    with_flag(base != nullptr, [&](auto has_base) {
      with_flag(residual != nullptr, [&](auto has_residual) {
        with_flag(stochastic, [&](auto is_stochastic) {
          k_pack<WT, has_base.value, has_residual.value, is_stochastic.value><<<grid, kThreads, 0, s.stream>>>(
              (const WT *)s.w, (const WT *)base, residual, messages, keys, q);
        });
      });
    });
  });
}

void launch_unpack(const PackedShape &s, const PackedRows &rows, const void *base, const uint8_t *messages) {
  UnpackParams q;
  q.rows = rows;
  q.rows_per_block = rows.n;
  q.n_params = s.n_params;
  q.stride = s.stride;
  q.scales_at = packed_scales_at(s.n_params);
  q.message_bytes = packed_bytes(s.n_params);
  const dim3 grid(column_blocks(s.n_params), (unsigned)((rows.n + q.rows_per_block - 1) / q.rows_per_block));
  with_storage(s.bf16, [&](auto wt) {
    using WT = typename decltype(wt)::type;
    with_flag(base != nullptr, [&](auto has_base) {
      k_unpack<WT, has_base.value><<<grid, kThreads, 0, s.stream>>>((WT *)s.w, (const WT *)base, messages, q);
    });
  });
}

void launch_aggregate_packed(const PackedShape &s, const PackedWeights &weights, const PackedRows &receivers, void *base,
                             bool move_base, const uint8_t *messages) {
  AggregateParams q;
  q.from = weights;
  q.to = receivers;
  q.move_base = move_base;
  q.n_params = s.n_params;
  q.stride = s.stride;
  q.scales_at = packed_scales_at(s.n_params);
  q.message_bytes = packed_bytes(s.n_params);
  with_storage(s.bf16, [&](auto wt) {
    using WT = typename decltype(wt)::type;
    with_flag(base != nullptr, [&](auto has_base) {
      k_aggregate_packed<WT, has_base.value><<<column_blocks(s.n_params), kThreads, 0, s.stream>>>((WT *)s.w, (WT *)base,
                                                                                                  messages, q);
    });
  });
}

size_t packed_dots_scratch_bytes(int sm_count) {
  return sizeof(double) * (size_t)sm_count * kPackedMaxRows * kPackedMaxRows;
}

cudaError_t launch_packed_dots(const PackedShape &s, const PackedRows &a_rows, const uint8_t *a, const PackedRows &b_rows,
                               const uint8_t *b, float *out, void *scratch) {
  DotsParams q;
  q.a = a_rows;
  q.b = b_rows;
  q.same = a == b && a_rows.n == b_rows.n && memcmp(a_rows.id, b_rows.id, sizeof(a_rows.id)) == 0;
  const int most = a_rows.n > b_rows.n ? a_rows.n : b_rows.n;
  q.rows = 1;
  while (q.rows < most) q.rows *= 2;
  q.segments = kDotsThreads / q.rows;
  q.blocks = (s.n_params + kPackedBlock - 1) / kPackedBlock;
  q.scales_at = packed_scales_at(s.n_params);
  q.message_bytes = packed_bytes(s.n_params);
  const int64_t pieces = (s.n_params + kDotsPiece - 1) / kDotsPiece;
  q.tiles = (pieces + q.segments - 1) / q.segments;
  const int blocks = (int)(q.tiles < s.sm_count ? q.tiles : s.sm_count);
  const int pairs = a_rows.n * b_rows.n;
  cudaError_t rc = cudaSuccess;
  with_flag(q.same != 0, [&](auto same) {
    auto kernel = k_packed_dots<same.value>;
    const int bytes = 1024 + (same.value ? kDotsMaxStages * kDotsSetBytes : 4 * 2 * kDotsSetBytes);
    rc = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (rc == cudaSuccess) kernel<<<blocks, kDotsThreads, bytes, s.stream>>>(a, b, (double *)scratch, q);
  });
  if (rc != cudaSuccess) return rc;
  k_packed_dots_finish<<<(pairs + kThreads / 32 - 1) / (kThreads / 32), kThreads, 0, s.stream>>>(
      (const double *)scratch, blocks, a_rows.n, b_rows.n, q.same, out);
  return cudaSuccess;
}

#ifdef HADFL_DEBUG
int packed_debug_publish(const void *table, size_t bytes) {
  return cudaMemcpyToSymbol(g_debug, table, bytes) == cudaSuccess ? 0 : 1;
}
int packed_debug_error(uint64_t *addr) {
  DebugRanges now;
  if (cudaMemcpyFromSymbol(&now, g_debug, sizeof(now)) != cudaSuccess) return 1;
  if (addr && now.error) *addr = now.bad_addr;
  return now.error ? 1 : 0;
}
#endif

}  // namespace hadfl
