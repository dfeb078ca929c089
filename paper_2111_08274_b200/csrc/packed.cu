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

// Blocks of kThreads threads that cover the columns.
unsigned column_blocks(bool bf16, int64_t columns) {
  const int64_t per_block = (int64_t)kThreads * (bf16 ? PackedE<__nv_bfloat16>::value : PackedE<float>::value);
  return (unsigned)((columns + per_block - 1) / per_block);
}

// A launch whose blocks may become resident while the kernel before it in the stream still runs (they wait for it
// themselves, see wait_for_stream): the start of a kernel passes under the end of the one before.  Measured, us, launches
// one after the other / so: products of 4 messages of 100,000 parameters 6.1 / 4.9, of 8 of 11.2 M 14.9 / 13.5; aggregate 4
// fp32 devices of 11.2 M 42.6 / 41.8, read the same 34.3 / 33.5.
template <typename... Params, typename... Args>
cudaError_t launch_dependent(void (*kernel)(Params...), unsigned grid, int threads, size_t shared_bytes, cudaStream_t stream,
                             Args... args) {
  cudaLaunchConfig_t config = {};
  config.gridDim = dim3(grid);
  config.blockDim = dim3((unsigned)threads);
  config.dynamicSmemBytes = shared_bytes;
  config.stream = stream;
  cudaLaunchAttribute early;
  early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  early.val.programmaticStreamSerializationAllowed = 1;
  config.attrs = &early;
  config.numAttrs = 1;
  const cudaError_t rc = cudaLaunchKernelEx(&config, kernel, static_cast<Params>(args)...);
  if (rc != cudaSuccess) cudaGetLastError();  // it is this call's, and not to be found by the next one
  return rc;
}

bool at_32(const void *p) { return ((uintptr_t)p & 31u) == 0; }

// The rows of a pack or unpack launch, and how many of them a block walks over: all, so that the base is loaded once, but
// fewer where the columns alone make less than two blocks per SM.  Measured, us, all rows / split: pack, 2 of 100,000 fp32
// parameters (25 or 49 blocks of columns) 2.40 / 1.96; 32 of 200,000 fp32 (98 blocks) 11.8 / 6.6; 16 of 300,000 bf16 (74)
// 6.3 / 5.7; from two blocks per SM on no split: 16 of 1 M fp32 (489) 33.1 / 37.1.
// together: no split, where one block may not write what another one reads.
template <typename Params>
unsigned split_rows(const PackedShape &s, const PackedRows &rows, int64_t columns, bool together, Params &q) {
  const unsigned blocks = column_blocks(s.bf16, columns);
  const unsigned sms = (unsigned)s.sm_count;
  const int split = blocks < 2 * sms && !together ? (int)((4 * sms + blocks - 1) / blocks) : 1;
  q.n = rows.n;
  q.rows_per_block = split < rows.n ? (rows.n + split - 1) / split : 1;
  q.row_blocks = (rows.n + q.rows_per_block - 1) / q.rows_per_block;
  q.n_params = s.n_params;
  q.scales_at = packed_scales_at(s.n_params);
  for (int j = 0; j < rows.n; ++j) {
    q.row_at[j] = rows.id[j] * s.stride;
    q.message_at[j] = rows.id[j] * packed_bytes(s.n_params);
  }
  return blocks * (unsigned)q.row_blocks;
}

}  // namespace

cudaError_t launch_pack(const PackedShape &s, const PackedRows &rows, const void *base, float *residual, bool stochastic,
                 uint64_t round, const PhiloxKeys &keys, uint8_t *messages) {
  PackParams q;
  const int64_t scales_at = packed_scales_at(s.n_params);
  q.code_columns = scales_at * 2;
  q.scale_columns = (packed_bytes(s.n_params) - scales_at) * kPackedBlock;
  const unsigned grid = split_rows(s, rows, q.scale_columns, false, q);
  q.tag = kTagPack | ((uint32_t)(round >> 32) & 0xFFFFFFu);
  for (int j = 0; j < rows.n; ++j) {
    // The rounds of the generator that the device takes part in alone (see random_words).
    const uint64_t p1 = (uint64_t)kPhiloxM1 * (uint32_t)rows.id[j];
    const uint64_t p0 = (uint64_t)kPhiloxM0 * ((uint32_t)(p1 >> 32) ^ (uint32_t)round ^ keys.a[0]);
    q.random[j] = RowRandom{(uint32_t)p1 ^ keys.a[1], (uint32_t)(p0 >> 32) ^ keys.b[1], (uint32_t)p0};
  }
  cudaError_t rc = cudaSuccess;
  with_storage(s.bf16, [&](auto wt) {
    using WT = typename decltype(wt)::type;
    with_flag(base != nullptr, [&](auto has_base) {
      with_flag(residual != nullptr, [&](auto has_residual) {
        with_flag(stochastic, [&](auto is_stochastic) {
          with_flag(at_32(residual), [&](auto is_at_32) {
            if constexpr (has_residual.value || is_at_32.value)  // without a residual there are no stores to rows
              rc = launch_dependent(k_pack<WT, has_base.value, has_residual.value, is_stochastic.value, is_at_32.value>, grid,
                                    kThreads, 0, s.stream, (const WT *)s.w, (const WT *)base, residual, messages, keys, q);
          });
        });
      });
    });
  });
  return rc;
}

cudaError_t launch_unpack(const PackedShape &s, const PackedRows &rows, const void *base, const uint8_t *messages) {
  UnpackParams q;
  // A base that is one of the rows to be written: a thread loads it before it writes any row of its columns.
  bool base_is_written = false;
  for (int j = 0; j < rows.n; ++j)
    base_is_written |= base == (const char *)s.w + rows.id[j] * s.stride * (s.bf16 ? 2 : 4);
  const unsigned grid = split_rows(s, rows, s.n_params, base_is_written, q);
  cudaError_t rc = cudaSuccess;
  with_storage(s.bf16, [&](auto wt) {
    using WT = typename decltype(wt)::type;
    with_flag(base != nullptr, [&](auto has_base) {
      with_flag(at_32(s.w) && s.stride % (int64_t)(32 / sizeof(WT)) == 0, [&](auto is_at_32) {
        rc = launch_dependent(k_unpack<WT, has_base.value, is_at_32.value>, grid, kThreads, 0, s.stream, (WT *)s.w,
                              (const WT *)base, messages, q);
      });
    });
  });
  return rc;
}

cudaError_t launch_aggregate_packed(const PackedShape &s, const PackedWeights &weights, const PackedRows &receivers, void *base,
                             bool move_base, const uint8_t *messages) {
  AggregateParams q;
  q.k = weights.k;
  q.n = receivers.n;
  q.move_base = move_base;
  q.n_params = s.n_params;
  q.scales_at = packed_scales_at(s.n_params);
  for (int j = 0; j < q.k; ++j) {
    q.a[j] = weights.a[j];
    q.message_at[j] = weights.id[j] * packed_bytes(s.n_params);
  }
  for (int j = 0; j < q.n; ++j) q.row_at[j] = receivers.id[j] * s.stride;
  const unsigned grid = column_blocks(s.bf16, s.n_params);
  cudaError_t rc = cudaSuccess;
  with_storage(s.bf16, [&](auto wt) {
    using WT = typename decltype(wt)::type;
    with_flag(base != nullptr, [&](auto has_base) {
      with_flag(at_32(s.w) && at_32(base) && s.stride % (int64_t)(32 / sizeof(WT)) == 0, [&](auto is_at_32) {
        rc = launch_dependent(k_aggregate_packed<WT, has_base.value, is_at_32.value>, grid, kThreads, 0, s.stream, (WT *)s.w,
                              (WT *)base, messages, q);
      });
    });
  });
  return rc;
}

namespace {

// Tiles of a launch, with `rows` the larger number of messages, and its blocks.
int64_t dots_tiles(int64_t n_params, int rows) {
  const int64_t pieces = (n_params + kDotsPiece - 1) / kDotsPiece;
  const int segments = kDotsRows / 32 * (32 / rows);
  return (pieces + segments - 1) / segments;
}
int dots_blocks(int64_t tiles, int sm_count) { return (int)(tiles < sm_count ? tiles : sm_count); }

}  // namespace

size_t packed_dots_scratch_bytes(int sm_count, int n_devices, int64_t n_params) {
  // Fewer messages make tiles of more parameters, and not more blocks.
  const int blocks = dots_blocks(dots_tiles(n_params, n_devices), sm_count);
  return sizeof(double) * (size_t)blocks * (size_t)n_devices * (size_t)n_devices;
}

cudaError_t launch_packed_dots(const PackedShape &s, const PackedRows &a_rows, const uint8_t *a, const PackedRows &b_rows,
                               const uint8_t *b, float *out, void *scratch, bool (&shared_allowed)[2]) {
  DotsParams q;
  q.a = a_rows;
  q.b = b_rows;
  const bool same = a == b && a_rows.n == b_rows.n && memcmp(a_rows.id, b_rows.id, sizeof(a_rows.id)) == 0;
  q.rows = a_rows.n > b_rows.n ? a_rows.n : b_rows.n;
  q.per_warp = 32 / q.rows;
  q.segments = kDotsRows / 32 * q.per_warp;
  q.blocks = (s.n_params + kPackedBlock - 1) / kPackedBlock;
  q.scales_at = packed_scales_at(s.n_params);
  q.message_bytes = packed_bytes(s.n_params);
  q.tiles = dots_tiles(s.n_params, q.rows);
  const int blocks = dots_blocks(q.tiles, s.sm_count);
  const int pairs = a_rows.n * b_rows.n;
  double *partials = (double *)scratch;
  cudaError_t rc = cudaSuccess;
  with_flag(same, [&](auto is_same) {
    using Stages = DotsStages<is_same.value>;
    auto kernel = k_packed_dots<is_same.value>;
    const int bytes = 1024 + Stages::value * Stages::bytes;
    bool &allowed = shared_allowed[is_same.value];
    if (!allowed) rc = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    allowed = rc == cudaSuccess;
    if (allowed)
      rc = launch_dependent(kernel, (unsigned)blocks, kDotsThreads, bytes, s.stream, a, b, partials, q);
    else
      cudaGetLastError();
  });
  if (rc != cudaSuccess) return rc;
  return launch_dependent(k_packed_dots_finish, (unsigned)((pairs + kThreads / 32 - 1) / (kThreads / 32)), kThreads, 0,
                          s.stream, (const double *)partials, blocks, (int)a_rows.n, (int)b_rows.n, (int)same, out);
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
