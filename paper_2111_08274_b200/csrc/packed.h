// Messages of microscaled 4-bit floating point: their layout (host arithmetic) and the launches of packed.cu.
// A launch only enqueues; the callers in hadfl.cu have checked every argument.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "philox.cuh"

namespace hadfl {

constexpr int kPackedBlock = 32;       // parameters that share a scale
constexpr int kPackedAlign = 128;      // codes and scales each fill up a multiple of this many bytes
constexpr int kPackedMaxRows = 32;
constexpr uint32_t kTagPack = 0x51000000u;  // 'Q': stochastic rounding of messages, counter (p / 8, round, device, tag|round>>32)

// Byte offset of the scales in a message of n_params parameters, and the message's bytes.
inline int64_t packed_scales_at(int64_t n_params) {
  const int64_t blocks = (n_params + kPackedBlock - 1) / kPackedBlock;
  return (blocks * (kPackedBlock / 2) + kPackedAlign - 1) / kPackedAlign * kPackedAlign;
}
inline int64_t packed_bytes(int64_t n_params) {
  const int64_t blocks = (n_params + kPackedBlock - 1) / kPackedBlock;
  return packed_scales_at(n_params) + (blocks + kPackedAlign - 1) / kPackedAlign * kPackedAlign;
}

struct PackedRows {
  int32_t n;
  int32_t id[kPackedMaxRows];
};

// What all launches are told of the arena and the messages.
struct PackedShape {
  void *w;            // arena
  int64_t stride;     // elements between its rows, and between those of the residual
  int64_t n_params;
  bool bf16;
  int sm_count;
  cudaStream_t stream;
};

struct PackedWeights {
  int32_t k;
  int32_t id[kPackedMaxRows];
  float a[kPackedMaxRows];
};

cudaError_t launch_pack(const PackedShape &s, const PackedRows &rows, const void *base, float *residual, bool stochastic,
                 uint64_t round, const PhiloxKeys &keys, uint8_t *messages);
cudaError_t launch_unpack(const PackedShape &s, const PackedRows &rows, const void *base, const uint8_t *messages);
cudaError_t launch_aggregate_packed(const PackedShape &s, const PackedWeights &weights, const PackedRows &receivers, void *base,
                             bool move_base, const uint8_t *messages);
// out[i * b_rows.n + j] = sum over the parameters of message a_rows.id[i] of a times message b_rows.id[j] of b.
// scratch: packed_dots_scratch_bytes() bytes.  shared_allowed: kept by the handle, false at first.
size_t packed_dots_scratch_bytes(int sm_count, int n_devices, int64_t n_params);
cudaError_t launch_packed_dots(const PackedShape &s, const PackedRows &a_rows, const uint8_t *a, const PackedRows &b_rows,
                               const uint8_t *b, float *out, void *scratch, bool (&shared_allowed)[2]);

// Debug build: this file's kernels have a range table of their own.
int packed_debug_publish(const void *table, size_t bytes);
int packed_debug_error(uint64_t *addr);

}  // namespace hadfl
