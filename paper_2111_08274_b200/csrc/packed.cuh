// sm_100a kernels of the exchange in messages of microscaled 4-bit floating point.
//
// A message of P parameters is ceil(P / 32) blocks of 32 codes (e2m1: sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6; two per
// byte, the even parameter in the low half) and one byte per block, the power-of-two scale 2^(byte - 127) (255: the block
// reads as NaN, as one with a value that is not finite or nearly so does).  With u the fp32 values to send and A the largest |u| of a block, the scale is the smallest power of two,
// 2^-127 or larger, with A <= 6 * scale: no value is cut off, so stochastic rounding is free of bias and the residual of
// a block at most one scale.
//
// All of it streams: 8 consecutive parameters per thread, four threads per block of 32, so that a warp's loads are 1 KB
// of fp32 parameters, its codes one line of 128 bytes, its scales 8 bytes.
#pragma once
#include <cuda_fp16.h>
#include <cuda_fp4.h>

#include "packed.h"
#include "storage.cuh"

namespace hadfl {

constexpr int kPackedE = 8;  // parameters per thread
constexpr uint32_t kPackedNan = 255;

// 2^(byte - 127), NaN for 255.
__device__ __forceinline__ float packed_scale(uint32_t byte) {
  const uint32_t bits = byte == 0u ? 0x00400000u : byte << 23;
  return __uint_as_float(byte == kPackedNan ? 0x7FC00000u : bits);
}

// The values of 8 codes, without their scale.
__device__ __forceinline__ void packed_values(uint32_t codes, float (&v)[kPackedE]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __half2_raw h = __nv_cvt_fp4x2_to_halfraw2((__nv_fp4x2_storage_t)(codes >> (8 * i)), __NV_E2M1);
    const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h));
    v[2 * i] = f.x;
    v[2 * i + 1] = f.y;
  }
}

__device__ __forceinline__ uint32_t packed_codes(const float (&y)[kPackedE]) {
  uint32_t codes = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    codes |= (uint32_t)__nv_cvt_float2_to_fp4x2(make_float2(y[2 * i], y[2 * i + 1]), __NV_E2M1, cudaRoundNearest)
             << (8 * i);
  return codes;
}

// |y| <= 6 to a neighbour on the e2m1 grid, away from zero with probability (way from the lower one) / (spacing): 16
// random bits are added to the upper 16 of the 22 mantissa bits that e2m1 does not have, and the 22 bits dropped.  Below
// 1 the grid is evenly spaced, as it is from 1 to 2, where the sum with 1 is.
__device__ __forceinline__ float packed_stochastic(float y, uint32_t r16) {
  const float t = fabsf(y);
  const bool small = t < 1.0f;
  float z = small ? __fadd_rn(t, 1.0f) : t;
  z = __uint_as_float((__float_as_uint(z) + (r16 << 6)) & 0xFFC00000u);
  return copysignf(small ? z - 1.0f : z, y);
}

struct PackParams {
  PackedRows rows;
  int rows_per_block;
  uint32_t round_lo, tag;  // words 1 and 3 of the rounding's counter
  int64_t n_params, stride;
  int64_t code_columns, scale_columns;  // columns that the message's codes and scales have room for
  int64_t scales_at, message_bytes;
};

// Quantisation.  A thread walks over the rows of its 8 columns with the base in registers.
template <typename WT, bool kBase, bool kResidual, bool kStochastic>
__global__ void __launch_bounds__(kThreads)
k_pack(const WT *__restrict__ w, const WT *base, float *__restrict__ residual, uint8_t *__restrict__ messages,
       PhiloxKeys keys, const __grid_constant__ PackParams q) {
  constexpr int E = kPackedE;
  const int64_t p = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int64_t column = E * p;
  if (column >= q.scale_columns) return;  // whole warps: scale_columns is a multiple of 32 * 128
  const int live = live_of(q.n_params, p, E);
  RawPack<WT, E> base_raw;
  zero_raw(base_raw);
  if (kBase && live > 0) ld_raw(base + column, live, base_raw);
  const int first = blockIdx.y * q.rows_per_block;
  const int end = min(first + q.rows_per_block, q.rows.n);
  for (int j = first; j < end; ++j) {
    const int dev = q.rows.id[j];
    const int64_t row = (int64_t)dev * q.stride;
    RawPack<WT, E> w_raw;
    RawPack<float, E> e_raw;
    zero_raw(w_raw);
    zero_raw(e_raw);
    if (live > 0) {
      ld_raw(w + row + column, live, w_raw);
      if (kResidual) ld_raw(residual + row + column, live, e_raw);
    }
    float u[E];
    unpack(w_raw, u);
    if (kBase) {
      float b[E];
      unpack(base_raw, b);
#pragma unroll
      for (int i = 0; i < E; ++i) u[i] = __fsub_rn(u[i], b[i]);
    }
    if (kResidual) {
#pragma unroll
      for (int i = 0; i < E; ++i) u[i] = __fadd_rn(u[i], e_raw.v[i]);
    }
    // The largest magnitude of the block, as bits: infinities and NaNs are above all finite values.
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < E; ++i) most = max(most, __float_as_uint(u[i]) & 0x7FFFFFFFu);
    most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, 1));
    most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, 2));
    const bool lost = most > 0x7F400000u;  // above 6 * 2^125: a larger scale's codes 4 to 6 would read as infinities
    // A = m 2^E: the scale's exponent is E - 2 for m <= 1.5, else E - 1; the sum carries into the exponent where m > 1.5.
    const int exponent = (int)((most + 0x3FFFFFu) >> 23) - 2;
    const uint32_t byte = lost ? kPackedNan : (uint32_t)max(exponent, 0);
    const float inverse = __uint_as_float((254u - byte) << 23);
    float y[E];
#pragma unroll
    for (int i = 0; i < E; ++i) y[i] = __fmul_rn(u[i], inverse);
    if (kStochastic) {
      uint32_t c0 = (uint32_t)p, c1 = q.round_lo, c2 = (uint32_t)dev, c3 = q.tag;
      philox4x32_10(c0, c1, c2, c3, keys);
      const uint32_t r[4] = {c0, c1, c2, c3};
#pragma unroll
      for (int i = 0; i < E; ++i) y[i] = packed_stochastic(y[i], i & 1 ? r[i / 2] >> 16 : r[i / 2] & 0xFFFFu);
    }
    const uint32_t codes = lost ? 0u : packed_codes(y);
    uint8_t *message = messages + (int64_t)dev * q.message_bytes;
    if (column < q.code_columns && access_ok(message + column / 2, 4)) *reinterpret_cast<uint32_t *>(message + column / 2) = codes;
    if ((threadIdx.x & 3) == 0) {
      uint8_t *at = message + q.scales_at + column / kPackedBlock;
      if (access_ok(at, 1)) *at = (uint8_t)byte;
    }
    if (kResidual && live > 0) {
      float v[E];
      packed_values(codes, v);
      const float scale = packed_scale(byte);
#pragma unroll
      for (int i = 0; i < E; ++i) v[i] = lost ? 0.f : __fsub_rn(u[i], v[i] * scale);
      st_pack_any(residual + row, p, live, v);
    }
  }
}

// The 8 codes and the scale byte of a message at a thread's columns (past the last block: zeros).
struct RawCodes {
  uint32_t codes, byte;
};
__device__ __forceinline__ RawCodes ld_codes(const uint8_t *message, int64_t column, int64_t scales_at) {
  RawCodes r{0u, 0u};
  if (access_ok(message + column / 2, 4)) r.codes = *reinterpret_cast<const uint32_t *>(message + column / 2);
  const uint8_t *at = message + scales_at + column / kPackedBlock;
  if (access_ok(at, 1)) r.byte = *at;
  return r;
}
__device__ __forceinline__ void packed_decode(const RawCodes &r, float (&d)[kPackedE]) {
  packed_values(r.codes, d);
  const float scale = packed_scale(r.byte);
#pragma unroll
  for (int i = 0; i < kPackedE; ++i) d[i] = __fmul_rn(d[i], scale);
}

struct UnpackParams {
  PackedRows rows;
  int rows_per_block;
  int64_t n_params, stride, scales_at, message_bytes;
};

// w[i] = base + d_i for the listed devices.
template <typename WT, bool kBase>
__global__ void __launch_bounds__(kThreads)
k_unpack(WT *w, const WT *base, const uint8_t *__restrict__ messages, const __grid_constant__ UnpackParams q) {
  constexpr int E = kPackedE;
  const int64_t p = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int64_t column = E * p;
  const int live = live_of(q.n_params, p, E);
  if (live == 0) return;
  float b[E];
  if (kBase) {
    RawPack<WT, E> raw;
    ld_raw(base + column, live, raw);
    unpack(raw, b);
  }
  const int first = blockIdx.y * q.rows_per_block;
  const int end = min(first + q.rows_per_block, q.rows.n);
  for (int j = first; j < end; ++j) {
    const int dev = q.rows.id[j];
    float d[E];
    packed_decode(ld_codes(messages + (int64_t)dev * q.message_bytes, column, q.scales_at), d);
    if (kBase) {
#pragma unroll
      for (int i = 0; i < E; ++i) d[i] = __fadd_rn(b[i], d[i]);
    }
    st_pack_any(w + (int64_t)dev * q.stride, p, live, d);
  }
}

struct AggregateParams {
  PackedWeights from;
  PackedRows to;
  int move_base;
  int64_t n_params, stride, scales_at, message_bytes;
};

// Eq. 5 from messages: acc = a_0 d_0, acc = fma(a_j, d_j, acc); base + acc to the receivers and, on request, the base.
template <typename WT, bool kBase>
__global__ void __launch_bounds__(kThreads)
k_aggregate_packed(WT *w, WT *base, const uint8_t *__restrict__ messages, const __grid_constant__ AggregateParams q) {
  constexpr int E = kPackedE, B = 4;
  const int64_t p = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int64_t column = E * p;
  const int live = live_of(q.n_params, p, E);
  if (live == 0) return;
  RawPack<WT, E> base_raw;
  if (kBase) ld_raw(base + column, live, base_raw);
  float acc[E];
  for (int j0 = 0; j0 < q.from.k; j0 += B) {
    RawCodes raw[B];
#pragma unroll
    for (int j = 0; j < B; ++j)
      if (j0 + j < q.from.k) raw[j] = ld_codes(messages + (int64_t)q.from.id[j0 + j] * q.message_bytes, column, q.scales_at);
#pragma unroll
    for (int j = 0; j < B; ++j) {
      if (j0 + j >= q.from.k) continue;
      const float a = q.from.a[j0 + j];
      float d[E];
      packed_decode(raw[j], d);
#pragma unroll
      for (int i = 0; i < E; ++i) acc[i] = j0 + j == 0 ? __fmul_rn(a, d[i]) : fmaf(a, d[i], acc[i]);
    }
  }
  if (kBase) {
    float b[E];
    unpack(base_raw, b);
#pragma unroll
    for (int i = 0; i < E; ++i) acc[i] = __fadd_rn(b[i], acc[i]);
  }
  for (int j = 0; j < q.to.n; ++j) st_pack_any(w + (int64_t)q.to.id[j] * q.stride, p, live, acc);
  if (kBase && q.move_base) st_pack_any(base, p, live, acc);
}

struct DotsParams {
  PackedRows a, b;
  int64_t n_params, scales_at, message_bytes;
};

// Products of messages.  A block takes tiles of 64 columns: the values of all rows as fp32 in shared memory, four of the
// up to 1024 pairs per thread, fp32 within a tile and 64 bits above; partials[block][pair].
constexpr int kDotsColumns = 64;
__global__ void __launch_bounds__(kThreads)
k_packed_dots(const uint8_t *__restrict__ a, const uint8_t *__restrict__ b, double *__restrict__ partials,
              const __grid_constant__ DotsParams q) {
  __shared__ float rows[2 * kPackedMaxRows][kDotsColumns + 1];
  const int pairs = q.a.n * q.b.n;
  double sum[4] = {};
  const int64_t tiles = (q.n_params + kDotsColumns - 1) / kDotsColumns;
  for (int64_t t = blockIdx.x; t < tiles; t += gridDim.x) {
    for (int i = threadIdx.x; i < (q.a.n + q.b.n) * (kDotsColumns / kPackedE); i += kThreads) {
      const int r = i / (kDotsColumns / kPackedE), c = i % (kDotsColumns / kPackedE) * kPackedE;
      const int64_t column = t * kDotsColumns + c;
      const uint8_t *m = r < q.a.n ? a + q.a.id[r] * q.message_bytes : b + q.b.id[r - q.a.n] * q.message_bytes;
      float d[kPackedE] = {};
      if (column < q.n_params) packed_decode(ld_codes(m, column, q.scales_at), d);
      const int at = r < q.a.n ? r : kPackedMaxRows + r - q.a.n;
#pragma unroll
      for (int k = 0; k < kPackedE; ++k) rows[at][c + k] = d[k];
    }
    __syncthreads();
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const int pair = threadIdx.x + s * kThreads;
      if (pair >= pairs) break;
      const float *x = rows[pair / q.b.n], *y = rows[kPackedMaxRows + pair % q.b.n];
      float dot = 0.f;
      for (int c = 0; c < kDotsColumns; ++c) dot = fmaf(x[c], y[c], dot);
      sum[s] += (double)dot;
    }
    __syncthreads();
  }
  for (int s = 0; s < 4; ++s) {
    const int pair = threadIdx.x + s * kThreads;
    if (pair < pairs) partials[(int64_t)blockIdx.x * pairs + pair] = sum[s];
  }
}

// out[pair] = sum of the blocks' partial sums, in their order.
__global__ void __launch_bounds__(kThreads)
k_packed_dots_finish(const double *__restrict__ partials, int n_blocks, int pairs, float *__restrict__ out) {
  const int pair = blockIdx.x * kThreads + threadIdx.x;
  if (pair >= pairs) return;
  double sum = 0;
  for (int i = 0; i < n_blocks; ++i) sum += partials[(int64_t)i * pairs + pair];
  if (access_ok(out + pair, 4)) out[pair] = (float)sum;
}

}  // namespace hadfl
