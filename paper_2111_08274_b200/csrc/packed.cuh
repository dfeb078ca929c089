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

// ------------------------------------------------------------------------------------------
// Products of messages, out = A B^T over the parameters, on the tensor cores: the codes and scales of a message are what
// tcgen05.mma kind::mxf4 takes (e2m1 with one ue8m0 scale per 32 along K), so they go from HBM to shared memory as they
// are and are never decoded.  A and B have up to 32 rows, the instruction 128 of each.  The K axis fills them: with R the
// rows rounded up to a power of two, row s R + i of a tile is message i at the s-th of 128 / R consecutive pieces of
// 256 parameters, in A and in B.  The accumulator's R x R blocks on the diagonal are then sums over 128 / R pieces at
// once, and the rest of it is not read.  (With the messages in rows 0 .. R-1 alone every instruction would read 128 rows
// of shared memory for R rows of data, which at R = 8 takes five times as long as HBM takes to deliver them.)
// Rows that no message fills hold whatever was there: a row of A or B reaches its own row or column of the product only.
// The accumulator is fp32 in TMEM, where a long sum of one sign loses bits, so that every kDotsFlush tiles it is added
// to sums in 64 bits.
// ------------------------------------------------------------------------------------------
constexpr int kDotsThreads = 128;   // also the rows of a tile
constexpr int kDotsPiece = 256;     // parameters of a row in a tile: 128 bytes of codes, 8 scales
constexpr int kDotsMaxStages = 6;
constexpr int kDotsFlush = 64;      // 2^14 parameters per row
constexpr int kDotsCodeBytes = kDotsThreads * kDotsPiece / 2;
constexpr int kDotsScaleBytes = kDotsThreads * kDotsPiece / kPackedBlock;
constexpr int kDotsSetBytes = kDotsCodeBytes + kDotsScaleBytes;
constexpr int kDotsTmemColumns = 256;  // 128 of the accumulator, 2 x 16 of scales
constexpr uint32_t kDotsWaitNs = 1000, kDotsMaxWaits = 1u << 20;  // a wait ends after a second or so

struct DotsParams {
  PackedRows a, b;
  int same;               // B is A: one tile, and only pairs i <= j
  int rows;               // R
  int segments;           // pieces of a tile, at most 128 / R

  int64_t tiles;
  int64_t blocks;         // blocks of 32 parameters
  int64_t scales_at, message_bytes;
};

__device__ __forceinline__ uint32_t shared_address(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void copy_async_16(uint32_t to, const void *from, uint32_t bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_async_4(uint32_t to, const void *from, uint32_t bytes) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// Waits for the barrier's phase, with a limit; false if it ran out.
__device__ __forceinline__ bool barrier_wait(uint32_t barrier, uint32_t parity) {
  for (uint32_t i = 0; i < kDotsMaxWaits; ++i) {
    uint32_t done;
    asm volatile(
        "{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\nselp.u32 %0, 1, 0, p;\n}"
        : "=r"(done)
        : "r"(barrier), "r"(parity), "r"(kDotsWaitNs)
        : "memory");
    if (done) return true;
  }
  return false;
}

// Shared-memory descriptors: codes in rows of 128 bytes, eight rows to a swizzle atom of 1024; scales in atoms of
// 8 x 16 bytes without swizzle.
__device__ __forceinline__ uint64_t codes_descriptor(uint32_t at) {
  return (uint64_t)((at & 0x3FFFFu) >> 4) | (uint64_t)1 << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 |
         (uint64_t)2 << 61;
}
__device__ __forceinline__ uint64_t scales_descriptor(uint32_t at) {
  return (uint64_t)((at & 0x3FFFFu) >> 4) | (uint64_t)(128 >> 4) << 32 | (uint64_t)1 << 46;
}
__device__ __forceinline__ void scales_to_tmem(uint32_t tmem, uint32_t at) {
  asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(scales_descriptor(at)) : "memory");
}

// 64 parameters of all rows; `half`: which two of the four scales that a 32-bit column holds.
__device__ __forceinline__ void dots_mma(uint32_t tmem, uint64_t a, uint64_t b, uint32_t scales_a, uint32_t scales_b,
                                         uint32_t half, uint32_t accumulate) {
  constexpr uint32_t kE2m1 = 1u << 7 | 1u << 10, kN = (128u >> 3) << 17, kM = (128u >> 7) << 27, kUe8m0 = 1u << 23;
  const uint32_t instruction = kE2m1 | kN | kM | kUe8m0 | (2 * half) << 4 | (2 * half) << 29;
  asm volatile(
      "{\n.reg .pred p;\nsetp.ne.b32 p, %6, 0;\n"
      "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n}" ::"r"(tmem),
      "l"(a), "l"(b), "r"(instruction), "r"(scales_a), "r"(scales_b), "r"(accumulate)
      : "memory");
}

__device__ __forceinline__ void tmem_load_32(uint32_t at, float (&v)[32]) {
  uint32_t r[32];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,"
      "%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
        "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
        "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(at));
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}

// One thread's part of a tile's copies: 8 pieces of 16 bytes of codes, and the scales of one row.
struct DotsLoader {
  int64_t row[8];         // of the row that piece i belongs to: byte offset of its message, -1 without one
  int64_t own;            // of row threadIdx.x
  const uint8_t *messages;

  __device__ __forceinline__ void start(const uint8_t *m, const PackedRows &ids, const DotsParams &q) {
    messages = m;
#pragma unroll
    for (int i = 0; i < 8; ++i) row[i] = offset(ids, q, i * 16 + (threadIdx.x >> 3));
    own = offset(ids, q, threadIdx.x);
  }
  static __device__ __forceinline__ int64_t offset(const PackedRows &ids, const DotsParams &q, int r) {
    const int i = r & (q.rows - 1);
    return i < ids.n && r < q.segments * q.rows ? ids.id[i] * q.message_bytes : -1;
  }
  // to: the set's place in a stage.  What lies behind the last block is filled with zeros.
  __device__ __forceinline__ void load(uint32_t to, int64_t tile, int log_rows, const DotsParams &q) const {
    const int c = threadIdx.x & 7;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (row[i] < 0) continue;
      const int r = i * 16 + (threadIdx.x >> 3);
      const int64_t block = (tile * q.segments + (r >> log_rows)) * 8 + c;
      const uint8_t *from = messages + row[i] + block * 16;
      const bool there = block < q.blocks && access_ok(from, 16);
      copy_async_16(to + r * 128 + ((c ^ (r & 7)) << 4), there ? from : messages, there ? 16u : 0u);
    }
    if (own < 0) return;
    const int r = threadIdx.x;
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      const int64_t block = (tile * q.segments + (r >> log_rows)) * 8 + 4 * g;
      const uint8_t *from = messages + own + q.scales_at + block;
      const int64_t left = q.blocks - block;
      uint32_t bytes = left >= 4 ? 4u : left > 0 ? (uint32_t)left : 0u;
      if (!access_ok(from, bytes)) bytes = 0;
      copy_async_4(to + kDotsCodeBytes + g * 512 + (r & 31) * 16 + (r >> 5) * 4, bytes ? from : messages, bytes);
    }
  }
};

// partials[pair][block]: 64-bit sums of this block's tiles.
template <bool kSame>
__global__ void __launch_bounds__(kDotsThreads)
k_packed_dots(const uint8_t *__restrict__ a, const uint8_t *__restrict__ b, double *__restrict__ partials,
              const __grid_constant__ DotsParams q) {
  extern __shared__ uint8_t shared[];
  __shared__ __align__(8) uint64_t barriers[kDotsMaxStages];
  __shared__ uint32_t tmem_base;
  __shared__ int failed;
  constexpr int kSets = kSame ? 1 : 2;
  constexpr int kStageBytes = kSets * kDotsSetBytes;
  constexpr int kStages = kSame ? kDotsMaxStages : 4;
  const uint32_t stages_at = (shared_address(shared) + 1023u) & ~1023u;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int log_rows = 31 - __clz(q.rows);
  if (warp == 0) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(shared_address(&tmem_base)),
                 "n"(kDotsTmemColumns)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  if (threadIdx.x == 0) {
    failed = 0;
    for (int i = 0; i < kStages; ++i)
      asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(shared_address(&barriers[i])) : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  DotsLoader from_a, from_b;
  from_a.start(a, q.a, q);
  if (!kSame) from_b.start(b, q.b, q);
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = tmem_base;

  const int n_tiles = (int)((q.tiles - blockIdx.x + gridDim.x - 1) / gridDim.x);
  auto load = [&](int t) {
    if (t < n_tiles) {
      const int64_t tile = blockIdx.x + (int64_t)t * gridDim.x;
      const uint32_t to = stages_at + (t % kStages) * kStageBytes;
      from_a.load(to, tile, log_rows, q);
      if (!kSame) from_b.load(to + kDotsSetBytes, tile, log_rows, q);
    }
    copy_async_commit();
  };
  // Tile t's stage takes tile t + kStages once the products of tile t are done; they are asked for two tiles later, when
  // they are (so that kStages - 2 tiles are in flight).
  constexpr int kAhead = kStages - 2;
  for (int t = 0; t < kAhead; ++t) load(t);
  double sum[32];
#pragma unroll
  for (int i = 0; i < 32; ++i) sum[i] = 0.0;
  int in_sum = 0;
  for (int t = 0; t < n_tiles; ++t) {
    if (t >= 2 && !barrier_wait(shared_address(&barriers[(t - 2) % kStages]), ((t - 2) / kStages) & 1)) failed = 1;
    load(t + kAhead);
    copy_async_wait<kAhead>();
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncthreads();
    if (failed) break;
    if (threadIdx.x == 0) {
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      const uint32_t stage = stages_at + (t % kStages) * kStageBytes;
      const uint32_t stage_b = kSame ? stage : stage + kDotsSetBytes;
      const uint32_t scales = tmem + 128 + (t & 1) * 16;  // not those that the tile before still uses
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        scales_to_tmem(scales + 4 * g, stage + kDotsCodeBytes + g * 512);
        if (!kSame) scales_to_tmem(scales + 8 + 4 * g, stage_b + kDotsCodeBytes + g * 512);
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t scales_a = scales + 4 * (k / 2), scales_b = kSame ? scales_a : scales_a + 8;
        dots_mma(tmem, codes_descriptor(stage + 32 * k), codes_descriptor(stage_b + 32 * k), scales_a, scales_b, k & 1,
                 in_sum > 0 || k > 0);
      }
      asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(
                       shared_address(&barriers[t % kStages]))
                   : "memory");
    }
    if (++in_sum == kDotsFlush || t + 1 == n_tiles) {
      if (!barrier_wait(shared_address(&barriers[t % kStages]), (t / kStages) & 1)) failed = 1;
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      // Row r needs columns r / R * R .. + R - 1: they lie among the 32 of its warp's rows.
      float v[32];
      tmem_load_32(tmem + ((uint32_t)(warp * 32) << 16) + warp * 32, v);
#pragma unroll
      for (int i = 0; i < 32; ++i) sum[i] += (double)v[i];
      in_sum = 0;
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      __syncthreads();
      if (failed) break;
    }
  }
  copy_async_wait<0>();
  if (failed) barrier_wait(shared_address(&barriers[(n_tiles - 1) % kStages]), ((n_tiles - 1) / kStages) & 1);
  __syncthreads();
  // The blocks on the diagonal, segment by segment, in the stages' place.
  double *mine = reinterpret_cast<double *>(shared + (stages_at - shared_address(shared)));
  const int row_in = threadIdx.x & (q.rows - 1), segment = threadIdx.x >> log_rows;
#pragma unroll
  for (int i = 0; i < 32; ++i)
    if ((i >> log_rows) == (lane >> log_rows)) mine[((segment << log_rows) + row_in << log_rows) + (i & (q.rows - 1))] = sum[i];
  __syncthreads();
  const int pairs = q.a.n * q.b.n;
  for (int p = threadIdx.x; p < pairs; p += kDotsThreads) {
    const int i = p / q.b.n, j = p - i * q.b.n;
    if (kSame && i > j) continue;
    double total = 0.0;
    for (int s = 0; s < q.segments; ++s) total += mine[((s << log_rows) + i << log_rows) + j];
    // A wait that ran out (which nothing is known to cause) shows as products that are no numbers.
    double *at = partials + (int64_t)p * gridDim.x + blockIdx.x;
    if (access_ok(at, 8)) *at = failed ? __longlong_as_double(0x7FF8000000000000ll) : total;
  }
  if (warp == 0)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(kDotsTmemColumns) : "memory");
}

// out[pair] = sum of the blocks' partial sums in a fixed order, a warp per pair; of a set with itself each sum is for two.
__global__ void __launch_bounds__(kThreads)
k_packed_dots_finish(const double *__restrict__ partials, int n_blocks, int m, int n, int same, float *__restrict__ out) {
  const int p = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (p >= m * n) return;
  const int i = p / n, j = p - i * n;
  if (same && i > j) return;
  double sum = 0.0;
  for (int k = lane; k < n_blocks; k += 32) sum += partials[(int64_t)p * n_blocks + k];
  sum = warp_sum(sum);
  if (lane) return;
  if (access_ok(out + p, 4)) out[p] = (float)sum;
  if (same && i < j && access_ok(out + j * n + i, 4)) out[j * n + i] = (float)sum;
}

}  // namespace hadfl
