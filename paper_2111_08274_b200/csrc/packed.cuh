// sm_100a kernels of the exchange in messages of microscaled 4-bit floating point.
//
// A message of P parameters is ceil(P / 32) blocks of 32 codes (e2m1: sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6; two per
// byte, the even parameter in the low half) and one byte per block, the power-of-two scale 2^(byte - 127) (255: the block
// reads as NaN, as one with a value that is not finite or nearly so does).  With u the fp32 values to send and A the
// largest |u| of a block, the scale is the smallest power of two, 2^-127 or larger, with A <= 6 * scale: no value is cut
// off, so stochastic rounding is free of bias, and what nearest rounding leaves out is at most one scale (stochastic
// rounding: below two).
//
// All of it streams: a thread has 32 bytes of a row of parameters, 8 fp32 or 16 bf16 values, and four or two
// threads a block of 32, so that a warp's codes are one or two lines of 128 bytes.
#pragma once
#include <cuda_fp16.h>
#include <cuda_fp4.h>

#include "packed.h"
#include "storage.cuh"

namespace hadfl {

constexpr uint32_t kPackedNan = 255;

// The kernels here are launched as dependents of what is before them in the stream (launch_dependent): their blocks may
// become resident while the kernel before still runs, and touch no memory before this.  It returns when that kernel is
// done and its writes are visible; as every kernel here begins with it, so is everything before that.  Data that the kernel
// before may write are read by ordinary loads (or cp.async) behind the wait: no kernel here has a __restrict__ pointer, which
// would promise that nobody writes the data while the kernel is there, and so allow loads through the read-only path or
// ahead of the wait.
__device__ __forceinline__ void wait_for_stream() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
// The kernel behind this one may become resident once all blocks are here.
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// Parameters per thread, in parts of 8.
template <typename WT>
struct PackedE {
  static constexpr int value = 32 / (int)sizeof(WT), parts = value / 8;
};

// E consecutive values of a row as they come from memory.
template <typename T, int kParts>
struct RawParts {
  RawPack<T, 8> part[kParts];
};
// live: how many of the values there are; FullPack<8 * kParts> where all are.
template <typename T, int kParts, typename Live>
__device__ __forceinline__ void ld_parts(const T *at, Live live, RawParts<T, kParts> &r) {
#pragma unroll
  for (int i = 0; i < kParts; ++i) {
    if constexpr (std::is_same_v<Live, int>) {
      const int here = min(max(live - 8 * i, 0), 8);
      zero_raw(r.part[i]);
      if (here > 0) ld_raw(at + 8 * i, here, r.part[i]);
    } else {
      ld_raw(at + 8 * i, 8, r.part[i]);
    }
  }
}
struct Eight {
  __device__ constexpr operator int() const { return 8; }
};
// Values to a row, rounded to its storage type.  k32: the row starts at a multiple of 32 bytes; whole 32 bytes then go out
// in one store (two of 16 write half of each 32-byte sector at a time, see st_full).
template <bool k32, typename T, int E, typename Live>
__device__ __forceinline__ void st_parts(T *at, Live live, const float (&v)[E]) {
  if constexpr (k32 && sizeof(T) == 2) {
    if (live >= E) {
      if (!access_ok(at, 2 * E)) return;
      uint32_t x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = floats_to_bf16x2(v[2 * i], v[2 * i + 1]);
      asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(at), "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]),
                   "r"(x[4]), "r"(x[5]), "r"(x[6]), "r"(x[7])
                   : "memory");
      return;
    }
  }
  if constexpr (std::is_same_v<Live, int> || !k32 || sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < E / 8; ++i) {
      const int here = min(live - 8 * i, 8);
      float x[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = v[8 * i + j];
      if (here == 8)
        st_pack_any(at + 8 * i, 0, std::conditional_t<k32, FullPack<8>, Eight>{}, x);
      else if (here > 0)
        st_pack_any(at + 8 * i, 0, here, x);
    }
  }
}
// Calls f(live) for a thread's columns, with FullPack where all columns of the block are there.
template <int E, typename F>
__device__ __forceinline__ void with_live(int64_t n_params, int64_t block, F &&f) {
  if (E * kThreads * (block + 1) <= n_params)
    f(FullPack<E>{});
  else
    f(live_of(n_params, block * kThreads + threadIdx.x, E));
}

// 2^(byte - 127), NaN for 255.
__device__ __forceinline__ float packed_scale(uint32_t byte) {
  const uint32_t bits = byte == 0u ? 0x00400000u : byte << 23;
  return __uint_as_float(byte == kPackedNan ? 0x7FC00000u : bits);
}

// The values of 8 codes, without their scale.
__device__ __forceinline__ void packed_values(uint32_t codes, float *v) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __half2_raw h = __nv_cvt_fp4x2_to_halfraw2((__nv_fp4x2_storage_t)(codes >> (8 * i)), __NV_E2M1);
    const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h));
    v[2 * i] = f.x;
    v[2 * i + 1] = f.y;
  }
}

// 8 values y (|y| <= 6) as codes, rounded to nearest, ties to even.
__device__ __forceinline__ uint32_t packed_codes(const float *y) {
  uint32_t codes = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    codes |= (uint32_t)__nv_cvt_float2_to_fp4x2(make_float2(y[2 * i], y[2 * i + 1]), __NV_E2M1, cudaRoundNearest)
             << (8 * i);
  return codes;
}

// ... rounded away from zero with probability (way from the lower value) / (distance of the two).  t = y * 2^-126 has |y| = 1
// at the smallest normal number, so that its bits have the spacing of e2m1 throughout - even below 1, where both formats
// are subnormal - and bits 22 to 24 are the code.  (t is rounded to 2^-23 of y's unit, as fl(|y| + 1) is.)  The 16
// random bits are added to the upper 16 of the 22 bits below, a carry is the step up.  Codes and signs are then gathered
// in 16-bit halves, parameters i and i + 4 in one word, so that a shift or a mask is for two of them.
__device__ __forceinline__ uint32_t packed_codes_stochastic(const float *t, const uint32_t (&r)[4]) {
  uint32_t up[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) up[i] = __float_as_uint(t[i]) + ((i & 1 ? r[i / 2] >> 16 : r[i / 2] & 0xFFFFu) << 6);
  uint32_t codes = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t two = __byte_perm(up[i], up[i + 4], 0x7632);  // in each half: the sign at 15, the code at 6 to 8
    const uint32_t magnitude = 4 * i < 6 ? two >> (6 - 4 * i) : two << (4 * i - 6);
    codes |= (magnitude & 0x00070007u << 4 * i) | (two >> (12 - 4 * i) & 0x00080008u << 4 * i);
  }
  return codes;
}

// Random words of the 8 parameters of a group: the first two rounds of Philox4x32-10 on the counter (group, round, device,
// tag), split into what depends on the group alone (once per thread), on the device alone (on the host: RowRandom) and
// the three exclusive ors of both.
struct RowRandom {
  uint32_t c0, c2, c3;
};
struct GroupRandom {
  uint32_t a, b, c;
};
__device__ __forceinline__ GroupRandom group_random(uint32_t group, uint32_t tag, const PhiloxKeys &k) {
  const unsigned long long p0 = (unsigned long long)kPhiloxM0 * group;
  const unsigned long long p1 = (unsigned long long)kPhiloxM1 * ((uint32_t)(p0 >> 32) ^ tag ^ k.b[0]);
  return GroupRandom{(uint32_t)(p1 >> 32), (uint32_t)p1, (uint32_t)p0};
}
__device__ __forceinline__ void random_words(const GroupRandom &g, const RowRandom &row, const PhiloxKeys &k,
                                             uint32_t (&r)[4]) {
  r[0] = g.a ^ row.c0;
  r[1] = g.b;
  r[2] = g.c ^ row.c2;
  r[3] = row.c3;
#pragma unroll
  for (int i = 2; i < 10; ++i) philox_round(r[0], r[1], r[2], r[3], k.a[i], k.b[i]);
}

// The largest magnitude; NaN if there is one.
__device__ __forceinline__ float max_magnitude(float a, float b, float c) {
  float d;
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

struct PackParams {
  int n, rows_per_block, row_blocks;
  uint32_t tag;  // word 3 of the rounding's counter
  int64_t n_params;
  int64_t code_columns, scale_columns;  // columns that the message's codes and scales have room for
  int64_t scales_at;
  int64_t row_at[kPackedMaxRows], message_at[kPackedMaxRows];
  RowRandom random[kPackedMaxRows];
};

// Quantisation.  A thread walks over the rows of its columns with the base in registers, and loads the next row while it
// works on one (with a residual, whose loads are twice as many bytes, other blocks do for that: 92 us instead of 111 for 4 of
// 11.2 M fp32 parameters with stochastic rounding, which then has room for more blocks).
//
// Bound by HBM, except with stochastic rounding and no residual, where the instructions bind (bf16: 18.6 per parameter,
// most of them the generator's, against 9.9 with rounding to nearest).  Measured, us, and of the copy bandwidth (of what has
// to be read and written): 4 of 11.2 M fp32, base, residual, stochastic 90 (102 %); 16 of 14.7 M bf16, base, nearest 105 (91 %),
// stochastic 174 (55 %; 72 % of the issue slots used); 4 of 2^27 fp32 alone 342 (109 %).
// Blocks per SM that the compiler is to leave registers for (0: it chooses, mostly few registers and many blocks).  Measured, us,
// packed and read, the compiler's choice / this one: bf16 without a residual, to nearest, 5 blocks with 48 registers
// instead of 64: 16 of 14.7 M 207 / 202; with a residual 4 blocks, whose loads then go out together: 8 of 2 M fp32 51.5 / 47.4, 8
// of 8.4 M 181 / 180.  Of the others, fp32 without a residual loses with fewer blocks (4 of 2^27 727; left to one block 780, to
// five 746); bf16 with stochastic rounding has not been measured with any other number (with a base it takes 71 registers,
// which are three blocks).
template <typename WT, bool kResidual, bool kStochastic>
constexpr int pack_min_blocks() {
  if (kResidual) return 4;
  return sizeof(WT) == 2 && !kStochastic ? 5 : 0;
}
template <typename WT, bool kBase, bool kResidual, bool kStochastic, bool k32>
__global__ void __launch_bounds__(kThreads, pack_min_blocks<WT, kResidual, kStochastic>())
k_pack(const WT *w, const WT *base, float *residual, uint8_t *messages,
       PhiloxKeys keys, const __grid_constant__ PackParams q) {
  constexpr int E = PackedE<WT>::value, kParts = PackedE<WT>::parts, kLanes = kPackedBlock / E;
  constexpr bool kPrefetch = !kResidual;
  const int64_t block = blockIdx.x / q.row_blocks;
  const int64_t group = block * kThreads + threadIdx.x;
  const int64_t column = E * group;
  let_next_start();
  wait_for_stream();
  if (column >= q.scale_columns) return;  // whole warps: scale_columns is a multiple of 32 * 128
  const int first = blockIdx.x % q.row_blocks * q.rows_per_block;
  const int end = min(first + q.rows_per_block, q.n);
  with_live<E>(q.n_params, block, [&](auto live) {
    RawParts<WT, kParts> base_raw;
    if (kBase) ld_parts(base + column, live, base_raw);
    GroupRandom group_part[kParts];
    if (kStochastic) {
#pragma unroll
      for (int i = 0; i < kParts; ++i) group_part[i] = group_random((uint32_t)(group * kParts + i), q.tag, keys);
    }
    struct Row {
      RawParts<WT, kParts> w;
      RawParts<float, kParts> e;
    };
    auto load = [&](int j, Row &r) {
      const int64_t at = q.row_at[j] + column;
      ld_parts(w + at, live, r.w);
      if (kResidual) ld_parts(residual + at, live, r.e);
    };
    Row next;
    if (kPrefetch) load(first, next);
#pragma unroll(kPrefetch ? 2 : 1)
    for (int j = first; j < end; ++j) {
      Row row;
      if (kPrefetch) {
        row = next;
        if (j + 1 < end) load(j + 1, next);
      } else {
        load(j, row);
      }
      float u[E];
#pragma unroll
      for (int i = 0; i < kParts; ++i) {
        float v[8];
        unpack(row.w.part[i], v);
        if (kBase) {
          float b[8];
          unpack(base_raw.part[i], b);
#pragma unroll
          for (int k = 0; k < 8; ++k) v[k] = __fsub_rn(v[k], b[k]);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) u[8 * i + k] = kResidual ? __fadd_rn(v[k], row.e.part[i].v[k]) : v[k];
      }
      // The largest magnitude of the block, as bits: infinities and NaNs are above all finite values.
      float most_here = 0.f;
#pragma unroll
      for (int i = 0; i < E; i += 2) most_here = max_magnitude(most_here, u[i], u[i + 1]);
      uint32_t most = __float_as_uint(most_here);
#pragma unroll
      for (int lanes = 1; lanes < kLanes; lanes *= 2) most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, lanes));
      const bool lost = most > 0x7F400000u;  // above 6 * 2^125: a larger scale's codes 4 to 6 would read as infinities
      // A = m 2^E: the scale's exponent is E - 2 for m <= 1.5, else E - 1; the sum carries into the exponent where m > 1.5.
      const int exponent = (int)((most + 0x3FFFFFu) >> 23) - 2;
      const uint32_t byte = lost ? kPackedNan : (uint32_t)max(exponent, 0);
      uint32_t codes[kParts];
      if (kStochastic) {
        // 2^-(s + 126); where that is no number of fp32 (s > 23), 2^-110 is taken off before.  (What then underflows is below
        // 2^-40 of the scale: 0 in t either way.)
        const bool large = byte > 127u + 23u;
        const float down = large ? 0x1p-110f : 1.0f;
        const uint32_t biased = 128u + (large ? 110u : 0u) - byte;  // exponent + 127 of what is left
        const float to_t = (int)biased > 0 ? __uint_as_float(biased << 23) : __uint_as_float(0x00400000u >> -(int)biased);
#pragma unroll
        for (int i = 0; i < kParts; ++i) {
          float t[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) t[k] = u[8 * i + k];
          if (__any_sync(0xFFFFFFFFu, large)) {  // (a branch: as a condition of each product it is 3 us of 176)
#pragma unroll
            for (int k = 0; k < 8; ++k) t[k] = __fmul_rn(t[k], down);
          }
#pragma unroll
          for (int k = 0; k < 8; ++k) t[k] = __fmul_rn(t[k], to_t);
          uint32_t r[4];
          random_words(group_part[i], q.random[j], keys, r);
          codes[i] = packed_codes_stochastic(t, r);
        }
      } else {
        const float inverse = __uint_as_float((254u - byte) << 23);
#pragma unroll
        for (int i = 0; i < kParts; ++i) {
          float y[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) y[k] = __fmul_rn(u[8 * i + k], inverse);
          codes[i] = packed_codes(y);
        }
      }
      if (lost) {
#pragma unroll
        for (int i = 0; i < kParts; ++i) codes[i] = 0;
      }
      uint8_t *message = messages + q.message_at[j];
      if (column < q.code_columns && access_ok(message + column / 2, 4 * kParts)) {
        if constexpr (kParts == 2)
          *reinterpret_cast<uint2 *>(message + column / 2) = make_uint2(codes[0], codes[1]);
        else
          *reinterpret_cast<uint32_t *>(message + column / 2) = codes[0];
      }
      if ((threadIdx.x & (kLanes - 1)) == 0) {
        uint8_t *at = message + q.scales_at + column / kPackedBlock;
        if (access_ok(at, 1)) *at = (uint8_t)byte;
      }
      if (kResidual && live > 0) {
        const float scale = packed_scale(byte);
        float v[E];
#pragma unroll
        for (int i = 0; i < kParts; ++i) packed_values(codes[i], v + 8 * i);
#pragma unroll
        for (int i = 0; i < E; ++i) v[i] = lost ? 0.f : fmaf(-v[i], scale, u[i]);  // the product is exact
        st_parts<k32>(residual + q.row_at[j] + column, live, v);
      }
    }
  });
}

// The codes and the scale byte of a message at a thread's columns.
template <int kParts>
struct RawCodes {
  uint32_t codes[kParts], byte;
};
template <int kParts>
__device__ __forceinline__ RawCodes<kParts> ld_codes(const uint8_t *message, int64_t column, int64_t scales_at) {
  RawCodes<kParts> r;
  memset(&r, 0, sizeof(r));
  if (access_ok(message + column / 2, 4 * kParts)) {
    if constexpr (kParts == 2) {
      const uint2 c = *reinterpret_cast<const uint2 *>(message + column / 2);
      r.codes[0] = c.x;
      r.codes[1] = c.y;
    } else {
      r.codes[0] = *reinterpret_cast<const uint32_t *>(message + column / 2);
    }
  }
  const uint8_t *at = message + scales_at + column / kPackedBlock;
  if (access_ok(at, 1)) r.byte = *at;
  return r;
}
template <int kParts>
__device__ __forceinline__ void packed_decode(const RawCodes<kParts> &r, float (&d)[8 * kParts]) {
#pragma unroll
  for (int i = 0; i < kParts; ++i) packed_values(r.codes[i], d + 8 * i);
  const float scale = packed_scale(r.byte);
#pragma unroll
  for (int i = 0; i < 8 * kParts; ++i) d[i] = __fmul_rn(d[i], scale);
}

// Messages whose loads are in flight together.  Measured, us, 4 / 8: 16 of 32 bf16 devices of 23.5 M parameters 168 / 190,
// 4 of 8 fp32 devices of 11.2 M 43.0 / 47.0, 32 fp32 devices of 4.2 M 112 / 111.
constexpr int kPackedBatch = 4;

struct UnpackParams {
  int n, rows_per_block, row_blocks;
  int64_t n_params, scales_at;
  int64_t row_at[kPackedMaxRows], message_at[kPackedMaxRows];
};

// w[i] = base + d_i for the listed devices.  Bound by HBM: 16 of 14.7 M bf16 98 us, 93 % of the copy bandwidth; 4 of 2^27 fp32
// 368 us, 101 %.
template <typename WT, bool kBase, bool k32>
__global__ void __launch_bounds__(kThreads)
k_unpack(WT *w, const WT *base, const uint8_t *messages, const __grid_constant__ UnpackParams q) {
  constexpr int E = PackedE<WT>::value, kParts = PackedE<WT>::parts, B = kPackedBatch;
  const int64_t block = blockIdx.x / q.row_blocks;
  const int64_t column = E * (block * kThreads + threadIdx.x);
  const int first = blockIdx.x % q.row_blocks * q.rows_per_block;
  const int end = min(first + q.rows_per_block, q.n);
  let_next_start();
  wait_for_stream();
  if (column >= q.n_params) return;
  with_live<E>(q.n_params, block, [&](auto live) {
    RawParts<WT, kParts> base_raw;
    if (kBase) ld_parts(base + column, live, base_raw);
    for (int j0 = first; j0 < end; j0 += B) {
      RawCodes<kParts> raw[B];
#pragma unroll
      for (int j = 0; j < B; ++j)
        if (j0 + j < end) raw[j] = ld_codes<kParts>(messages + q.message_at[j0 + j], column, q.scales_at);
#pragma unroll
      for (int j = 0; j < B; ++j) {
        if (j0 + j >= end) continue;
        float d[E];
        packed_decode(raw[j], d);
        if (kBase) {
#pragma unroll
          for (int i = 0; i < kParts; ++i) {
            float b[8];
            unpack(base_raw.part[i], b);
#pragma unroll
            for (int k = 0; k < 8; ++k) d[8 * i + k] = __fadd_rn(b[k], d[8 * i + k]);
          }
        }
        st_parts<k32>(w + q.row_at[j0 + j] + column, live, d);
      }
    }
  });
}

struct AggregateParams {
  int k, n, move_base;
  int64_t n_params, scales_at;
  float a[kPackedMaxRows];
  int64_t row_at[kPackedMaxRows], message_at[kPackedMaxRows];
};

// Eq. 5 from messages: acc = a_0 d_0, acc = fma(a_j, d_j, acc); base + acc to the receivers and, on request, the base.  Bound by
// HBM: 4 of 8 fp32 devices of 11.2 M parameters 42 us, 90 % of the copy bandwidth; 16 of 32 bf16 devices of 23.5 M 166 us,
// 92 %; 4 of 16 fp32 devices of 2^25 to all 386 us, 98 %.
template <typename WT, bool kBase, bool k32>
__global__ void __launch_bounds__(kThreads)
k_aggregate_packed(WT *w, WT *base, const uint8_t *messages, const __grid_constant__ AggregateParams q) {
  constexpr int E = PackedE<WT>::value, kParts = PackedE<WT>::parts, B = kPackedBatch;
  const int64_t block = blockIdx.x;
  const int64_t column = E * (block * kThreads + threadIdx.x);
  let_next_start();
  wait_for_stream();
  if (column >= q.n_params) return;
  with_live<E>(q.n_params, block, [&](auto live) {
    RawParts<WT, kParts> base_raw;
    if (kBase) ld_parts((const WT *)base + column, live, base_raw);
    float acc[E];
    for (int j0 = 0; j0 < q.k; j0 += B) {
      RawCodes<kParts> raw[B];
#pragma unroll
      for (int j = 0; j < B; ++j)
        if (j0 + j < q.k) raw[j] = ld_codes<kParts>(messages + q.message_at[j0 + j], column, q.scales_at);
#pragma unroll
      for (int j = 0; j < B; ++j) {
        if (j0 + j >= q.k) continue;
        const float a = q.a[j0 + j];
        float d[E];
        packed_decode(raw[j], d);
#pragma unroll
        for (int i = 0; i < E; ++i) acc[i] = j0 + j == 0 ? __fmul_rn(a, d[i]) : fmaf(a, d[i], acc[i]);
      }
    }
    if (kBase) {
#pragma unroll
      for (int i = 0; i < kParts; ++i) {
        float b[8];
        unpack(base_raw.part[i], b);
#pragma unroll
        for (int k = 0; k < 8; ++k) acc[8 * i + k] = __fadd_rn(b[k], acc[8 * i + k]);
      }
    }
    for (int j = 0; j < q.n; ++j) st_parts<k32>(w + q.row_at[j] + column, live, acc);
    if (kBase && q.move_base) st_parts<k32>(base + column, live, acc);
  });
}

// ------------------------------------------------------------------------------------------
// Products of messages, out = A B^T over the parameters, on the tensor cores: the codes and scales of a message are what
// tcgen05.mma kind::mxf4 takes (e2m1 with one ue8m0 scale per 32 along K), so they go from HBM to shared memory as they
// are and are never decoded.  A and B have up to 32 rows, the instruction 128 of each.  The K axis fills them: with R the
// larger number of rows and g = floor(32 / R), each 32 rows of a tile are all messages at g of 4 g consecutive pieces of
// 256 parameters, one after the other, in A and in B.  The accumulator's R x R blocks on the diagonal are then sums over
// as many pieces at once, each within the 32 x 32 of one warp's lanes, and the rest of it is not read.  (R rounded up to a
// power of two instead, with 128 / R pieces: 5 messages of 26.8 M parameters 19.9 us, against 15.4.  Blocks that go on
// across the bounds of the 32 rows, 128 / R of them whatever R: the scales of a piece then no longer begin at a sector, and
// sums cannot stay in registers: 17 messages of 7.9 M 23.3 us, against 21.4.)  (With the messages in rows 0 .. R-1 alone every instruction would read 128 rows
// of shared memory for R rows of data, which at R = 8 takes five times as long as HBM takes to deliver them.)
// Rows that no message fills hold whatever was there: a row of A or B reaches its own row or column of the product only.
// The accumulator is fp32 in TMEM, where a long sum of one sign loses bits, so that every kDotsFlush tiles it is added
// to sums in 64 bits.
// ------------------------------------------------------------------------------------------
// Warps for the copies, for the accumulators' rows, and to ask for the products, each of the latter with an accumulator.
constexpr int kDotsLoadWarps = 8, kDotsSumWarps = 4, kDotsMmaWarps = 2;
constexpr int kDotsThreads = 32 * (kDotsLoadWarps + kDotsSumWarps + kDotsMmaWarps);
constexpr int kDotsRows = 128;      // of a tile
constexpr int kDotsPiece = 256;     // parameters of a row in a tile: 128 bytes of codes, 8 scales
constexpr int kDotsFlush = 64;      // 2^14 parameters per row
constexpr int kDotsCodeBytes = kDotsRows * kDotsPiece / 2;
constexpr int kDotsScaleBytes = kDotsRows * kDotsPiece / kPackedBlock;
constexpr int kDotsSetBytes = kDotsCodeBytes + kDotsScaleBytes;
constexpr int kDotsTmemColumns = 512;  // the accumulators, 128 each, and the scales of the tiles, 64
// Tiles in shared memory: a multiple of kDotsMmaWarps, so that a stage's tiles are asked for by one thread, one after the
// other, and the parity of a phase tells which one is there.  Measured, us: one set of 32 messages of 23.5 M parameters with 4 /
// 6 / 8 stages 78 / 67 / 65; two sets of 32 of 16.8 M with 4 / 6 89 / 134 (six leave the L1 18 KB, and the scales' copies of
// 4 bytes share their sectors there).
template <bool kSame>
struct DotsStages {
  static constexpr int value = kSame ? 8 : 4;
  static_assert(value % kDotsMmaWarps == 0);
  static constexpr int bytes = (kSame ? 1 : 2) * kDotsSetBytes;
};
constexpr uint32_t kDotsWaitNs = 1000, kDotsMaxWaits = 1u << 20;  // a wait ends after a second or so

struct DotsParams {
  PackedRows a, b;
  int rows;               // R
  int per_warp;           // pieces that 32 rows hold, g
  int segments;           // pieces of a tile, 4 g
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
// The barrier gets this thread's arrival once its copies so far are there.
__device__ __forceinline__ void copy_async_arrive(uint64_t *barrier) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(shared_address(barrier)) : "memory");
}
__device__ __forceinline__ void copy_async_wait_all() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// Waits for the barrier's phase, with a limit; false if it ran out.
__device__ __forceinline__ bool barrier_wait(uint64_t *barrier, uint32_t parity) {
  for (uint32_t i = 0; i < kDotsMaxWaits; ++i) {
    uint32_t done;
    asm volatile(
        "{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\nselp.u32 %0, 1, 0, p;\n}"
        : "=r"(done)
        : "r"(shared_address(barrier)), "r"(parity), "r"(kDotsWaitNs)
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

// Tensor memory.  These instructions are aligned, that is undefined where the lanes of a warp are apart (behind a wait, a
// loop or a branch that each lane takes by itself), so that the lanes meet before each; all of them come here or none.
__device__ __forceinline__ void tmem_alloc(uint32_t *base) {
  __syncwarp();
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(shared_address(base)),
               "n"(kDotsTmemColumns)
               : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_free(uint32_t base) {
  __syncwarp();
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(base), "n"(kDotsTmemColumns) : "memory");
}
__device__ __forceinline__ void tmem_load_32(uint32_t at, float (&v)[32]) {
  uint32_t r[32];
  __syncwarp();
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

// What row r of a tile holds: a message and one of the tile's pieces, -1 where it holds none.
struct DotsRow {
  int message, segment;
};
__device__ __forceinline__ DotsRow dots_row(int r, const DotsParams &q) {
  const int s = (r & 31) / q.rows;
  return DotsRow{(r & 31) - s * q.rows, s < q.per_warp ? (r >> 5) * q.per_warp + s : -1};
}

// One thread's part of a tile's copies: four pieces of 16 bytes of codes, and four scales.
struct DotsLoader {
  static constexpr int kThreadsOf = 32 * kDotsLoadWarps, kPieces = kDotsRows * 8 / kThreadsOf;
  const uint8_t *codes[kPieces], *scales;  // in tile 0; null where no message fills the row
  int64_t block[kPieces], scale_block;     // and which block of 32 parameters that is
  uint32_t to[kPieces], scales_to;         // places in a set

  __device__ __forceinline__ void start(const uint8_t *messages, const PackedRows &ids, const DotsParams &q) {
    const int c = threadIdx.x & 7;
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int r = i * (kThreadsOf / 8) + (threadIdx.x >> 3);
      const DotsRow row = dots_row(r, q);
      block[i] = (int64_t)row.segment * 8 + c;
      codes[i] = start_of(messages, row, ids, q, block[i] * 16);
      to[i] = r * 128 + ((c ^ (r & 7)) << 4);  // 16-byte pieces change places within a row, the 128-byte swizzle
    }
    const int r = threadIdx.x & (kDotsRows - 1), g = threadIdx.x / kDotsRows;
    const DotsRow row = dots_row(r, q);
    scale_block = (int64_t)row.segment * 8 + 4 * g;
    scales = start_of(messages, row, ids, q, q.scales_at + scale_block);
    scales_to = kDotsCodeBytes + g * 512 + (r & 31) * 16 + (r >> 5) * 4;
  }
  static __device__ __forceinline__ const uint8_t *start_of(const uint8_t *messages, const DotsRow &row,
                                                            const PackedRows &ids, const DotsParams &q, int64_t offset) {
    return row.segment >= 0 && row.message < ids.n ? messages + ids.id[row.message] * q.message_bytes + offset : nullptr;
  }
  // at: the set's place in a stage.  What lies behind the last block is filled with zeros.
  __device__ __forceinline__ void load(uint32_t at, int64_t tile, const DotsParams &q) const {
    const int64_t first = tile * q.segments * 8;  // block of the tile
    if (first + q.segments * 8 <= q.blocks) {
#pragma unroll
      for (int i = 0; i < kPieces; ++i)
        if (codes[i] && access_ok(codes[i] + first * 16, 16)) copy_async_16(at + to[i], codes[i] + first * 16, 16u);
      if (scales && access_ok(scales + first, 4)) copy_async_4(at + scales_to, scales + first, 4u);
      return;
    }
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      if (!codes[i]) continue;
      const bool there = first + block[i] < q.blocks && access_ok(codes[i] + first * 16, 16);
      copy_async_16(at + to[i], there ? codes[i] + first * 16 : codes[i], there ? 16u : 0u);
    }
    if (!scales) return;
    const int64_t left = q.blocks - first - scale_block;
    uint32_t bytes = left >= 4 ? 4u : left > 0 ? (uint32_t)left : 0u;
    if (!access_ok(scales + first, bytes)) bytes = 0;
    copy_async_4(at + scales_to, bytes ? scales + first : scales, bytes);
  }
};

__device__ __forceinline__ void barrier_init(uint64_t *barrier, int count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(shared_address(barrier)), "r"(count) : "memory");
}
__device__ __forceinline__ void barrier_arrive(uint64_t *barrier) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(shared_address(barrier)) : "memory");
}
// The barrier gets an arrival once all products so far are done.
__device__ __forceinline__ void barrier_commit(uint64_t *barrier) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(shared_address(barrier))
               : "memory");
}

// A ring of tiles in shared memory between the warps that copy and the threads that ask for the products, an accumulator
// between each of those and the warps that add them up.  partials[pair][block]: 64-bit sums of the block's tiles.
// Bound by HBM for long messages, else by the way from the first copy to the last sum (about 4 us with the finish).  Measured,
// us, and of the copy bandwidth: 32 of 23.5 M parameters 65 (94 %; 75 to 80 in a long run, under the power limit), two sets
// of 32 of 16.8 M 89 (98 %), 8 of 11.2 M 12.3 (59 %), 4 of 100,000 3.9; of 2^27 parameters in all, 5 messages 15.4 (71 %), 9
// 15.9, and 17, which leave the lower half of every 32 rows empty, 21.4 (51 %).  One thread that asks for products instead of
// two: 103, 102, 17.6 us for these three (what each tile waits for then adds up to more than its copies take); three:
// 66 to 75, no gain.
template <bool kSame>
__global__ void __launch_bounds__(kDotsThreads)
k_packed_dots(const uint8_t *a, const uint8_t *b, double *partials,
              const __grid_constant__ DotsParams q) {
  using Stages = DotsStages<kSame>;
  constexpr int kStages = Stages::value;
  extern __shared__ uint8_t shared[];
  __shared__ __align__(8) uint64_t full[kStages], empty[kStages];
  __shared__ __align__(8) uint64_t sum_full[kDotsMmaWarps], sum_empty[kDotsMmaWarps], drained[kDotsMmaWarps];
  __shared__ uint32_t tmem_base;
  __shared__ int failed;
  const uint32_t stages_at = (shared_address(shared) + 1023u) & ~1023u;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int n_tiles = (int)((q.tiles - blockIdx.x + gridDim.x - 1) / gridDim.x);
  if (warp == kDotsLoadWarps) tmem_alloc(&tmem_base);
  if (warp == kDotsLoadWarps + 1 && lane == 0) {
    failed = 0;
    for (int i = 0; i < kStages; ++i) {
      barrier_init(&full[i], 32 * kDotsLoadWarps);
      barrier_init(&empty[i], 1);
    }
    for (int i = 0; i < kDotsMmaWarps; ++i) {
      barrier_init(&sum_full[i], 1);
      barrier_init(&sum_empty[i], kDotsSumWarps);
      barrier_init(&drained[i], 1);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  DotsLoader from_a, from_b;
  auto load = [&](int t) {
    const int64_t tile = blockIdx.x + (int64_t)t * gridDim.x;
    const uint32_t to = stages_at + (t % kStages) * Stages::bytes;
    from_a.load(to, tile, q);
    if (!kSame) from_b.load(to + kDotsSetBytes, tile, q);
  };
  if (warp < kDotsLoadWarps) {
    from_a.start(a, q.a, q);
    if (!kSame) from_b.start(b, q.b, q);
    wait_for_stream();
    load(0);
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = tmem_base;
  let_next_start();  // all blocks have their tensor memory by then, so that those of the next call cannot be in their way
  double sum[32];

  if (warp < kDotsLoadWarps) {
    copy_async_arrive(&full[0]);
    for (int t = 1; t < n_tiles; ++t) {
      // The stage's last tile was t - kStages; its products are done.
      if (t >= kStages && !barrier_wait(&empty[t % kStages], (t / kStages - 1) & 1)) {
        failed = 1;
        break;
      }
      load(t);
      copy_async_arrive(&full[t % kStages]);
    }
    copy_async_wait_all();
  } else if (warp < kDotsLoadWarps + kDotsSumWarps) {
#pragma unroll
    for (int i = 0; i < 32; ++i) sum[i] = 0.0;
    // What a row needs of the accumulator lies among the columns with its warp's 32 rows' numbers.
    const uint32_t rows = (warp - kDotsLoadWarps) * 32;
    const int n_sums = (n_tiles + kDotsMmaWarps * kDotsFlush - 1) / (kDotsMmaWarps * kDotsFlush);
    bool there = true;
    for (int f = 0; f < n_sums && there; ++f) {
      for (int m = 0; m < kDotsMmaWarps; ++m) {
        if (n_tiles <= m + f * kDotsMmaWarps * kDotsFlush) break;
        // One answer for the warp: its lanes go on, or stop, together.
        there = __all_sync(0xFFFFFFFFu, barrier_wait(&sum_full[m], f & 1));
        if (!there) {
          failed = 1;
          break;
        }
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        float v[32];
        tmem_load_32(tmem + (rows << 16) + m * kDotsRows + rows, v);
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncwarp();
        if (lane == 0) barrier_arrive(&sum_empty[m]);
#pragma unroll
        for (int i = 0; i < 32; ++i) sum[i] += (double)v[i];
      }
    }
  } else if (lane == 0) {
    // Warp m takes the tiles t = m, m + kDotsMmaWarps, ...: what one tile has to wait for (its copies, the fence, its
    // scales) passes under the products of another.
    const int m = warp - kDotsLoadWarps - kDotsSumWarps;
    const uint32_t accumulator = tmem + m * kDotsRows;
    int in_sum = 0, f = 0;
    for (int t = m; t < n_tiles; t += kDotsMmaWarps) {
      if (in_sum == 0 && f > 0 && !barrier_wait(&sum_empty[m], (f - 1) & 1)) {
        failed = 1;
        break;
      }
      const int stage = t % kStages;
      if (!barrier_wait(&full[stage], (t / kStages) & 1)) {
        failed = 1;
        break;
      }
      // The copies were made through the generic proxy, the tensor core reads through the asynchronous one.  (The threads
      // that copy would wait here for all their copies in flight.)
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      const uint32_t at = stages_at + stage * Stages::bytes, at_b = kSame ? at : at + kDotsSetBytes;
      // The scales have a place per stage: it is free when the stage is.
      const uint32_t scales = tmem + kDotsMmaWarps * kDotsRows + stage * (kSame ? 8 : 16);
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        scales_to_tmem(scales + 4 * g, at + kDotsCodeBytes + g * 512);
        if (!kSame) scales_to_tmem(scales + 8 + 4 * g, at_b + kDotsCodeBytes + g * 512);
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t scales_a = scales + 4 * (k / 2), scales_b = kSame ? scales_a : scales_a + 8;
        dots_mma(accumulator, codes_descriptor(at + 32 * k), codes_descriptor(at_b + 32 * k), scales_a, scales_b, k & 1,
                 in_sum > 0 || k > 0);
      }
      barrier_commit(&empty[stage]);
      if (++in_sum == kDotsFlush || t + kDotsMmaWarps >= n_tiles) {
        barrier_commit(&sum_full[m]);
        in_sum = 0;
        ++f;
      }
    }
    // Nothing is in flight when the tensor memory is given back, even if some wait above ran out.
    barrier_commit(&drained[m]);
    if (!barrier_wait(&drained[m], 0)) failed = 1;
  }
  __syncthreads();
  wait_for_stream();  // (done long since) what follows writes where the call before may have read
  // The blocks on the diagonal, [segment][j][i], in the stages' place (whose last products are in the sums).
  double *mine = reinterpret_cast<double *>(shared + (stages_at - shared_address(shared)));
  if (warp >= kDotsLoadWarps && warp < kDotsLoadWarps + kDotsSumWarps) {
    const DotsRow row = dots_row(threadIdx.x - 32 * kDotsLoadWarps, q);
    const int begin = lane - row.message;  // of the row's block among the warp's columns
#pragma unroll
    for (int c = 0; c < 32; ++c) {
      const int j = c - begin;
      if (row.segment >= 0 && j >= 0 && j < q.rows) mine[(row.segment * q.rows + j) * q.rows + row.message] = sum[c];
    }
  }
  __syncthreads();
  // A lane has every `lanes`-th segment of a pair, four to six of them; then a butterfly over a pair's lanes.
  const int log_lanes = 31 - __clz(q.per_warp), per_warp = 32 >> log_lanes, part = lane >> (5 - log_lanes);
  const int all = q.rows * q.rows;
  for (int e0 = warp * per_warp; e0 < all; e0 += kDotsThreads / 32 * per_warp) {
    const int e = e0 + (lane & (per_warp - 1)), j = e / q.rows, i = e - j * q.rows;
    double total = 0.0;
    if (e < all)
      for (int s = part; s < q.segments; s += 1 << log_lanes) total += mine[s * all + e];
    for (int off = 16; off >= per_warp; off >>= 1) total += __shfl_xor_sync(0xFFFFFFFFu, total, off);
    if (part || e >= all || i >= q.a.n || j >= q.b.n || (kSame && i > j)) continue;
    // A wait that ran out (which nothing is known to cause) shows as products that are no numbers.
    double *at = partials + (int64_t)(i * q.b.n + j) * gridDim.x + blockIdx.x;
    if (access_ok(at, 8)) *at = failed ? __longlong_as_double(0x7FF8000000000000ll) : total;
  }
  if (warp == kDotsLoadWarps) tmem_free(tmem);
}

// out[pair] = sum of the blocks' partial sums in a fixed order, a warp per pair; of a set with itself each sum is for two.
__global__ void __launch_bounds__(kThreads)
k_packed_dots_finish(const double *partials, int n_blocks, int m, int n, int same, float *out) {
  const int p = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  const int i = p / n, j = p - i * n;
  let_next_start();
  wait_for_stream();
  if (p >= m * n || (same && i > j)) return;
  double sum = 0.0;
  for (int k = lane; k < n_blocks; k += 32) sum += __ldcg(partials + (int64_t)p * n_blocks + k);
  sum = warp_sum(sum);
  if (lane) return;
  if (access_ok(out + p, 4)) out[p] = (float)sum;
  if (same && i < j && access_ok(out + j * n + i, 4)) out[j * n + i] = (float)sum;
}

}  // namespace hadfl
