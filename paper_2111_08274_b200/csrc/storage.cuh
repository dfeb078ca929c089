// How the kernels read and write rows of parameters: packs of consecutive values held by one thread, fp32 or bf16
// in memory, whole or ragged at the end of a row.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>
#include <string.h>

#include <type_traits>

#include "debug_check.cuh"

namespace hadfl {

constexpr int kMaxDevices = 32;
constexpr int kThreads = 256;

// ------------------------------------------------------------------------------------------
// Storage access by element and by column group (used by the initial-model kernel and by the
// ragged last pack of a row).
// ------------------------------------------------------------------------------------------
__device__ __forceinline__ void st_group(float *row, int64_t g, float4 v) {
  if (!access_ok(row + 4 * g, 16)) return;
  *reinterpret_cast<float4 *>(row + 4 * g) = v;
}
__device__ __forceinline__ void st_group(__nv_bfloat16 *row, int64_t g, float4 v) {
  if (!access_ok(row + 4 * g, 8)) return;
  const __nv_bfloat162 lo = __floats2bfloat162_rn(v.x, v.y);
  const __nv_bfloat162 hi = __floats2bfloat162_rn(v.z, v.w);
  uint2 raw;
  raw.x = *reinterpret_cast<const uint32_t *>(&lo);
  raw.y = *reinterpret_cast<const uint32_t *>(&hi);
  *reinterpret_cast<uint2 *>(row + 4 * g) = raw;
}
__device__ __forceinline__ void st_elem(float *row, int64_t p, float v) {
  if (access_ok(row + p, 4)) row[p] = v;
}
__device__ __forceinline__ void st_elem(__nv_bfloat16 *row, int64_t p, float v) {
  if (access_ok(row + p, 2)) row[p] = __float2bfloat16_rn(v);
}

// ------------------------------------------------------------------------------------------
// Packs: E consecutive parameters held by one thread (E = 4 or 8).  fp32: E/4 128-bit accesses;
// bf16: one 64-bit (E = 4) or 128-bit (E = 8) access.  A pack of 8 is two column groups, i.e.
// two Philox blocks.  `live` < E only in the ragged last pack of a row.
// ------------------------------------------------------------------------------------------
template <typename WT>
struct Pack16 {  // the pack that is 16 bytes of storage
  static constexpr int E = sizeof(WT) == 2 ? 8 : 4;
};

template <int E>
__device__ __forceinline__ void st_pack(float *row, int64_t p, const float (&v)[E]) {
  if (!access_ok(row + E * p, 4 * E)) return;
#pragma unroll
  for (int i = 0; i < E / 4; ++i)
    *reinterpret_cast<float4 *>(row + E * p + 4 * i) =
        make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
}
__device__ __forceinline__ void bf16x2_to_floats(uint32_t raw, float &lo, float &hi) {
  lo = __uint_as_float(raw << 16);
  hi = __uint_as_float(raw & 0xFFFF0000u);
}
__device__ __forceinline__ uint32_t floats_to_bf16x2(float lo, float hi) {
  const __nv_bfloat162 t = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t *>(&t);
}
template <int E>
__device__ __forceinline__ void st_pack(__nv_bfloat16 *row, int64_t p, const float (&v)[E]) {
  if (!access_ok(row + E * p, 2 * E)) return;
  if (E == 8) {
    uint4 raw;
    raw.x = floats_to_bf16x2(v[0], v[1]);
    raw.y = floats_to_bf16x2(v[2], v[3]);
    raw.z = floats_to_bf16x2(v[E - 4], v[E - 3]);
    raw.w = floats_to_bf16x2(v[E - 2], v[E - 1]);
    *reinterpret_cast<uint4 *>(row + 8 * p) = raw;
  } else {
    uint2 raw;
    raw.x = floats_to_bf16x2(v[0], v[1]);
    raw.y = floats_to_bf16x2(v[2], v[3]);
    *reinterpret_cast<uint2 *>(row + 4 * p) = raw;
  }
}
// A loaded pack as it came from memory.  Loads fill a RawPack and nothing else, so that a thread
// can issue all the loads of a batch (or both loads of a row) without an instruction that
// depends on the data in between; `unpack` widens to fp32 registers at the point of use.
template <typename WT, int E>
struct RawPack;
template <int E>
struct RawPack<float, E> {
  float v[E];
};
template <>
struct RawPack<__nv_bfloat16, 8> {
  uint4 q;
};
template <>
struct RawPack<__nv_bfloat16, 4> {
  uint2 q;
};

template <int E>
__device__ __forceinline__ void unpack(const RawPack<float, E> &r, float (&v)[E]) {
#pragma unroll
  for (int i = 0; i < E; ++i) v[i] = r.v[i];
}
__device__ __forceinline__ void unpack(const RawPack<__nv_bfloat16, 8> &r, float (&v)[8]) {
  bf16x2_to_floats(r.q.x, v[0], v[1]);
  bf16x2_to_floats(r.q.y, v[2], v[3]);
  bf16x2_to_floats(r.q.z, v[4], v[5]);
  bf16x2_to_floats(r.q.w, v[6], v[7]);
}
__device__ __forceinline__ void unpack(const RawPack<__nv_bfloat16, 4> &r, float (&v)[4]) {
  bf16x2_to_floats(r.q.x, v[0], v[1]);
  bf16x2_to_floats(r.q.y, v[2], v[3]);
}

// fp32 values as a pack in storage form (bf16: to nearest even).
template <int E>
__device__ __forceinline__ void pack_raw(const float (&v)[E], RawPack<float, E> &r) {
#pragma unroll
  for (int i = 0; i < E; ++i) r.v[i] = v[i];
}
__device__ __forceinline__ void pack_raw(const float (&v)[8], RawPack<__nv_bfloat16, 8> &r) {
  r.q = make_uint4(floats_to_bf16x2(v[0], v[1]), floats_to_bf16x2(v[2], v[3]), floats_to_bf16x2(v[4], v[5]),
                   floats_to_bf16x2(v[6], v[7]));
}

// `at` points to the first element of the pack.  live == E: vector load; otherwise (the ragged
// last pack of a row) element by element, dead lanes read as 0.
template <int E>
__device__ __forceinline__ void ld_raw(const float *at, int live, RawPack<float, E> &r) {
  if (!access_ok(at, 4 * (size_t)live)) {  // debug build only: a skipped load reads as zeros
#pragma unroll
    for (int i = 0; i < E; ++i) r.v[i] = 0.f;
    return;
  }
  if (live == E) {
#pragma unroll
    for (int i = 0; i < E / 4; ++i) {
      const float4 t = *reinterpret_cast<const float4 *>(at + 4 * i);
      r.v[4 * i] = t.x; r.v[4 * i + 1] = t.y; r.v[4 * i + 2] = t.z; r.v[4 * i + 3] = t.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < E; ++i) r.v[i] = i < live ? at[i] : 0.f;
  }
}
__device__ __forceinline__ uint32_t ld_bf16_bits(const __nv_bfloat16 *at, int i, int live) {
  return i < live ? (uint32_t)*reinterpret_cast<const unsigned short *>(at + i) : 0u;
}
__device__ __forceinline__ void ld_raw(const __nv_bfloat16 *at, int live, RawPack<__nv_bfloat16, 8> &r) {
  if (!access_ok(at, 2 * (size_t)live)) {
    r.q = make_uint4(0u, 0u, 0u, 0u);
    return;
  }
  if (live == 8) {
    r.q = *reinterpret_cast<const uint4 *>(at);
  } else {
    r.q.x = ld_bf16_bits(at, 0, live) | (ld_bf16_bits(at, 1, live) << 16);
    r.q.y = ld_bf16_bits(at, 2, live) | (ld_bf16_bits(at, 3, live) << 16);
    r.q.z = ld_bf16_bits(at, 4, live) | (ld_bf16_bits(at, 5, live) << 16);
    r.q.w = ld_bf16_bits(at, 6, live) | (ld_bf16_bits(at, 7, live) << 16);
  }
}
__device__ __forceinline__ void ld_raw(const __nv_bfloat16 *at, int live, RawPack<__nv_bfloat16, 4> &r) {
  if (!access_ok(at, 2 * (size_t)live)) {
    r.q = make_uint2(0u, 0u);
    return;
  }
  if (live == 4) {
    r.q = *reinterpret_cast<const uint2 *>(at);
  } else {
    r.q.x = ld_bf16_bits(at, 0, live) | (ld_bf16_bits(at, 1, live) << 16);
    r.q.y = ld_bf16_bits(at, 2, live) | (ld_bf16_bits(at, 3, live) << 16);
  }
}
// The same pack back to memory as it is.
template <int E>
__device__ __forceinline__ void st_raw(float *at, int live, const RawPack<float, E> &r) {
  if (!access_ok(at, 4 * (size_t)live)) return;
  if (live == E) {
#pragma unroll
    for (int i = 0; i < E / 4; ++i)
      *reinterpret_cast<float4 *>(at + 4 * i) = make_float4(r.v[4 * i], r.v[4 * i + 1], r.v[4 * i + 2], r.v[4 * i + 3]);
  } else {
#pragma unroll
    for (int i = 0; i < E; ++i)
      if (i < live) at[i] = r.v[i];
  }
}
__device__ __forceinline__ void st_raw(__nv_bfloat16 *at, int live, const RawPack<__nv_bfloat16, 8> &r) {
  if (!access_ok(at, 2 * (size_t)live)) return;
  if (live == 8) {
    *reinterpret_cast<uint4 *>(at) = r.q;
  } else {
    const uint32_t words[4] = {r.q.x, r.q.y, r.q.z, r.q.w};
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < live) reinterpret_cast<unsigned short *>(at)[i] = (unsigned short)(words[i / 2] >> (16 * (i & 1)));
  }
}
template <typename WT, int E>
__device__ __forceinline__ void zero_raw(RawPack<WT, E> &r) {
  memset(&r, 0, sizeof(r));
}
template <typename T, int E>
__device__ __forceinline__ void st_pack_any(T *row, int64_t p, int live, const float (&v)[E]) {
  if (live == E) {
    st_pack<E>(row, p, v);
  } else {
#pragma unroll
    for (int i = 0; i < E; ++i)
      if (i < live) st_elem(row, E * p + i, v[i]);
  }
}
// Full packs (`live` is a compile-time E) of an arena whose rows start at multiples of 32 bytes: 8 fp32 values
// in one 32-byte store.  Two 16-byte stores of a warp cover half of each sector, and where L1 does not hold
// the line they reach L2 as two partial writes (30 % more write sectors in a batch that overwrites all
// devices).  Measured, us, two stores / one: resident batches, 16 devices, 2^24, one step 428 / 405 per round,
// 32 devices, 23.5 M 1602 / 1572; fused round, 8 devices, 11.2 M, one step 238.7 / 232.4; 16 devices, 2^25,
// one step 1300 / 1292.  A test of the address at each store cost what it gave (8 steps 578 -> 584 .. 588),
// hence the compile-time choice.  32-byte loads gain nothing (the line stays in L1 between the two halves)
// and cost bf16 rounds of 8 steps 2 %.
__device__ __forceinline__ void st_full(float *at, const float (&v)[8]) {
  if (!access_ok(at, 32)) return;
  asm volatile("st.global.v8.f32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(at), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]),
               "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]) : "memory");
}
template <int E>
struct FullPack {  // a number of live lanes that is E at compile time
  __device__ constexpr operator int() const { return E; }
};
template <typename T, int E>
__device__ __forceinline__ void st_pack_any(T *row, int64_t p, FullPack<E>, const float (&v)[E]) {
  if constexpr (sizeof(T) == 4 && E == 8)
    st_full(row + E * p, v);
  else
    st_pack<E>(row, p, v);
}
template <typename T>
__device__ __forceinline__ void st_raw(T *at, FullPack<8>, const RawPack<T, 8> &r) {
  if constexpr (sizeof(T) == 4)
    st_full(at, r.v);
  else
    st_raw(at, 8, r);
}
// Whether the fp32 rows behind w and m (their distance is a multiple of 32 bytes) start at multiples of 32.
template <typename WT, typename MT>
__device__ __forceinline__ bool rows_at_32(const WT *w, const MT *m) {
  const uintptr_t at = (sizeof(WT) == 4 ? (uintptr_t)w : 0) | (sizeof(MT) == 4 ? (uintptr_t)m : 0);
  return (at & 31) == 0;
}
// The value a parameter has once stored: itself for fp32, rounded to nearest even for bf16.
__device__ __forceinline__ float as_stored(float v, const float *) { return v; }
__device__ __forceinline__ float as_stored(float v, const __nv_bfloat16 *) {
  return __bfloat162float(__float2bfloat16_rn(v));
}
__device__ __forceinline__ int live_of(int64_t n_params, int64_t p, int E) {
  const int64_t left = n_params - (int64_t)E * p;
  return left >= E ? E : (left > 0 ? (int)left : 0);
}
template <int E>
__device__ __forceinline__ FullPack<E> live_of(std::true_type, int64_t, int64_t) {
  return {};
}
template <int E>
__device__ __forceinline__ int live_of(std::false_type, int64_t n_params, int64_t p) {
  return live_of(n_params, p, E);
}

__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, off);
  return v;
}

// Whether this block draws the last of n tickets; what it wrote before is visible to the block that does.
__device__ __forceinline__ bool is_last_block(unsigned int *__restrict__ ticket, unsigned int n, bool *s_last) {
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) *s_last = (atomicAdd(ticket, 1u) == n - 1u);
  __syncthreads();
  if (!*s_last) return false;
  __threadfence();
  return true;
}

}  // namespace hadfl
