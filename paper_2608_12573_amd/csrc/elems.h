// Neighbouring elements of a row to and from fp32, and sums over a wave.
//
// Lanes take 16 bytes of the widest type at hand in an access, so that a wave's is
// one run of memory: 4 elements where one of the tensors is fp32, else 8.
#pragma once

#include <type_traits>

#include "device_common.h"
#include "profk.h"

namespace profk {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
// (rows start at any element: 16-byte accesses need no alignment but the element's)
typedef uint32_t u32x4h __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x2h __attribute__((ext_vector_type(2), aligned(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), bf16x2));
}

// E elements (4, or 8 of bf16) as they are in memory.
template <int DT, int E> struct Raw {
  static constexpr int W = DT == PROFK_F32 ? E : E / 2;
  uint32_t q[W];
};
template <int W> struct Words;
template <> struct Words<2> { typedef u32x2h type; };
template <> struct Words<4> { typedef u32x4h type; };

// Elements i .. i + E - 1 of a row of D; those from D on are 0.
template <int DT, int E> __device__ __forceinline__ Raw<DT, E> load_raw(const void* row, uint32_t i, uint32_t D) {
  Raw<DT, E> r;
  constexpr int W = Raw<DT, E>::W, S = W < 4 ? W : 4;
  using V = typename Words<S>::type;
  if constexpr (DT == PROFK_F32) {
    const uint32_t* const p = static_cast<const uint32_t*>(row) + i;
    if (i + E <= D) {
#pragma unroll
      for (int w = 0; w < W; w += S) {
        const V v = *reinterpret_cast<const V*>(p + w);
#pragma unroll
        for (int s = 0; s < S; ++s) r.q[w + s] = v[s];
      }
    } else {
#pragma unroll
      for (uint32_t e = 0; e < E; ++e) r.q[e] = i + e < D ? p[e] : 0u;
    }
  } else {
    const uint16_t* const p = static_cast<const uint16_t*>(row) + i;
    if (i + E <= D) {
      const V v = *reinterpret_cast<const V*>(p);
#pragma unroll
      for (int s = 0; s < S; ++s) r.q[s] = v[s];
    } else {
#pragma unroll
      for (uint32_t e = 0; e < E / 2; ++e) {
        const uint32_t lo = i + 2 * e < D ? p[2 * e] : 0u, hi = i + 2 * e + 1 < D ? p[2 * e + 1] : 0u;
        r.q[e] = lo | hi << 16;
      }
    }
  }
  return r;
}

template <int DT, int E> __device__ __forceinline__ void to_f32(const Raw<DT, E>& r, float (&v)[E]) {
#pragma unroll
  for (int e = 0; e < E; ++e) {
    if constexpr (DT == PROFK_F32) v[e] = __uint_as_float(r.q[e]);
    else v[e] = __uint_as_float(e & 1 ? r.q[e / 2] & 0xFFFF0000u : r.q[e / 2] << 16);
  }
}

template <int DT, int E> __device__ __forceinline__ void load(const void* row, uint32_t i, uint32_t D, float (&v)[E]) {
  to_f32<DT, E>(load_raw<DT, E>(row, i, D), v);
}

// E values as they are in memory, each rounded once.
template <int DT, int E> __device__ __forceinline__ Raw<DT, E> pack(const float (&v)[E]) {
  Raw<DT, E> r;
#pragma unroll
  for (int w = 0; w < Raw<DT, E>::W; ++w)
    r.q[w] = DT == PROFK_F32 ? __float_as_uint(v[w % E]) : pack_bf16(v[2 * w % E], v[(2 * w + 1) % E]);
  return r;
}

// Of E elements as they are in memory those that lie in the row.
template <int DT, int E> __device__ __forceinline__ void store_raw(void* row, uint32_t i, uint32_t D, const Raw<DT, E>& r) {
  constexpr int W = Raw<DT, E>::W, S = W < 4 ? W : 4;
  using V = typename Words<S>::type;
  using O = std::conditional_t<DT == PROFK_F32, uint32_t, uint16_t>;
  O* const p = static_cast<O*>(row) + i;
  if (i + E <= D) {
#pragma unroll
    for (int w = 0; w < W; w += S) {
      V o;
#pragma unroll
      for (int s = 0; s < S; ++s) o[s] = r.q[w + s];
      *reinterpret_cast<V*>(p + w * (DT == PROFK_F32 ? 1 : 2)) = o;
    }
  } else {
#pragma unroll
    for (uint32_t e = 0; e < E; ++e)
      if (i + e < D) p[e] = static_cast<O>(DT == PROFK_F32 ? r.q[e % W] : r.q[e / 2] >> e % 2 * 16);
  }
}

// Of E values those that lie in the row, each rounded once.
template <int DT, int E> __device__ __forceinline__ void store(void* row, uint32_t i, uint32_t D, const float (&v)[E]) {
  store_raw<DT, E>(row, i, D, pack<DT, E>(v));
}

// Element i of a row, as fp32.
__device__ __forceinline__ float load1(const void* row, uint32_t i, int dtype) {
  return dtype == PROFK_F32 ? static_cast<const float*>(row)[i]
                            : __uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t*>(row)[i]) << 16);
}

template <int CTRL> __device__ __forceinline__ float dpp_add(float x) {
  return x + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xF, 0xF, false));
}
// The sum over each row of 16 lanes, in every one of them: quad swaps, then half-row
// and row mirrors.
__device__ __forceinline__ float sum16(float x) {
  x = dpp_add<0xB1>(x);
  x = dpp_add<0x4E>(x);
  x = dpp_add<0x141>(x);
  return dpp_add<0x140>(x);
}
// The sum over the wave, in every lane.
__device__ __forceinline__ float wave_sum(float x) {
  x = sum16(x);
  const int i = __float_as_int(x);
  return (__int_as_float(__builtin_amdgcn_readlane(i, 0)) + __int_as_float(__builtin_amdgcn_readlane(i, 16))) +
         (__int_as_float(__builtin_amdgcn_readlane(i, 32)) + __int_as_float(__builtin_amdgcn_readlane(i, 48)));
}

}  // namespace profk
