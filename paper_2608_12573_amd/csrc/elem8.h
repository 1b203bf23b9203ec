// Eight neighbouring elements of a row to and from fp32, and sums over a wave.
#pragma once

#include "device_common.h"
#include "profk.h"

namespace profk {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
// (rows start at any element: 16-byte accesses need no alignment but the element's)
typedef uint32_t u32x4h __attribute__((ext_vector_type(4), aligned(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), bf16x2));
}

// 8 elements as they are in memory.
template <int DT> struct Raw8 { u32x4 q[DT == PROFK_F32 ? 2 : 1]; };

// Elements i .. i + 7 of a row of D; those from D on are 0.
template <int DT> __device__ __forceinline__ Raw8<DT> load_raw8(const void* row, uint32_t i, uint32_t D) {
  Raw8<DT> r;
  if constexpr (DT == PROFK_F32) {
    const uint32_t* const p = static_cast<const uint32_t*>(row) + i;
    if (i + 8 <= D) {
      r.q[0] = *reinterpret_cast<const u32x4h*>(p);
      r.q[1] = *reinterpret_cast<const u32x4h*>(p + 4);
    } else {
#pragma unroll
      for (uint32_t e = 0; e < 8; ++e) r.q[e / 4][e % 4] = i + e < D ? p[e] : 0u;
    }
  } else {
    const uint16_t* const p = static_cast<const uint16_t*>(row) + i;
    if (i + 8 <= D) {
      r.q[0] = *reinterpret_cast<const u32x4h*>(p);
    } else {
#pragma unroll
      for (uint32_t e = 0; e < 4; ++e) {
        const uint32_t lo = i + 2 * e < D ? p[2 * e] : 0u, hi = i + 2 * e + 1 < D ? p[2 * e + 1] : 0u;
        r.q[0][e] = lo | hi << 16;
      }
    }
  }
  return r;
}

template <int DT> __device__ __forceinline__ void to_f32(const Raw8<DT>& r, float (&v)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if constexpr (DT == PROFK_F32) v[e] = __uint_as_float(r.q[e / 4][e % 4]);
    else v[e] = __uint_as_float(e & 1 ? r.q[0][e / 2] & 0xFFFF0000u : r.q[0][e / 2] << 16);
  }
}

template <int DT> __device__ __forceinline__ void load8(const void* row, uint32_t i, uint32_t D, float (&v)[8]) {
  to_f32<DT>(load_raw8<DT>(row, i, D), v);
}

// Of eight values those that lie in the row, each rounded once.
template <int DT> __device__ __forceinline__ void store8(void* row, uint32_t i, uint32_t D, const float (&v)[8]) {
  if constexpr (DT == PROFK_F32) {
    float* const p = static_cast<float*>(row) + i;
    if (i + 8 <= D) {
      *reinterpret_cast<u32x4h*>(p) = u32x4h{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
      *reinterpret_cast<u32x4h*>(p + 4) = u32x4h{__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7])};
    } else {
#pragma unroll
      for (uint32_t e = 0; e < 8; ++e)
        if (i + e < D) p[e] = v[e];
    }
  } else {
    __bf16* const p = static_cast<__bf16*>(row) + i;
    if (i + 8 <= D) {
      *reinterpret_cast<u32x4h*>(p) = u32x4h{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
    } else {
#pragma unroll
      for (uint32_t e = 0; e < 8; ++e)
        if (i + e < D) p[e] = static_cast<__bf16>(v[e]);
    }
  }
}

// Element i of a row, as fp32.
__device__ __forceinline__ float load1(const void* row, uint32_t i, int dtype) {
  return dtype == PROFK_F32 ? static_cast<const float*>(row)[i]
                            : __uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t*>(row)[i]) << 16);
}

template <int CTRL> __device__ __forceinline__ float dpp_add(float x) {
  return x + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xF, 0xF, false));
}
// The sum over the wave, in every lane: exchanges inside each row of 16 lanes,
// then the four rows'.
__device__ __forceinline__ float wave_sum(float x) {
  x = dpp_add<0xB1>(x);
  x = dpp_add<0x4E>(x);
  x = dpp_add<0x141>(x);
  x = dpp_add<0x140>(x);
  const int i = __float_as_int(x);
  return (__int_as_float(__builtin_amdgcn_readlane(i, 0)) + __int_as_float(__builtin_amdgcn_readlane(i, 16))) +
         (__int_as_float(__builtin_amdgcn_readlane(i, 32)) + __int_as_float(__builtin_amdgcn_readlane(i, 48)));
}

}  // namespace profk
