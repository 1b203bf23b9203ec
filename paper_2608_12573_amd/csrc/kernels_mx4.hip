// Microscaled 4-bit floating point: quantisation, its inverse, and the
// product x W^T of two quantised matrices.
//
// A block of 32 consecutive values of a row has one scale 2^s, held as the
// byte s + 127; a value is a code of 4 bits, a sign and one of 0, 0.5, 1,
// 1.5, 2, 3, 4, 6 (E2M1).  s = floor(log2 m) - 2 within [-127, 127] for the
// block's largest magnitude m, which puts m / 2^s in [4, 8): the top of the
// codes' range, with 6 the largest (the formula of the OCP Microscaling
// Formats specification, version 1.0).  v / 2^s is rounded to nearest, ties
// to even.  Byte 255 is NaN: a block that holds an infinity or NaN.
//
// Layout: K is padded to Kp, whole steps of 128 values (zero codes).  Codes
// [R, Kp / 2] bytes, the even value of a pair in the low half; scales
// [R, Kp / 32] bytes.  A row's codes start at a multiple of 64 bytes, and the
// four scales of a step are one word: a lane of the 32x32x64 matrix
// instruction takes 32 values of a row (16 bytes) and their scale.
#include <type_traits>

#include "device_common.h"
#include "launch.h"

namespace profk {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4u __attribute__((ext_vector_type(4), aligned(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2u __attribute__((ext_vector_type(2), aligned(2)));

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), bf16x2));
}

// ------------------------------------------------------------- quantise ---
// A lane takes 8 values, four lanes a block.  The convert instruction divides
// by its scale and rounds; small blocks are scaled up by 2^64 first, so that
// neither the values nor the scale are subnormal.
constexpr int kMxBS = 256;
constexpr uint32_t kMxSmall = 64;             // scale bytes below this are taken 2^64 larger

template <int DT> __device__ __forceinline__ void mx_load8(const void* row, uint32_t k, uint32_t K, float (&v)[8]) {
  if (k + 8 <= K) {
    if constexpr (DT == PROFK_F32) {
      const float* const p = static_cast<const float*>(row) + k;
      const f32x4 a = *reinterpret_cast<const f32x4u*>(p), b = *reinterpret_cast<const f32x4u*>(p + 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[e] = a[e];
        v[4 + e] = b[e];
      }
    } else {
      const u32x4 a = *reinterpret_cast<const u32x4u*>(static_cast<const uint16_t*>(row) + k);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(e & 1 ? a[e / 2] & 0xFFFF0000u : a[e / 2] << 16);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      v[e] = 0.0f;
      if (k + e < K) v[e] = __uint_as_float(DT == PROFK_F32 ? load_raw<0>(row, k + e) : load_raw<1>(row, k + e) << 16);
    }
  }
}

// The codes of a lane's 8 values and its block's scale byte; the four lanes
// of a block call it together.
__device__ __forceinline__ uint32_t mx_quant8(const float (&v)[8], uint32_t& byte) {
  uint32_t m = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(v[e]) & 0x7FFFFFFFu);
  m = max(m, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(m), 0xB1, 0xF, 0xF, false)));
  m = max(m, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(m), 0x4E, 0xF, 0xF, false)));
  const uint32_t ex = m >> 23;                      // floor(log2 m) + 127, 0 for subnormals
  if (ex == 255) {
    byte = 255;
    return 0;
  }
  byte = max(ex, 2u) - 2;
  const bool small = byte < kMxSmall;
  const float f = small ? 0x1p64f : 1.0f;
  const float scale = __uint_as_float((small ? byte + 64 : byte) << 23);
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0] * f, v[1] * f, scale, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2] * f, v[3] * f, scale, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4] * f, v[5] * f, scale, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6] * f, v[7] * f, scale, 3);
  return c;
}

struct MxQuantArgs {
  const void* x;
  uint64_t stride;
  uint32_t rows, K, lanes;   // lanes of a row (Kp / 8)
  uint32_t* codes;
  uint8_t* scales;
};

template <int DT> __global__ __launch_bounds__(kMxBS) void k_mx_quantize(MxQuantArgs a) {
  const uint32_t t = blockIdx.x * kMxBS + threadIdx.x;
  const uint32_t r = t / a.lanes, c = t - r * a.lanes;
  if (r >= a.rows) return;                          // (whole quads: a row has a multiple of 16 lanes)
  float v[8];
  mx_load8<DT>(static_cast<const char*>(a.x) + r * a.stride * (DT == PROFK_F32 ? 4 : 2), 8 * c, a.K, v);
  uint32_t byte;
  a.codes[t] = mx_quant8(v, byte);
  if ((c & 3) == 0) a.scales[t >> 2] = static_cast<uint8_t>(byte);
}

struct MxDequantArgs {
  const uint32_t* codes;
  const uint8_t* scales;
  uint32_t rows, K, lanes;
  void* out;
};

template <int DT> __global__ __launch_bounds__(kMxBS) void k_mx_dequantize(MxDequantArgs a) {
  const uint32_t t = blockIdx.x * kMxBS + threadIdx.x;
  const uint32_t r = t / a.lanes, k = 8 * (t - r * a.lanes);
  if (r >= a.rows || k >= a.K) return;
  const uint32_t code = a.codes[t], byte = a.scales[t >> 2];
  const bool small = byte < kMxSmall;
  const float scale = __uint_as_float((small ? byte + 64 : byte) << 23);
  const float f = byte == 255 ? __builtin_nanf("") : small ? 0x1p-64f : 1.0f;
  const f32x2 p0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, scale, 0);
  const f32x2 p1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, scale, 1);
  const f32x2 p2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, scale, 2);
  const f32x2 p3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, scale, 3);
  const float v[8] = {p0.x * f, p0.y * f, p1.x * f, p1.y * f, p2.x * f, p2.y * f, p3.x * f, p3.y * f};
  const size_t o = static_cast<size_t>(r) * a.K + k;
  if constexpr (DT == PROFK_F32) {
    float* const out = static_cast<float*>(a.out) + o;
    if (k + 8 <= a.K) {
      *reinterpret_cast<f32x4u*>(out) = f32x4{v[0], v[1], v[2], v[3]};
      *reinterpret_cast<f32x4u*>(out + 4) = f32x4{v[4], v[5], v[6], v[7]};
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (k + e < a.K) out[e] = v[e];
    }
  } else {
    __bf16* const out = static_cast<__bf16*>(a.out) + o;
    if (k + 8 <= a.K) {
      *reinterpret_cast<u32x4u*>(out) =
          u32x4{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (k + e < a.K) out[e] = static_cast<__bf16>(v[e]);
    }
  }
}

// -------------------------------------------------------------- product ---
__device__ __forceinline__ i32x8 mx_frag(const u32x4& v) {
  return i32x8{static_cast<int>(v.x), static_cast<int>(v.y), static_cast<int>(v.z), static_cast<int>(v.w), 0, 0, 0, 0};
}
// One 32x32x64 step; the scales are bytes 2 * KS of sa and sb.
template <int KS> __device__ __forceinline__ f32x16 mx_mma(const u32x4& a, const u32x4& b, f32x16 c, int sa, int sb) {
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(mx_frag(a), mx_frag(b), c, 4, 4, 2 * KS, sa, 2 * KS, sb);
}

struct MxGemmArgs {
  const uint8_t *a, *b;       // codes [M, Kp / 2], [N, Kp / 2]
  const uint8_t *as, *bs;     // scales [M, Kp / 32], [N, Kp / 32]
  uint32_t M, N, steps;       // steps of 128 values
  void* out;                  // [M, N]
};

// Values n .. n + 3 of an output row.
template <int DT> __device__ __forceinline__ void mx_store4(void* out, size_t row, uint32_t n, uint32_t N, f32x4 v) {
  const size_t o = row * N + n;
  if (n + 4 <= N) {
    if constexpr (DT == PROFK_F32) *reinterpret_cast<f32x4u*>(static_cast<float*>(out) + o) = v;
    else *reinterpret_cast<u32x2u*>(static_cast<uint16_t*>(out) + o) = u32x2u{pack_bf16(v.x, v.y), pack_bf16(v.z, v.w)};
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (n + e < N) {
        if constexpr (DT == PROFK_F32) static_cast<float*>(out)[o + e] = v[e];
        else static_cast<__bf16*>(out)[o + e] = static_cast<__bf16>(v[e]);
      }
  }
}

// A simple product: a wave computes 32 x 128 outputs straight from memory.
// Column n = 128 w + 4 (lane % 32) + j is in fragment j, so that a lane's four
// results of a row are neighbours.
template <int DT> __global__ __launch_bounds__(256) void k_mx_simple(MxGemmArgs g) {
  const uint32_t lane = threadIdx.x & (kWave - 1), w = threadIdx.x / kWave;
  const uint32_t c = lane & 31, h = lane >> 5;
  const uint32_t m0 = blockIdx.y * 32, n0 = (blockIdx.x * 4 + w) * 128;
  if (n0 >= g.N) return;
  const size_t cb = static_cast<size_t>(g.steps) * 64, sb = static_cast<size_t>(g.steps) * 4;
  const uint32_t m = min(m0 + c, g.M - 1);
  const uint8_t* const pa = g.a + m * cb + h * 16;
  f32x16 acc[4] = {};
  for (uint32_t k = 0; k < g.steps; ++k) {
    const int sa = static_cast<int>(reinterpret_cast<const uint32_t*>(g.as + m * sb)[k] >> (8 * h));
    const u32x4 a0 = *reinterpret_cast<const u32x4*>(pa + k * 64), a1 = *reinterpret_cast<const u32x4*>(pa + k * 64 + 32);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t n = min(n0 + 4 * c + j, g.N - 1);
      const uint8_t* const pb = g.b + n * cb + h * 16 + k * 64;
      const int sw = static_cast<int>(reinterpret_cast<const uint32_t*>(g.bs + n * sb)[k] >> (8 * h));
      acc[j] = mx_mma<0>(a0, *reinterpret_cast<const u32x4*>(pb), acc[j], sa, sw);
      acc[j] = mx_mma<1>(a1, *reinterpret_cast<const u32x4*>(pb + 32), acc[j], sa, sw);
    }
  }
#pragma unroll
  for (int v = 0; v < 16; ++v) {
    const uint32_t r = m0 + 8 * (v / 4) + 4 * h + (v % 4);
    if (r < g.M) mx_store4<DT>(g.out, r, n0 + 4 * c, g.N, f32x4{acc[0][v], acc[1][v], acc[2][v], acc[3][v]});
  }
}

}  // namespace

uint64_t mx_steps(int64_t K) { return (static_cast<uint64_t>(K) + 127) / 128; }

hipError_t launch_mx_quantize(int dtype, const void* x, uint64_t stride, int64_t R, int64_t K, uint8_t* codes,
                              uint8_t* scales, hipStream_t s) {
  const uint64_t lanes = mx_steps(K) * 16;
  const int64_t step = static_cast<int64_t>((uint64_t{1} << 31) / lanes);
  (void)hipGetLastError();
  for (int64_t r = 0; r < R; r += step) {
    const uint64_t rows = static_cast<uint64_t>(R - r < step ? R - r : step);
    const MxQuantArgs a{static_cast<const uint8_t*>(x) + static_cast<uint64_t>(r) * stride * (dtype == PROFK_F32 ? 4 : 2),
                        stride, static_cast<uint32_t>(rows), static_cast<uint32_t>(K), static_cast<uint32_t>(lanes),
                        reinterpret_cast<uint32_t*>(codes + r * lanes * 4), scales + r * (lanes / 4)};
    const uint32_t grid = static_cast<uint32_t>((rows * lanes + kMxBS - 1) / kMxBS);
    if (dtype == PROFK_F32) k_mx_quantize<PROFK_F32><<<grid, kMxBS, 0, s>>>(a);
    else k_mx_quantize<PROFK_BF16><<<grid, kMxBS, 0, s>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_mx_dequantize(int dtype, const uint8_t* codes, const uint8_t* scales, int64_t R, int64_t K, void* out,
                                hipStream_t s) {
  const uint64_t lanes = mx_steps(K) * 16;
  const int64_t step = static_cast<int64_t>((uint64_t{1} << 31) / lanes);
  (void)hipGetLastError();
  for (int64_t r = 0; r < R; r += step) {
    const uint64_t rows = static_cast<uint64_t>(R - r < step ? R - r : step);
    const MxDequantArgs a{reinterpret_cast<const uint32_t*>(codes + r * lanes * 4), scales + r * (lanes / 4),
                          static_cast<uint32_t>(rows), static_cast<uint32_t>(K), static_cast<uint32_t>(lanes),
                          static_cast<uint8_t*>(out) + static_cast<uint64_t>(r) * K * (dtype == PROFK_F32 ? 4 : 2)};
    const uint32_t grid = static_cast<uint32_t>((rows * lanes + kMxBS - 1) / kMxBS);
    if (dtype == PROFK_F32) k_mx_dequantize<PROFK_F32><<<grid, kMxBS, 0, s>>>(a);
    else k_mx_dequantize<PROFK_BF16><<<grid, kMxBS, 0, s>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_mx_matmul(const MxMatmulCall& c) {
  const MxGemmArgs g{c.a, c.b, c.as, c.bs, static_cast<uint32_t>(c.M), static_cast<uint32_t>(c.N),
                     static_cast<uint32_t>(mx_steps(c.K)), c.out};
  (void)hipGetLastError();
  const dim3 grid((g.N + 511) / 512, (g.M + 31) / 32);
  if (c.out_dtype == PROFK_F32) k_mx_simple<PROFK_F32><<<grid, 256, 0, c.stream>>>(g);
  else k_mx_simple<PROFK_BF16><<<grid, 256, 0, c.stream>>>(g);
  return hipGetLastError();
}

}  // namespace profk
