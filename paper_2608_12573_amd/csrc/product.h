// The dense product P[i, j] = sum_k A(i, k) B(j, k) of bf16 operands: its
// arguments, epilogue and launches (kernels_product.hip, kernels_product_grad.hip,
// kernels_linear.hip).
#pragma once

#include "elems.h"

namespace profk {

// An operand lies "along" k, a row of K neighbours for each i (or j), or
// "across" it, a row of neighbouring i for each k.
struct ProdArgs {
  const __bf16 *a, *b;
  const __bf16* a_low;              // a second operand to be added to a, laid out as it is, or null
  uint64_t as, bs;                  // elements from row to row
  uint32_t I, J, K;
  const float* bias;                // [J]
  int act, out_dtype;
  const void* residual;             // [I, J] of out_dtype
  uint64_t residual_stride;
  void *out, *pre;                  // [I, J]
  uint32_t i0, j0;                  // kernel of any sizes: first row and column of this launch
  uint32_t parts, part_k;           // tiled kernels: K in parts of part_k, their fp32 sums to out [parts, I, J]
  bool a_padded, b_padded;          // rows end in whole granules of 8, zeros past their end
};

// s_waitcnt vmcnt(N) lgkmcnt(0) (gfx9 encoding: vmcnt in bits 3:0 and 15:14,
// expcnt in 6:4, lgkmcnt in 11:8): all but this wave's N newest loads are done,
// and so are its LDS reads.
template <int N> __device__ __forceinline__ void prod_wait() {
  static_assert(N >= 0 && N < 64, "vmcnt");
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((N & 0xF) | ((N >> 4) << 14) | (0x7 << 4));
  asm volatile("" ::: "memory");
}

// ------------------------------------------------------------ activations ---
// An infinite z gives the limit, NaN stays NaN.
//
// gelu's normal distribution function: with t = 1 / (1 + 0.2325 |z|),
//   Phi(-|z|) = t P(t) e^(-z^2 / 2),
// P a polynomial of degree 7 fitted to Phi(-a) e^(a^2 / 2) / t over a from 0 to 13.5
// for the least greatest relative error (9.2e-8, before its coefficients' rounding).
// The exponent's roundings are summed beside it, so that small results are as near
// as large ones: Phi is within 2^-20 of itself down to z = -12.5, below which it is
// 0 to 1e-36.  The library's erf has two branches and many more instructions a value.
struct Normal {
  float cdf, density;               // density: e^(-z^2 / 2)
};
// 2^(h + l) for an l of the size of h's roundings
__device__ __forceinline__ float exp2_sum(float h, float l) {
  const float e = __builtin_amdgcn_exp2f(h);
  return fmaf(e * l, 0.69314718055994531f, e);
}
__device__ __forceinline__ Normal normal_of(float z) {
  const float a = fminf(fabsf(z), 40.0f);
  const float t = __builtin_amdgcn_rcpf(fmaf(0.2325f, a, 1.0f));
  // -z^2 / (2 ln 2), the constant as a sum of two numbers
  constexpr float kHi = -0.7213475108146667f, kLo = -9.629815e-9f;
  const float s = a * a, h = s * kHi;
  const float e = exp2_sum(h, fmaf(fmaf(a, a, -s), kHi, fmaf(s, kLo, fmaf(s, kHi, -h))));
  float q = fmaf(t, -0.06940309137311834f, 0.24030702839907406f);
  q = fmaf(t, q, -0.19107164775638127f);
  q = fmaf(t, q, 0.21710237380367514f);
  q = fmaf(t, q, 0.01726995487392053f);
  q = fmaf(t, q, 0.10205930278671793f);
  q = fmaf(t, q, 0.09087767547070454f);
  q = fmaf(t, q, 0.09285843157661314f);
  q *= t * e;
  return {z < 0.0f ? q : 1.0f - q, e};
}
// (below -87, where e^-z leaves fp32, 0: within 2e-36 of z sigmoid(z))
__device__ __forceinline__ float sigmoid_of(float z) {
  const float c = fminf(fmaxf(z, -87.0f), 87.0f);
  constexpr float kHi = -1.4426950216293335f, kLo = -1.9259630e-8f;   // -1 / ln 2
  const float h = c * kHi;
  const float p = __builtin_amdgcn_rcpf(1.0f + exp2_sum(h, fmaf(c, kLo, fmaf(c, kHi, -h))));
  return z < -87.0f ? 0.0f : p;
}
template <int ACT> __device__ __forceinline__ float act_of(float z) {
  if constexpr (ACT == PROFK_ACT_RELU) return z < 0.0f ? 0.0f : z;
  if constexpr (ACT == PROFK_ACT_GELU) return (z < -40.0f ? -40.0f : z) * normal_of(z).cdf;
  if constexpr (ACT == PROFK_ACT_SILU) return (z < -200.0f ? -200.0f : z) * sigmoid_of(z);
  return z;
}
template <int ACT> __device__ __forceinline__ float slope_of(float z) {
  if constexpr (ACT == PROFK_ACT_RELU) return z > 0.0f ? 1.0f : 0.0f;
  if constexpr (ACT == PROFK_ACT_GELU) {
    const float c = z < -40.0f ? -40.0f : z > 40.0f ? 40.0f : z;
    const Normal n = normal_of(c);
    return fmaf(c * n.density, 0.39894228040143268f, n.cdf);
  }
  if constexpr (ACT == PROFK_ACT_SILU) {
    const float c = z < -200.0f ? -200.0f : z > 200.0f ? 200.0f : z;
    const float p = sigmoid_of(c);
    return p * fmaf(c, 1.0f - p, 1.0f);
  }
  return 1.0f;
}

// f(std::integral_constant<int, ACT>) for an activation known at run time.
template <class F> void with_act(int act, F f) {
  if (act == PROFK_ACT_RELU) f(std::integral_constant<int, PROFK_ACT_RELU>{});
  else if (act == PROFK_ACT_GELU) f(std::integral_constant<int, PROFK_ACT_GELU>{});
  else if (act == PROFK_ACT_SILU) f(std::integral_constant<int, PROFK_ACT_SILU>{});
  else f(std::integral_constant<int, PROFK_ACT_NONE>{});
}

// How the tiled product goes about a size: tiles of 256 x 256 on a CU each, or
// two of 128 x 128, and K in parts whose sums are joined by another kernel.
struct ProdPlan {
  bool large;
  uint32_t parts, part_k;
  double us;                        // its cost
};
ProdPlan plan_product(uint64_t I, uint64_t J, uint64_t K, uint32_t cus);
// Both products of a gradient in one launch are the faster way.
bool plan_pair(uint64_t M, uint64_t N, uint64_t K, uint32_t cus);

// The rows that the kernel of few rows takes.  From 17 it reads a as often as b, and
// is the faster one where the tiles of 128 columns do not fill the CUs (us, 32 rows
// here and 33 there: 4096 x 4096 10.6 and 14.9; 4096 x 12288 31.4 and 27.0, 1024 x
// 50000 36.0 and 25.8).
inline bool few_rows(uint64_t I, uint64_t J, uint32_t cus) { return I <= 16 || (I <= 32 && J < 32 * cus); }

// Up to kFewAny rows of operands along k of any stride and alignment; false: more.
constexpr uint32_t kFewAny = 4;
bool launch_product_few_any(const ProdArgs& g, uint32_t cus, hipStream_t s);
// The product of few rows, and the tiled one; false: these operands are not
// aligned as they need them.
bool launch_product_few(const ProdArgs& g, uint32_t cus, hipStream_t s);                // A and B along k, few_rows
bool launch_product_along(ProdArgs g, const ProdPlan& p, float* sums, uint32_t cus, hipStream_t s);   // A and B along k
bool launch_product_grad(ProdArgs g, bool a_across, const ProdPlan& p, float* sums, uint32_t cus,
                         hipStream_t s);                                               // B across k, A as said

// ... B across k: dx (A along) and dW (A across) at once, unsplit, in small tiles.
bool launch_product_pair(const ProdArgs& dx, const ProdArgs& dw, hipStream_t s);

// Operands that the tiled product takes: rows of whole 16-byte granules.  `len`
// is the length of a row.
inline bool granules(const void* p, uint64_t stride, uint32_t len, bool padded) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride % 8 == 0 && (padded || len % 8 == 0) && stride <= (1u << 21);
}

}  // namespace profk
