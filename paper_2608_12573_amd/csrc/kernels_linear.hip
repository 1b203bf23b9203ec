// The dense product of bf16 matrices with bias, activation and residual in its
// epilogue, and its gradients.
//
//   z = x W^T + b,  y = act(z) + residual,  dz = dy act'(z)
//   dx = dz W,  dW = dz^T x,  db = sum over the rows of dz.
// Products are exact in fp32 and summed in it on the matrix cores; bias,
// activation and residual are fp32, and y (and z, where it is kept) is rounded
// once.  Where dz is no bf16 number by itself (dy in fp32, or the slope of gelu or
// silu), it enters the two products as the sum of two, within 2^-16 of itself: as
// many matrix instructions again.  A caller may have it rounded to one instead,
// within 2^-8 of each term, which the products average over their sums (4096 x 2048 x
// 12288 with gelu 826 us as two, 455 rounded).  db is summed from dz itself.
//
// All three products are P[i, j] = sum_k A(i, k) B(j, k) with either operand's k
// neighbouring in memory ("along") or a whole row apart ("across").
#include <type_traits>

#include "join.h"
#include "launch.h"
#include "linear.h"
#include "product.h"
#include "product_put.h"

namespace profk {

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// ------------------------------------------------- product of any operands ---
// Any sizes, strides and alignments: tiles of 128 x 128 on four waves of 64 x 64, 32
// of k at a time through registers to LDS, its rows 80 bytes apart.  One workgroup a
// tile takes all of k: 4096 x 4096 x 12288 742 us on rows at odd elements, against 296
// of the tiled product on whole granules; where the tiles are few the more (8 x 4096 x
// 4096 102 and 9.3, 256 rows 129 and 21; gradients of 64 x 4096 x 4096 257 and 33).
constexpr uint32_t kAnyB = 128, kAnyK = 32, kAnyRow = 40;

// 8 neighbours in memory, those from `left` on 0.
__device__ __forceinline__ u32x4 load_part8(const __bf16* p, uint32_t left) {
  return __builtin_bit_cast(u32x4, load_raw<PROFK_BF16, 8>(p, 0, left));
}

template <bool ACROSS> struct AnyTile {
  u32x4 v[2];
  // rows r0 .. r0 + 127 of R, k0 .. k0 + 31 of K
  __device__ __forceinline__ void load(const __bf16* p, uint64_t stride, uint32_t r0, uint32_t R, uint32_t k0, uint32_t K) {
#pragma unroll
    for (uint32_t q = 0; q < 2; ++q) {
      const uint32_t t = threadIdx.x + q * 256;
      const uint32_t r = r0 + (ACROSS ? t % 16 * 8 : t / 4), k = k0 + (ACROSS ? t / 16 : t % 4 * 8);
      v[q] = u32x4{};
      if (r < R && k < K) v[q] = ACROSS ? load_part8(p + k * stride + r, R - r) : load_part8(p + r * stride + k, K - k);
    }
  }
  __device__ __forceinline__ void store(uint16_t* s) const {
#pragma unroll
    for (uint32_t q = 0; q < 2; ++q) {
      const uint32_t t = threadIdx.x + q * 256;
      if constexpr (ACROSS) {
#pragma unroll
        for (uint32_t e = 0; e < 8; ++e)
          s[(t % 16 * 8 + e) * kAnyRow + t / 16] = static_cast<uint16_t>(v[q][e / 2] >> (16 * (e % 2)));
      } else {
        *reinterpret_cast<u32x4*>(s + t / 4 * kAnyRow + t % 4 * 8) = v[q];
      }
    }
  }
};

template <bool TA, bool TB> __global__ __launch_bounds__(256) void k_prod_any(ProdArgs g, uint32_t tiles_i) {
  __shared__ __align__(16) uint16_t sa[kAnyB * kAnyRow], sb[kAnyB * kAnyRow];
  const uint32_t i0 = g.i0 + blockIdx.x % tiles_i * kAnyB, j0 = g.j0 + blockIdx.x / tiles_i * kAnyB;
  const uint32_t lane = threadIdx.x & (kWave - 1), w = threadIdx.x / kWave;
  const uint32_t c = lane & 31, h = lane >> 5, wi = w / 2 * 64, wj = w % 2 * 64;
  AnyTile<TA> ta;
  AnyTile<TB> tb;
  f32x16 acc[2][2] = {};
  ta.load(g.a, g.as, i0, g.I, 0, g.K);
  tb.load(g.b, g.bs, j0, g.J, 0, g.K);
  // (a second term of a: its steps of k follow)
  const uint32_t steps = (g.K + kAnyK - 1) / kAnyK, all = g.a_low ? 2 * steps : steps;
  for (uint32_t t = 0; t < all; ++t) {
    __syncthreads();
    ta.store(sa);
    tb.store(sb);
    __syncthreads();
    if (t + 1 < all) {
      const uint32_t k = (t + 1 < steps ? t + 1 : t + 1 - steps) * kAnyK;
      ta.load(t + 1 < steps ? g.a : g.a_low, g.as, i0, g.I, k, g.K);
      tb.load(g.b, g.bs, j0, g.J, k, g.K);
    }
#pragma unroll
    for (uint32_t q = 0; q < 2; ++q) {
      bf16x8 fa[2], fb[2];
#pragma unroll
      for (uint32_t u = 0; u < 2; ++u) {
        fa[u] = *reinterpret_cast<const bf16x8*>(sa + (wi + u * 32 + c) * kAnyRow + q * 16 + h * 8);
        fb[u] = *reinterpret_cast<const bf16x8*>(sb + (wj + u * 32 + c) * kAnyRow + q * 16 + h * 8);
      }
#pragma unroll
      for (uint32_t u = 0; u < 2; ++u)
#pragma unroll
        for (uint32_t v = 0; v < 2; ++v)
          acc[u][v] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[u], fb[v], acc[u][v], 0, 0, 0);
    }
  }
#pragma unroll
  for (uint32_t u = 0; u < 2; ++u)
#pragma unroll
    for (uint32_t v = 0; v < 2; ++v)
#pragma unroll
      for (uint32_t e = 0; e < 16; ++e) {
        const uint32_t i = i0 + wi + u * 32 + 8 * (e / 4) + 4 * h + e % 4, j = j0 + wj + v * 32 + c;
        if (i < g.I && j < g.J) put(g, i, j, acc[u][v][e]);
      }
}

template <bool TA, bool TB> hipError_t launch_any(ProdArgs g, hipStream_t s) {
  const uint64_t ti = (g.I + kAnyB - 1) / kAnyB, tj = (g.J + kAnyB - 1) / kAnyB;
  (void)hipGetLastError();
  constexpr uint64_t kMost = 2048;   // tiles a side of a launch (fewer than 2^32 threads)
  for (uint64_t j = 0; j < tj; j += kMost) {
    for (uint64_t i = 0; i < ti; i += kMost) {
      g.i0 = static_cast<uint32_t>(i * kAnyB);
      g.j0 = static_cast<uint32_t>(j * kAnyB);
      const uint32_t ni = static_cast<uint32_t>(ti - i < kMost ? ti - i : kMost);
      const uint32_t nj = static_cast<uint32_t>(tj - j < kMost ? tj - j : kMost);
      k_prod_any<TA, TB><<<ni * nj, 256, 0, s>>>(g, ni);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
  }
  return hipSuccess;
}

// --------------------------------------------------------------------- dz ---
// dz = dy act'(z) to bf16, or to a sum of two bf16 numbers, and the sums of its
// columns over a part of the rows.  A workgroup has cols threads for 8 columns each,
// and as many rows at a time as fit.
struct DzArgs {
  const void *dy, *pre;
  uint64_t dy_stride;
  uint32_t M, N, cols, parts;       // cols: a power of two
  __bf16 *dz, *low;                 // rows dz_stride apart; null: only the sums; low null: one number
  uint64_t dz_stride;
  float* part;                      // [parts, N], or null
};
constexpr uint32_t kDzBS = 256;

// The bf16 number next to a finite x (the largest, where that is infinite), so that x
// less it is finite; infinities and NaN as they are.
__device__ __forceinline__ float top_term(float x) {
  const float hi = static_cast<float>(static_cast<__bf16>(x));
  return fabsf(hi) == INFINITY && fabsf(x) < INFINITY ? copysignf(0x1.FEp127f, x) : hi;
}

template <int DT, int ACT> __device__ __forceinline__ void dz_body(const DzArgs& a, uint32_t slab, uint32_t p) {
  __shared__ float s[kDzBS][8];
  constexpr uint32_t ES = DT == PROFK_F32 ? 4 : 2;
  const uint32_t rows = kDzBS / a.cols, sub = threadIdx.x / a.cols;
  const uint32_t j = (slab * a.cols + threadIdx.x % a.cols) * 8;
  const uint32_t r0 = static_cast<uint32_t>(static_cast<uint64_t>(a.M) * p / a.parts);
  const uint32_t r1 = static_cast<uint32_t>(static_cast<uint64_t>(a.M) * (p + 1) / a.parts);
  float sum[8] = {}, d[8], z[8];
  for (uint32_t r = j < a.N ? r0 + sub : r1; r < r1; r += rows) {
    load<DT, 8>(static_cast<const char*>(a.dy) + r * a.dy_stride * ES, j, a.N, d);
    if constexpr (ACT != PROFK_ACT_NONE) {
      load<DT, 8>(static_cast<const char*>(a.pre) + static_cast<uint64_t>(r) * a.N * ES, j, a.N, z);
#pragma unroll
      for (int e = 0; e < 8; ++e) d[e] *= slope_of<ACT>(z[e]);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] += d[e];
    if (a.low) {
      float low[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float hi = top_term(d[e]);
        low[e] = fabsf(d[e]) < INFINITY ? d[e] - hi : 0.0f;
        d[e] = hi;
      }
      store<PROFK_BF16, 8>(a.low + r * a.dz_stride, j, static_cast<uint32_t>(a.dz_stride), low);
    }
    if (a.dz) store<PROFK_BF16, 8>(a.dz + r * a.dz_stride, j, static_cast<uint32_t>(a.dz_stride), d);   // (0 past N)
  }
  if (!a.part) return;
  if (rows > 1) {
#pragma unroll
    for (int e = 0; e < 8; ++e) s[threadIdx.x][e] = sum[e];
    __syncthreads();
    if (sub == 0) {
      for (uint32_t k = 1; k < rows; ++k) {
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] += s[k * a.cols + threadIdx.x][e];
      }
    }
  }
  if (sub == 0 && j < a.N) store<PROFK_F32, 8>(a.part + static_cast<size_t>(p) * a.N, j, a.N, sum);
}

// Two matrices (either may have no rows) of any stride and alignment, to rows of
// whole 16-byte granules, zeros past K.
struct PadArgs {
  const __bf16* x[2];
  uint64_t stride[2];
  uint32_t R[2], K;
  __bf16* out[2];
};
__device__ __forceinline__ void pad_body(const PadArgs& a, uint32_t block, uint32_t blocks) {
  const uint32_t per = (a.K + 7) / 8;
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    const uint64_t n = static_cast<uint64_t>(a.R[m]) * per;
    for (uint64_t i = block * uint64_t{256} + threadIdx.x; i < n; i += blocks * uint64_t{256}) {
      const uint32_t r = static_cast<uint32_t>(i / per), k = static_cast<uint32_t>(i % per) * 8;
      reinterpret_cast<u32x4*>(a.out[m])[i] =
          __builtin_bit_cast(u32x4, load_raw<PROFK_BF16, 8>(a.x[m] + r * a.stride[m], k, a.K));
    }
  }
}
__global__ __launch_bounds__(256) void k_pad(PadArgs a) { pad_body(a, blockIdx.x, gridDim.x); }

// dz, in dz_blocks workgroups, and the copies beside it.
template <int DT, int ACT> __global__ __launch_bounds__(kDzBS) void k_dz(DzArgs a, uint32_t slabs, uint32_t dz_blocks, PadArgs p) {
  static_assert(kDzBS == 256, "pad_body");
  if (blockIdx.x < dz_blocks) dz_body<DT, ACT>(a, blockIdx.x % slabs, blockIdx.x / slabs);
  else pad_body(p, blockIdx.x - dz_blocks, gridDim.x - dz_blocks);
}

__global__ __launch_bounds__(kJoinBS) void k_db_join(const float* part, uint32_t parts, uint32_t N, float* db) {
  for (uint32_t b = blockIdx.x; b < (N + kJoinCols - 1) / kJoinCols; b += gridDim.x) {
    const float sum = join_parts(part, parts, N, b);
    const uint32_t j = b * kJoinCols + threadIdx.x;
    if (threadIdx.x < kJoinCols && j < N) db[j] = sum;
  }
}

// Threads of 8 columns of a workgroup of k_dz.
uint32_t dz_cols(int64_t N) {
  uint32_t cols = 1;
  while (cols < kDzBS && cols * 8 < N) cols *= 2;
  return cols;
}
// Parts of the rows: each thread has a few of them, and no more workgroups than
// the CUs hold.  (The sums of few rows are one part, and need no join.)
uint32_t dz_parts(int64_t M, int64_t N, int num_cus) {
  const int64_t cols = dz_cols(N), rows = kDzBS / cols;
  const int64_t slabs = N > 0 ? (N + cols * 8 - 1) / (cols * 8) : 1, most = (static_cast<int64_t>(num_cus) * 8 + slabs - 1) / slabs;
  const int64_t want = (M + rows * 4 - 1) / (rows * 4), parts = want < most ? want : most;
  return parts < 1 ? 1u : static_cast<uint32_t>(parts);
}

size_t align256(size_t n) { return (n + 255) / 256 * 256; }

uint64_t padded(int64_t K) { return (static_cast<uint64_t>(K) + 7) / 8 * 8; }
size_t pad_bytes(int64_t R, int64_t K) { return K % 8 ? align256(static_cast<size_t>(R) * padded(K) * 2) : 0; }

// Operands whose rows are not whole granules (K % 8) are copied, a pass over
// them, for the tiled product (gradients of 509 x 1001 x 777: with the product of
// any operands 140 us, with the copies 43).
PadArgs pad_args(const void* x, uint64_t x_stride, int64_t M, __bf16* x_out, const void* w, uint64_t w_stride, int64_t N,
                 __bf16* w_out, int64_t K) {
  return {{static_cast<const __bf16*>(x), static_cast<const __bf16*>(w)},
          {x_stride, w_stride},
          {static_cast<uint32_t>(M), static_cast<uint32_t>(N)},
          static_cast<uint32_t>(K),
          {x_out, w_out}};
}
uint32_t pad_blocks(const PadArgs& a) {
  const uint64_t blocks = (static_cast<uint64_t>(a.R[0] > a.R[1] ? a.R[0] : a.R[1]) * ((a.K + 7) / 8) + 255) / 256;
  return blocks < 8192 ? static_cast<uint32_t>(blocks) : 8192;
}

// Bytes of the sums of K's parts of an I x J product.
size_t sums_bytes(int64_t I, int64_t J, int64_t K, uint32_t cus) {
  if (I < 1 || J < 1 || K < 1) return 0;
  const ProdPlan p = plan_product(static_cast<uint64_t>(I), static_cast<uint64_t>(J), static_cast<uint64_t>(K), cus);
  return p.parts == 1 ? 0 : align256(static_cast<size_t>(p.parts) * static_cast<size_t>(I) * static_cast<size_t>(J) * 4);
}

struct GradLayout {
  size_t dz, low, part, x, w, sums, bytes;   // offsets
  uint64_t dz_stride;
  uint32_t parts;
};
GradLayout grad_layout(int64_t M, int64_t N, int64_t K, int num_cus) {
  GradLayout L{};
  L.dz_stride = (static_cast<uint64_t>(N) + 7) / 8 * 8;
  L.parts = dz_parts(M, N, num_cus);
  L.low = align256(static_cast<size_t>(M) * L.dz_stride * 2);
  L.part = 2 * L.low;
  L.x = L.part + align256(static_cast<size_t>(L.parts) * N * 4);
  L.w = L.x + pad_bytes(M, K);
  L.sums = L.w + pad_bytes(N, K);
  const uint32_t cus = static_cast<uint32_t>(num_cus);
  const size_t dx = sums_bytes(M, K, N, cus), dw = sums_bytes(N, K, M, cus);   // (one after the other)
  L.bytes = L.sums + (dx > dw ? dx : dw);
  return L;
}

}  // namespace

// Each way to go about a product costs the stages of the tiles that a CU takes
// one after the other, and the join that writes and reads the parts' sums; the
// least is taken.  A stage is of 64 of k: 1.5 us for a tile of 256 x 256, 0.95 for
// two of 128 x 128, 0.55 for one (measured with K of 4096 and more; the choices are
// close: 4096 x 12288 by 2048 takes 193 us as two parts with their join, 197 as
// small tiles).
ProdPlan plan_product(uint64_t I, uint64_t J, uint64_t K, uint32_t cus) {
  ProdPlan best{false, 1, 0, 0.0};
  if (!I || !J || !K) return best;
  double least = 0.0;
  for (int large = 0; large < 2; ++large) {
    if (large && (I <= 128 || J <= 128)) continue;
    const uint64_t b = large ? 256 : 128, tiles = ((I + b - 1) / b) * ((J + b - 1) / b);
    for (uint32_t parts = 1; parts <= 16; parts *= 2) {
      const uint64_t part_k = ((K + parts - 1) / parts + 127) / 128 * 128, used = (K + part_k - 1) / part_k;
      if (parts > 1 && (part_k < 256 || used != parts)) break;
      const uint64_t items = tiles * parts, slots = (large ? 1 : 2) * uint64_t{cus};
      const double stage = large ? 1.5 : items <= cus ? 0.55 : 0.95;
      double us = static_cast<double>((items + slots - 1) / slots) * static_cast<double>(part_k / 64) * stage;
      if (parts > 1) us += 4.0 + static_cast<double>(parts) * static_cast<double>(I) * static_cast<double>(J) * 8.0 / 6e6;
      if ((!large && parts == 1) || us < least) {
        least = us;
        best = {large == 1, parts, static_cast<uint32_t>(part_k), us};
      }
    }
  }
  return best;
}

// The two products of a gradient whose small tiles the CUs hold all at once cost
// the longer one's stages, and a launch less (3 us).
bool plan_pair(uint64_t M, uint64_t N, uint64_t K, uint32_t cus) {
  if (!M || !N || !K) return false;
  const auto tiles = [](uint64_t a, uint64_t b) { return ((a + 127) / 128 + 7) / 8 * 8 * ((b + 127) / 128); };
  const uint64_t items = tiles(M, K) + tiles(N, K);
  if (items > 2 * uint64_t{cus}) return false;
  const double pair = static_cast<double>(((M > N ? M : N) + 127) / 128 * 2) * (items <= cus ? 0.55 : 0.95);
  return pair <= plan_product(M, K, N, cus).us + plan_product(N, K, M, cus).us + 3.0;
}

size_t lin_workspace(int64_t M, int64_t N, int64_t K, int num_cus) {
  const uint32_t cus = static_cast<uint32_t>(num_cus);
  const bool few = few_rows(static_cast<uint64_t>(M), static_cast<uint64_t>(N), cus);
  if (M <= kFewAny) return 0;
  return pad_bytes(M, K) + pad_bytes(N, K) + (few ? 0 : sums_bytes(M, N, K, cus));
}

size_t lin_grad_workspace(int64_t M, int64_t N, int64_t K, int num_cus) { return grad_layout(M, N, K, num_cus).bytes; }

hipError_t launch_linear(const LinCall& c, hipStream_t s) {
  ProdArgs g{static_cast<const __bf16*>(c.x), static_cast<const __bf16*>(c.w), nullptr, c.x_stride, c.w_stride,
             static_cast<uint32_t>(c.M), static_cast<uint32_t>(c.N), static_cast<uint32_t>(c.K), c.bias, c.act,
             c.out_dtype, c.residual, c.residual_stride, c.out, c.pre, 0, 0, 1, 0, false, false};
  const uint32_t cus = static_cast<uint32_t>(device_cu_count());
  (void)hipGetLastError();
  uint8_t* const ws = static_cast<uint8_t*>(c.ws);
  if (launch_product_few(g, cus, s) || launch_product_few_any(g, cus, s)) return hipGetLastError();
  if (c.K % 8) {
    __bf16* const x = reinterpret_cast<__bf16*>(ws);
    __bf16* const w = reinterpret_cast<__bf16*>(ws + pad_bytes(c.M, c.K));
    const PadArgs p = pad_args(c.x, c.x_stride, c.M, x, c.w, c.w_stride, c.N, w, c.K);
    k_pad<<<pad_blocks(p), 256, 0, s>>>(p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    g.a = x;
    g.b = w;
    g.as = g.bs = padded(c.K);
    g.a_padded = g.b_padded = true;
  }
  if (launch_product_few(g, cus, s)) return hipGetLastError();
  float* const sums = reinterpret_cast<float*>(ws + pad_bytes(c.M, c.K) + pad_bytes(c.N, c.K));
  // (few rows that are not aligned have no workspace for parts)
  const ProdPlan p = few_rows(g.I, g.J, cus) ? ProdPlan{false, 1, 0, 0.0} : plan_product(g.I, g.J, g.K, cus);
  if (launch_product_along(g, p, sums, cus, s)) return hipGetLastError();
  return launch_any<false, false>(g, s);
}

hipError_t launch_linear_grad(const LinGradCall& c, hipStream_t s) {
  const uint32_t cus = static_cast<uint32_t>(device_cu_count());
  const GradLayout L = grad_layout(c.M, c.N, c.K, static_cast<int>(cus));
  uint8_t* const ws = static_cast<uint8_t*>(c.ws);
  const uint32_t M = static_cast<uint32_t>(c.M), N = static_cast<uint32_t>(c.N), K = static_cast<uint32_t>(c.K);
  __bf16* const dz = reinterpret_cast<__bf16*>(ws + L.dz);
  // (dz is a bf16 number where dy is and the slope is 0 or 1)
  const bool slope = c.act == PROFK_ACT_GELU || c.act == PROFK_ACT_SILU;
  __bf16* const low = !c.round_dz && (slope || c.dtype == PROFK_F32) ? reinterpret_cast<__bf16*>(ws + L.low) : nullptr;
  float* const part = reinterpret_cast<float*>(ws + L.part);
  // (without an activation, dy in bf16 is dz)
  const bool given = c.act == PROFK_ACT_NONE && c.dtype == PROFK_BF16 && granules(c.dy, c.dy_stride, N, false);
  const bool dx = c.dx && M, dw = c.dw && N;
  const uint32_t cols = dz_cols(N);
  const DzArgs d{c.dy, c.pre, c.dy_stride, M, N, cols, L.parts, (dx || dw) && !given ? dz : nullptr,
                 dx || dw ? low : nullptr, L.dz_stride, !c.db ? nullptr : L.parts == 1 ? c.db : part};
  // the copies of W and x, where their rows are not whole granules, beside dz
  const PadArgs p = pad_args(c.x, c.x_stride, K % 8 && dw ? M : 0, reinterpret_cast<__bf16*>(ws + L.x), c.w, c.w_stride,
                             K % 8 && dx ? N : 0, reinterpret_cast<__bf16*>(ws + L.w), K);
  const uint32_t slabs = N && (d.dz || d.part) ? (N + cols * 8 - 1) / (cols * 8) : 0, dz_blocks = slabs * L.parts;
  (void)hipGetLastError();
  hipError_t e = hipSuccess;
  if (const uint32_t blocks = dz_blocks + pad_blocks(p)) {
    with_act(c.act, [&](auto act) {
      if (c.dtype == PROFK_F32) k_dz<PROFK_F32, decltype(act)::value><<<blocks, kDzBS, 0, s>>>(d, slabs, dz_blocks, p);
      else k_dz<PROFK_BF16, decltype(act)::value><<<blocks, kDzBS, 0, s>>>(d, slabs, dz_blocks, p);
    });
    e = hipGetLastError();
  }
  if (e == hipSuccess && c.db && N && L.parts > 1) {
    const uint32_t blocks = (N + kJoinCols - 1) / kJoinCols;   // (a launch holds fewer than 2^32 threads)
    k_db_join<<<blocks < 65536 ? blocks : 65536, kJoinBS, 0, s>>>(part, L.parts, N, c.db);
    e = hipGetLastError();
  }
  float* const sums = reinterpret_cast<float*>(ws + L.sums);
  ProdArgs g{};
  g.parts = 1;
  g.a = given ? static_cast<const __bf16*>(c.dy) : dz;
  g.a_low = low;
  g.as = given ? c.dy_stride : L.dz_stride;
  g.a_padded = !given;
  g.b_padded = K % 8 != 0;
  g.J = K;
  g.act = PROFK_ACT_NONE;
  g.out_dtype = PROFK_BF16;
  // b: W or x, or its copy
  auto product = [&](const void* b, uint64_t stride, size_t copy, uint32_t I, uint32_t k, void* out) {
    ProdArgs o = g;
    o.b = g.b_padded ? reinterpret_cast<const __bf16*>(ws + copy) : static_cast<const __bf16*>(b);
    o.bs = g.b_padded ? padded(K) : stride;
    o.I = I;
    o.K = k;
    o.out = out;
    return o;
  };
  const ProdArgs gx = product(c.w, c.w_stride, L.w, M, N, c.dx), gw = product(c.x, c.x_stride, L.x, N, M, c.dw);
  if (e == hipSuccess && dx && dw && plan_pair(M, N, K, cus) && launch_product_pair(gx, gw, s)) return hipGetLastError();
  if (e == hipSuccess && dx)
    e = launch_product_grad(gx, false, plan_product(M, K, N, cus), sums, cus, s) ? hipGetLastError() : launch_any<false, true>(gx, s);
  if (e == hipSuccess && dw)
    e = launch_product_grad(gw, true, plan_product(N, K, M, cus), sums, cus, s) ? hipGetLastError() : launch_any<true, true>(gw, s);
  return e;
}

}  // namespace profk
