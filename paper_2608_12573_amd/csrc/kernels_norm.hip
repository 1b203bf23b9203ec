// Layer norm of rows, and its gradients.
//
// Of one row of D values, m = mean x, r = 1 / sqrt(mean (x - m)^2 + eps),
// n = (x - m) r:
//   y = n w + b.
// The variance is summed from differences c to the mean m0 that the row's first
// sum gave, both from registers: no cancellation for rows far from 0, and one
// read.  m0 is off by its sum's rounding; with d = mean c, summed beside it,
//   m = m0 + d,  variance = mean c^2 - d^2,  x - m = c - d,
// where d is of the size of m0's last bits, so that rows of equal values give 0.
// With g = dy w:
//   dx = r (g - mean g - n mean(g n)),
// which takes out of g its parts along 1 and along n, and over the rows
//   dw = sum dy n,  db = sum dy.
// All in fp32; every output is rounded once.
//
// Bound by memory.  Measured (a copy of 1 GiB reaches 5.2 TB/s): 16384 x 8192 bf16
// 98 us (5.5 TB/s), 8192 x 8192 fp32 100 us (5.4); gradients 16384 x 4096 bf16 76
// us and 7 for the join of the workgroups' sums (4.8), 65536 x 1024 fp32 150 us
// (5.4).  1 x 4096 2.8 us.  Rows past 16384 elements, which are read again from the
// caches: 2048 x 32768 bf16 76 us, gradient 162.
#include "elems.h"
#include "join.h"
#include "launch.h"
#include "norm.h"

namespace profk {

namespace {

// Sums over the GS threads of a row, a wave or more, in every one of them.  Rows
// of more than a wave: the workgroup's rows go together, and `slot` [waves of the
// workgroup] alternates between successive sums, so that one barrier each is enough.
template <int GS, int N> __device__ __forceinline__ void row_sum(float (&v)[N], float (*slot)[N]) {
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] = wave_sum(v[k]);
  if constexpr (GS > kWave) {
    constexpr uint32_t NW = GS / kWave;
    const uint32_t w = threadIdx.x / kWave, first = w / NW * NW;
    if ((threadIdx.x & (kWave - 1)) == 0) {
#pragma unroll
      for (int k = 0; k < N; ++k) slot[w][k] = v[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) {
      float s = slot[first][k];
#pragma unroll
      for (uint32_t q = 1; q < NW; ++q) s += slot[first + q][k];
      v[k] = s;
    }
  }
}

// (rounding may leave a variance of equal values below 0; NaN passes)
__device__ __forceinline__ float row_rstd(float sq, float d, float eps) {
  const float var = fmaf(-d, d, sq);
  return 1.0f / sqrtf((var < 0.0f ? 0.0f : var) + eps);
}

template <int E>
__device__ __forceinline__ void load_param(const void* p, int dtype, uint32_t i, uint32_t D, float none, float (&v)[E]) {
  if (!p) {
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = none;
  } else if (dtype == PROFK_F32) {
    if constexpr (E == 8) {
      float lo[4], hi[4];
      load<PROFK_F32, 4>(p, i, D, lo);
      load<PROFK_F32, 4>(p, i + 4, D, hi);
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = e < 4 ? lo[e % 4] : hi[e % 4];
    } else {
      load<PROFK_F32, E>(p, i, D, v);
    }
  } else {
    load<PROFK_BF16, E>(p, i, D, v);
  }
}

// Elements of one of a thread's accesses.
template <int XDT, int YDT> constexpr int kElems = XDT == PROFK_F32 || YDT == PROFK_F32 ? 4 : 8;

template <int DT> __device__ __forceinline__ const void* row_at(const void* x, uint64_t stride, uint32_t r) {
  return static_cast<const char*>(x) + r * stride * (DT == PROFK_F32 ? 4 : 2);
}
template <int DT> __device__ __forceinline__ void* row_at(void* x, uint64_t stride, uint32_t r) {
  return static_cast<char*>(x) + r * stride * (DT == PROFK_F32 ? 4 : 2);
}

template <int E> __device__ __forceinline__ void store_sums(float* row, uint32_t i, uint32_t D, const float (&v)[E]) {
#pragma unroll
  for (int k = 0; k < E; k += 4) store<PROFK_F32, 4>(row, i + k, D, {v[k], v[k + 1], v[k + 2], v[k + 3]});
}

template <int E>
__device__ __forceinline__ void store_param(void* p, int dtype, uint32_t i, uint32_t D, const float (&v)[E]) {
  if (!p) return;
  if (dtype == PROFK_F32) store_sums<E>(static_cast<float*>(p), i, D, v);
  else store<PROFK_BF16, E>(p, i, D, v);
}

// A row in the registers of GS threads, C8 times 8 elements each, R rows a
// workgroup; workgroups go through the rows, the scale and shift kept in
// registers and the next row loaded under this one.
template <int XDT, int YDT, int GS, int R, int C8> __global__ __launch_bounds__(GS * R) void k_norm(NormArgs a) {
  constexpr uint32_t BS = GS * R;
  constexpr int E = kElems<XDT, YDT>, C = C8 * 8 / E;
  static_assert(GS == kWave || R == 1, "a row that is left out meets no barrier");
  __shared__ float s_red[BS / kWave][1], s_sq[BS / kWave][2];
  const uint32_t t = threadIdx.x % GS;
  const uint32_t step = gridDim.x * R;
  uint32_t row = blockIdx.x * R + threadIdx.x / GS;
  if (row >= a.T) return;      // (a whole wave, or the workgroup)
  float w[C][E], b[C][E];
  Raw<XDT, E> next[C];
#pragma unroll
  for (int c = 0; c < C; ++c) next[c] = load_raw<XDT, E>(row_at<XDT>(a.x, a.stride, row), (c * GS + t) * E, a.D);
#pragma unroll
  for (int c = 0; c < C; ++c) {
    load_param(a.w, a.p_dtype, (c * GS + t) * E, a.D, 1.0f, w[c]);
    load_param(a.b, a.p_dtype, (c * GS + t) * E, a.D, 0.0f, b[c]);
  }
  const float inv = 1.0f / static_cast<float>(a.D);
  for (; row < a.T; row += step) {
    float v[C][E], s[1] = {0.0f};
#pragma unroll
    for (int c = 0; c < C; ++c) {
      to_f32<XDT, E>(next[c], v[c]);
#pragma unroll
      for (int e = 0; e < E; ++e) s[0] += v[c][e];
    }
    if (a.T - row > step) {
#pragma unroll
      for (int c = 0; c < C; ++c) next[c] = load_raw<XDT, E>(row_at<XDT>(a.x, a.stride, row + step), (c * GS + t) * E, a.D);
    }
    row_sum<GS>(s, s_red);
    const float m = s[0] * inv;
    float q[2] = {0.0f, 0.0f};
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const uint32_t i = (c * GS + t) * E;
#pragma unroll
      for (uint32_t e = 0; e < E; ++e) {
        v[c][e] = i + e < a.D ? v[c][e] - m : 0.0f;
        q[0] += v[c][e];
        q[1] = fmaf(v[c][e], v[c][e], q[1]);
      }
    }
    row_sum<GS>(q, s_sq);
    const float d = q[0] * inv, r = row_rstd(q[1] * inv, d, a.eps);
    void* const out = row_at<YDT>(a.out, a.out_stride, row);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      float y[E];
#pragma unroll
      for (int e = 0; e < E; ++e) y[e] = fmaf((v[c][e] - d) * r, w[c][e], b[c][e]);
      store<YDT, E>(out, (c * GS + t) * E, a.D, y);
    }
    if (t == 0) {
      if (a.mean) a.mean[row] = m + d;
      if (a.rstd) a.rstd[row] = r;
    }
  }
}

// Rows too long for registers: a workgroup reads its row three times, twice
// from the caches.
template <int XDT, int YDT> __global__ __launch_bounds__(1024) void k_norm_long(NormArgs a) {
  constexpr uint32_t BS = 1024;
  constexpr int E = kElems<XDT, YDT>;
  __shared__ float s_red[BS / kWave][1], s_sq[BS / kWave][2];
  const float inv = 1.0f / static_cast<float>(a.D);
  for (uint32_t row = blockIdx.x; row < a.T; row += gridDim.x) {
    const void* const x = row_at<XDT>(a.x, a.stride, row);
    float s[1] = {0.0f}, v[E];
    for (uint32_t i = threadIdx.x * E; i < a.D; i += BS * E) {
      load<XDT, E>(x, i, a.D, v);
#pragma unroll
      for (int e = 0; e < E; ++e) s[0] += v[e];
    }
    row_sum<BS>(s, s_red);
    const float m = s[0] * inv;
    float q[2] = {0.0f, 0.0f};
    for (uint32_t i = threadIdx.x * E; i < a.D; i += BS * E) {
      load<XDT, E>(x, i, a.D, v);
#pragma unroll
      for (uint32_t e = 0; e < E; ++e) {
        const float c = i + e < a.D ? v[e] - m : 0.0f;
        q[0] += c;
        q[1] = fmaf(c, c, q[1]);
      }
    }
    row_sum<BS>(q, s_sq);
    const float d = q[0] * inv, r = row_rstd(q[1] * inv, d, a.eps);
    void* const out = row_at<YDT>(a.out, a.out_stride, row);
    for (uint32_t i = threadIdx.x * E; i < a.D; i += BS * E) {
      float w[E], b[E];
      load<XDT, E>(x, i, a.D, v);
      load_param(a.w, a.p_dtype, i, a.D, 1.0f, w);
      load_param(a.b, a.p_dtype, i, a.D, 0.0f, b);
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = fmaf((v[e] - m - d) * r, w[e], b[e]);
      store<YDT, E>(out, i, a.D, v);
    }
    if (threadIdx.x == 0) {
      if (a.mean) a.mean[row] = m + d;
      if (a.rstd) a.rstd[row] = r;
    }
  }
}

// The gradients of rows in registers: one sum of two numbers a row, and the sums
// of dy n and dy over a thread's rows kept in registers until its end, when the
// workgroup's R rows of threads are added.
template <int XDT, int YDT, int GS, int R, int C8> __global__ __launch_bounds__(GS * R) void k_norm_grad(NormGradArgs a) {
  constexpr uint32_t BS = GS * R;
  constexpr int E = kElems<XDT, YDT>, C = C8 * 8 / E;
  __shared__ float s_red[2][BS / kWave][2];
  __shared__ float s_sum[R > 1 ? 2 * GS * C * E : 1];
  // (1024 threads have 128 registers each: no row ahead, the scale from the caches)
  constexpr bool kLean = BS == 1024 && C8 > 1;
  const uint32_t t = threadIdx.x % GS, sub = threadIdx.x / GS;
  const uint32_t step = gridDim.x * R;
  float w[kLean ? 1 : C][E], dw[C][E] = {}, db[C][E] = {};
  Raw<XDT, E> nx[C];
  Raw<YDT, E> ny[C];
  float nm, nr;
  // (a row that is not there has a gradient of 0)
  auto load = [&](uint32_t r) {
    const uint32_t D = r < a.T ? a.D : 0;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      nx[c] = load_raw<XDT, E>(row_at<XDT>(a.x, a.stride, r), (c * GS + t) * E, D);
      ny[c] = load_raw<YDT, E>(row_at<YDT>(a.dy, a.dy_stride, r), (c * GS + t) * E, D);
    }
    nm = D ? a.mean[r] : 0.0f;
    nr = D ? a.rstd[r] : 0.0f;
  };
  uint32_t row0 = blockIdx.x * R;
  if constexpr (!kLean) {
    load(row0 + sub);
#pragma unroll
    for (int c = 0; c < C; ++c) load_param(a.w, a.p_dtype, (c * GS + t) * E, a.D, 1.0f, w[c]);
  }
  const float inv = 1.0f / static_cast<float>(a.D);
  uint32_t slot = 0;
  for (; row0 < a.T; row0 += step, slot ^= 1) {
    const uint32_t row = row0 + sub;
    float n[C][E], g[C][E], s[2] = {0.0f, 0.0f};
    if constexpr (kLean) load(row);
    const float m = nm, r = nr;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      to_f32<XDT, E>(nx[c], n[c]);
      to_f32<YDT, E>(ny[c], g[c]);
      if constexpr (kLean) load_param(a.w, a.p_dtype, (c * GS + t) * E, a.D, 1.0f, w[0]);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        // (past the row's end dy is 0)
        n[c][e] = (n[c][e] - m) * r;
        dw[c][e] = fmaf(g[c][e], n[c][e], dw[c][e]);
        db[c][e] += g[c][e];
        g[c][e] *= w[kLean ? 0 : c][e];
        s[0] += g[c][e];
        s[1] = fmaf(g[c][e], n[c][e], s[1]);
      }
    }
    if (!kLean && a.T - row0 > step) load(row + step);
    if (a.dx) {       // (the same for all: the barrier is met by the whole workgroup)
      row_sum<GS>(s, s_red[slot]);
      s[0] *= inv;
      s[1] *= inv;
      if (R == 1 || row < a.T) {
        void* const out = row_at<XDT>(a.dx, a.dx_stride, row);
#pragma unroll
        for (int c = 0; c < C; ++c) {
#pragma unroll
          for (int e = 0; e < E; ++e) g[c][e] = r * (g[c][e] - s[0] - n[c][e] * s[1]);
          store<XDT, E>(out, (c * GS + t) * E, a.D, g[c]);
        }
      }
    }
  }
  if (!a.part) return;
  float* const part = a.part + static_cast<size_t>(blockIdx.x) * 2 * a.D;
  if constexpr (R > 1) {
#pragma unroll
    for (uint32_t k = 1; k < R; ++k) {
      if (sub == k) {
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const uint32_t i = (c * E + e) * GS + t;
            s_sum[i] = k > 1 ? s_sum[i] + dw[c][e] : dw[c][e];
            s_sum[GS * C * E + i] = k > 1 ? s_sum[GS * C * E + i] + db[c][e] : db[c][e];
          }
      }
      __syncthreads();
    }
    if (sub != 0) return;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        dw[c][e] += s_sum[(c * E + e) * GS + t];
        db[c][e] += s_sum[GS * C * E + (c * E + e) * GS + t];
      }
  }
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const uint32_t i = (c * GS + t) * E;
    if (a.parts == 1) {           // (no join follows)
      store_param<E>(a.dw, a.p_dtype, i, a.D, dw[c]);
      store_param<E>(a.db, a.p_dtype, i, a.D, db[c]);
    } else {
      store_sums<E>(part, i, a.D, dw[c]);
      store_sums<E>(part + a.D, i, a.D, db[c]);
    }
  }
}

// Long rows: dx by a workgroup a row, read twice; the sums over the rows by
// workgroups of some columns and a part of the rows.
template <int XDT, int YDT> __global__ __launch_bounds__(1024) void k_norm_grad_long(NormGradArgs a) {
  constexpr uint32_t BS = 1024;
  constexpr int E = kElems<XDT, YDT>;
  __shared__ float s_red[2][BS / kWave][2];
  const float inv = 1.0f / static_cast<float>(a.D);
  uint32_t slot = 0;
  for (uint32_t row = blockIdx.x; row < a.T; row += gridDim.x, slot ^= 1) {
    const void* const x = row_at<XDT>(a.x, a.stride, row);
    const void* const dy = row_at<YDT>(a.dy, a.dy_stride, row);
    void* const out = row_at<XDT>(a.dx, a.dx_stride, row);
    const float m = a.mean[row], r = a.rstd[row];
    float s[2] = {0.0f, 0.0f}, n[E], g[E], w[E];
    for (uint32_t i = threadIdx.x * E; i < a.D; i += BS * E) {
      load<XDT, E>(x, i, a.D, n);
      load<YDT, E>(dy, i, a.D, g);
      load_param(a.w, a.p_dtype, i, a.D, 1.0f, w);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float q = g[e] * w[e];
        s[0] += q;
        s[1] = fmaf(q, (n[e] - m) * r, s[1]);
      }
    }
    row_sum<BS>(s, s_red[slot]);
    s[0] *= inv;
    s[1] *= inv;
    for (uint32_t i = threadIdx.x * E; i < a.D; i += BS * E) {
      load<XDT, E>(x, i, a.D, n);
      load<YDT, E>(dy, i, a.D, g);
      load_param(a.w, a.p_dtype, i, a.D, 1.0f, w);
#pragma unroll
      for (int e = 0; e < E; ++e) g[e] = r * (g[e] * w[e] - s[0] - (n[e] - m) * r * s[1]);
      store<XDT, E>(out, i, a.D, g);
    }
  }
}

template <int XDT, int YDT> __global__ __launch_bounds__(256) void k_norm_cols(NormGradArgs a) {
  constexpr int E = kElems<XDT, YDT>;
  const uint32_t i = (blockIdx.x * 256 + threadIdx.x) * E;
  if (i >= a.D) return;
  const uint32_t p = blockIdx.y;
  const uint32_t r0 = static_cast<uint32_t>(static_cast<uint64_t>(a.T) * p / a.parts);
  const uint32_t r1 = static_cast<uint32_t>(static_cast<uint64_t>(a.T) * (p + 1) / a.parts);
  float dw[E] = {}, db[E] = {}, n[E], g[E];
  for (uint32_t row = r0; row < r1; ++row) {
    load<XDT, E>(row_at<XDT>(a.x, a.stride, row), i, a.D, n);
    load<YDT, E>(row_at<YDT>(a.dy, a.dy_stride, row), i, a.D, g);
    const float m = a.mean[row], r = a.rstd[row];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      dw[e] = fmaf(g[e], (n[e] - m) * r, dw[e]);
      db[e] += g[e];
    }
  }
  float* const part = a.part + static_cast<size_t>(p) * 2 * a.D;
  if (a.parts == 1) {
    store_param<E>(a.dw, a.p_dtype, i, a.D, dw);
    store_param<E>(a.db, a.p_dtype, i, a.D, db);
  } else {
    store_sums<E>(part, i, a.D, dw);
    store_sums<E>(part + a.D, i, a.D, db);
  }
}

// The parts' sums to dw and db.
__global__ __launch_bounds__(kJoinBS) void k_norm_join(NormGradArgs a) {
  const float sum = join_parts(a.part, a.parts, 2 * a.D, blockIdx.x);
  const uint32_t col = blockIdx.x * kJoinCols + threadIdx.x;
  if (threadIdx.x >= kJoinCols || col >= 2 * a.D) return;
  void* const out = col < a.D ? a.dw : a.db;
  const uint32_t i = col < a.D ? col : col - a.D;
  if (!out) return;
  if (a.p_dtype == PROFK_F32) static_cast<float*>(out)[i] = sum;
  else static_cast<__bf16*>(out)[i] = static_cast<__bf16>(sum);
}

// Longest rows that are kept in registers.
constexpr uint32_t kBlockD = 16384;

// f(threads of a row, chunks of 8 elements of a thread) for rows of D <= kBlockD.
// (16384 x 6000 bf16 with 512 threads took 89 us, with 384 80.)  The gradient holds
// four numbers for each of the forward call's three, and has 8 elements a thread
// where that does: with 16, a SIMD had registers for three waves (16384 x 6000 bf16
// 184 and 165 us, 8192 x 8192 92 and 86).
template <class F> void with_shape(uint32_t D, F f) {
  using std::integral_constant;
  if (D <= 512) f(integral_constant<int, 64>{}, integral_constant<int, 1>{});
  else if (D <= 1024) f(integral_constant<int, 64>{}, integral_constant<int, 2>{});
  else if (D <= 2048) f(integral_constant<int, 256>{}, integral_constant<int, 1>{});
  else if (D <= 4096) f(integral_constant<int, 256>{}, integral_constant<int, 2>{});
  else if (D <= 6144) f(integral_constant<int, 384>{}, integral_constant<int, 2>{});
  else if (D <= 8192) f(integral_constant<int, 512>{}, integral_constant<int, 2>{});
  else if (D <= 12288) f(integral_constant<int, 768>{}, integral_constant<int, 2>{});
  else f(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
}

template <class F> void with_grad_shape(uint32_t D, F f) {
  using std::integral_constant;
  if (D <= 512) f(integral_constant<int, 64>{}, integral_constant<int, 1>{});
  else if (D <= 1024) f(integral_constant<int, 128>{}, integral_constant<int, 1>{});
  else if (D <= 2048) f(integral_constant<int, 256>{}, integral_constant<int, 1>{});
  else if (D <= 4096) f(integral_constant<int, 512>{}, integral_constant<int, 1>{});
  else if (D <= 6144) f(integral_constant<int, 768>{}, integral_constant<int, 1>{});
  else if (D <= 8192) f(integral_constant<int, 1024>{}, integral_constant<int, 1>{});
  else if (D <= 12288) f(integral_constant<int, 768>{}, integral_constant<int, 2>{});
  else f(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
}

// Rows of a workgroup of the two kernels, and its workgroups a CU.
constexpr int norm_rows_of(int gs) { return gs == 64 ? 4 : 1; }
constexpr int grad_rows_of(int gs) { return gs == 64 ? 8 : gs == 128 ? 4 : gs == 256 ? 2 : 1; }
uint32_t row_grid(uint32_t T, uint32_t rows, uint32_t threads, uint32_t cus) {
  const uint32_t need = (T + rows - 1) / rows, most = (threads <= 256 ? 4 : threads <= 512 ? 2 : 1) * cus;
  return need < most ? need : most;
}

template <int XDT, int YDT> void norm_rows(const NormArgs& a, uint32_t cus, hipStream_t s) {
  if (a.D > kBlockD) {
    k_norm_long<XDT, YDT><<<a.T < 2 * cus ? a.T : 2 * cus, 1024, 0, s>>>(a);
    return;
  }
  with_shape(a.D, [&](auto gs, auto c) {
    constexpr int GS = decltype(gs)::value, R = norm_rows_of(GS);
    k_norm<XDT, YDT, GS, R, decltype(c)::value><<<row_grid(a.T, R, GS * R, cus), GS * R, 0, s>>>(a);
  });
}

template <int XDT, int YDT> void norm_grad_rows(const NormGradArgs& a, uint32_t cus, hipStream_t s) {
  if (a.D > kBlockD) {
    if (a.dx && a.T) k_norm_grad_long<XDT, YDT><<<a.T < 2 * cus ? a.T : 2 * cus, 1024, 0, s>>>(a);
    if (a.part) k_norm_cols<XDT, YDT><<<dim3((a.D + 256 * kElems<XDT, YDT> - 1) / (256 * kElems<XDT, YDT>), a.parts), 256, 0, s>>>(a);
    return;
  }
  with_grad_shape(a.D, [&](auto gs, auto c) {
    constexpr int GS = decltype(gs)::value, R = grad_rows_of(GS);
    k_norm_grad<XDT, YDT, GS, R, decltype(c)::value><<<a.parts, GS * R, 0, s>>>(a);
  });
}

}  // namespace

uint32_t norm_grad_parts(int64_t T, int64_t D, int num_cus) {
  const uint32_t cus = static_cast<uint32_t>(num_cus);
  if (T <= 0) return 1;
  if (D <= static_cast<int64_t>(kBlockD)) {
    uint32_t parts = 0;
    with_grad_shape(static_cast<uint32_t>(D), [&](auto gs, auto) {
      constexpr int GS = decltype(gs)::value, R = grad_rows_of(GS);
      parts = row_grid(static_cast<uint32_t>(T), R, GS * R, cus);
    });
    return parts;
  }
  const uint32_t slabs = static_cast<uint32_t>((D + 2047) / 2048), most = (4 * cus + slabs - 1) / slabs;
  return static_cast<uint32_t>(T < most ? T : most);
}

hipError_t launch_norm(const NormArgs& a, int dtype, int out_dtype, hipStream_t s) {
  const uint32_t cus = static_cast<uint32_t>(device_cu_count());
  (void)hipGetLastError();
  if (dtype == PROFK_F32) {
    if (out_dtype == PROFK_F32) norm_rows<PROFK_F32, PROFK_F32>(a, cus, s);
    else norm_rows<PROFK_F32, PROFK_BF16>(a, cus, s);
  } else {
    if (out_dtype == PROFK_F32) norm_rows<PROFK_BF16, PROFK_F32>(a, cus, s);
    else norm_rows<PROFK_BF16, PROFK_BF16>(a, cus, s);
  }
  return hipGetLastError();
}

hipError_t launch_norm_grad(const NormGradArgs& a, int dtype, int dy_dtype, hipStream_t s) {
  const uint32_t cus = static_cast<uint32_t>(device_cu_count());
  (void)hipGetLastError();
  if (dtype == PROFK_F32) {
    if (dy_dtype == PROFK_F32) norm_grad_rows<PROFK_F32, PROFK_F32>(a, cus, s);
    else norm_grad_rows<PROFK_F32, PROFK_BF16>(a, cus, s);
  } else {
    if (dy_dtype == PROFK_F32) norm_grad_rows<PROFK_BF16, PROFK_F32>(a, cus, s);
    else norm_grad_rows<PROFK_BF16, PROFK_BF16>(a, cus, s);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.part || a.parts == 1) return e;
  k_norm_join<<<(2 * a.D + kJoinCols - 1) / kJoinCols, kJoinBS, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace profk
