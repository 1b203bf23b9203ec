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
#include "elem8.h"
#include "launch.h"
#include "norm.h"

namespace profk {

namespace {

constexpr uint32_t kJoinCols = 64, kJoinRows = 16;   // join: columns and rows of partial sums of a workgroup

// Sums over the threads of a row: a wave's, or all BS.  `slot` alternates
// between successive sums, so that one barrier each is enough.
template <int BS, bool WAVE, int N> __device__ __forceinline__ void row_sum(float (&v)[N], float (*slot)[N]) {
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] = wave_sum(v[k]);
  if constexpr (!WAVE) {
    constexpr int NW = BS / kWave;
    if ((threadIdx.x & (kWave - 1)) == 0) {
#pragma unroll
      for (int k = 0; k < N; ++k) slot[threadIdx.x / kWave][k] = v[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) {
      float s = slot[0][k];
#pragma unroll
      for (int w = 1; w < NW; ++w) s += slot[w][k];
      v[k] = s;
    }
  }
}

// (rounding may leave a variance of equal values below 0; NaN passes)
__device__ __forceinline__ float row_rstd(float sq, float d, float eps) {
  const float var = fmaf(-d, d, sq);
  return 1.0f / sqrtf((var < 0.0f ? 0.0f : var) + eps);
}

__device__ __forceinline__ void load_param8(const void* p, int dtype, uint32_t i, uint32_t D, float none, float (&v)[8]) {
  if (!p) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = none;
  } else if (dtype == PROFK_F32) {
    load8<PROFK_F32>(p, i, D, v);
  } else {
    load8<PROFK_BF16>(p, i, D, v);
  }
}

template <int DT> __device__ __forceinline__ const void* row_at(const void* x, uint64_t stride, uint32_t r) {
  return static_cast<const char*>(x) + r * stride * (DT == PROFK_F32 ? 4 : 2);
}
template <int DT> __device__ __forceinline__ void* row_at(void* x, uint64_t stride, uint32_t r) {
  return static_cast<char*>(x) + r * stride * (DT == PROFK_F32 ? 4 : 2);
}

// A row in the registers of one wave or of a workgroup, C chunks of 8 elements
// a thread; workgroups go through the rows, the scale and shift kept in
// registers and the next row loaded under this one.
template <int XDT, int YDT, int BS, int C, bool WAVE> __global__ __launch_bounds__(BS) void k_norm(NormArgs a) {
  constexpr uint32_t GS = WAVE ? kWave : BS, R = BS / GS;
  __shared__ float s_red[BS / kWave][1], s_sq[BS / kWave][2];
  const uint32_t t = WAVE ? threadIdx.x & (kWave - 1) : threadIdx.x;
  const uint32_t step = gridDim.x * R;
  uint32_t row = blockIdx.x * R + (WAVE ? threadIdx.x / kWave : 0);
  if (row >= a.T) return;      // (a whole wave, or the workgroup)
  float w[C][8], b[C][8];
  Raw8<XDT> next[C];
#pragma unroll
  for (int c = 0; c < C; ++c) next[c] = load_raw8<XDT>(row_at<XDT>(a.x, a.stride, row), (c * GS + t) * 8, a.D);
#pragma unroll
  for (int c = 0; c < C; ++c) {
    load_param8(a.w, a.p_dtype, (c * GS + t) * 8, a.D, 1.0f, w[c]);
    load_param8(a.b, a.p_dtype, (c * GS + t) * 8, a.D, 0.0f, b[c]);
  }
  const float inv = 1.0f / static_cast<float>(a.D);
  for (; row < a.T; row += step) {
    float v[C][8], s[1] = {0.0f};
#pragma unroll
    for (int c = 0; c < C; ++c) {
      to_f32<XDT>(next[c], v[c]);
#pragma unroll
      for (int e = 0; e < 8; ++e) s[0] += v[c][e];
    }
    if (a.T - row > step) {
#pragma unroll
      for (int c = 0; c < C; ++c) next[c] = load_raw8<XDT>(row_at<XDT>(a.x, a.stride, row + step), (c * GS + t) * 8, a.D);
    }
    row_sum<BS, WAVE>(s, s_red);
    const float m = s[0] * inv;
    float q[2] = {0.0f, 0.0f};
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const uint32_t i = (c * GS + t) * 8;
#pragma unroll
      for (uint32_t e = 0; e < 8; ++e) {
        v[c][e] = i + e < a.D ? v[c][e] - m : 0.0f;
        q[0] += v[c][e];
        q[1] = fmaf(v[c][e], v[c][e], q[1]);
      }
    }
    row_sum<BS, WAVE>(q, s_sq);
    const float d = q[0] * inv, r = row_rstd(q[1] * inv, d, a.eps);
    void* const out = row_at<YDT>(a.out, a.out_stride, row);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      float y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = fmaf((v[c][e] - d) * r, w[c][e], b[c][e]);
      store8<YDT>(out, (c * GS + t) * 8, a.D, y);
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
  __shared__ float s_red[BS / kWave][1], s_sq[BS / kWave][2];
  const float inv = 1.0f / static_cast<float>(a.D);
  for (uint32_t row = blockIdx.x; row < a.T; row += gridDim.x) {
    const void* const x = row_at<XDT>(a.x, a.stride, row);
    float s[1] = {0.0f}, v[8];
    for (uint32_t i = threadIdx.x * 8; i < a.D; i += BS * 8) {
      load8<XDT>(x, i, a.D, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) s[0] += v[e];
    }
    row_sum<BS, false>(s, s_red);
    const float m = s[0] * inv;
    float q[2] = {0.0f, 0.0f};
    for (uint32_t i = threadIdx.x * 8; i < a.D; i += BS * 8) {
      load8<XDT>(x, i, a.D, v);
#pragma unroll
      for (uint32_t e = 0; e < 8; ++e) {
        const float c = i + e < a.D ? v[e] - m : 0.0f;
        q[0] += c;
        q[1] = fmaf(c, c, q[1]);
      }
    }
    row_sum<BS, false>(q, s_sq);
    const float d = q[0] * inv, r = row_rstd(q[1] * inv, d, a.eps);
    void* const out = row_at<YDT>(a.out, a.out_stride, row);
    for (uint32_t i = threadIdx.x * 8; i < a.D; i += BS * 8) {
      float w[8], b[8];
      load8<XDT>(x, i, a.D, v);
      load_param8(a.w, a.p_dtype, i, a.D, 1.0f, w);
      load_param8(a.b, a.p_dtype, i, a.D, 0.0f, b);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = fmaf((v[e] - m - d) * r, w[e], b[e]);
      store8<YDT>(out, i, a.D, v);
    }
    if (threadIdx.x == 0) {
      if (a.mean) a.mean[row] = m + d;
      if (a.rstd) a.rstd[row] = r;
    }
  }
}

// The gradients of rows in registers: one sum of two numbers a row, and each
// workgroup's sums of dy n and dy over its rows kept in registers until its end.
template <int XDT, int YDT, int BS, int C, bool WAVE> __global__ __launch_bounds__(BS) void k_norm_grad(NormGradArgs a) {
  constexpr uint32_t GS = WAVE ? kWave : BS, R = BS / GS;
  __shared__ float s_red[2][BS / kWave][2];
  const uint32_t t = WAVE ? threadIdx.x & (kWave - 1) : threadIdx.x;
  const uint32_t step = gridDim.x * R;
  uint32_t row = blockIdx.x * R + (WAVE ? threadIdx.x / kWave : 0);
  float w[C][8], dw[C][8] = {}, db[C][8] = {};
  Raw8<XDT> nx[C];
  Raw8<YDT> ny[C];
  float nm = 0.0f, nr = 0.0f;
  auto load = [&](uint32_t r) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      nx[c] = load_raw8<XDT>(row_at<XDT>(a.x, a.stride, r), (c * GS + t) * 8, a.D);
      ny[c] = load_raw8<YDT>(row_at<YDT>(a.dy, a.dy_stride, r), (c * GS + t) * 8, a.D);
    }
    nm = a.mean[r];
    nr = a.rstd[r];
  };
  if (row < a.T) load(row);
#pragma unroll
  for (int c = 0; c < C; ++c) load_param8(a.w, a.p_dtype, (c * GS + t) * 8, a.D, 1.0f, w[c]);
  const float inv = 1.0f / static_cast<float>(a.D);
  uint32_t slot = 0;
  for (; row < a.T; row += step, slot ^= 1) {
    float n[C][8], g[C][8], s[2] = {0.0f, 0.0f};
    const float m = nm, r = nr;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      to_f32<XDT>(nx[c], n[c]);
      to_f32<YDT>(ny[c], g[c]);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        // (past the row's end dy is 0)
        n[c][e] = (n[c][e] - m) * r;
        dw[c][e] = fmaf(g[c][e], n[c][e], dw[c][e]);
        db[c][e] += g[c][e];
        g[c][e] *= w[c][e];
        s[0] += g[c][e];
        s[1] = fmaf(g[c][e], n[c][e], s[1]);
      }
    }
    if (a.T - row > step) load(row + step);
    if (a.dx) {       // (the same for all: the barrier is met by the whole workgroup)
      row_sum<BS, WAVE>(s, s_red[slot]);
      s[0] *= inv;
      s[1] *= inv;
      void* const out = row_at<XDT>(a.dx, a.dx_stride, row);
#pragma unroll
      for (int c = 0; c < C; ++c) {
#pragma unroll
        for (int e = 0; e < 8; ++e) g[c][e] = r * (g[c][e] - s[0] - n[c][e] * s[1]);
        store8<XDT>(out, (c * GS + t) * 8, a.D, g[c]);
      }
    }
  }
  if (!a.part) return;
  float* const part = a.part + static_cast<size_t>(blockIdx.x) * 2 * a.D;
  if constexpr (WAVE) {
    // the waves' sums, in wave order
    __shared__ float s_sum[2][C * kWave * 8];
    for (uint32_t k = 0; k < R; ++k) {
      if (threadIdx.x / kWave == k) {
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const uint32_t i = (c * 8 + e) * kWave + t;
            s_sum[0][i] = k ? s_sum[0][i] + dw[c][e] : dw[c][e];
            s_sum[1][i] = k ? s_sum[1][i] + db[c][e] : db[c][e];
          }
      }
      __syncthreads();
    }
    for (uint32_t i = threadIdx.x; i < C * kWave * 8; i += BS) {
      const uint32_t col = (i / (8 * kWave) * kWave + i % kWave) * 8 + i / kWave % 8;
      if (col < a.D) {
        part[col] = s_sum[0][i];
        part[a.D + col] = s_sum[1][i];
      }
    }
  } else {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      store8<PROFK_F32>(part, (c * GS + t) * 8, a.D, dw[c]);
      store8<PROFK_F32>(part + a.D, (c * GS + t) * 8, a.D, db[c]);
    }
  }
}

// Long rows: dx by a workgroup a row, read twice; the sums over the rows by
// workgroups of 2048 columns and a part of the rows.
template <int XDT, int YDT> __global__ __launch_bounds__(1024) void k_norm_grad_long(NormGradArgs a) {
  constexpr uint32_t BS = 1024;
  __shared__ float s_red[2][BS / kWave][2];
  const float inv = 1.0f / static_cast<float>(a.D);
  uint32_t slot = 0;
  for (uint32_t row = blockIdx.x; row < a.T; row += gridDim.x, slot ^= 1) {
    const void* const x = row_at<XDT>(a.x, a.stride, row);
    const void* const dy = row_at<YDT>(a.dy, a.dy_stride, row);
    void* const out = row_at<XDT>(a.dx, a.dx_stride, row);
    const float m = a.mean[row], r = a.rstd[row];
    float s[2] = {0.0f, 0.0f}, n[8], g[8], w[8];
    for (uint32_t i = threadIdx.x * 8; i < a.D; i += BS * 8) {
      load8<XDT>(x, i, a.D, n);
      load8<YDT>(dy, i, a.D, g);
      load_param8(a.w, a.p_dtype, i, a.D, 1.0f, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float q = g[e] * w[e];
        s[0] += q;
        s[1] = fmaf(q, (n[e] - m) * r, s[1]);
      }
    }
    row_sum<BS, false>(s, s_red[slot]);
    s[0] *= inv;
    s[1] *= inv;
    for (uint32_t i = threadIdx.x * 8; i < a.D; i += BS * 8) {
      load8<XDT>(x, i, a.D, n);
      load8<YDT>(dy, i, a.D, g);
      load_param8(a.w, a.p_dtype, i, a.D, 1.0f, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) g[e] = r * (g[e] * w[e] - s[0] - (n[e] - m) * r * s[1]);
      store8<XDT>(out, i, a.D, g);
    }
  }
}

template <int XDT, int YDT> __global__ __launch_bounds__(256) void k_norm_cols(NormGradArgs a) {
  const uint32_t i = (blockIdx.x * 256 + threadIdx.x) * 8;
  if (i >= a.D) return;
  const uint32_t p = blockIdx.y;
  const uint32_t r0 = static_cast<uint32_t>(static_cast<uint64_t>(a.T) * p / a.parts);
  const uint32_t r1 = static_cast<uint32_t>(static_cast<uint64_t>(a.T) * (p + 1) / a.parts);
  float dw[8] = {}, db[8] = {}, n[8], g[8];
  for (uint32_t row = r0; row < r1; ++row) {
    load8<XDT>(row_at<XDT>(a.x, a.stride, row), i, a.D, n);
    load8<YDT>(row_at<YDT>(a.dy, a.dy_stride, row), i, a.D, g);
    const float m = a.mean[row], r = a.rstd[row];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      dw[e] = fmaf(g[e], (n[e] - m) * r, dw[e]);
      db[e] += g[e];
    }
  }
  float* const part = a.part + static_cast<size_t>(p) * 2 * a.D;
  store8<PROFK_F32>(part, i, a.D, dw);
  store8<PROFK_F32>(part + a.D, i, a.D, db);
}

// The parts' sums, in a fixed order, to dw and db.
__global__ __launch_bounds__(kJoinCols * kJoinRows) void k_norm_join(NormGradArgs a) {
  __shared__ float s[kJoinRows][kJoinCols];
  const uint32_t c = threadIdx.x % kJoinCols, k = threadIdx.x / kJoinCols;
  const uint32_t col = blockIdx.x * kJoinCols + c;     // of 2 D
  float sum = 0.0f;
  if (col < 2 * a.D)
    for (uint32_t p = k; p < a.parts; p += kJoinRows) sum += a.part[static_cast<size_t>(p) * 2 * a.D + col];
  s[k][c] = sum;
  __syncthreads();
  if (k != 0 || col >= 2 * a.D) return;
#pragma unroll
  for (uint32_t j = 1; j < kJoinRows; ++j) sum += s[j][c];
  void* const out = col < a.D ? a.dw : a.db;
  const uint32_t i = col < a.D ? col : col - a.D;
  if (!out) return;
  if (a.p_dtype == PROFK_F32) static_cast<float*>(out)[i] = sum;
  else static_cast<__bf16*>(out)[i] = static_cast<__bf16>(sum);
}

// Longest rows that are kept in registers.
constexpr uint32_t kWaveD = 1024, kBlockD = 16384;
// Workgroups a CU of the kernels that go through the rows.
constexpr uint32_t kPerCu = 4;

// f(BS, C, WAVE) for rows of D <= kBlockD.
template <class F> void with_shape(uint32_t D, F f) {
  using std::integral_constant;
  auto shape = [&](auto bs, auto c, auto wave) { f(bs, c, wave); };
  if (D <= 512) shape(integral_constant<int, 256>{}, integral_constant<int, 1>{}, std::true_type{});
  else if (D <= 1024) shape(integral_constant<int, 256>{}, integral_constant<int, 2>{}, std::true_type{});
  else if (D <= 2048) shape(integral_constant<int, 256>{}, integral_constant<int, 1>{}, std::false_type{});
  else if (D <= 4096) shape(integral_constant<int, 256>{}, integral_constant<int, 2>{}, std::false_type{});
  else if (D <= 8192) shape(integral_constant<int, 512>{}, integral_constant<int, 2>{}, std::false_type{});
  else shape(integral_constant<int, 1024>{}, integral_constant<int, 2>{}, std::false_type{});
}

// Workgroups that go through T rows of D.
uint32_t row_grid(uint32_t T, uint32_t D, uint32_t cus) {
  const uint32_t rows = D <= kWaveD ? 4 : 1;
  const uint32_t per_cu = D <= 4096 ? kPerCu : D <= 8192 ? kPerCu / 2 : 1;
  const uint32_t need = (T + rows - 1) / rows;
  return need < per_cu * cus ? need : per_cu * cus;
}

template <int XDT, int YDT> void norm_rows(const NormArgs& a, uint32_t cus, hipStream_t s) {
  if (a.D > kBlockD) {
    k_norm_long<XDT, YDT><<<a.T < 2 * cus ? a.T : 2 * cus, 1024, 0, s>>>(a);
    return;
  }
  with_shape(a.D, [&](auto bs, auto c, auto wave) {
    k_norm<XDT, YDT, decltype(bs)::value, decltype(c)::value, decltype(wave)::value>
        <<<row_grid(a.T, a.D, cus), decltype(bs)::value, 0, s>>>(a);
  });
}

template <int XDT, int YDT> void norm_grad_rows(const NormGradArgs& a, uint32_t cus, hipStream_t s) {
  if (a.D > kBlockD) {
    if (a.dx && a.T) k_norm_grad_long<XDT, YDT><<<a.T < 2 * cus ? a.T : 2 * cus, 1024, 0, s>>>(a);
    if (a.part) k_norm_cols<XDT, YDT><<<dim3((a.D + 2047) / 2048, a.parts), 256, 0, s>>>(a);
    return;
  }
  with_shape(a.D, [&](auto bs, auto c, auto wave) {
    k_norm_grad<XDT, YDT, decltype(bs)::value, decltype(c)::value, decltype(wave)::value>
        <<<a.parts, decltype(bs)::value, 0, s>>>(a);
  });
}

}  // namespace

uint32_t norm_grad_parts(int64_t T, int64_t D, int num_cus) {
  const uint32_t cus = static_cast<uint32_t>(num_cus);
  if (T <= 0) return 1;
  if (D <= static_cast<int64_t>(kBlockD)) return row_grid(static_cast<uint32_t>(T), static_cast<uint32_t>(D), cus);
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
  if (e != hipSuccess || !a.part) return e;
  k_norm_join<<<(2 * a.D + kJoinCols - 1) / kJoinCols, kJoinCols * kJoinRows, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace profk
