// The product of few rows along k, bound by reading b once.
//
// A wave takes groups of NG x 16 rows of b, 64 of k (whole lines of 128 bytes a
// row) at a time, and the rows of a beside them, loaded straight to a part of LDS
// of its own, four stages deep, so that no barrier is needed and the loads of the
// next group start before this one ends.  Granule g of row r is at position g ^
// (r / 2 % 8) of its eight.  a comes from the caches: one load of 8 rows more for
// each 16 or 32 rows of b.
// Measured: 1 x 4096 x 12288 18 us (5.6 TB/s; a plain read of large arrays reaches
// 7), where the tiles took 71.
// KSPLIT: the workgroup's waves each take a part of K of the same groups, and
// their sums are added in wave order.
#include <type_traits>

#include "launch.h"
#include "product.h"
#include "product_put.h"

namespace profk {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kFewBS = 256, kFewNW = kFewBS / kWave;
constexpr uint32_t kFewK = 64, kCuLds = 160 * 1024;

__device__ const uint4 g_few_zero = {0, 0, 0, 0};

// Granules of a wave's stage; LDS of a workgroup.
constexpr uint32_t few_gran(int ng, int xl) { return (ng * 16 + xl * 8) * 8; }
constexpr uint32_t few_sums(int ng, int xl, bool ksplit) { return ksplit ? (kFewNW - 1) * ng * (xl > 2 ? 2 : 1) * 4 * kWave : 1; }
constexpr uint32_t few_lds(int ng, int xl, bool ksplit) { return 4 * kFewNW * few_gran(ng, xl) * 16 + few_sums(ng, xl, ksplit) * 4; }
constexpr uint32_t few_per_cu(int ng, int xl, bool ksplit) {
  return kCuLds / few_lds(ng, xl, ksplit) < 8 ? kCuLds / few_lds(ng, xl, ksplit) : 8;
}

// XL: loads of a's rows, 8 each.
template <int NG, int XL, bool KSPLIT> __global__ __launch_bounds__(kFewBS) void k_prod_few(ProdArgs g) {
  constexpr int MG = XL > 2 ? 2 : 1, kLoads = NG * 2 + XL;
  constexpr uint32_t kQ = few_gran(NG, XL), kX = NG * 16 * 8;   // granules of a stage; first of a
  __shared__ __align__(16) uint4 s0[kFewNW * kQ], s1[kFewNW * kQ], s2[kFewNW * kQ], s3[kFewNW * kQ];
  __shared__ float s_sum[few_sums(NG, XL, KSPLIT)];
  const uint32_t tid = threadIdx.x, lane = tid & (kWave - 1);
  const uint32_t w = __builtin_amdgcn_readfirstlane(tid / kWave);
  const uint32_t c = lane & 15, h = lane >> 4;
  const uint32_t groups = (g.J + NG * 16 - 1) / (NG * 16), steps = (g.K + kFewK - 1) / kFewK;
  // this wave's groups and its part of K
  const uint32_t g0 = KSPLIT ? blockIdx.x : blockIdx.x * kFewNW + w, gs = KSPLIT ? gridDim.x : gridDim.x * kFewNW;
  const uint32_t p0 = KSPLIT ? steps * w / kFewNW : 0, p1 = KSPLIT ? steps * (w + 1) / kFewNW : steps;
  const uint32_t mine = g0 < groups ? (groups - g0 + gs - 1) / gs : 0;
  const uint32_t total = mine * (p1 - p0);

  // the step to load next: group ig, step ip
  uint32_t ig = g0, ip = p0, issued = 0;
  auto issue = [&](uint4* stage) {
    uint4* const st = stage + w * kQ;
    auto part = [&](const __bf16* p, uint64_t stride, uint32_t row, uint32_t r, uint4* at) {
      const uint32_t k = ip * kFewK + ((lane & 7) ^ (r >> 1 & 7)) * 8;
      const void* const q = k < g.K ? static_cast<const void*>(p + row * stride + k) : &g_few_zero;
      __builtin_amdgcn_global_load_lds(static_cast<const uint32_t*>(q), at, 16, 0, 0);
    };
#pragma unroll
    for (uint32_t q = 0; q < NG * 2; ++q) {
      const uint32_t r = q * 8 + lane / 8;
      part(g.b, g.bs, min(ig * (NG * 16) + r, g.J - 1), r, st + q * kWave);
    }
#pragma unroll
    for (uint32_t q = 0; q < XL; ++q) {
      const uint32_t r = q * 8 + lane / 8;
      part(g.a, g.as, min(r, g.I - 1), r, st + kX + q * kWave);
    }
    if (++issued < total) {      // (past the last one: it again)
      if (++ip == p1) {
        ip = p0;
        ig += gs;
      }
    }
  };
  if (total) {
    issue(s0);
    issue(s1);
    issue(s2);
  }
  f32x4 acc[MG][NG] = {};
  uint32_t cg = g0, cp = p0;     // the step at hand
  auto finish = [&]() {
    if (KSPLIT) {
      if (w > 0) {
#pragma unroll
        for (int m = 0; m < MG; ++m)
#pragma unroll
          for (int n = 0; n < NG; ++n)
#pragma unroll
            for (int v = 0; v < 4; ++v) s_sum[(((w - 1) * MG + m) * NG + n) * 4 * kWave + v * kWave + lane] = acc[m][n][v];
      }
      __syncthreads();
      if (w == 0) {
#pragma unroll
        for (int o = 0; o < kFewNW - 1; ++o)
#pragma unroll
          for (int m = 0; m < MG; ++m)
#pragma unroll
            for (int n = 0; n < NG; ++n)
#pragma unroll
              for (int v = 0; v < 4; ++v) acc[m][n][v] += s_sum[((o * MG + m) * NG + n) * 4 * kWave + v * kWave + lane];
      }
      __syncthreads();
    }
    if (!KSPLIT || w == 0) {
#pragma unroll
      for (int m = 0; m < MG; ++m)
#pragma unroll
        for (int n = 0; n < NG; ++n)
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            const uint32_t i = m * 16 + 4 * h + v, j = cg * (NG * 16) + n * 16 + c;
            if (i < g.I && j < g.J) put(g, i, j, acc[m][n][v]);
          }
    }
#pragma unroll
    for (int m = 0; m < MG; ++m)
#pragma unroll
      for (int n = 0; n < NG; ++n) acc[m][n] = f32x4{};
  };
  const uint32_t xr = XL == 1 ? c & 7 : c;      // (rows past a's last load are not stored)
  auto step = [&](uint4* cur, uint4* old) {
    // (this wave's own loads and reads: no barrier)
    prod_wait<2 * kLoads>();
    issue(old);
    const uint4* const st = cur + w * kQ;
#pragma unroll
    for (uint32_t q = 0; q < 2; ++q) {
      bf16x8 fa[MG], fb[NG];
#pragma unroll
      for (uint32_t n = 0; n < NG; ++n)
        fb[n] = __builtin_bit_cast(bf16x8, st[(n * 16 + c) * 8 + ((4 * q + h) ^ (c >> 1 & 7))]);
#pragma unroll
      for (uint32_t m = 0; m < MG; ++m)
        fa[m] = __builtin_bit_cast(bf16x8, st[kX + (m * 16 + xr) * 8 + ((4 * q + h) ^ (xr >> 1 & 7))]);
#pragma unroll
      for (int m = 0; m < MG; ++m)
#pragma unroll
        for (int n = 0; n < NG; ++n) acc[m][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fa[m], fb[n], acc[m][n], 0, 0, 0);
    }
    if (++cp == p1) {
      finish();
      cp = p0;
      cg += gs;
    }
  };
  for (uint32_t t = 0; t < total; t += 4) {
    step(s0, s3);
    if (t + 1 < total) step(s1, s0);
    if (t + 2 < total) step(s2, s1);
    if (t + 3 < total) step(s3, s2);
  }
  prod_wait<0>();   // (no load may reach LDS after the workgroup's end)
}

template <int NG, int XL> void few_launch(const ProdArgs& g, uint32_t cus, hipStream_t s) {
  const uint32_t groups = (g.J + NG * 16 - 1) / (NG * 16), steps = (g.K + kFewK - 1) / kFewK;
  // The waves share K where the groups are few, and where K is long (1 x K x N, us,
  // shared and not: 1024 x 12288 8.2 and 8.9, x 50000 22.9 and 23.0, x 131072 52.5 and
  // 48.1; 512 x 131072 33.0 and 26.9; 2048 x 131072 90.7 and 110.0).  (Each then has a
  // step: all meet at the barriers, whose number is that of the groups.)
  if (steps >= 32 || (steps >= 8 && groups < 4 * cus)) {
    const uint32_t most = few_per_cu(NG, XL, true) * cus;
    k_prod_few<NG, XL, true><<<groups < most ? groups : most, kFewBS, 0, s>>>(g);
  } else {
    const uint32_t quads = (groups + kFewNW - 1) / kFewNW, most = few_per_cu(NG, XL, false) * cus;
    k_prod_few<NG, XL, false><<<quads < most ? quads : most, kFewBS, 0, s>>>(g);
  }
}

// Up to kFewAny rows of any stride and alignment, with nothing copied: a wave takes
// four rows of b, its lanes neighbouring eights of k, so that each access is a run of
// memory whatever it starts at, and sums over its lanes at the end.  The next eights
// are on their way under the products of these.  Measured: 1 x 4097 x 12288 21 us, 1 x
// 2049 x 131072 101 us (5.3 TB/s); on the matrix cores, whose fragments are 64 bytes
// of 16 rows, 48 and 224, and with b copied first 55 and more.
// L: lanes of a row; 16 where rows are short (1 x 101 x 50001 with 64 17 us).
constexpr int kDotRows = 4;
template <int M, int L> __global__ __launch_bounds__(kFewBS) void k_prod_dot(ProdArgs g) {
  const uint32_t lane = threadIdx.x & (kWave - 1);
  const uint32_t w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  constexpr uint32_t kAt = kWave / L, kRows = kDotRows * kAt, kChunk = L * 8;   // rows of an access, of a wave; k of an access
  const uint32_t quads = (g.J + kRows - 1) / kRows, chunks = (g.K + kChunk - 1) / kChunk, l = lane % L;
  for (uint32_t q = blockIdx.x * kFewNW + w; q < quads; q += gridDim.x * kFewNW) {
    const __bf16* b[kDotRows];
#pragma unroll
    for (uint32_t r = 0; r < kDotRows; ++r) b[r] = g.b + min(q * kRows + r * kAt + lane / L, g.J - 1) * g.bs;
    Raw<PROFK_BF16, 8> nb[kDotRows], na[M];
    auto fetch = [&](uint32_t p) {
      const uint32_t k = (p * L + l) * 8;
      // (only the last chunk may be a part: no check in the others, behind which loads
      // would wait)
      if ((p + 1) * kChunk <= g.K) {
#pragma unroll
        for (int r = 0; r < kDotRows; ++r) nb[r] = __builtin_bit_cast(Raw<PROFK_BF16, 8>, *reinterpret_cast<const u32x4h*>(b[r] + k));
#pragma unroll
        for (uint32_t m = 0; m < M; ++m)
          na[m] = __builtin_bit_cast(Raw<PROFK_BF16, 8>, *reinterpret_cast<const u32x4h*>(g.a + m * g.as + k));
      } else {
#pragma unroll
        for (int r = 0; r < kDotRows; ++r) nb[r] = load_raw<PROFK_BF16, 8>(b[r], k, g.K);
#pragma unroll
        for (uint32_t m = 0; m < M; ++m) na[m] = load_raw<PROFK_BF16, 8>(g.a + m * g.as, k, g.K);
      }
    };
    float acc[kDotRows][M] = {};
    fetch(0);
    for (uint32_t p = 0; p < chunks; ++p) {
      float vb[kDotRows][8], va[M][8];
#pragma unroll
      for (int r = 0; r < kDotRows; ++r) to_f32<PROFK_BF16, 8>(nb[r], vb[r]);
#pragma unroll
      for (int m = 0; m < M; ++m) to_f32<PROFK_BF16, 8>(na[m], va[m]);
      if (p + 1 < chunks) fetch(p + 1);
#pragma unroll
      for (int r = 0; r < kDotRows; ++r)
#pragma unroll
        for (int m = 0; m < M; ++m)
#pragma unroll
          for (int e = 0; e < 8; ++e) acc[r][m] = fmaf(vb[r][e], va[m][e], acc[r][m]);
    }
#pragma unroll
    for (uint32_t r = 0; r < kDotRows; ++r)
#pragma unroll
      for (uint32_t m = 0; m < M; ++m) {
        const float sum = L == kWave ? wave_sum(acc[r][m]) : sum16(acc[r][m]);
        const uint32_t j = q * kRows + r * kAt + lane / L;
        if (l == r * M + m && j < g.J) put(g, m, j, sum);
      }
  }
}

}  // namespace

bool launch_product_few_any(const ProdArgs& g, uint32_t cus, hipStream_t s) {
  if (g.I > kFewAny) return false;
  const auto launch = [&](auto m, auto lanes) {
    constexpr uint32_t kRows = kDotRows * kWave / decltype(lanes)::value * kFewNW;
    const uint32_t blocks = (g.J + kRows - 1) / kRows, most = 8 * cus;
    k_prod_dot<decltype(m)::value, decltype(lanes)::value><<<blocks < most ? blocks : most, kFewBS, 0, s>>>(g);
  };
  const auto rows = [&](auto m) {
    if (g.K <= 256) launch(m, std::integral_constant<int, 16>{});
    else launch(m, std::integral_constant<int, 64>{});
  };
  if (g.I == 1) rows(std::integral_constant<int, 1>{});
  else if (g.I == 2) rows(std::integral_constant<int, 2>{});
  else if (g.I == 3) rows(std::integral_constant<int, 3>{});
  else rows(std::integral_constant<int, 4>{});
  return true;
}

bool launch_product_few(const ProdArgs& g, uint32_t cus, hipStream_t s) {
  if (!few_rows(g.I, g.J, cus) || !granules(g.a, g.as, g.K, g.a_padded) || !granules(g.b, g.bs, g.K, g.b_padded)) return false;
  // groups of 32 rows of b where every wave has one, which reads a half as often,
  // else of 16, which more workgroups share (us, 16 and 32: 1 x 4096 x 12288 19.3 and
  // 22.0, x 32768 51.2 and 50.3, x 131072 184 and 174)
  const bool wide = g.J >= 32 * 4 * cus;
  if (g.I <= 8) wide ? few_launch<2, 1>(g, cus, s) : few_launch<1, 1>(g, cus, s);
  else if (g.I <= 16) wide ? few_launch<2, 2>(g, cus, s) : few_launch<1, 2>(g, cus, s);
  else few_launch<1, 4>(g, cus, s);
  return true;
}

}  // namespace profk
