// Token log probabilities, entropy and top alternatives of rows of logits,
// and their gradient.
//
// With x a row of V logits, p_j = exp(x_j - lse):
//   lse = log sum_j exp(x_j),   logprob = x_y - lse,
//   H   = -sum_j p_j log p_j   (terms with p_j = 0 are 0),
//   alternatives: the n largest x_j as (x_j - lse, j), in the total order of
//   the library's other selections (larger key first, then smaller index).
//
// k_lp reads a row once.  A lane keeps s = sum 2^t and q = sum 2^t t over
// t = x L - c, L = log2(e) in fp32, with c of its wave, so that
//   log2 sum = c + log2 s  and  H = ln 2 (log2 s - q / s).
// c is the whole number nearest to the wave's largest x L so far; fp32 holds it
// exactly, so t is rounded once (one fma), and dividing the final c + log2 s by
// the same L leaves of L's own rounding (a relative 1.3e-8, as if the row had
// another temperature) no more than 1.3e-8 H in lse.  No t passes 1/2: where c
// is left behind, log2 s and q / s grow by as much as it is behind, and their
// difference loses what they were rounded by (16 powers of two: 2e-6 of H).
//
// Alternatives need no second pass.  Of each of the NW waves the n / NW-th best
// of its lanes' maxima of the first step is taken; the least of them bounds the
// row's n-th best from below, so that only logits at or above it are appended
// to a list in LDS; after 2, 4, 8... steps the list is cut to its best n, which
// raises the bound.  The steps take the row
// in pieces spread over all of it, so that the first is like the others where
// logits depend on their place (a range of forbidden tokens).  A list that
// overflows all the same is replaced by n sweeps that take the row's best of
// what is left, 4096 x 131072 bf16 with 20 alternatives then 13.7 ms in place of
// 0.2: one wave whose first step has fewer than n / NW good lanes is enough, and
// so these are rows of equal logits, of sorted ones, of a few allowed ones under
// a finite mask, or with the last eighth alone allowed.
//
// Measured: 4096 x 131072 bf16 with 20 alternatives 195 us (5.5 TB/s), without
// 179 (6.0): 9 and 7 vector instructions a logit keep the SIMDs busy for 78 and
// 68 % of the time beside the loads, so that 16-bit rows are bound by both;
// 32-bit rows by memory.  16384 x 512 fp32
// with 8 alternatives 18 us, without 10: the selection's instructions.  64 x
// 100003 fp32 14 us and 5 for the join, 1 x 131072 8 and 5: latency.
#include <type_traits>

#include "device_common.h"
#include "launch.h"
#include "logprobs.h"

namespace profk {

namespace {

constexpr float kL2E = 1.44269504088896340736f;   // log2(e), rounded to fp32
constexpr double kLn2 = 0.69314718055994530942;
constexpr float kNegInf = -__builtin_inff();
constexpr float kLpFloor = -300.0f;  // least exponent: 2^-300 is 0 in fp32, and 0 * -300 is no NaN
// Rows with a logit past this (or +inf, or NaN) are summed by the careful
// path, as are rows of nothing above its negative: x L must not overflow, and
// c / L is exact enough for x - lse only while c is small.  (That path reads the
// row twice more, an element a lane: 4096 x 131072 bf16 with one logit of 2e6 in
// each row 1.2 ms.)
constexpr float kLpLarge = 1e6f;
constexpr float kLpHuge = 1e38f;     // above its negative, x L - c is finite

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// IEEE 754-2019 maximum: NaN if either is.
__device__ __forceinline__ float max_nan(float a, float b) { return __builtin_elementwise_maximum(a, b); }
__device__ __forceinline__ float min_nan(float a, float b) { return __builtin_elementwise_minimum(a, b); }
__device__ __forceinline__ float exp2_fast(float t) { return __builtin_amdgcn_exp2f(t); }

template <int DT> struct LpElem;
template <> struct LpElem<PROFK_F32> {
  static constexpr int ES = 4, EPV = 4;
  static constexpr uint32_t kNegInfWord = 0xFF800000u;
  static __device__ __forceinline__ float get(const u32x4& v, int e) { return __uint_as_float(v[e]); }
  static __device__ __forceinline__ float load(const char* row, uint32_t i) {
    return reinterpret_cast<const float*>(row)[i];
  }
};
template <> struct LpElem<PROFK_BF16> {
  static constexpr int ES = 2, EPV = 8;
  static constexpr uint32_t kNegInfWord = 0xFF80FF80u;
  static __device__ __forceinline__ float get(const u32x4& v, int e) {
    return __uint_as_float(e & 1 ? v[e / 2] & 0xFFFF0000u : v[e / 2] << 16);
  }
  static __device__ __forceinline__ float load(const char* row, uint32_t i) {
    return __uint_as_float(static_cast<uint32_t>(reinterpret_cast<const uint16_t*>(row)[i]) << 16);
  }
};

// A candidate as one integer that orders as (value descending, index
// ascending) does; 0 is none.  Values at or below -inf are never candidates.
constexpr uint32_t kKeyNegInf = 0x007FFFFFu;
constexpr uint64_t kCandMin = static_cast<uint64_t>(kKeyNegInf + 1) << 32;
__device__ __forceinline__ uint64_t cand(float x, uint32_t i) {
  return static_cast<uint64_t>(key_f32(__float_as_uint(x))) << 32 | (0xFFFFFFFFu - i);
}
__device__ __forceinline__ uint32_t cand_index(uint64_t c) { return 0xFFFFFFFFu - static_cast<uint32_t>(c); }
__device__ __forceinline__ float cand_value(uint64_t c) {
  return __uint_as_float(bits_from_key_f32(static_cast<uint32_t>(c >> 32)));
}

// Wave-wide reductions with a uniform result: DPP exchanges inside each
// 16-lane row (quad swaps, half-row and row mirrors), then the four rows'.
template <int CTRL> __device__ __forceinline__ float dpp_f(float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xF, 0xF, false));
}
__device__ __forceinline__ float lane_f(float x, int lane) {
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), lane));
}
__device__ __forceinline__ float wave_max_f(float x) {
  x = fmaxf(x, dpp_f<0xB1>(x));
  x = fmaxf(x, dpp_f<0x4E>(x));
  x = fmaxf(x, dpp_f<0x141>(x));
  x = fmaxf(x, dpp_f<0x140>(x));
  return fmaxf(fmaxf(lane_f(x, 0), lane_f(x, 16)), fmaxf(lane_f(x, 32), lane_f(x, 48)));
}
__device__ __forceinline__ float wave_sum_f(float x) {
  x += dpp_f<0xB1>(x);
  x += dpp_f<0x4E>(x);
  x += dpp_f<0x141>(x);
  x += dpp_f<0x140>(x);
  return (lane_f(x, 0) + lane_f(x, 16)) + (lane_f(x, 32) + lane_f(x, 48));
}
__device__ __forceinline__ uint64_t wave_max_u64(uint64_t x) {
#pragma unroll
  for (int o = kWave / 2; o > 0; o >>= 1) {
    const uint64_t y = __shfl_xor(static_cast<unsigned long long>(x), o, kWave);
    x = y > x ? y : x;
  }
  return x;
}

// Running statistics of a set of logits; odd: some passed kLpLarge.
struct Stats {
  float c, s, q;
  uint32_t odd;
};
// s and q of c's reference to another one (d = c - c', at most about 0).
__device__ __forceinline__ void shift(float& s, float& q, float d) {
  d = fmaxf(d, kLpFloor);
  const float f = exp2_fast(d);
  q = f * fmaf(d, s, q);
  s *= f;
}

template <int BS> struct LpReduce {
  float c[BS / kWave], s[BS / kWave], q[BS / kWave];
  uint32_t odd[BS / kWave];
};

// The block's statistics, in every thread; a wave's lanes have one c.
template <int BS> __device__ __forceinline__ Stats block_stats(const Stats& a, LpReduce<BS>& r) {
  constexpr int NW = BS / kWave;
  const uint32_t lane = threadIdx.x & (kWave - 1), w = threadIdx.x / kWave;
  Stats t{a.c, wave_sum_f(a.s), wave_sum_f(a.q), __ballot(a.odd != 0) != 0 ? 1u : 0u};
  if (NW == 1) return t;
  if (lane == 0) {
    r.c[w] = t.c;
    r.s[w] = t.s;
    r.q[w] = t.q;
    r.odd[w] = t.odd;
  }
  __syncthreads();
  t.c = r.c[0];
#pragma unroll
  for (int i = 1; i < NW; ++i) t.c = fmaxf(t.c, r.c[i]);
  t.s = t.q = 0.0f;
  t.odd = 0;
#pragma unroll
  for (int i = 0; i < NW; ++i) {
    float s = r.s[i], q = r.q[i];
    shift(s, q, r.c[i] - t.c);
    t.s += s;
    t.q += q;
    t.odd |= r.odd[i];
  }
  __syncthreads();
  return t;
}

// Where c is near the largest x L, the sum is at least 2^-0.5.
__device__ __forceinline__ bool needs_care(const Stats& t) { return t.odd || !(t.s >= 0.5f); }

// What a row's outputs need, in 64 bits: lse = m + ls (log p = (x - m) - ls:
// beside an m of the lowest value the sum would lose ls) and H.
struct RowStats {
  double m, ls;
  float h;
  __device__ __forceinline__ float logp(float x) const {
    return m == -__builtin_inf() ? kNegInf : static_cast<float>((static_cast<double>(x) - m) - ls);
  }
};
// log2 of a positive s: the exponent exactly, and the logarithm of a
// significand in [0.75, 1.5), which is off by 2^-24 or so.
__device__ __forceinline__ double log2_of(float s) {
  int e;
  float f = frexpf(s, &e);
  if (f < 0.75f) {
    f *= 2.0f;
    --e;
  }
  return static_cast<double>(e) + static_cast<double>(__builtin_amdgcn_logf(f));
}
// (the roundings of q and s may leave a row of one logit just below 0)
__device__ __forceinline__ float entropy_of(double l2, float q, float s) {
  const float h = static_cast<float>(kLn2 * (l2 - static_cast<double>(q / s)));
  return h < 0.0f ? 0.0f : h;
}
__device__ __forceinline__ RowStats row_stats(const Stats& t) {
  constexpr double kInv = 1.0 / static_cast<double>(kL2E);
  const double l2 = log2_of(t.s);
  return {static_cast<double>(t.c) * kInv, l2 * kInv, entropy_of(l2, t.q, t.s)};
}

// The careful path: two sweeps of the row, x - m formed before the scale.
template <int DT, int BS>
__device__ __forceinline__ RowStats careful_stats(const char* row, uint32_t V, LpReduce<BS>& r) {
  constexpr int NW = BS / kWave;
  using E = LpElem<DT>;
  const uint32_t lane = threadIdx.x & (kWave - 1), w = threadIdx.x / kWave;
  float m = kNegInf;
  uint32_t bad = 0;   // NaN or +inf
  for (uint32_t i = threadIdx.x; i < V; i += BS) {
    const float x = E::load(row, i);
    bad |= !(x < __builtin_inff());
    m = fmaxf(m, x);
  }
  m = wave_max_f(m);
  const uint32_t wbad = __ballot(bad != 0) != 0;
  if (lane == 0) {
    r.c[w] = m;
    r.odd[w] = wbad;
  }
  __syncthreads();
  bad = 0;
#pragma unroll
  for (int i = 0; i < NW; ++i) {
    m = fmaxf(m, r.c[i]);
    bad |= r.odd[i];
  }
  __syncthreads();
  if (bad) return {__builtin_nan(""), __builtin_nan(""), __builtin_nanf("")};
  if (m == kNegInf) return {-__builtin_inf(), 0.0, 0.0f};   // nothing is allowed
  float s = 0.0f, q = 0.0f;
  for (uint32_t i = threadIdx.x; i < V; i += BS) {
    const float t = fmaxf((E::load(row, i) - m) * kL2E, kLpFloor);
    const float e = exp2_fast(t);
    s += e;
    q = fmaf(e, t, q);
  }
  s = wave_sum_f(s);
  q = wave_sum_f(q);
  if (lane == 0) {
    r.s[w] = s;
    r.q[w] = q;
  }
  __syncthreads();
  s = q = 0.0f;
#pragma unroll
  for (int i = 0; i < NW; ++i) {
    s += r.s[i];
    q += r.q[i];
  }
  __syncthreads();
  const double l2 = log2_of(s);
  return {static_cast<double>(m), kLn2 * l2, entropy_of(l2, q, s)};
}

// The n best of elements [0, V) of a row, by n sweeps, into list (sorted,
// 0 past the last).
template <int DT, int BS>
__device__ __forceinline__ void sweep_top(const char* row, uint32_t V, uint32_t base, uint32_t n, uint64_t* list,
                                       uint64_t* red) {
  constexpr int NW = BS / kWave;
  const uint32_t lane = threadIdx.x & (kWave - 1), w = threadIdx.x / kWave;
  uint64_t last = ~0ull;
  for (uint32_t k = 0; k < n; ++k) {
    uint64_t best = 0;
    for (uint32_t i = threadIdx.x; i < V; i += BS) {
      const uint64_t c = cand(LpElem<DT>::load(row, i), base + i);
      if (c < last && c >= kCandMin && c > best) best = c;
    }
    best = wave_max_u64(best);
    if (lane == 0) red[w] = best;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NW; ++i) best = red[i] > best ? red[i] : best;
    __syncthreads();
    if (threadIdx.x == 0) list[k] = best;
    last = best;   // (0: no element is left, and none is found again)
  }
  __syncthreads();
}

// The list's best n, sorted, in its first entries; returns how many there
// are.  cnt <= CAP entries, all different; the list has room for four more.
template <int BS, int CAP>
__device__ __forceinline__ uint32_t cut_list(uint64_t* list, uint32_t cnt, uint32_t n) {
  constexpr int P = CAP / BS;
  if (threadIdx.x < 4) list[cnt + threadIdx.x] = 0;   // (read with the last ones, above none)
  __syncthreads();
  auto rank_of = [&](auto turns) {
    constexpr int Q = decltype(turns)::value;
    uint64_t mine[Q];
    uint32_t rank[Q];
#pragma unroll
    for (int p = 0; p < Q; ++p) {
      const uint32_t i = p * BS + threadIdx.x;
      mine[p] = i < cnt ? list[i] : 0ull;
      rank[p] = 0;
    }
    // (a wave without an entry has nothing to rank)
    const uint32_t end = __ballot(mine[0] != 0) ? cnt : 0u;
    for (uint32_t j = 0; j < end; j += 4) {
      uint64_t o[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) o[k] = list[j + k];
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int p = 0; p < Q; ++p) rank[p] += o[k] > mine[p];
    }
    __syncthreads();
#pragma unroll
    for (int p = 0; p < Q; ++p)
      if (mine[p] && rank[p] < n) list[rank[p]] = mine[p];
  };
  if (cnt <= static_cast<uint32_t>(BS)) rank_of(std::integral_constant<int, 1>{});
  else rank_of(std::integral_constant<int, P>{});
  __syncthreads();
  return cnt < n ? cnt : n;
}

__device__ __forceinline__ uint32_t wave_min_u32(uint32_t x) { return ~wave_max_u32(~x); }

// The r-th largest x of the wave's lanes with `in` (0 if they are fewer); left:
// how many are at least as large.  Found from its highest bit, a ballot a bit,
// until a prefix is reached by r lanes alone, of which it is the least.
// (Ranking 64 lanes by comparing all with all goes through LDS 64 times.)
__device__ __forceinline__ uint32_t wave_kth(uint32_t x, bool in, uint32_t r, uint32_t& left) {
  uint32_t p = 0;
  left = static_cast<uint32_t>(__popcll(__ballot(in)));
  if (left < r) return 0;
  for (uint32_t bit = 0x80000000u; bit != 0 && left != r; bit >>= 1) {
    const uint32_t n = static_cast<uint32_t>(__popcll(__ballot(in && x >= (p | bit))));
    if (n >= r) {
      p |= bit;
      left = n;
    }
  }
  return left == r ? wave_min_u32(in && x >= p ? x : 0xFFFFFFFFu) : p;
}

// A lower bound of the n-th best of the candidates that the block's lanes have
// the best ones of (0: none): of each wave the n / NW-th best, and the least
// of those.
template <int BS> __device__ __forceinline__ uint64_t bound_of(uint64_t best, uint32_t n, uint64_t* red) {
  constexpr int NW = BS / kWave;
  const uint32_t r = (n + NW - 1) / NW;
  const uint32_t key = static_cast<uint32_t>(best >> 32), low = static_cast<uint32_t>(best);
  uint32_t left;
  const uint32_t k = wave_kth(key, best != 0, r, left);
  uint64_t bound = static_cast<uint64_t>(k) << 32;
  // those that have the r-th key itself: by index
  if (k) bound |= wave_kth(low, key == k, r - static_cast<uint32_t>(__popcll(__ballot(key > k))), left);
  if (bound < kCandMin) bound = kCandMin;
  if (NW == 1) return bound;
  if ((threadIdx.x & (kWave - 1)) == 0) red[threadIdx.x / kWave] = bound;
  __syncthreads();
  bound = red[0];
#pragma unroll
  for (int i = 1; i < NW; ++i) bound = red[i] < bound ? red[i] : bound;
  return bound;
}

// Outputs of a row, by the whole block; list holds its n best, sorted.
__device__ __forceinline__ void write_row(const LpArgs& a, uint32_t r, const RowStats& t, const uint64_t* list,
                                          uint32_t found, float xy, int64_t y) {
  if (threadIdx.x == 0) {
    const float lse = static_cast<float>(t.m + t.ls);
    a.lse[r] = lse;
    // (from m first: beside an m of the lowest value the sum has lost ls)
    if (a.lse_low) {
      const bool finite = fabsf(lse) < __builtin_inff();
      a.lse_low[r] = finite ? static_cast<float>((t.m - static_cast<double>(lse)) + t.ls) : 0.0f;
    }
    a.entropy[r] = t.h;
    float lp = 0.0f;                                              // no token
    if (y >= static_cast<int64_t>(a.V)) lp = __builtin_nanf("");  // not a token
    else if (y >= 0) lp = t.logp(xy);
    a.logprob[r] = lp;
  }
  for (uint32_t i = threadIdx.x; i < a.n; i += blockDim.x) {
    const uint64_t c = i < found ? list[i] : 0ull;
    const size_t o = static_cast<size_t>(r) * a.n + i;
    a.top[o] = c ? t.logp(cand_value(c)) : kNegInf;
    a.top_idx[o] = c ? static_cast<int64_t>(cand_index(c)) : -1;
  }
}

template <int DT> __device__ __forceinline__ float token_logit(const char* row, uint32_t V, int64_t y) {
  return y >= 0 && y < static_cast<int64_t>(V) ? LpElem<DT>::load(row, static_cast<uint32_t>(y)) : 0.0f;
}

// One workgroup of BS threads, U 16-byte vectors per lane and step, per row
// or per chunk of a row (SPLIT: its statistics and its n best go to the
// workspace, for k_lp_join).
template <int DT, int BS, int U, bool TOP, bool SPLIT>
__global__ __launch_bounds__(BS) void k_lp(LpArgs a) {
  using E = LpElem<DT>;
  constexpr int ES = E::ES, EPV = E::EPV, NW = BS / kWave;
  constexpr int CAP = TOP ? (BS == kWave ? 512 : 1024) : BS;
  __shared__ __align__(16) uint64_t s_list[CAP + 4];
  __shared__ uint64_t s_red[NW];
  __shared__ uint32_t s_cnt;
  __shared__ LpReduce<BS> s_stats;
  const uint32_t tid = threadIdx.x, lane = tid & (kWave - 1);
  const uint32_t w = __builtin_amdgcn_readfirstlane(tid / kWave);
  const uint32_t r = a.row + (SPLIT ? blockIdx.x / a.G : blockIdx.x);
  const uint32_t g = SPLIT ? blockIdx.x % a.G : 0u;
  const char* const row = static_cast<const char*>(a.x) + static_cast<size_t>(r) * a.stride * ES;
  const uint32_t base = g * a.chunk;                                 // first element of this block
  const uint32_t D = SPLIT ? min(a.chunk, a.V - base) : a.V;
  const char* const x = row + static_cast<size_t>(base) * ES;

  uint32_t head = static_cast<uint32_t>(((16 - (reinterpret_cast<uintptr_t>(x) & 15)) & 15) / ES);
  if (head > D) head = D;
  const uint32_t nvec = (D - head) / EPV;
  const u32x4* const vec = reinterpret_cast<const u32x4*>(x + static_cast<size_t>(head) * ES);
  const uint32_t pieces = (nvec + kWave - 1) / kWave;                // of 64 vectors
  const uint32_t steps = (pieces + NW * U - 1) / (NW * U);
  // Piece u of step `step` of this wave starts at vector `first`; a lane reads
  // vector `at` + lane: a piece that ends past the last vector is read as the
  // row's last 64, and blanked where it is not those (a row of fewer vectors:
  // past the last).  All of it is scalar, and the lane's offset is the same
  // for every load.
  auto first_of = [&](uint32_t step, int u) { return ((u * NW + w) * steps + step) * kWave; };
  const uint32_t last_at = nvec > static_cast<uint32_t>(kWave) ? nvec - kWave : 0u;
  const uint32_t lane_off = min(lane, nvec - 1);
  auto at_of = [&](uint32_t step, int u) { return min(first_of(step, u), last_at); };
  using Vecs = u32x4[U];
  auto load = [&](uint32_t step, Vecs& v) {
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = __builtin_nontemporal_load(vec + at_of(step, u) + lane_off);
  };
  auto blank = [&](uint32_t step, Vecs& v) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t first = first_of(step, u), i = at_of(step, u) + lane;
      if (__builtin_expect(first + kWave > nvec, 0)) {
        if (i < first || i >= nvec) v[u] = u32x4{E::kNegInfWord, E::kNegInfWord, E::kNegInfWord, E::kNegInfWord};
      }
    }
  };
  auto vec_max = [](const u32x4& v) {
    float m = E::get(v, 0);
#pragma unroll
    for (int e = 1; e < EPV; ++e) m = max_nan(m, E::get(v, e));
    return m;
  };
  Vecs v0, v1;     // a step, and the next one, loaded meanwhile
  if (steps) load(0, v0);
  const int64_t y = SPLIT ? -1 : a.tokens[r];
  const float xy = SPLIT ? 0.0f : token_logit<DT>(row, a.V, y);
  // elements before the first and after the last whole vector, one a lane
  const uint32_t tail0 = head + nvec * EPV, ns = head + (D - tail0);
  const uint32_t own_i = tid < head ? tid : tail0 + (tid - head);
  const float own = tid < ns ? E::load(x, own_i) : kNegInf;

  Stats st{-kLpLarge * kL2E, 0.0f, 0.0f, 0u};   // c: the wave's
  float lim = -kLpLarge;                        // the largest logit that c has been set for
  // some lane's m passed lim, or is NaN; the whole wave calls it
  auto rebase = [&](float m) {
    if (__ballot(!(m <= kLpLarge))) {
      st.odd = 1;
      return;
    }
    m = wave_max_f(m);
    const float c = lane_f(rintf(fmaxf(m, -kLpLarge) * kL2E), 0);
    shift(st.s, st.q, st.c - c);
    st.c = c;
    lim = lane_f(m, 0);
  };
  // z's term; FLOOR: z may be -inf, or as low as makes t -inf
  auto term = [&](float z, auto floor) {
    float t = fmaf(z, kL2E, -st.c);
    if (decltype(floor)::value) t = fmaxf(t, kLpFloor);
    const float e = exp2_fast(t);
    st.s += e;
    st.q = fmaf(e, t, st.q);
  };
  uint64_t bound = kCandMin;                    // candidates are at or above it
  float boundf = cand_value(kCandMin);
  bool over = false;
  auto offer = [&](float z, uint32_t i) {
    if (!(z < boundf)) {
      const uint64_t c = cand(z, i);
      if (c >= bound) {
        const uint32_t slot = atomicAdd(&s_cnt, 1u);
        if (slot < static_cast<uint32_t>(CAP)) s_list[slot] = c;
      }
    }
  };

  if (TOP && tid == 0) s_cnt = 0;
  {
    // the first step's maxima: c, and the bound
    float bm = own;
    uint64_t best = 0;
    if (steps) {
      blank(0, v0);
      float vm[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        vm[u] = vec_max(v0[u]);
        bm = max_nan(bm, vm[u]);
      }
      if (TOP) {
        // a lane's maximum at an index no smaller than its own (the last of its
        // vector); a maximum of 0 may be either zero, so it counts as -0
        float top = vm[0];
        uint32_t at = at_of(0, 0);
#pragma unroll
        for (int u = 1; u < U; ++u)
          if (vm[u] > top) {
            top = vm[u];
            at = at_of(0, u);
          }
        if (top > kNegInf) best = cand(top == 0.0f ? -0.0f : top, base + head + (at + lane) * EPV + EPV - 1);
      }
    }
    if (__ballot(!(bm <= lim))) rebase(bm);
    if (TOP && steps) {
      bound = bound_of<BS>(best, a.n, s_red);
      boundf = cand_value(bound);
    }
    if (TOP && (NW == 1 || !steps)) __syncthreads();   // (s_cnt)
  }
  auto take = [&](uint32_t step, Vecs& v, Vecs& next) {
    if (BS > kWave && step + 1 < steps) load(step + 1, next);
    if (BS > kWave && step) blank(step, v);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      // one compare for both: a larger logit than c is set for, or a candidate
      const float m = vec_max(v[u]);
      if (__ballot(!(m < (TOP ? fminf(lim, boundf) : lim)))) {
        if (__ballot(!(m <= lim))) rebase(m);
        if (TOP && !over && !(m < boundf)) {
#pragma unroll
          for (int e = 0; e < EPV; ++e)
            offer(E::get(v[u], e), base + head + (at_of(step, u) + lane) * EPV + e);
        }
      }
      // 16-bit rows are bound by the instructions of a term, of which the floor
      // is one: half a one for the least logit decides whether it is needed
      bool low = true;
      if (DT == PROFK_BF16) {
        float mn = E::get(v[u], 0);
#pragma unroll
        for (int e = 1; e < EPV; ++e) mn = min_nan(mn, E::get(v[u], e));
        low = __ballot(!(mn > -kLpHuge)) != 0;
      }
      if (low) {
#pragma unroll
        for (int e = 0; e < EPV; ++e) term(E::get(v[u], e), std::true_type{});
      } else {
#pragma unroll
        for (int e = 0; e < EPV; ++e) term(E::get(v[u], e), std::false_type{});
      }
    }
    // the list is cut after 2, 4, 8... steps
    if (BS > kWave && TOP && step > 0 && (step & (step + 1)) == 0 && step + 1 < steps) {
      __syncthreads();
      const uint32_t cnt = s_cnt;
      over = cnt > static_cast<uint32_t>(CAP);
      if (!over && cnt > a.n) {
        cut_list<BS, CAP>(s_list, cnt, a.n);
        bound = s_list[a.n - 1];
        boundf = cand_value(bound);
        if (tid == 0) s_cnt = a.n;
      }
      __syncthreads();
    }
  };
  if constexpr (BS == kWave) {
    if (steps) take(0, v0, v0);      // (a wave's rows and chunks are one step)
  } else {
    for (uint32_t step = 0; step < steps; step += 2) {
      take(step, v0, v1);
      if (step + 1 < steps) take(step + 1, v1, v0);
    }
  }
  if (tid < ns) {
    term(own, std::true_type{});
    if (TOP && !over) offer(own, base + own_i);
  }
  uint32_t found = 0;
  if (TOP) {
    __syncthreads();
    const uint32_t cnt = s_cnt;
    if (cnt > static_cast<uint32_t>(CAP)) {
      sweep_top<DT, BS>(x, D, base, a.n, s_list, s_red);
      found = a.n;
    } else {
      found = cut_list<BS, CAP>(s_list, cnt, a.n);
    }
  }
  const Stats t = block_stats<BS>(st, s_stats);
  if (SPLIT) {
    const size_t o = static_cast<size_t>(blockIdx.x);
    if (tid == 0) {
      float* const p = a.part + o * kLpPart;
      p[0] = t.c;
      p[1] = t.s;
      p[2] = t.q;
      p[3] = t.odd ? 1.0f : 0.0f;
    }
    if (TOP)
      for (uint32_t i = tid; i < a.n; i += BS) a.part_top[o * a.n + i] = i < found ? s_list[i] : 0ull;
    return;
  }
  RowStats rs;
  if (needs_care(t)) rs = careful_stats<DT, BS>(row, a.V, s_stats);
  else rs = row_stats(t);
  write_row(a, r, rs, s_list, found, xy, y);
}

// Joins a row's G chunks, of whose candidates the best n are selected as k_lp
// selects them from a step's.
template <int DT, bool TOP> __global__ __launch_bounds__(kLpJoinBS) void k_lp_join(LpArgs a) {
  constexpr int BS = kLpJoinBS, CAP = TOP ? 1024 : BS, U = 8;
  __shared__ __align__(16) uint64_t s_list[CAP + 4];
  __shared__ uint64_t s_red[BS / kWave];
  __shared__ uint32_t s_cnt;
  __shared__ LpReduce<BS> s_stats;
  const uint32_t tid = threadIdx.x, r = a.row + blockIdx.x;
  const char* const row = static_cast<const char*>(a.x) + static_cast<size_t>(r) * a.stride * LpElem<DT>::ES;
  const size_t first = static_cast<size_t>(blockIdx.x) * a.G;
  Stats st{-kLpLarge * kL2E, 0.0f, 0.0f, 0u};
  static_assert(kLpMaxChunks <= BS, "one chunk a thread");
  if (tid < a.G) {
    const f32x4 p = *reinterpret_cast<const f32x4*>(a.part + (first + tid) * kLpPart);
    st = Stats{p[0], p[1], p[2], p[3] != 0.0f ? 1u : 0u};
  }
  const uint64_t* const top = a.part_top + first * a.n;
  const uint32_t total = TOP ? a.G * a.n : 0u;
  // the first BS * U candidates stay in registers, the others are read twice
  uint64_t mine[U];
  uint64_t best = 0;
  if (TOP) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t i = u * BS + tid;
      mine[u] = i < total ? top[i] : 0ull;
    }
  }
  const int64_t y = a.tokens[r];
  const float xy = token_logit<DT>(row, a.V, y);
  uint32_t found = 0;
  if (TOP) {
#pragma unroll
    for (int u = 0; u < U; ++u) best = mine[u] > best ? mine[u] : best;
    for (uint32_t i = U * BS + tid; i < total; i += BS) best = top[i] > best ? top[i] : best;
    if (tid == 0) s_cnt = 0;
    const uint64_t bound = bound_of<BS>(best, a.n, s_red);
    auto offer = [&](uint64_t c) {
      if (c < bound) return;
      const uint32_t slot = atomicAdd(&s_cnt, 1u);
      if (slot < static_cast<uint32_t>(CAP)) s_list[slot] = c;
    };
#pragma unroll
    for (int u = 0; u < U; ++u) offer(mine[u]);
    for (uint32_t i = U * BS + tid; i < total; i += BS) offer(top[i]);
    __syncthreads();
    const uint32_t cnt = s_cnt;
    if (cnt > static_cast<uint32_t>(CAP)) {
      sweep_top<DT, BS>(row, a.V, 0, a.n, s_list, s_red);
      found = a.n;
    } else {
      found = cut_list<BS, CAP>(s_list, cnt, a.n);
    }
  }
  // the lanes of a wave to one c
  const float c = wave_max_f(st.c);
  shift(st.s, st.q, st.c - c);
  st.c = c;
  const Stats t = block_stats<BS>(st, s_stats);
  RowStats rs;
  if (needs_care(t)) rs = careful_stats<DT, BS>(row, a.V, s_stats);
  else rs = row_stats(t);
  write_row(a, r, rs, s_list, found, xy, y);
}

// ------------------------------------------------------------ gradient ----
// With p = exp(x - lse), G = g + sum_i t_i - l (g only where y is a token; l of
// lse itself, whose gradient is p):
//   dx_j = -p_j (G + h (log p_j + H))  +  g [j = y] + sum_i t_i [j = a_i].
// One workgroup per piece of a row: the first term for all of it, then the
// few elements that take the second are written again, behind a barrier.
// Bound by memory: 4096 x 131072 bf16 361 us (5.9 TB/s read and written; a copy
// of 1 GiB 5.2), 509 x 50001 fp32 with 16 alternatives 36 us (5.6).
constexpr int kGradBS = 256;
constexpr int kGradU = 4;

typedef uint32_t u32x4u __attribute__((ext_vector_type(4), aligned(2)));   // at any element's address

// An lse rounded to fp32 alone leaves all of a row's p off by half a unit in its
// last place, 2^-24 of |lse| at most; with what the rounding left (lse_low) they
// are as exact as x - lse is.  Without it, from this size on lse is too coarse
// (2^-10 of p off, and useless beside a row of the lowest value), and the row's
// statistics are taken from its logits again, by each of its workgroups.
constexpr float kCoarseLse = 16384.0f;

struct GradRow {
  float m, ls;       // log p = (x - m) - ls
  float a, b;        // dx = p (a + b log p): a = -(G + h H), b = -h
  bool empty;        // no logit is allowed: the gradient is 0
};
__device__ __forceinline__ float grad_at(const GradRow& g, float x) {
  const float l = fmaxf((x - g.m) - g.ls, -200.0f);   // 2^(-200 L) is 0 in fp32
  return exp2_fast(l * kL2E) * fmaf(g.b, l, g.a);
}

template <int DT> __global__ __launch_bounds__(kGradBS) void k_lp_grad(LpGradArgs a) {
  using E = LpElem<DT>;
  constexpr int ES = E::ES, EPV = E::EPV, BS = kGradBS;
  constexpr uint32_t kPiece = BS * kGradU * EPV;
  __shared__ LpReduce<BS> s_stats;
  const uint32_t tid = threadIdx.x;
  const uint32_t rl = blockIdx.x / a.pieces, piece = blockIdx.x - rl * a.pieces;
  const size_t r = static_cast<size_t>(a.row) + rl;
  const char* const x = static_cast<const char*>(a.x) + r * a.stride * ES;
  char* const out = static_cast<char*>(a.out) + r * a.out_stride * ES;
  // pieces are whole vectors of the output; the first takes the elements
  // before its first aligned one, the last those after its last
  uint32_t head = static_cast<uint32_t>(((16 - (reinterpret_cast<uintptr_t>(out) & 15)) & 15) / ES);
  if (head > a.V) head = a.V;
  const uint32_t lo = piece == 0 ? 0u : head + piece * kPiece;
  const uint32_t body = head + piece * kPiece;
  const uint32_t hi = piece + 1 == a.pieces || a.V - body < kPiece ? a.V : body + kPiece;
  if (lo >= a.V) return;
  // the piece's logits first: what follows waits for loads of its own
  const uint32_t nvec = hi > body ? (hi - body) / EPV : 0u;
  u32x4 v[kGradU];
#pragma unroll
  for (int u = 0; u < kGradU; ++u) {
    const uint32_t i = u * BS + tid;
    v[u] = u32x4{};
    if (i < nvec) v[u] = *reinterpret_cast<const u32x4u*>(x + (static_cast<size_t>(body) + i * EPV) * ES);
  }

  GradRow g;
  g.m = a.lse[r];
  g.ls = a.lse_low ? a.lse_low[r] : 0.0f;
  const float h = a.g_entropy ? a.g_entropy[r] : 0.0f;
  const int64_t y = a.tokens ? a.tokens[r] : -1;
  float gy = a.g_logprob && y >= 0 ? a.g_logprob[r] : 0.0f;
  if (y >= static_cast<int64_t>(a.V)) gy = __builtin_nanf("");
  float G = a.g_lse ? gy - a.g_lse[r] : gy;
  const float* const gt = a.n ? a.g_top + r * a.n : nullptr;
  const int64_t* const at = a.n ? a.top_idx + r * a.n : nullptr;
  for (uint32_t i = 0; i < a.n; ++i)
    if (at[i] >= 0 && at[i] < static_cast<int64_t>(a.V)) G += gt[i];
  g.empty = g.m == kNegInf;
  if (!a.lse_low && fabsf(g.m) >= kCoarseLse && fabsf(g.m) < __builtin_inff()) {
    const RowStats t = careful_stats<DT, BS>(x, a.V, s_stats);
    g.m = static_cast<float>(t.m);
    g.ls = static_cast<float>(t.ls);
  }
  g.a = -G;
  g.b = -h;
  if (a.g_entropy) g.a = -fmaf(h, a.entropy[r], G);
  if (!(g.m == g.m)) g.a = __builtin_nanf("");
  if (g.empty) {
    g.m = g.ls = 0.0f;
    g.a = g.b = 0.0f;
  }
  // the elements of this piece that take a gradient of their own
  float fix = 0.0f;
  int64_t j = -1;
  if (tid <= a.n && !g.empty) {
    j = tid < a.n ? at[tid] : y;
    if (j < static_cast<int64_t>(lo) || j >= static_cast<int64_t>(hi)) j = -1;
    if (j >= 0) {
      float own = y == j ? gy : 0.0f;
      for (uint32_t i = 0; i < a.n; ++i)
        if (at[i] == j) own += gt[i];
      fix = own + grad_at(g, E::load(x, static_cast<uint32_t>(j)));
    }
  }

#pragma unroll
  for (int u = 0; u < kGradU; ++u) {
    const uint32_t i = u * BS + tid;
    if (i >= nvec) continue;
    float d[EPV];
#pragma unroll
    for (int e = 0; e < EPV; ++e) d[e] = grad_at(g, E::get(v[u], e));
    u32x4 o;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (DT == PROFK_F32) {
        o[e] = __float_as_uint(d[e]);
      } else {
        o[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{d[2 * e], d[2 * e + 1]}), bf16x2));
      }
    }
    __builtin_nontemporal_store(o, reinterpret_cast<u32x4*>(out + (static_cast<size_t>(body) + i * EPV) * ES));
  }
  auto put = [&](uint32_t i, float d) {
    if constexpr (DT == PROFK_F32) reinterpret_cast<float*>(out)[i] = d;
    else reinterpret_cast<__bf16*>(out)[i] = static_cast<__bf16>(d);
  };
  const uint32_t tail = body + nvec * EPV;
  const uint32_t nh = min(body, hi) - lo, nt = hi > tail ? hi - tail : 0u;
  if (tid < nh + nt) {
    const uint32_t i = tid < nh ? lo + tid : tail + (tid - nh);
    put(i, grad_at(g, E::load(x, i)));
  }
  if (a.n || a.tokens) {
    __syncthreads();   // (completes the stores above before those below)
    if (j >= 0) put(static_cast<uint32_t>(j), fix);
  }
}

template <int DT, int BS, int U>
void launch_lp(const LpArgs& a, uint32_t rows, hipStream_t s) {
  if (a.G > 1) {
    if (a.n) k_lp<DT, BS, U, true, true><<<rows * a.G, BS, 0, s>>>(a);
    else k_lp<DT, BS, U, false, true><<<rows * a.G, BS, 0, s>>>(a);
  } else {
    if (a.n) k_lp<DT, BS, U, true, false><<<rows, BS, 0, s>>>(a);
    else k_lp<DT, BS, U, false, false><<<rows, BS, 0, s>>>(a);
  }
}

template <int DT> void launch_lp_dt(const LpArgs& a, uint32_t rows, hipStream_t s) {
  // Rows that a wave holds (two vectors a lane, or eight) take one wave: no
  // barriers; longer ones 256 threads and a step of 16 KB in turn, the next one
  // loaded meanwhile.  (16384 x 512 fp32 with eight vectors a lane 29 us, with
  // two 17; 4096 x 131072 bf16 with steps of 32 KB, none loaded ahead, 206 us,
  // with these 194.)
  const uint64_t bytes = static_cast<uint64_t>(a.G > 1 ? a.chunk : a.V) * LpElem<DT>::ES;
  if (bytes <= 2 * kWave * 16) launch_lp<DT, kWave, 2>(a, rows, s);
  else if (bytes <= static_cast<uint64_t>(kLpWaveBytes)) launch_lp<DT, kWave, 8>(a, rows, s);
  else launch_lp<DT, 256, 4>(a, rows, s);
  if (a.G > 1) {
    if (a.n) k_lp_join<DT, true><<<rows, kLpJoinBS, 0, s>>>(a);
    else k_lp_join<DT, false><<<rows, kLpJoinBS, 0, s>>>(a);
  }
}

}  // namespace

LpLayout lp_layout(int64_t T, int64_t V, int64_t n, int num_cus) {
  LpLayout L;
  // Rows too few for four workgroups a CU are split over that many (64 x
  // 100003 fp32 19 us, over eight a CU 21; 1000 x 131072 bf16 73 and 77), in
  // chunks of no less than a wave's step (1 x 131072: 13.4 us, also with half).
  const int64_t want = 4 * static_cast<int64_t>(num_cus);
  int64_t G = T < want ? (want + T - 1) / T : 1;
  const int64_t most = (V + kLpMinChunk - 1) / kLpMinChunk;
  if (G > most) G = most;
  if (G > kLpMaxChunks) G = kLpMaxChunks;
  int64_t chunk = (V + G - 1) / G;
  chunk = (chunk + 63) / 64 * 64;      // (whole 16-byte vectors: chunks are aligned alike)
  L.chunk = static_cast<uint32_t>(chunk);
  L.G = static_cast<uint32_t>((V + chunk - 1) / chunk);
  if (L.G > 1) {
    L.off_top = (static_cast<size_t>(T) * L.G * kLpPart * sizeof(float) + 255) / 256 * 256;
    L.bytes = L.off_top + static_cast<size_t>(T) * L.G * static_cast<size_t>(n) * sizeof(uint64_t);
  }
  return L;
}

hipError_t launch_logprobs(LpCall c) {
  const LpLayout& L = c.L;
  LpArgs a = c.a;
  a.G = L.G;
  a.chunk = L.chunk;
  a.part = reinterpret_cast<float*>(c.ws);
  a.part_top = reinterpret_cast<uint64_t*>(c.ws + L.off_top);
  const int64_t step = rows_per_launch(256) / L.G;
  (void)hipGetLastError();
  for (int64_t r = 0; r < c.T; r += step) {
    const uint32_t rows = static_cast<uint32_t>(c.T - r < step ? c.T - r : step);
    a.row = static_cast<uint32_t>(r);
    if (c.dtype == PROFK_F32) launch_lp_dt<PROFK_F32>(a, rows, c.stream);
    else launch_lp_dt<PROFK_BF16>(a, rows, c.stream);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_logprobs_grad(LpGradArgs a, int dtype, int64_t T, hipStream_t s) {
  const uint32_t piece = kGradBS * kGradU * (dtype == PROFK_F32 ? 4 : 8);
  // (a row's unaligned head is its first piece's)
  a.pieces = static_cast<uint32_t>((static_cast<uint64_t>(a.V) + piece - 1) / piece);
  const int64_t step = rows_per_launch(kGradBS) / a.pieces;
  (void)hipGetLastError();
  for (int64_t r = 0; r < T; r += step) {
    const uint32_t rows = static_cast<uint32_t>(T - r < step ? T - r : step);
    a.row = static_cast<uint32_t>(r);
    if (dtype == PROFK_F32) k_lp_grad<PROFK_F32><<<rows * a.pieces, kGradBS, 0, s>>>(a);
    else k_lp_grad<PROFK_BF16><<<rows * a.pieces, kGradBS, 0, s>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace profk
