// The tiled product on the matrix cores (kernels_product.hip,
// kernels_product_grad.hip).
//
// A workgroup of WM x WN waves computes tiles of BM x BN outputs, a wave MI x NJ
// accumulators of 32 x 32 with the 32x32x16 instruction.  A stage is 64 of k of
// both operands, loaded straight to LDS in granules of 16 bytes; there are two,
// and one is filled, on into the workgroup's next tile, while the other is
// multiplied.  Fragments are read a quarter of a stage (16 of k, one instruction
// for each accumulator) ahead, under the matrix instructions of the one before.
//
// An operand along k is 128 bytes a row in a stage, whole lines; granule g of row
// r is at position g ^ (r / 2 % 8) of its eight, so that a fragment's read of
// sixteen rows covers all 64 banks once.  One across k is BM (or BN) neighbours
// for each of the 64 k; a fragment is two transposing reads, in which sixteen
// lanes take 4 k of 16 neighbours.  Granule g of row k is at position g ^ (4 (k %
// 4)): the four rows of a read then cover all banks once.
//
// Rows past I or J are read as the last and not stored; granules past K are read
// from zeros, of both operands (a product of what lies there may be NaN).
//
// Output column n of a wave's slab is in fragment n % NJ, lane n / NJ, where B is
// along k (its rows are in LDS in that order), so that a lane's NJ results of a
// row are neighbours; where it is across, in fragment n / 32, lane n % 32.
//
// 256 x 256 tiles on eight waves of 64 x 128: a stage moves 64 KB for 32 matrix
// instructions a wave, of 32 cycles, two waves a SIMD.  Measured: 8192^3 to bf16
// 774 us (1.42 PFLOP/s; the library's 669-700), 4096 x 4096 x 12288 296-330 us (1.25
// to 1.39, by clock; the library's 272-325), with silu and a residual 326-341.  At 8192^3 the matrix cores are busy for 84 % of
// the cycles (the library's for 88), at a clock that falls to 1.5 GHz under both;
// this kernel reads LDS half as much again as a wave of 128 x 128 would.  What it
// took: the last two fragments of a stage read ahead, which frees its LDS half way
// and gives loads a stage and a quarter (846 -> 772 us at 8192^3); panels of
// tiles (4096 x 2048 of K = 12288, B across, 250 -> 192 us).  Not kept: four waves
// of 128 x 128 (821 us: one wave a SIMD hides no wait), a load a wave that brings
// the lines of the stage after the next into L2 (883 us: the loads' own rate).
#pragma once

#include <type_traits>

#include "launch.h"
#include "product.h"

namespace profk {

namespace {

typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
typedef float f32x2u __attribute__((ext_vector_type(2), aligned(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2u __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t __attribute__((aligned(2))) u32u;
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr uint32_t kProdXcds = 8;
constexpr uint32_t kStageK = 64;
constexpr uint32_t kPanel = 8;      // column tiles of a panel

__device__ const uint4 g_zero_granule = {0, 0, 0, 0};

// A workgroup barrier that waits for nothing else, across which the compiler
// moves no memory access.
__device__ __forceinline__ void prod_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

template <int WM, int WN, int MI, int NJ> struct ProdTile {
  static constexpr int NW = WM * WN, BS = NW * kWave, BM = WM * MI * 32, BN = WN * NJ * 32;
  static constexpr int QA = BM * 8 / BS, QB = BN * 8 / BS;   // loads of a lane
  static constexpr int kB = BM * 8, kGran = (BM + BN) * 8;   // first granule of b; granules of a stage
  static_assert(BM * 8 % BS == 0 && BN * 8 % BS == 0 && (NJ == 2 || NJ == 4), "whole loads, neighbouring results of a lane");
};

// One operand's part of a stage: what a lane loads, and where it reads.  BW
// neighbours (BM or BN), Q loads a lane, F fragments a wave, PERM: its rows are in
// LDS in the order of the outputs.
template <bool ACROSS, int BW, int Q, int F, bool PERM, bool WHOLE> struct ProdSide {
  static_assert(!(ACROSS && PERM), "granules of neighbours stay together");
  const uint8_t* base;
  uint32_t off[Q], w, lane;
  uint32_t K, adv;                  // k of a stage's row, and bytes from stage to stage
  uint64_t row_bytes;
  uint32_t rd0;
  __device__ __forceinline__ static uint32_t order(uint32_t r) {
    return PERM ? r / (F * 32) * (F * 32) + r % 32 * F + r % (F * 32) / 32 : r;
  }
  // wave, its first fragment's rows and its lane
  __device__ __forceinline__ void init(uint32_t wave, uint32_t l, uint32_t first, uint64_t stride, uint32_t k) {
    w = wave;
    lane = l;
    K = k;
    row_bytes = stride * 2;
    adv = ACROSS ? static_cast<uint32_t>(row_bytes) * kStageK : kStageK * 2;
    if constexpr (ACROSS) {
      const uint32_t t = lane & 15, b = lane >> 4 & 1, h = lane >> 5;
      rd0 = (8 * h + t / 4) * (BW * 2) + ((first / 32 ^ t / 4) * 4 + b * 2 + t % 4 / 2) * 16 + t % 2 * 8;
    } else {
      const uint32_t c = lane & 31, h = lane >> 5;
      rd0 = (first + c) * 128 + (h ^ (c >> 1 & 7)) * 16;
    }
  }
  // granule of load q: its k (across) or its first k (along)
  __device__ __forceinline__ uint32_t k_of(int q) const {
    const uint32_t p = (w * Q + q) * kWave + lane;
    if constexpr (ACROSS) return p / (BW / 8);
    else return ((p & 7) ^ (p >> 4 & 7)) * 8;
  }
  __device__ __forceinline__ void start(const __bf16* p, uint32_t r0, uint32_t R) {
    if constexpr (ACROSS) {
      base = reinterpret_cast<const uint8_t*>(p + r0);
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        const uint32_t at = (w * Q + q) * kWave + lane, k = at / (BW / 8), g = at % (BW / 8) ^ (k & 3) * 4;
        off[q] = k * static_cast<uint32_t>(row_bytes) + min(g, (R - r0 + 7) / 8 - 1) * 16;
      }
    } else {
      base = reinterpret_cast<const uint8_t*>(p) + r0 * row_bytes;
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        const uint32_t r = order((w * Q + q) * 8 + lane / 8);
        off[q] = min(r, R - 1 - r0) * static_cast<uint32_t>(row_bytes) + k_of(q) * 2;
      }
    }
  }
  // on to a tile's first k, with `left` from there
  __device__ __forceinline__ void skip(uint32_t k, uint32_t left) {
    base += k * (ACROSS ? row_bytes : uint64_t{2});
    K = left;
  }
  // stage `next` of the tile to LDS, of the operand `plane` bytes behind this one
  __device__ __forceinline__ void issue(uint4* st, uint32_t next, int64_t plane = 0) const {
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const uint8_t* p = base + plane + off[q];
      if constexpr (!WHOLE) p = next * kStageK + k_of(q) < K ? p : reinterpret_cast<const uint8_t*>(&g_zero_granule);
      __builtin_amdgcn_global_load_lds(reinterpret_cast<const uint32_t*>(p), st + (w * Q + q) * kWave, 16, 0, 0);
    }
  }
  // fragments of quarter q of a stage
  __device__ __forceinline__ void read(const uint4* st, uint32_t q, u32x4 (&f)[F]) {
    // (taken anew, or the compiler keeps an address for each read)
    asm volatile("" : "+v"(rd0));
    if constexpr (ACROSS) {
      typedef __attribute__((address_space(3))) s16x4* lds4;
      typedef const __attribute__((address_space(3))) uint8_t* lds8;
      const lds8 p = (lds8)reinterpret_cast<const uint8_t*>(st);
#pragma unroll
      for (int u = 0; u < F; ++u) {
        const uint32_t at = (rd0 ^ (u * 64)) + q * (16 * BW * 2);
        const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(p + at)));
        const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(p + at + 4 * BW * 2)));
        f[u] = u32x4{lo[0], lo[1], hi[0], hi[1]};
      }
    } else {
      const uint8_t* const p = reinterpret_cast<const uint8_t*>(st);
#pragma unroll
      for (int u = 0; u < F; ++u) f[u] = *reinterpret_cast<const u32x4*>(p + (rd0 ^ (q * 32)) + u * 4096);
    }
  }
};

// WHOLE: K is a multiple of two stages (TWO: of one).  SPLIT: K is taken in g.parts
// parts of g.part_k, a whole number of two stages (the last may hold less), each a
// tile of its own whose sums go to g.out [parts, I, J].  TWO: a is the sum of g.a and
// g.a_low; the 64 of k of a stage come by twice, first of g.a, then of g.a_low.
template <bool TA, bool TB, int ACT, int DT, int WM, int WN, int MI, int NJ, bool WHOLE, bool SPLIT, bool TWO>
__device__ __forceinline__ void prod_body(const ProdArgs& g, uint32_t tiles_i, uint32_t tiles, uint32_t block,
                                          uint32_t blocks, uint4* s0, uint4* s1) {
  static_assert(!SPLIT || (!WHOLE && ACT == PROFK_ACT_NONE && DT == PROFK_F32), "sums of parts");
  using T = ProdTile<WM, WN, MI, NJ>;
  // workgroup b runs on XCD b % 8: each XCD takes a run of tiles, and goes through
  // panels of kPanel column tiles row by row, so that what it works on at a time
  // is near a square, which shares most in its L2
  const uint32_t xcd = block % kProdXcds, per_xcd = blocks / kProdXcds;   // (a multiple of 8)
  const uint32_t end = static_cast<uint32_t>(static_cast<uint64_t>(tiles) * (xcd + 1) / kProdXcds);
  const uint32_t tile0 = static_cast<uint32_t>(static_cast<uint64_t>(tiles) * xcd / kProdXcds) + block / kProdXcds;
  if (tile0 >= end) return;
  // a tile takes an even number of stages, so that each starts at the same one
  const uint32_t tile_k = SPLIT ? g.part_k : g.K, of_part = SPLIT ? tiles / g.parts : tiles;
  const uint32_t stages =
      TWO ? (tile_k + kStageK - 1) / kStageK * 2 : (tile_k + 2 * kStageK - 1) / (2 * kStageK) * 2;
  const int64_t low = TWO ? reinterpret_cast<const uint8_t*>(g.a_low) - reinterpret_cast<const uint8_t*>(g.a) : 0;
  const uint32_t tid = threadIdx.x, lane = tid & (kWave - 1);
  const uint32_t w = __builtin_amdgcn_readfirstlane(tid / kWave);
  const uint32_t c = lane & 31, h = lane >> 5, wm = w / WN, wn = w % WN;

  ProdSide<TA, T::BM, T::QA, MI, false, WHOLE> sa;
  ProdSide<TB, T::BN, T::QB, NJ, !TB, WHOLE> sb;
  sa.init(w, lane, wm * MI * 32, g.as, g.K);
  sb.init(w, lane, wn * NJ * 32, g.bs, g.K);
  const uint32_t tiles_j = (g.J + T::BN - 1) / T::BN;
  auto place = [&](uint32_t tile, uint32_t& i, uint32_t& j) {
    if (SPLIT) tile %= of_part;
    const uint32_t p = tile / (kPanel * tiles_i), rest = tile - p * (kPanel * tiles_i);
    const uint32_t width = min(kPanel, tiles_j - p * kPanel);
    i = rest / width * T::BM;
    j = (p * kPanel + rest % width) * T::BN;
  };
  auto start = [&](uint32_t tile) {
    uint32_t i, j;
    place(tile, i, j);
    sa.start(g.a, i, g.I);
    sb.start(g.b, j, g.J);
    if constexpr (SPLIT) {
      const uint32_t k = tile / of_part * g.part_k;
      sa.skip(k, g.K - k);
      sb.skip(k, g.K - k);
    }
  };
  uint32_t next_k = 0, next_tile = tile0;
  // (past the last tile: its last stage again)
  auto of_k = [](uint32_t stage) { return TWO ? stage / 2 : stage; };
  auto issue_a = [&](uint4* st) { sa.issue(st, of_k(next_k), next_k % 2 ? low : 0); };
  auto issue_b = [&](uint4* st) {
    sb.issue(st + T::kB, of_k(next_k));
    ++next_k;
    if (TWO && next_k % 2) return;
    if (next_k < stages && (WHOLE || of_k(next_k) * kStageK < sa.K)) {
      sa.base += sa.adv;
      sb.base += sb.adv;
    }
  };
  // after a tile's last stage
  auto turn = [&]() {
    if (next_k == stages) {
      if (next_tile + per_xcd < end) {
        next_k = 0;
        next_tile += per_xcd;
        start(next_tile);
      } else {
        next_k = stages - 1;
      }
    }
  };
  struct Frag {
    u32x4 a[MI], b[NJ];
  };
  auto rd = [&](const uint4* st, uint32_t q, Frag& f) {
    sa.read(st, q, f.a);
    sb.read(st + T::kB, q, f.b);
  };
  f32x16 acc[MI][NJ];
  auto mma = [&](const Frag& f) {
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NJ; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, f.a[i]),
                                                            __builtin_bit_cast(bf16x8, f.b[j]), acc[i][j], 0, 0, 0);
  };
  // The accumulators exist here: a quarter's instructions, which touch no
  // memory, would else be moved past the barriers to where they are stored.
  auto pin = [&]() {
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NJ; ++j) asm volatile("" : "+v"(acc[i][j]));
  };
  // LDS reads and loads between the matrix instructions of a quarter: the first
  // one waits for the reads before, and loads issued one after the other keep
  // the wave from its matrix instructions while they are taken
  constexpr int kReads = MI * (TA ? 2 : 1) + NJ * (TB ? 2 : 1);
  auto weave = [&](auto reads) {
    constexpr int M = MI * NJ, per = (decltype(reads)::value + M - 2) / (M - 1);
    pin();
#pragma unroll
    for (int i = 0; i < M; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, per, 0);
      __builtin_amdgcn_sched_group_barrier(0x010, 1, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  auto clear = [&]() {
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NJ; ++j) acc[i][j] = f32x16{};
  };
  using O = std::conditional_t<DT == PROFK_F32, float, __bf16>;
  auto store = [&](uint32_t tile) {
    uint32_t ti, tj;
    place(tile, ti, tj);
    const uint32_t mw = ti + wm * MI * 32, nw = tj + wn * NJ * 32;
    const uint32_t m = mw + 4 * h, n = nw + (TB ? c : NJ * c);
    O* const out = static_cast<O*>(g.out) + (SPLIT ? static_cast<size_t>(tile / of_part) * g.I * g.J : 0);
    // f(row, v) for the rows of eight of a lane's results of fragment i, from v0 on
    auto rows = [&](auto check, int i, int v0, auto f) {
      uint32_t first = m + i * 32;
      // (no row's address or mask is kept through the steps)
      asm volatile("" : "+v"(first));
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int v = v0; v < v0 + 8; ++v) {
        const uint32_t r = first + 8 * (v / 4) + v % 4;
        if (!decltype(check)::value || r < g.I) f(r, v);
      }
    };
    auto both = [&](auto f) {
      if (mw + MI * 32 <= g.I && nw + NJ * 32 <= g.J) f(std::false_type{});
      else f(std::true_type{});
    };
    if constexpr (TB) {
      // (no epilogue: a gradient) neighbouring lanes hold neighbouring columns
      both([&](auto check) {
#pragma unroll
        for (int q = 0; q < 2 * MI; ++q) {
          const int i = q / 2;
          rows(check, i, q % 2 * 8, [&](uint32_t r, int v) {
            O* const p = out + static_cast<size_t>(r) * g.J + n;
#pragma unroll
            for (int j = 0; j < NJ; ++j)
              if (!decltype(check)::value || n + j * 32 < g.J) p[j * 32] = static_cast<O>(acc[i][j][v]);
          });
        }
      });
    } else {
      float bias[NJ];
#pragma unroll
      for (uint32_t j = 0; j < NJ; ++j) bias[j] = !SPLIT && g.bias && n + j < g.J ? g.bias[n + j] : 0.0f;
      both([&](auto check) {
        constexpr bool kCheck = decltype(check)::value;
        if (kCheck && n >= g.J) return;
        const bool whole = !kCheck || n + NJ <= g.J;
        auto put_all = [&](O* p, const float (&y)[NJ]) {
          if (whole) {
            if constexpr (DT == PROFK_F32) {
              if constexpr (NJ == 4) *reinterpret_cast<f32x4u*>(p) = f32x4u{y[0], y[1], y[2], y[3]};
              else *reinterpret_cast<f32x2u*>(p) = f32x2u{y[0], y[1]};
            } else if constexpr (NJ == 4) {
              *reinterpret_cast<u32x2u*>(p) = u32x2u{pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3])};
            } else {
              *reinterpret_cast<u32u*>(p) = pack_bf16(y[0], y[1]);
            }
          } else {
#pragma unroll
            for (uint32_t j = 0; j < NJ - 1; ++j)
              if (n + j < g.J) p[j] = static_cast<O>(y[j]);
          }
        };
#pragma unroll
        for (int h2 = 0; h2 < 2 * MI; ++h2) {
          const int i = h2 / 2, v0 = h2 % 2 * 8;
          // (eight rows' loads go out before the first is used)
          float add[8][NJ];
          if (!SPLIT && g.residual) {
            rows(check, i, v0, [&](uint32_t r, int v) {
              const O* const q = static_cast<const O*>(g.residual) + r * g.residual_stride + n;
              if (whole) {
#pragma unroll
                for (int j = 0; j < NJ; j += 2) {
                  if constexpr (DT == PROFK_F32) {
                    const f32x2u u = *reinterpret_cast<const f32x2u*>(q + j);
                    add[v - v0][j] = u[0];
                    add[v - v0][j + 1] = u[1];
                  } else {
                    const uint32_t u = *reinterpret_cast<const u32u*>(q + j);
                    add[v - v0][j] = __uint_as_float(u << 16);
                    add[v - v0][j + 1] = __uint_as_float(u & 0xFFFF0000u);
                  }
                }
              } else {
#pragma unroll
                for (uint32_t j = 0; j < NJ - 1; ++j) add[v - v0][j] = n + j < g.J ? static_cast<float>(q[j]) : 0.0f;
                add[v - v0][NJ - 1] = 0.0f;
              }
            });
          }
          rows(check, i, v0, [&](uint32_t r, int v) {
            const size_t at = static_cast<size_t>(r) * g.J + n;
            float z[NJ];
#pragma unroll
            for (int j = 0; j < NJ; ++j) z[j] = acc[i][j][v] + bias[j];
            if (!SPLIT && g.pre) put_all(static_cast<O*>(g.pre) + at, z);
#pragma unroll
            for (int j = 0; j < NJ; ++j) z[j] = act_of<ACT>(z[j]);
            if (!SPLIT && g.residual) {
#pragma unroll
              for (int j = 0; j < NJ; ++j) z[j] += add[v - v0][j];
            }
            put_all(out + at, z);
          });
        }
      });
    }
  };
  using R0 = std::integral_constant<int, 0>;
  using R1 = std::integral_constant<int, kReads>;
  using R2 = std::integral_constant<int, 2 * kReads>;
  start(tile0);
  issue_a(s0);
  issue_b(s0);
  issue_a(s1);
  issue_b(s1);
  Frag f0, f1, f2;
  prod_wait<T::QA + T::QB>();
  prod_barrier();
  rd(s0, 0, f0);
  // One stage; its first quarter's fragments are in fa.  Its last two are read
  // under the second, so that all waves are done with its part of LDS half way, and
  // the loads of the stage after the next have a stage and a quarter to arrive.
  auto stage = [&](uint4* cur, uint4* nxt, Frag& fa, Frag& fb, auto last) {
    __builtin_amdgcn_sched_barrier(0);
    rd(cur, 1, fb);
    mma(fa);
    weave(R1{});
    rd(cur, 2, fa);
    rd(cur, 3, f2);
    mma(fb);
    weave(R2{});
    if (decltype(last)::value) turn();
    prod_wait<63>();
    prod_barrier();
    issue_a(cur);
    mma(fa);
    weave(R0{});
    // the next stage has arrived
    prod_wait<T::QA>();
    prod_barrier();
    issue_b(cur);
    rd(nxt, 0, fb);
    mma(f2);
    weave(R1{});
  };
  for (uint32_t tile = tile0; tile < end; tile += per_xcd) {
    clear();
    for (uint32_t k = 0; k < stages; k += 2) {
      stage(s0, s1, f0, f1, std::true_type{});
      stage(s1, s0, f1, f0, std::false_type{});
    }
    store(tile);
  }
  prod_wait<0>();   // (no load may reach LDS after the workgroup's end)
}

template <bool TA, bool TB, int ACT, int DT, int WM, int WN, int MI, int NJ, int WAVES, bool WHOLE, bool SPLIT, bool TWO>
__global__ __launch_bounds__(WM * WN * 64, WAVES) void k_prod(ProdArgs g, uint32_t tiles_i, uint32_t tiles) {
  using T = ProdTile<WM, WN, MI, NJ>;
  // distinct arrays, so that the compiler can tell the stage being read from the
  // one being filled
  __shared__ __align__(16) uint4 s0[T::kGran], s1[T::kGran];
  prod_body<TA, TB, ACT, DT, WM, WN, MI, NJ, WHOLE, SPLIT, TWO>(g, tiles_i, tiles, blockIdx.x, gridDim.x, s0, s1);
}

// Workgroups of a launch over `tiles`.
inline uint32_t prod_grid(uint32_t tiles, uint32_t most) {
  const uint32_t grid = (tiles + kProdXcds - 1) / kProdXcds * kProdXcds;
  return grid > most ? most / kProdXcds * kProdXcds : grid;
}

// PER: workgroups a CU holds.
template <bool TA, bool TB, int ACT, int DT, int WM, int WN, int MI, int NJ, int PER, bool SPLIT, bool TWO>
void launch_tiles(const ProdArgs& g, uint32_t cus, hipStream_t s) {
  using T = ProdTile<WM, WN, MI, NJ>;
  const uint32_t ti = (g.I + T::BM - 1) / T::BM, tj = (g.J + T::BN - 1) / T::BN, tiles = ti * tj * (SPLIT ? g.parts : 1);
  const uint32_t grid = prod_grid(tiles, PER * cus);
  constexpr int kWaves = PER * WM * WN / 4;
  if constexpr (SPLIT) {
    k_prod<TA, TB, ACT, DT, WM, WN, MI, NJ, kWaves, false, true, TWO><<<grid, T::BS, 0, s>>>(g, ti, tiles);
  } else if (g.K % ((TWO ? 1 : 2) * kStageK) == 0) {
    k_prod<TA, TB, ACT, DT, WM, WN, MI, NJ, kWaves, true, false, TWO><<<grid, T::BS, 0, s>>>(g, ti, tiles);
  } else {
    k_prod<TA, TB, ACT, DT, WM, WN, MI, NJ, kWaves, false, false, TWO><<<grid, T::BS, 0, s>>>(g, ti, tiles);
  }
}

template <bool TA, bool TB, int ACT, int DT, bool SPLIT, bool TWO>
void launch_shape(const ProdArgs& g, const ProdPlan& p, uint32_t cus, hipStream_t s) {
  if (p.large) launch_tiles<TA, TB, ACT, DT, 4, 2, 2, 4, 1, SPLIT, TWO>(g, cus, s);
  else launch_tiles<TA, TB, ACT, DT, 2, 2, 2, 2, 2, SPLIT, TWO>(g, cus, s);
}

// Tiles are counted in 32 bits.
inline bool tiles_fit(const ProdArgs& g) {
  return static_cast<uint64_t>((g.I + 127) / 128) * ((g.J + 127) / 128) < (uint64_t{1} << 31);
}

// The sums of K's parts, in their order, with the epilogue: 8 neighbours a
// thread.
template <int DT, int ACT> __global__ __launch_bounds__(256) void k_prod_join(ProdArgs g, const float* sums) {
  const uint32_t per = (g.J + 7) / 8;
  const uint64_t n = static_cast<uint64_t>(g.I) * per, size = static_cast<uint64_t>(g.I) * g.J;
  for (uint64_t t = blockIdx.x * uint64_t{256} + threadIdx.x; t < n; t += gridDim.x * uint64_t{256}) {
    const uint32_t i = static_cast<uint32_t>(t / per), j = static_cast<uint32_t>(t % per) * 8;
    const uint64_t at = static_cast<uint64_t>(i) * g.J;
    float z[8], v[8];
    load<PROFK_F32, 8>(sums + at, j, g.J, z);
    for (uint32_t p = 1; p < g.parts; ++p) {
      load<PROFK_F32, 8>(sums + p * size + at, j, g.J, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) z[e] += v[e];
    }
    if (g.bias) {
      load<PROFK_F32, 8>(g.bias, j, g.J, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) z[e] += v[e];
    }
    using O = std::conditional_t<DT == PROFK_F32, float, __bf16>;
    if (g.pre) store<DT, 8>(static_cast<O*>(g.pre) + at, j, g.J, z);
#pragma unroll
    for (int e = 0; e < 8; ++e) z[e] = act_of<ACT>(z[e]);
    if (g.residual) {
      load<DT, 8>(static_cast<const O*>(g.residual) + i * g.residual_stride, j, g.J, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) z[e] += v[e];
    }
    store<DT, 8>(static_cast<O*>(g.out) + at, j, g.J, z);
  }
}

template <bool TA, bool TB, int ACT, int DT, bool TWO>
void launch_planned(ProdArgs g, const ProdPlan& p, float* sums, uint32_t cus, hipStream_t s) {
  if (p.parts == 1) {
    launch_shape<TA, TB, ACT, DT, false, TWO>(g, p, cus, s);
    return;
  }
  g.parts = p.parts;
  g.part_k = p.part_k;
  ProdArgs part = g;
  part.out = sums;
  launch_shape<TA, TB, PROFK_ACT_NONE, PROFK_F32, true, TWO>(part, p, cus, s);
  const uint64_t blocks = (static_cast<uint64_t>(g.I) * ((g.J + 7) / 8) + 255) / 256;
  k_prod_join<DT, ACT><<<blocks < 8192 ? static_cast<uint32_t>(blocks) : 8192, 256, 0, s>>>(g, sums);
}

}  // namespace

}  // namespace profk
