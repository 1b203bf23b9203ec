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
// [R, Kp / 2] bytes, the even value of a pair in the low half: a row's codes
// start at a multiple of 64 bytes, and a lane of the 32x32x64 matrix
// instruction takes 32 values of a row (16 bytes) and their scale.  Scales
// [R / 32, Kp / 128, 32, 4] bytes, R padded to whole groups of 32 rows: the
// four scales of a row's step are a word, and a group's step is one line of 128
// bytes.  (With a row's scales one after the other, a step's loads of a 256 x
// 256 tile touched 512 lines for 2 KB, as many as its 32 KB of codes did, and
// a product of 4096 x 4096 x 65536 took 805 us.)
#include <type_traits>

#include "device_common.h"
#include "launch.h"
#include "mx4.h"

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
// Bound by memory: 131072 x 2048 fp32 to codes 248 us (4.9 TB/s read and
// written), codes to bf16 121 us (5.6 TB/s); a copy of 1 GiB reaches 5.2.
//
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

// A workgroup takes 32 rows and kMxPairs steps: whole lines of scales.
constexpr uint32_t kMxPairs = 2;

struct MxQuantArgs {
  const void* x;
  uint64_t stride;
  uint32_t rows, K, steps;
  uint8_t *codes, *scales;
};

// Word of a row's four scales of step k, in words from the first.
__device__ __forceinline__ size_t mx_scale_word(uint32_t r, uint32_t k, uint32_t steps) {
  return (static_cast<size_t>(r >> 5) * steps + k) * 32 + (r & 31);
}

template <int DT> __global__ __launch_bounds__(kMxBS) void k_mx_quantize(MxQuantArgs a) {
  constexpr int P = 32 * 16 / kMxBS;                 // turns to 32 rows of a step, 16 lanes a row
  const uint32_t parts = (a.steps + kMxPairs - 1) / kMxPairs;
  const uint32_t group = blockIdx.x / parts, k0 = (blockIdx.x - group * parts) * kMxPairs;
  const uint32_t c = threadIdx.x & 15;
  float v[kMxPairs][P][8];
#pragma unroll
  for (uint32_t u = 0; u < kMxPairs; ++u)
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const uint32_t r = group * 32 + p * (kMxBS / 16) + threadIdx.x / 16, k = (k0 + u) * 128 + 8 * c;
      // (past the rows or the row's values: zeros)
      const bool in = r < a.rows;
      mx_load8<DT>(static_cast<const char*>(a.x) + (in ? r : 0) * a.stride * (DT == PROFK_F32 ? 4 : 2), k,
                   in ? a.K : 0, v[u][p]);
    }
#pragma unroll
  for (uint32_t u = 0; u < kMxPairs; ++u) {
    const uint32_t k = k0 + u;
    if (k >= a.steps) break;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const uint32_t r = group * 32 + p * (kMxBS / 16) + threadIdx.x / 16;
      uint32_t byte;
      const uint32_t code = mx_quant8(v[u][p], byte);
      if (r < a.rows)
        *reinterpret_cast<uint32_t*>(a.codes + (static_cast<size_t>(r) * a.steps + k) * 64 + 4 * c) = code;
      // the row's four bytes, from lanes 0, 4, 8 and 12 of its sixteen
      uint32_t word = byte;
      word |= static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(byte), 0x104, 0xF, 0xF, false)) << 8;
      word |= static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(byte), 0x108, 0xF, 0xF, false)) << 16;
      word |= static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(byte), 0x10C, 0xF, 0xF, false)) << 24;
      if (c == 0) reinterpret_cast<uint32_t*>(a.scales)[mx_scale_word(r, k, a.steps)] = word;
    }
  }
}

struct MxDequantArgs {
  const uint32_t* codes;
  const uint8_t* scales;
  uint32_t rows, K, lanes;   // lanes of a row (Kp / 8)
  void* out;
};

template <int DT> __global__ __launch_bounds__(kMxBS) void k_mx_dequantize(MxDequantArgs a) {
  const uint32_t t = blockIdx.x * kMxBS + threadIdx.x;
  const uint32_t r = t / a.lanes, c = t - r * a.lanes, k = 8 * c;
  if (r >= a.rows || k >= a.K) return;
  const uint32_t code = a.codes[t], byte = a.scales[4 * mx_scale_word(r, c / 16, a.lanes / 16) + c % 16 / 4];
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
  const uint8_t *as, *bs;     // scales [M / 32, steps, 32, 4], [N / 32, steps, 32, 4]
  uint32_t M, N, steps;       // steps of 128 values
  void* out;                  // [M, N]
  const void* x;              // few rows: a before it is quantised (a, as unused)
  uint64_t x_stride;
  uint32_t K;
};

// s_waitcnt vmcnt(N) lgkmcnt(0) (gfx9 encoding: vmcnt in bits 3:0 and 15:14,
// expcnt in 6:4, lgkmcnt in 11:8): all but this wave's N newest loads are
// done, and so are its LDS reads.
template <int N> __device__ __forceinline__ void wait_loads_lds() {
  static_assert(N >= 0 && N < 64, "vmcnt");
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((N & 0xF) | ((N >> 4) << 14) | (0x7 << 4));
}
// A workgroup barrier that waits for nothing else, across which the compiler
// moves no memory access.
__device__ __forceinline__ void bare_barrier() {
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// The tiled product.  A workgroup of WM x WN waves computes tiles of BM x BN
// outputs, a wave MI x NJ accumulators of 32 x 32.  A stage, two steps (256
// values of K), is 128 bytes of codes a row, whole lines, and two words of
// four scales, loaded straight to LDS; there are two, and one is filled, on
// into the workgroup's next tile, while the other is multiplied.  Fragments
// are read half a step ahead, under the matrix instructions of the half
// before.  16-byte granule g of a row r is at position g ^ (r / 2 % 8) of its
// eight: sixteen neighbouring rows' granules g then cover all 64 banks once.
//
// Output column n of a wave's slab is in fragment n % NJ, lane n / NJ (the
// codes of b are in LDS in that order), so that a lane's NJ results of a row are
// neighbours and are stored together.
//
// Rows past M or N are read as the last one and not stored.
//
// 256 x 256 tiles on eight waves of 64 x 128: a stage moves 68 KB for 32 matrix
// instructions a wave, of 32 cycles, two waves a SIMD.  Measured: 4096 x 4096 x
// 65536 to bf16 566 us (3.9 PFLOP/s), 4096 x 2048 x 131072 636 to 665 us (3.5 to
// 3.3, as the clock falls), 4096 x 512 x 12288 to fp32 41 us (4.9 TB/s of output,
// near a copy's rate).  The same instructions on random codes in registers alone
// reach 6.3 PFLOP/s, at about 1.6 GHz (8.8 on zeros); the library's bf16 product
// of 8192^3 1.2.  Of short K it is bound by the stores.  Of long K by no unit
// alone: at 4096 x 4096 x 65536 the matrix cores are busy for 54 % of the cycles,
// and waves wait for 40 % of theirs, at each stage's barrier and for its loads;
// a tile's first stage waits for the stores of the tile before as well, which
// are counted with the loads (the same operations with twice the outputs, 4096 x
// 2048 x 131072, take about 90 us more).
// Four waves of 128 x 128 read a third less from LDS and were slower (631 us at
// 4096 x 4096 x 65536: one wave a SIMD hides no wait).
template <int WM, int WN, int MI, int NJ> struct MxTile {
  static constexpr int NW = WM * WN, BS = NW * kWave, BM = WM * MI * 32, BN = WN * NJ * 32;
  static constexpr int QA = BM * 8 / BS, QB = BN * 8 / BS;     // loads of a lane: codes
  static constexpr int QS = (BM + BN) / 32 / NW;               // ... scales, 32 rows and two steps each
  static constexpr int kB = BM * 8, kS = (BM + BN) * 8;        // first granule of b, of the scales
  static constexpr int kGran = kS + (BM + BN) / 2;             // granules of a stage
  static_assert(BM * 8 % BS == 0 && BN * 8 % BS == 0 && (BM + BN) / 32 % NW == 0, "whole loads");
  static_assert(NJ == 4, "four neighbouring results a lane");
};

// WHOLE: the steps are a multiple of four, so that no part of a stage is
// skipped and the reads and the matrix instructions of a half step are one run
// of code.
template <int DT, int WM, int WN, int MI, int NJ, bool WHOLE>
__device__ __forceinline__ void mx_gemm_body(const MxGemmArgs& g, uint32_t tiles_m, uint32_t tiles) {
  using T = MxTile<WM, WN, MI, NJ>;
  // distinct arrays, so that the compiler can tell the stage being read from
  // the one being filled
  __shared__ __align__(16) uint4 s0[T::kGran], s1[T::kGran];
  // workgroup b runs on XCD b % 8: each XCD takes a run of tiles, the row
  // tiles of a column tile one after the other, so that its L2 holds what
  // they share
  const uint32_t xcd = blockIdx.x % kXcds, per_xcd = gridDim.x / kXcds;   // (the grid is a multiple of 8)
  const uint32_t end = static_cast<uint32_t>(static_cast<uint64_t>(tiles) * (xcd + 1) / kXcds);
  const uint32_t tile0 = static_cast<uint32_t>(static_cast<uint64_t>(tiles) * xcd / kXcds) + blockIdx.x / kXcds;
  if (tile0 >= end) return;
  // a tile takes an even number of stages, so that each starts at the same
  // one; what is past its last step is not multiplied
  const uint32_t stages = WHOLE ? g.steps / 2 : (g.steps + 3) / 4 * 2;
  const uint32_t tid = threadIdx.x, lane = tid & (kWave - 1);
  const uint32_t w = __builtin_amdgcn_readfirstlane(tid / kWave);
  const uint32_t c = lane & 31, h = lane >> 5, wm = w / WN, wn = w % WN;
  const uint32_t cb = g.steps * 64;

  auto col_of = [](uint32_t r) { return r / (NJ * 32) * (NJ * 32) + r % 32 * NJ + r % (NJ * 32) / 32; };
  // The stage to load next: a lane's offsets from the first row of its tile
  // (within 256 rows of at most 2^19 bytes), to which a stage adds.
  auto gran = [&](uint32_t q) { return (lane & 7) ^ ((q * 8 + lane / 8) >> 1 & 7); };   // granule of load q
  const uint8_t *base_a, *base_b, *base_s[T::QS];
  uint32_t oa[T::QA], ob[T::QB], os[T::QS];
  auto start = [&](uint32_t tile) {
    const uint32_t m0 = tile % tiles_m * T::BM, n0 = tile / tiles_m * T::BN;
    const uint32_t last_m = g.M - 1 - m0, last_n = g.N - 1 - n0;
    base_a = g.a + static_cast<size_t>(m0) * cb;
    base_b = g.b + static_cast<size_t>(n0) * cb;
#pragma unroll
    for (int q = 0; q < T::QA; ++q) {
      oa[q] = min((w * T::QA + q) * 8 + lane / 8, last_m) * cb + gran(w * T::QA + q) * 16;
    }
#pragma unroll
    for (int q = 0; q < T::QB; ++q) {
      ob[q] = min(col_of((w * T::QB + q) * 8 + lane / 8), last_n) * cb + gran(w * T::QB + q) * 16;
    }
    // (groups past the last one read the last one)
#pragma unroll
    for (int q = 0; q < T::QS; ++q) {
      const uint32_t gr = w * T::QS + q;
      const bool of_a = gr < T::BM / 32;
      const uint32_t first = of_a ? m0 / 32 + min(gr, last_m / 32) : n0 / 32 + min(gr - T::BM / 32, last_n / 32);
      base_s[q] = (of_a ? g.as : g.bs) + static_cast<size_t>(first) * g.steps * 128;
      os[q] = lane * 4;
    }
  };
  uint32_t next_k = 0, next_tile = tile0;
  // (past a tile's last step, and the last tile: the last again)
  auto issue_a = [&](uint4* st) {
    // the last of an odd number of steps: its granules and scales twice
    const bool half = !WHOLE && 2 * next_k + 1 >= g.steps;
#pragma unroll
    for (int q = 0; q < T::QA; ++q)
      __builtin_amdgcn_global_load_lds(
          reinterpret_cast<const uint32_t*>(base_a + oa[q] - (half ? (gran(w * T::QA + q) & 4) * 16 : 0u)),
          st + (w * T::QA + q) * kWave, 16, 0, 0);
  };
  auto issue_b = [&](uint4* st) {
    const bool half = !WHOLE && 2 * next_k + 1 >= g.steps;
#pragma unroll
    for (int q = 0; q < T::QB; ++q)
      __builtin_amdgcn_global_load_lds(
          reinterpret_cast<const uint32_t*>(base_b + ob[q] - (half ? (gran(w * T::QB + q) & 4) * 16 : 0u)),
          st + T::kB + (w * T::QB + q) * kWave, 16, 0, 0);
  };
  auto issue_s = [&](uint4* st) {
    const bool half = !WHOLE && 2 * next_k + 1 >= g.steps;
#pragma unroll
    for (int q = 0; q < T::QS; ++q)
      __builtin_amdgcn_global_load_lds(reinterpret_cast<const uint32_t*>(base_s[q] + (half ? os[q] & 127u : os[q])),
                                       st + T::kS + (w * T::QS + q) * (kWave / 4), 4, 0, 0);
    ++next_k;
    if (2 * next_k < g.steps) {
      base_a += 128;
      base_b += 128;
#pragma unroll
      for (int q = 0; q < T::QS; ++q) base_s[q] += 256;
    }
  };
  // after a tile's last stage
  auto turn = [&]() {
    if (next_k == stages && next_tile + per_xcd < end) {
      next_k = 0;
      next_tile += per_xcd;
      start(next_tile);
    }
  };
  struct Frag {
    u32x4 a[MI], b[NJ];
  };
  struct Scale {
    int a[MI], b[NJ];
  };
  // byte offsets of a lane's fragments and scales in a stage; taken anew at
  // each read, or the compiler keeps one for each
  const uint32_t sw = (h ^ (c >> 1 & 7)) * 16;
  uint32_t la = (wm * MI * 32 + c) * 128 + sw, lb = T::kB * 16 + (wn * NJ * 32 + c) * 128 + sw;
  uint32_t lsa = T::kS * 16 + (wm * MI * 64 + c) * 4;
  uint32_t lsb = T::kS * 16 + (T::BM * 2 + (wn * NJ + c / 8) * 64 + (NJ * c & 31)) * 4;
  auto rd = [&](const uint4* st, uint32_t q, Frag& f) {   // half step q of a stage
    asm volatile("" : "+v"(la), "+v"(lb));
    const uint8_t* const p = reinterpret_cast<const uint8_t*>(st);
#pragma unroll
    for (int i = 0; i < MI; ++i) f.a[i] = *reinterpret_cast<const u32x4*>(p + (la ^ (q * 32)) + i * 4096);
#pragma unroll
    for (int j = 0; j < NJ; ++j) f.b[j] = *reinterpret_cast<const u32x4*>(p + (lb ^ (q * 32)) + j * 4096);
  };
  auto rd_scale = [&](const uint4* st, uint32_t t, Scale& sc) {   // step t of a stage
    asm volatile("" : "+v"(lsa), "+v"(lsb));
    const uint8_t* const p = reinterpret_cast<const uint8_t*>(st) + t * 128;
#pragma unroll
    for (int i = 0; i < MI; ++i) sc.a[i] = *reinterpret_cast<const int*>(p + lsa + i * 256);
    // (b's scales are in the order of its rows: a lane's are neighbours)
    const u32x4 b = *reinterpret_cast<const u32x4*>(p + lsb);
#pragma unroll
    for (int j = 0; j < NJ; ++j) sc.b[j] = static_cast<int>(b[j]);
  };
  // the scales that this half of the wave takes, to bytes 0 and 2
  auto own_scale = [&](const Scale& raw, Scale& sc) {
#pragma unroll
    for (int i = 0; i < MI; ++i) sc.a[i] = static_cast<int>(static_cast<uint32_t>(raw.a[i]) >> (8 * h));
#pragma unroll
    for (int j = 0; j < NJ; ++j) sc.b[j] = static_cast<int>(static_cast<uint32_t>(raw.b[j]) >> (8 * h));
  };
  f32x16 acc[MI][NJ];
  auto mma = [&](auto KS, const Frag& f, const Scale& sc) {
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NJ; ++j)
        acc[i][j] = mx_mma<decltype(KS)::value>(f.a[i], f.b[j], acc[i][j], sc.a[i], sc.b[j]);
  };
  // The accumulators exist here: a half step's instructions, which touch no
  // memory, would else be moved past the barriers to where they are stored.
  auto pin = [&]() {
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NJ; ++j) asm volatile("" : "+v"(acc[i][j]));
  };
  // LDS reads and loads between the matrix instructions of a half step: the
  // first one waits for the reads before, and loads issued one after the other
  // keep the wave from its matrix instructions while they are taken
  auto weave = [&](auto reads) {
    constexpr int R = decltype(reads)::value, M = MI * NJ, per = (R + M - 2) / (M - 1);
    pin();
#pragma unroll
    for (int i = 0; i < M; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, per, 0);
      __builtin_amdgcn_sched_group_barrier(0x010, 1, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  using I0 = std::integral_constant<int, 0>;
  using I1 = std::integral_constant<int, 1>;
  using Reads = std::integral_constant<int, MI + NJ>;
  using ReadsScale = std::integral_constant<int, 2 * MI + NJ + 1>;
  auto clear = [&]() {
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NJ; ++j) acc[i][j] = f32x16{};
  };
  // (the stores address the output itself: through a pointer of no known
  // address space each would wait for the loads to LDS and for the store before)
  auto store = [&](uint32_t tile) {
    using O = std::conditional_t<DT == PROFK_F32, float, __bf16>;
    const uint32_t mw = tile % tiles_m * T::BM + wm * MI * 32, nw = tile / tiles_m * T::BN + wn * NJ * 32;
    const uint32_t m = mw + 4 * h, n = nw + NJ * c;
    size_t at = static_cast<size_t>(m) * g.N + n;
    O* const out = static_cast<O*>(g.out);
    auto put4 = [&](size_t o, int i, int v) {
      if constexpr (DT == PROFK_F32)
        *reinterpret_cast<f32x4u*>(out + o) = f32x4{acc[i][0][v], acc[i][1][v], acc[i][2][v], acc[i][3][v]};
      else
        *reinterpret_cast<u32x2u*>(out + o) = u32x2u{pack_bf16(acc[i][0][v], acc[i][1][v]), pack_bf16(acc[i][2][v], acc[i][3][v])};
    };
    auto rows = [&](auto put) {
#pragma unroll
      for (int i = 0; i < MI; ++i) {
        // (no row's address or mask is kept through the steps)
        asm volatile("" : "+v"(at));
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const uint32_t r = i * 32 + 8 * (v / 4) + (v % 4);
          put(at + static_cast<size_t>(r) * g.N, r, i, v);
        }
      }
    };
    if (mw + MI * 32 <= g.M && nw + NJ * 32 <= g.N) {
      rows([&](size_t o, uint32_t, int i, int v) { put4(o, i, v); });
    } else {
      rows([&](size_t o, uint32_t r, int i, int v) {
        if (m + r >= g.M || n >= g.N) return;
        if (n + NJ <= g.N) {
          put4(o, i, v);
        } else {
          out[o] = static_cast<O>(acc[i][0][v]);
          if (n + 1 < g.N) out[o + 1] = static_cast<O>(acc[i][1][v]);
          if (n + 2 < g.N) out[o + 2] = static_cast<O>(acc[i][2][v]);
        }
      });
    }
  };
  start(tile0);
  issue_a(s0);
  issue_b(s0);
  issue_s(s0);
  issue_a(s1);
  Frag f0, f1;
  Scale sc, raw;
  wait_loads_lds<T::QA>();
  bare_barrier();
  rd_scale(s0, 0, raw);
  rd(s0, 0, f0);
  // One stage; its first half step's fragments are in f0, its first step's
  // scales in raw, and the loads of a for the next have been issued.
  auto stage = [&](uint4* cur, uint4* nxt, uint32_t k, auto last) {
    const bool one = WHOLE || 2 * k < g.steps, two = WHOLE || 2 * k + 1 < g.steps;
    __builtin_amdgcn_sched_barrier(0);
    own_scale(raw, sc);
    issue_b(nxt);
    rd(cur, 1, f1);
    if (one) mma(I0{}, f0, sc);
    weave(Reads{});
    issue_s(nxt);
    rd_scale(cur, 1, raw);
    rd(cur, 2, f0);
    if (one) mma(I1{}, f1, sc);
    weave(ReadsScale{});
    if (decltype(last)::value) turn();
    own_scale(raw, sc);
    rd(cur, 3, f1);
    if (two) mma(I0{}, f0, sc);
    weave(Reads{});
    // this wave has read its stage and its loads of the next have arrived; by
    // the barrier, so have the others
    wait_loads_lds<0>();
    bare_barrier();
    issue_a(cur);
    rd_scale(nxt, 0, raw);
    rd(nxt, 0, f0);
    if (two) mma(I1{}, f1, sc);
    weave(ReadsScale{});
  };
  for (uint32_t tile = tile0; tile < end; tile += per_xcd) {
    clear();
    for (uint32_t k = 0; k < stages; k += 2) {
      stage(s0, s1, k, std::true_type{});     // (loads the tile's next odd stage)
      stage(s1, s0, k + 1, std::false_type{});
    }
    store(tile);
  }
  wait_loads_lds<0>();   // (no load may reach LDS after the workgroup's end)
}

template <int DT, int WM, int WN, int MI, int NJ, int WAVES, bool WHOLE>
__global__ __launch_bounds__(WM * WN * 64, WAVES) void k_mx_gemm(MxGemmArgs g, uint32_t tiles_m, uint32_t tiles) {
  mx_gemm_body<DT, WM, WN, MI, NJ, WHOLE>(g, tiles_m, tiles);
}

// The product of few rows (M <= 32), bound by reading b once.  A wave takes
// groups of 32 rows of b, two steps (128 bytes a row) at a time: whole lines,
// loaded straight to a part of LDS of its own, four stages deep, so that no
// barrier is needed and the loads of the next group start before this one
// ends.  Granule g of row r is at position g ^ (r / 2 % 8) of its eight.  a
// sits in LDS, its rows 16 bytes apart from a whole number of banks.
// KSPLIT: the workgroup's waves each take a part of the steps of the same
// groups, and their sums are added in wave order.
// Measured: 1 x 4096 x 131072 45 us (6.4 TB/s; a plain read reaches 7).  Loads
// straight to registers, 32 rows of 32 bytes each, took 81 us, and 114 past
// the caches.
constexpr int kMxFewBS = 256;
constexpr int kMxCodes = -1;                          // a's type where it is quantised already
constexpr uint32_t kMxFewStage = 32 * 128 + 32 * 8;   // bytes of a wave's stage: codes, then scales
constexpr int kMxFewLoads = 5;                        // loads of a stage
// LDS for a.  With the smaller one, two workgroups fit a CU where each wave
// takes its own groups; the sums of waves that share them take their place.
constexpr uint32_t kMxFewLdsSmall = 10 * 1024, kMxFewLds = 64 * 1024;
constexpr uint32_t kCuLds = 160 * 1024;
// Workgroups of a kernel that a CU holds, by their LDS: a, the waves' four
// stages, and the sums of all waves but one.
constexpr uint32_t mx_few_per_cu(bool ksplit, uint32_t lds) {
  return kCuLds / (lds + kMxFewBS / kWave * 4 * kMxFewStage + (ksplit ? (kMxFewBS / kWave - 1) * 16 * kWave * 4 : 4));
}
static_assert(mx_few_per_cu(false, kMxFewLdsSmall) == 2 && mx_few_per_cu(true, kMxFewLdsSmall) == 1 &&
              mx_few_per_cu(true, kMxFewLds) == 1, "LDS of the kernel of few rows");
__host__ __device__ constexpr uint32_t mx_few_row(uint32_t steps) { return steps * 64 + 16; }   // LDS bytes of a row of a
__host__ __device__ constexpr uint32_t mx_few_lds(uint32_t M, uint32_t steps) { return M * (mx_few_row(steps) + steps * 4); }
// a fits `lds` bytes.
constexpr bool mx_few(uint64_t M, uint64_t steps, uint32_t lds) {
  return M <= 32 && steps <= lds / 64 && mx_few_lds(static_cast<uint32_t>(M), static_cast<uint32_t>(steps)) <= lds;
}

template <int DT, int XDT, bool KSPLIT, int LDS> __device__ __forceinline__ void mx_few_body(const MxGemmArgs& g) {
  constexpr int NW = kMxFewBS / kWave;
  constexpr uint32_t kQ = kMxFewStage / 16;
  __shared__ __align__(16) uint8_t smem[LDS];   // a: codes, then scales
  __shared__ __align__(16) uint4 s0[NW * kQ], s1[NW * kQ], s2[NW * kQ], s3[NW * kQ];
  __shared__ float s_sum[KSPLIT ? (NW - 1) * 16 * kWave : 1];
  const uint32_t tid = threadIdx.x, lane = tid & (kWave - 1);
  const uint32_t w = __builtin_amdgcn_readfirstlane(tid / kWave);
  const uint32_t c = lane & 31, h = lane >> 5;
  const uint32_t groups = (g.N + 31) / 32, pairs = (g.steps + 1) / 2;
  // this wave's groups and its pairs of steps
  const uint32_t g0 = KSPLIT ? blockIdx.x : blockIdx.x * NW + w, gs = KSPLIT ? gridDim.x : gridDim.x * NW;
  const uint32_t p0 = KSPLIT ? pairs * w / NW : 0, p1 = KSPLIT ? pairs * (w + 1) / NW : pairs;
  const uint32_t mine = g0 < groups ? (groups - g0 + gs - 1) / gs : 0;
  const uint32_t total = mine * (p1 - p0);
  const uint32_t rb = mx_few_row(g.steps);
  const size_t cb = static_cast<size_t>(g.steps) * 64;

  // the pair to load next: group ig, pair ip
  uint32_t ig = g0, ip = p0, issued = 0;
  auto issue = [&](uint4* stage) {
    uint4* const st = stage + w * kQ;
    const uint32_t n0 = ig * 32, last = g.N - 1 - n0;
    const uint32_t half = 2 * ip + 1 < g.steps ? 1u : 0u;   // 0: the pair's second step is past the end
    const uint8_t* const codes = g.b + n0 * cb + ip * 128;
    const uint8_t* const scales = g.bs + (static_cast<size_t>(ig) * g.steps + 2 * ip) * 128;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const uint32_t r = q * 8 + lane / 8, gr = (lane & 7) ^ (r >> 1 & 7);
      const uint32_t o = min(r, last) * static_cast<uint32_t>(cb) + (half ? gr : gr & 3) * 16;
      __builtin_amdgcn_global_load_lds(reinterpret_cast<const uint32_t*>(codes + o), st + q * kWave, 16, 0, 0);
    }
    const uint32_t o = (half ? lane : lane & 31) * 4;
    __builtin_amdgcn_global_load_lds(reinterpret_cast<const uint32_t*>(scales + o), st + 4 * kWave, 4, 0, 0);
    if (++issued < total) {
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
  // a to LDS meanwhile, quantised here where it is not yet
  uint32_t* const s_scale = reinterpret_cast<uint32_t*>(smem + g.M * rb);
  if constexpr (XDT == kMxCodes) {
    for (uint32_t i = tid; i < g.M * g.steps * 4; i += kMxFewBS) {
      const uint32_t r = i / (g.steps * 4), q = i - r * g.steps * 4;
      *reinterpret_cast<uint4*>(smem + r * rb + q * 16) = reinterpret_cast<const uint4*>(g.a)[i];
    }
    for (uint32_t i = tid; i < g.steps * 32; i += kMxFewBS)
      if ((i & 31) < g.M) s_scale[(i & 31) * g.steps + (i >> 5)] = reinterpret_cast<const uint32_t*>(g.as)[i];
  } else {
    const uint32_t lanes = g.steps * 16;
    for (uint32_t i = tid; i < g.M * lanes; i += kMxFewBS) {   // (whole quads of lanes)
      const uint32_t r = i / lanes, q = i - r * lanes;
      float v[8];
      mx_load8<XDT>(static_cast<const char*>(g.x) + r * g.x_stride * (XDT == PROFK_F32 ? 4 : 2), 8 * q, g.K, v);
      uint32_t byte;
      *reinterpret_cast<uint32_t*>(smem + r * rb + q * 4) = mx_quant8(v, byte);
      if ((q & 3) == 0) reinterpret_cast<uint8_t*>(s_scale)[i >> 2] = static_cast<uint8_t>(byte);
    }
  }
  __syncthreads();

  const uint32_t m = min(c, g.M - 1);
  const uint8_t* const xa = smem + m * rb + h * 16;
  const uint32_t* const xs = s_scale + m * g.steps;
  f32x16 acc = {};
  uint32_t cg = g0, cp = p0;      // the pair at hand
  auto finish = [&]() {
    const uint32_t n = cg * 32 + c;
    if (KSPLIT) {
      if (w > 0) {
#pragma unroll
        for (int v = 0; v < 16; ++v) s_sum[((w - 1) * 16 + v) * kWave + lane] = acc[v];
      }
      __syncthreads();
      if (w == 0) {
#pragma unroll
        for (int o = 0; o < NW - 1; ++o)
#pragma unroll
          for (int v = 0; v < 16; ++v) acc[v] += s_sum[(o * 16 + v) * kWave + lane];
      }
      __syncthreads();
    }
    if ((!KSPLIT || w == 0) && n < g.N) {
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const uint32_t r = 8 * (v / 4) + 4 * h + (v % 4);
        if (r < g.M) {
          const size_t o = static_cast<size_t>(r) * g.N + n;
          if constexpr (DT == PROFK_F32) static_cast<float*>(g.out)[o] = acc[v];
          else static_cast<__bf16*>(g.out)[o] = static_cast<__bf16>(acc[v]);
        }
      }
    }
    acc = f32x16{};
  };
  auto step = [&](uint4* cur, uint4* old) {
    // (this wave's own loads and reads: no barrier)
    wait_loads_lds<2 * kMxFewLoads>();
    issue(old);
    const uint4* const st = cur + w * kQ;
    const uint32_t* const sc = reinterpret_cast<const uint32_t*>(st + 4 * kWave);
    const uint32_t x = c >> 1 & 7;
    auto one = [&](uint32_t k, uint32_t hi, uint32_t scale) {
      const u32x4 b0 = __builtin_bit_cast(u32x4, st[c * 8 + ((4 * hi + h) ^ x)]);
      const u32x4 b1 = __builtin_bit_cast(u32x4, st[c * 8 + ((4 * hi + 2 + h) ^ x)]);
      const u32x4 a0 = *reinterpret_cast<const u32x4*>(xa + k * 64), a1 = *reinterpret_cast<const u32x4*>(xa + k * 64 + 32);
      const int sa = static_cast<int>(xs[k] >> (8 * h)), sw = static_cast<int>(scale >> (8 * h));
      acc = mx_mma<0>(a0, b0, acc, sa, sw);
      acc = mx_mma<1>(a1, b1, acc, sa, sw);
    };
    one(2 * cp, 0, sc[c]);
    if (2 * cp + 1 < g.steps) one(2 * cp + 1, 1, sc[32 + c]);
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
  wait_loads_lds<0>();   // (no load may reach LDS after the workgroup's end)
}

template <int DT, int XDT, bool KSPLIT, int LDS> __global__ __launch_bounds__(kMxFewBS) void k_mx_few(MxGemmArgs g) {
  mx_few_body<DT, XDT, KSPLIT, LDS>(g);
}

// PER: workgroups a CU holds.
template <int DT, int WM, int WN, int MI, int NJ, int PER> void launch_gemm(const MxGemmArgs& g, uint32_t cus, hipStream_t s) {
  using T = MxTile<WM, WN, MI, NJ>;
  const uint32_t tm = (g.M + T::BM - 1) / T::BM, tn = (g.N + T::BN - 1) / T::BN, tiles = tm * tn;
  uint32_t grid = (tiles + kXcds - 1) / kXcds * kXcds;
  if (grid > PER * cus) grid = PER * cus / kXcds * kXcds;
  constexpr int kWaves = PER * WM * WN / 4;
  if (g.steps % 4 == 0) k_mx_gemm<DT, WM, WN, MI, NJ, kWaves, true><<<grid, T::BS, 0, s>>>(g, tm, tiles);
  else k_mx_gemm<DT, WM, WN, MI, NJ, kWaves, false><<<grid, T::BS, 0, s>>>(g, tm, tiles);
}

// The kernel of few rows, true, or none (false: the tiled product's case).
// Where a fits beside a second workgroup's stages it is the faster one, and it
// quantises a itself (K = 4096, N = 131072, with the quantisation: M = 1 50 us).
// With a larger a it is so where the waves of a workgroup share the steps of a
// group, as they do where the groups are few (M = 8, K = 4096, N = 8192: 9
// against 13 us); without sharing it is not (M = 16 and 32, N = 131072: 61 and
// 71 against 57 and 62 us).  The grid is what the CUs hold at once: workgroups
// past that fill their stages and quantise a again when the first ones end (K =
// 4096, M = 4, one and two a CU where one fits: N = 10000 12.9 and 17.1 us, 16384
// 14.1 and 18.1, 32000 21.9 and 25.4).
template <int DT, int XDT> bool launch_few(const MxGemmArgs& g, uint32_t cus, hipStream_t s) {
  const uint32_t groups = (g.N + 31) / 32;
  const bool share = groups < 4 * cus && g.steps >= 8;
  if (mx_few(g.M, g.steps, kMxFewLdsSmall)) {
    if (share) {
      const uint32_t most = mx_few_per_cu(true, kMxFewLdsSmall) * cus;
      k_mx_few<DT, XDT, true, kMxFewLdsSmall><<<groups < most ? groups : most, kMxFewBS, 0, s>>>(g);
    } else {
      const uint32_t quads = (groups + 3) / 4, most = mx_few_per_cu(false, kMxFewLdsSmall) * cus;
      k_mx_few<DT, XDT, false, kMxFewLdsSmall><<<quads < most ? quads : most, kMxFewBS, 0, s>>>(g);
    }
    return true;
  }
  if constexpr (XDT == kMxCodes) {
    if (share && mx_few(g.M, g.steps, kMxFewLds)) {
      k_mx_few<DT, XDT, true, kMxFewLds><<<groups < cus ? groups : cus, kMxFewBS, 0, s>>>(g);
      return true;
    }
  }
  return false;
}

template <int DT> void launch_product(const MxGemmArgs& g, int x_dtype, uint32_t cus, hipStream_t s) {
  if (!g.x ? launch_few<DT, kMxCodes>(g, cus, s)
           : x_dtype == PROFK_F32 ? launch_few<DT, PROFK_F32>(g, cus, s) : launch_few<DT, PROFK_BF16>(g, cus, s))
    return;
  // Tiles of 256 x 256 where every CU has one, else two workgroups a CU of 128 x
  // 128 (M x K x N, us with the larger and the smaller: 2048 x 4096 x 4096, 128
  // large tiles, 29 and 23; 2048 x 4096 x 8192, 256 of them, 36 and 42; 512 x 2048
  // x 50000, 392, 33 and 35; 128 x 4096 x 131072, half of each empty, 91 and 70).
  // The rule does not see a second round of large tiles that is nearly empty: from
  // 257 to about 320 of them the smaller ones would be faster (2304 x 4096 x 7680,
  // 270, 54 and 51; 4096 x 512 x 4352, 272, 16 and 12; at 376, 57 and 62).
  const uint64_t large = static_cast<uint64_t>((g.M + 255) / 256) * ((g.N + 255) / 256);
  if (g.M > 128 && large >= cus) launch_gemm<DT, 4, 2, 2, 4, 1>(g, cus, s);
  else launch_gemm<DT, 4, 1, 1, 4, 2>(g, cus, s);
}

}  // namespace

uint64_t mx_steps(int64_t K) { return (static_cast<uint64_t>(K) + 127) / 128; }

hipError_t launch_mx_quantize(int dtype, const void* x, uint64_t stride, int64_t R, int64_t K, uint8_t* codes,
                              uint8_t* scales, hipStream_t s) {
  const uint64_t steps = mx_steps(K), parts = (steps + kMxPairs - 1) / kMxPairs;
  const int64_t step = static_cast<int64_t>(rows_per_launch(kMxBS) / static_cast<int64_t>(parts)) * 32;
  (void)hipGetLastError();
  for (int64_t r = 0; r < R; r += step) {
    const uint64_t rows = static_cast<uint64_t>(R - r < step ? R - r : step);
    const MxQuantArgs a{static_cast<const uint8_t*>(x) + static_cast<uint64_t>(r) * stride * (dtype == PROFK_F32 ? 4 : 2),
                        stride, static_cast<uint32_t>(rows), static_cast<uint32_t>(K), static_cast<uint32_t>(steps),
                        codes + r * steps * 64, scales + r * steps * 4};
    const uint32_t grid = static_cast<uint32_t>((rows + 31) / 32 * parts);
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
  const int64_t step = static_cast<int64_t>((uint64_t{1} << 31) / lanes / 32 * 32);   // (whole groups of rows)
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

// A workgroup that quantises a for itself saves a launch (about 4 us); where a
// is larger, that every workgroup does so costs more (K = 4096, N = 131072:
// M = 4 59.2 us against 55.2 and the launch, M = 16 77.9 against 63.7 and it).
bool mx_quantizes_x(int64_t M, int64_t K) {
  return mx_few(static_cast<uint64_t>(M), mx_steps(K), kMxFewLdsSmall);
}

hipError_t launch_mx_matmul(const MxMatmulCall& c) {
  const MxGemmArgs g{c.a, c.b, c.as, c.bs, static_cast<uint32_t>(c.M), static_cast<uint32_t>(c.N),
                     static_cast<uint32_t>(mx_steps(c.K)), c.out, c.x, c.x_stride, static_cast<uint32_t>(c.K)};
  const uint32_t cus = static_cast<uint32_t>(device_cu_count());
  (void)hipGetLastError();
  if (c.out_dtype == PROFK_F32) launch_product<PROFK_F32>(g, c.x_dtype, cus, c.stream);
  else launch_product<PROFK_BF16>(g, c.x_dtype, cus, c.stream);
  return hipGetLastError();
}

}  // namespace profk
