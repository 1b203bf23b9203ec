// Penalties for repeated tokens, biases and masks of allowed tokens on rows of
// logits, and the gradient with respect to the logits.
//
// Of a row x with its history (the first n_prompt tokens of it a prompt), c_v
// the occurrences of v after the prompt:
//   u_v = x_v / repetition if x_v > 0, x_v repetition otherwise, where v is in
//         the history, else x_v
//   y_v = u_v - [c_v > 0] presence - c_v frequency + bias_v, or -inf where the
//         row's mask forbids v
//   dx_v = dy_v (1 / repetition, repetition or 1), or 0 where it is forbidden.
// The division is a product with repetition's reciprocal, rounded to fp32: 1.5
// units in the last place at most.
//
// A workgroup takes a piece of a row, 64 bytes a thread, loaded under the search of
// the lists.  It counts the history's tokens that fall into its piece in a table in
// LDS (integer atomics: their order changes nothing), lists the biases of its
// tokens, and marks both in a bitmap.  The marked tokens, few as a rule, are then
// adjusted from their logits, and their values take the place of their counts, as
// they are in memory; the piece goes by with two selections an element, by the
// bitmap and by the mask.  (With each element looked up and adjusted in place, 256
// x 131072 bf16 took 44 us, instructions.)  Every piece reads the whole history
// again, from the caches.
//
// The table is as large as the piece, so that it does not limit the workgroups of
// a CU: of 16-bit logits it has two flags and 14 bits of count, of 32-bit ones 30.
// Rows with longer histories than 14 bits count, and pieces with more biases than
// are listed, take a piece of 16-bit logits in two halves, 32 bits a token, each
// element from its registers: first the counts, then, in the same table, the number
// of each token's last bias, by an integer maximum.  Every step is a pass over a
// list: no token searches a long one (256 x 131072 bf16 with 5000 biases a row 95 us,
// with one for every token 985).
//
// The gradient needs no counts, but the sign of the history's logits, which it
// reads when it comes upon their tokens and notes beside the flag.
#include <type_traits>

#include "adjust.h"
#include "elems.h"
#include "launch.h"

namespace profk {

namespace {

// Of a token's word, in its upper half where it has 32 bits: it is in the prompt
// (of the gradient: in the history); it has a bias (its logit is above 0).
constexpr uint32_t kAdjSeen = 0x8000u, kAdjBias = 0x4000u, kAdjCount = 0x3FFFu;
// Biases of a piece that are listed in LDS: each of their tokens goes through that
// list (us, 256 x 131072 bf16, by the list and by element: 200 spread biases a row 38
// and 52, 15 neighbouring ones 75 and 49, 50 of them 360 and 49).
constexpr uint32_t kAdjList = 16;
constexpr uint32_t kAdjBytes = 64;             // of a thread's elements, 16 at a time
constexpr uint32_t kAdjBS = 512;               // most threads

// Bytes of the table for each element of a thread.
template <int DT, bool GRAD> constexpr uint32_t kAdjWord = DT == PROFK_F32 && !GRAD ? 4 : 2;

// All ones in the half of a pair, or the element, whose bit is set.
template <int DT> __device__ __forceinline__ uint32_t mask_of(uint32_t bits, int w) {
  if constexpr (DT == PROFK_F32) return static_cast<uint32_t>(__builtin_amdgcn_sbfe(bits, w, 1));
  const uint32_t lo = __builtin_amdgcn_sbfe(bits, 2 * w, 1), hi = __builtin_amdgcn_sbfe(bits, 2 * w + 1, 1);
  return (lo & 0xFFFFu) | (hi & 0xFFFF0000u);
}

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ int64_t clamp64(int64_t x, int64_t lo, int64_t hi) { return x < lo ? lo : x > hi ? hi : x; }

template <int DT, bool GRAD> __global__ __launch_bounds__(kAdjBS) void k_adjust(AdjustArgs a) {
  extern __shared__ __align__(16) uint32_t s_word[];     // the table
  __shared__ uint32_t s_bits[GRAD ? 1 : kAdjBS * kAdjBytes / (DT == PROFK_F32 ? 4 : 2) / 32];
  const uint32_t row = a.row + blockIdx.x / a.pieces, p = blockIdx.x % a.pieces;
  const uint32_t v0 = p * a.piece, n = min(a.piece, a.V - v0);
  constexpr uint32_t ES = DT == PROFK_F32 ? 4 : 2;
  constexpr int E = 16 / ES, C = kAdjBytes / 16;
  const uint32_t tid = threadIdx.x, BS = blockDim.x;
  const char* const x = static_cast<const char*>(a.x) + (row * a.stride + v0) * ES;
  const char* const src = GRAD ? static_cast<const char*>(a.dy) + (row * a.dy_stride + v0) * ES : x;
  char* const out = static_cast<char*>(a.out) + (row * a.out_stride + v0) * ES;
  // the piece first: nothing of it waits for the lists
  Raw<DT, E> raw[C];
#pragma unroll
  for (uint32_t q = 0; q < C; ++q) raw[q] = load_raw<DT, E>(src, (q * BS + tid) * E, n);
  // (a list's offsets may be anything: none reaches past the list)
  const int64_t *tokens = nullptr, *ids = nullptr;
  const float* values = nullptr;
  uint32_t n_hist = 0, n_bias = 0;
  if (a.tokens) {
    const int64_t h0 = clamp64(a.offsets[row], 0, a.n_tokens);
    n_hist = static_cast<uint32_t>(clamp64(a.offsets[row + 1], h0, a.n_tokens) - h0);
    tokens = a.tokens + h0;
  }
  if (!GRAD && a.bias_ids) {
    const int64_t b0 = clamp64(a.bias_offsets[row], 0, a.n_bias);
    n_bias = static_cast<uint32_t>(clamp64(a.bias_offsets[row + 1], b0, a.n_bias) - b0);
    ids = a.bias_ids + b0;
    values = a.bias_values + b0;
  }
  const uint32_t* words = nullptr;
  bool lost = false;                 // the row names a mask that is not there
  if (a.allowed) {
    const int64_t k = a.mask ? a.mask[row] : a.n_masks == 1 ? 0 : row;
    lost = k >= a.n_masks;
    if (k >= 0 && !lost) words = a.allowed + static_cast<uint64_t>(k) * a.allowed_stride;
  }
  const bool lists = n_hist || n_bias;
  const uint32_t made = a.n_prompt && n_hist ? static_cast<uint32_t>(clamp64(a.n_prompt[row], 0, n_hist)) : 0;
  const float rep = a.repetition ? a.repetition[row] : 1.0f, inv = 1.0f / rep;
  const float pres = !GRAD && a.presence ? a.presence[row] : 0.0f;
  const float freq = !GRAD && a.frequency ? a.frequency[row] : 0.0f;
  // (a piece starts at a multiple of 32 tokens)
  uint32_t ok[C];
#pragma unroll
  for (uint32_t q = 0; q < C; ++q) {
    const uint32_t i = (q * BS + tid) * E;
    ok[q] = words && i < n ? words[(v0 + i) / 32] >> (i % 32) : 0xFFu;
  }
  // (eight tokens at a time: a load waits for none before it)
  constexpr uint32_t TB = 8;
  int64_t tok[TB];
  auto load_tokens = [&](uint32_t i) {
#pragma unroll
    for (uint32_t q = 0; q < TB; ++q) tok[q] = i + q * BS < n_hist ? tokens[i + q * BS] : -1;
  };
  // an entry's place in the piece, n or more where it has none
  auto in_piece = [&](int64_t v) { return v >> 32 == 0 ? static_cast<uint32_t>(v) - v0 : ~0u; };
  load_tokens(tid);
  int64_t id = tid < n_bias ? ids[tid] : -1;
  __shared__ uint32_t s_n, s_tok[kAdjList], s_at[kAdjList];
  // the last bias of token v of the piece, from the list in LDS, whose order may be
  // any
  auto bias_of = [&](uint32_t v) {
    uint32_t at = 0;
    for (uint32_t k = 0; k < s_n; ++k)
      if (s_tok[k] == v && s_at[k] > at) at = s_at[k];
    return values[at];
  };
  auto clear = [&]() {
    for (uint32_t i = tid * 4; i < BS * (kAdjBytes / ES) * kAdjWord<DT, GRAD> / 4; i += BS * 4)
      *reinterpret_cast<u32x4*>(s_word + i) = u32x4{};
  };
  // the history's tokens of the piece's places from lo on to the table, 32 bits a
  // place or 16; and, where they are to be listed, the biases
  auto search = [&](auto wide, uint32_t lo, uint32_t len, bool list) {
    constexpr bool kWide = decltype(wide)::value;
    auto at_word = [&](uint32_t v) { return s_word + (kWide ? v : v / 2); };
    auto flag = [&](uint32_t v, uint32_t f) { return kWide ? f << 16 : f << (v & 1) * 16; };
    auto mark = [&](uint32_t v) {
      if constexpr (!GRAD) atomicOr(s_bits + v / 32, 1u << v % 32);
    };
    clear();
    if constexpr (!GRAD) {
      for (uint32_t i = tid; i < BS * (kAdjBytes / ES) / 32; i += BS) s_bits[i] = 0;
    }
    if (tid == 0) s_n = 0;
    __syncthreads();
    for (uint32_t i = tid; i < n_hist; i += TB * BS) {
      uint32_t v[TB];
      [[maybe_unused]] float z[TB];
#pragma unroll
      for (uint32_t q = 0; q < TB; ++q) {
        v[q] = in_piece(tok[q]);
        v[q] = v[q] < n ? v[q] - lo : ~0u;
        if constexpr (GRAD) {
          z[q] = 0.0f;
          if (v[q] < len) z[q] = load1(x, v[q] + lo, DT);
        }
      }
#pragma unroll
      for (uint32_t q = 0; q < TB; ++q) {
        if (v[q] < len) {
          if constexpr (GRAD) {
            atomicOr(at_word(v[q]), flag(v[q], kAdjSeen | (z[q] > 0.0f ? kAdjBias : 0u)));
          } else if (i + q * BS < made) {
            atomicOr(at_word(v[q]), flag(v[q], kAdjSeen));
          } else {
            atomicAdd(at_word(v[q]), kWide ? 1u : 1u << (v[q] & 1) * 16);
          }
          mark(v[q]);
        }
      }
      load_tokens(i + TB * BS);
    }
    for (uint32_t i = tid; list && i < n_bias; i += BS) {
      const uint32_t v = in_piece(id);
      if (v < n) {
        atomicOr(at_word(v), flag(v, kAdjBias));
        mark(v);
        const uint32_t k = atomicAdd(&s_n, 1u);
        if (k < kAdjList) {
          s_tok[k] = v;
          s_at[k] = i;
        }
      }
      id = i + BS < n_bias ? ids[i + BS] : -1;
    }
    __syncthreads();
  };
  // one element's penalties: its flags and count
  auto adjust = [&](float y, uint32_t flags, uint32_t count) {
    if (flags & kAdjSeen || count) {
      y *= y > 0.0f ? inv : rep;
      y -= count ? fmaf(static_cast<float>(count), freq, pres) : 0.0f;
    }
    return y;
  };
  constexpr uint32_t kNan = DT == PROFK_F32 ? 0x7FC00000u : 0x7FC07FC0u;
  constexpr uint32_t kForbidden = GRAD ? 0u : DT == PROFK_F32 ? 0xFF800000u : 0xFF80FF80u;
  auto finish = [&](uint32_t q, Raw<DT, E>& y) {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const uint32_t m = mask_of<DT>(ok[q], w);
      y.q[w] = lost ? kNan : (y.q[w] & m) | (kForbidden & ~m);
    }
    store_raw<DT, E>(out, (q * BS + tid) * E, n, y);
  };
  if constexpr (GRAD) {
    if (lists) search(std::false_type{}, 0, n, false);
#pragma unroll
    for (uint32_t q = 0; q < C; ++q) {
      const uint32_t i = (q * BS + tid) * E;
      if (i >= n) return;
      if (lists) {
        float y[E];
        to_f32<DT, E>(raw[q], y);
        // (the words past the row's end stay 0)
        const uint32_t* const c = s_word + i / 2;
#pragma unroll
        for (uint32_t e = 0; e < E; ++e) {
          const uint32_t f = c[e / 2] >> e % 2 * 16;
          y[e] *= f & kAdjSeen ? (f & kAdjBias ? inv : rep) : 1.0f;
        }
        raw[q] = pack<DT, E>(y);
      }
      finish(q, raw[q]);
    }
    return;
  }
  // (more biases than all pieces could list: a pass over them less)
  bool by_element = (DT != PROFK_F32 && n_hist > kAdjCount) || n_bias / kAdjList >= a.pieces;
  constexpr bool kWide = DT == PROFK_F32;
  if (lists && !by_element) {
    search(std::integral_constant<bool, kWide>{}, 0, n, true);
    by_element = s_n > kAdjList;
  }
  if (!by_element) {
    using O = std::conditional_t<DT == PROFK_F32, float, __bf16>;
    if (lists) {
      // a word of the bitmap a thread, or a part of one where the words are fewer:
      // marked tokens of a thread are adjusted one after the other (4 x 256 fp32, most
      // of them marked and 50 biases a row: 95 us by words, 15 so)
      uint32_t span = 32;
      while (span > 1 && n * 2 <= BS * span) span /= 2;
      for (uint32_t u = tid; u * span < n; u += BS) {
        const uint32_t first = u * span;
        uint32_t bits = s_bits[first / 32] >> first % 32;
        if (span < 32) bits &= (1u << span) - 1;
        for (; bits; bits &= bits - 1) {
          const uint32_t v = first + static_cast<uint32_t>(__builtin_ctz(bits));
          const uint32_t c = kWide ? s_word[v] : s_word[v / 2] >> v % 2 * 16, flags = kWide ? c >> 16 : c;
          float y = adjust(load1(x, v, DT), flags, kWide ? c & 0x3FFFFFFFu : c & kAdjCount);
          if (flags & kAdjBias) y += bias_of(v);
          reinterpret_cast<O*>(s_word)[v] = static_cast<O>(y);
        }
      }
      __syncthreads();
    }
#pragma unroll
    for (uint32_t q = 0; q < C; ++q) {
      const uint32_t i = (q * BS + tid) * E;
      if (i >= n) return;
      if (lists) {
        const uint32_t bits = s_bits[i / 32] >> i % 32;
        const u32x4 c = *reinterpret_cast<const u32x4*>(s_word + i * ES / 4);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const uint32_t m = mask_of<DT>(bits, w);
          raw[q].q[w] = (c[w] & m) | (raw[q].q[w] & ~m);
        }
      }
      finish(q, raw[q]);
    }
    return;
  }
  constexpr uint32_t kParts = kWide ? 1 : 2, CP = C / kParts;
  const uint32_t part = BS * E * CP;
#pragma unroll
  for (uint32_t h = 0; h < kParts; ++h) {
    const uint32_t lo = h * part;
    if (lo >= n) return;                  // (the whole workgroup)
    const uint32_t len = min(part, n - lo);
    __syncthreads();
    load_tokens(tid);
    search(std::true_type{}, lo, len, false);
    float y[CP][E];
#pragma unroll
    for (uint32_t q = 0; q < CP; ++q) {
      to_f32<DT, E>(raw[h * CP + q], y[q]);
#pragma unroll
      for (uint32_t e = 0; e < E; ++e) {
        const uint32_t c = s_word[(q * BS + tid) * E + e];
        y[q][e] = adjust(y[q][e], c >> 16, c & 0x3FFFFFFFu);
      }
    }
    if (n_bias) {
      __syncthreads();
      clear();
      __syncthreads();
      for (uint32_t i = tid; i < n_bias; i += BS) {
        const uint32_t p = in_piece(ids[i]), v = p < n ? p - lo : ~0u;
        if (v < len) atomicMax(s_word + v, i + 1);
      }
      __syncthreads();
#pragma unroll
      for (uint32_t q = 0; q < CP; ++q) {
#pragma unroll
        for (uint32_t e = 0; e < E; ++e) {
          const uint32_t c = s_word[(q * BS + tid) * E + e];
          if (c) y[q][e] += values[c - 1];
        }
      }
    }
#pragma unroll
    for (uint32_t q = 0; q < CP; ++q) {
      raw[h * CP + q] = pack<DT, E>(y[q]);
      if (lo + (q * BS + tid) * E < n) finish(h * CP + q, raw[h * CP + q]);
    }
  }
}

}  // namespace

hipError_t launch_adjust(AdjustArgs a, int dtype, int64_t T, hipStream_t s) {
  const uint32_t cus = static_cast<uint32_t>(device_cu_count());
  const uint32_t elems = kAdjBytes / (dtype == PROFK_F32 ? 4 : 2);      // of a thread
  // pieces of whole words of the mask; more of them where the rows are few
  uint32_t piece = kAdjBS * elems;
  while (piece > 1024 && static_cast<uint64_t>(T) * ((a.V + piece - 1) / piece) < 2 * cus) piece /= 2;
  if (a.V < piece) piece = (a.V + 31) / 32 * 32;
  a.piece = piece;
  a.pieces = (a.V + piece - 1) / piece;
  // threads for the piece, and no fewer than go through an average history in one
  // step
  const int64_t history = a.tokens ? a.n_tokens / T : 0;
  uint32_t bs = kAdjBS;
  while (bs > 64 && bs * elems >= 2 * piece && bs * 8 >= 2 * history) bs /= 2;
  const uint32_t word = dtype == PROFK_F32 ? (a.dy ? kAdjWord<PROFK_F32, true> : kAdjWord<PROFK_F32, false>) : 2;
  const uint32_t lds = a.tokens || (!a.dy && a.bias_ids) ? bs * elems * word : 0;
  const int64_t step = ((int64_t{1} << 31) - 1) / bs / a.pieces < 1 ? 1 : ((int64_t{1} << 31) - 1) / bs / a.pieces;
  (void)hipGetLastError();
  for (int64_t r = 0; r < T; r += step) {
    a.row = static_cast<uint32_t>(r);
    const uint32_t grid = static_cast<uint32_t>(T - r < step ? T - r : step) * a.pieces;
    if (dtype == PROFK_F32) {
      if (a.dy) k_adjust<PROFK_F32, true><<<grid, bs, lds, s>>>(a);
      else k_adjust<PROFK_F32, false><<<grid, bs, lds, s>>>(a);
    } else {
      if (a.dy) k_adjust<PROFK_BF16, true><<<grid, bs, lds, s>>>(a);
      else k_adjust<PROFK_BF16, false><<<grid, bs, lds, s>>>(a);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace profk
