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
// A workgroup takes a piece of a row.  It counts the history's tokens that fall
// into its piece in LDS, a word a token (integer atomics: their order changes
// nothing), lists the biases of its tokens, and streams the piece once.  Every piece reads the whole history again, from the caches.
#include "adjust.h"
#include "elems.h"
#include "launch.h"

namespace profk {

namespace {

// Of a token's word: it is in the prompt, it has a bias; the rest counts it after
// the prompt.
constexpr uint32_t kAdjPrompt = 0x80000000u, kAdjBias = 0x40000000u;
constexpr uint32_t kAdjList = 256;             // biases of a piece that are kept in LDS
constexpr uint32_t kAdjElems = 16;             // of a thread, 16 bytes at a time
constexpr uint32_t kAdjPiece = 8192;           // most elements of a piece (LDS: a word each)

__device__ __forceinline__ int64_t clamp64(int64_t x, int64_t lo, int64_t hi) { return x < lo ? lo : x > hi ? hi : x; }

template <int DT, bool GRAD> __global__ __launch_bounds__(512) void k_adjust(AdjustArgs a) {
  extern __shared__ __align__(16) uint32_t s_word[];     // [piece]
  const uint32_t row = a.row + blockIdx.x / a.pieces, p = blockIdx.x % a.pieces;
  const uint32_t v0 = p * a.piece, n = min(a.piece, a.V - v0);
  constexpr uint32_t ES = DT == PROFK_F32 ? 4 : 2;
  constexpr int E = 16 / ES, C = kAdjElems / E;
  const uint32_t tid = threadIdx.x, BS = blockDim.x;
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
  const char* const x = static_cast<const char*>(a.x) + (row * a.stride + v0) * ES;
  const char* const src = GRAD ? static_cast<const char*>(a.dy) + (row * a.dy_stride + v0) * ES : x;
  char* const out = static_cast<char*>(a.out) + (row * a.out_stride + v0) * ES;
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
  // the piece and its part of the mask, and the first of the lists, loaded
  // together (a piece starts at a multiple of 32 tokens)
  Raw<DT, E> raw[C];
  uint32_t ok[C];
#pragma unroll
  for (uint32_t q = 0; q < C; ++q) {
    const uint32_t i = (q * BS + tid) * E;
    raw[q] = load_raw<DT, E>(src, i, n);
    ok[q] = words && i < n ? words[(v0 + i) / 32] >> (i % 32) : 0xFFu;
  }
  // (four tokens at a time: a load waits for none before it)
  int64_t tok[4];
  auto load_tokens = [&](uint32_t i) {
#pragma unroll
    for (uint32_t q = 0; q < 4; ++q) tok[q] = i + q * BS < n_hist ? tokens[i + q * BS] : -1;
  };
  // an entry's place in the piece, n or more where it has none
  auto in_piece = [&](int64_t v) { return v >> 32 == 0 ? static_cast<uint32_t>(v) - v0 : ~0u; };
  load_tokens(tid);
  int64_t id = tid < n_bias ? ids[tid] : -1;
  __shared__ uint32_t s_n, s_tok[kAdjList], s_at[kAdjList];
  if (lists) {
    for (uint32_t i = tid * 4; i < a.piece; i += BS * 4) *reinterpret_cast<u32x4*>(s_word + i) = u32x4{};
    if (tid == 0) s_n = 0;
    __syncthreads();
    for (uint32_t i = tid; i < n_hist; i += 4 * BS) {
#pragma unroll
      for (uint32_t q = 0; q < 4; ++q) {
        const uint32_t v = in_piece(tok[q]);
        if (v < n) {
          if (i + q * BS < made) atomicOr(s_word + v, kAdjPrompt);
          else atomicAdd(s_word + v, 1u);
        }
      }
      load_tokens(i + 4 * BS);
    }
    for (uint32_t i = tid; i < n_bias; i += BS) {
      const uint32_t v = in_piece(id);
      if (v < n) {
        atomicOr(s_word + v, kAdjBias);
        const uint32_t k = atomicAdd(&s_n, 1u);
        if (k < kAdjList) {
          s_tok[k] = v;
          s_at[k] = i;
        }
      }
      id = i + BS < n_bias ? ids[i + BS] : -1;
    }
    __syncthreads();
  }
  // the last bias of token v of the piece: from the list in LDS, whose order may
  // be any, or, where that did not hold them all, from the row's
  auto bias_of = [&](uint32_t v) {
    uint32_t at = 0;
    if (s_n <= kAdjList) {
      for (uint32_t k = 0; k < s_n; ++k)
        if (s_tok[k] == v && s_at[k] > at) at = s_at[k];
    } else {
      for (at = n_bias - 1; in_piece(ids[at]) != v;) --at;
    }
    return values[at];
  };
  // (the words past the row's end stay 0)
  auto words_of = [&](uint32_t i, uint32_t (&c)[E]) {
#pragma unroll
    for (uint32_t w = 0; w < E; w += 4) {
      const u32x4 c4 = lists && i < n ? *reinterpret_cast<const u32x4*>(s_word + i + w) : u32x4{};
#pragma unroll
      for (uint32_t e = 0; e < 4; ++e) c[w + e] = c4[e];
    }
  };
  // the gradient needs the logits of the history's tokens alone: all of a thread's
  // are on their way before the first is used
  float seen[C][E];
  if constexpr (GRAD) {
#pragma unroll
    for (uint32_t q = 0; q < C; ++q) {
      const uint32_t i = (q * BS + tid) * E;
      uint32_t c[E];
      words_of(i, c);
#pragma unroll
      for (uint32_t e = 0; e < E; ++e) {
        seen[q][e] = 0.0f;
        if (c[e]) seen[q][e] = load1(x, i + e, DT);
      }
    }
  }
#pragma unroll
  for (uint32_t q = 0; q < C; ++q) {
    const uint32_t i = (q * BS + tid) * E;
    if (i >= n) return;
    float y[E];
    to_f32<DT, E>(raw[q], y);
    uint32_t c[E];
    words_of(i, c);
#pragma unroll
    for (uint32_t e = 0; e < E; ++e) {
      if constexpr (GRAD) {
        y[e] *= c[e] ? (seen[q][e] > 0.0f ? inv : rep) : 1.0f;
      } else {
        if (c[e] & ~kAdjBias) {
          y[e] *= y[e] > 0.0f ? inv : rep;
          const uint32_t m = c[e] & ~(kAdjPrompt | kAdjBias);
          y[e] -= m ? fmaf(static_cast<float>(m), freq, pres) : 0.0f;
        }
        if (c[e] & kAdjBias) y[e] += bias_of(i + e);
      }
    }
#pragma unroll
    for (uint32_t e = 0; e < E; ++e) y[e] = ok[q] >> e & 1 ? y[e] : GRAD ? 0.0f : -__builtin_inff();
    if (lost) {
#pragma unroll
      for (uint32_t e = 0; e < E; ++e) y[e] = __builtin_nanf("");
    }
    store<DT, E>(out, i, n, y);
  }
}

}  // namespace

hipError_t launch_adjust(AdjustArgs a, int dtype, int64_t T, hipStream_t s) {
  const uint32_t cus = static_cast<uint32_t>(device_cu_count());
  // pieces of whole words of the mask; more of them where the rows are few
  uint32_t piece = kAdjPiece;
  while (piece > 1024 && static_cast<uint64_t>(T) * ((a.V + piece - 1) / piece) < 2 * cus) piece /= 2;
  if (a.V < piece) piece = (a.V + 31) / 32 * 32;
  a.piece = piece;
  a.pieces = (a.V + piece - 1) / piece;
  // threads for the piece, and no fewer than go through an average history in one
  // step
  const int64_t history = a.tokens ? a.n_tokens / T : 0;
  uint32_t bs = 512;
  while (bs > 64 && bs * kAdjElems >= 2 * piece && bs * 4 >= 2 * history) bs /= 2;
  const uint32_t lds = a.tokens || (!a.dy && a.bias_ids) ? piece * 4 : 0;
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
