// Token log probabilities, entropy and alternatives of rows of logits, and
// their gradient (kernels_logprobs.hip): what the C ABI needs of the kernels.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

namespace profk {

constexpr int64_t kLpMaxTop = 64;             // most alternatives of a row
constexpr int kLpWaveBytes = 8192;            // longest row (or chunk) that one wave takes
constexpr int64_t kLpMinChunk = 2048;         // shortest chunk of a row split over workgroups
constexpr int64_t kLpMaxChunks = 256;
constexpr int kLpJoinBS = 256;
constexpr int kLpPart = 4;                    // words of a chunk's statistics

struct LpArgs {
  const void* x;
  uint64_t stride;      // elements between row starts
  uint32_t V, n;        // n: alternatives (0: none)
  const int64_t* tokens;
  float *logprob, *entropy, *lse, *lse_low, *top;   // lse_low: null, or what lse's rounding leaves
  int64_t* top_idx;
  uint32_t row;         // first row of this launch
  uint32_t G, chunk;    // chunks of a row, and their elements
  float* part;          // G > 1: the chunks' statistics
  uint64_t* part_top;   // ... and their n best
};

struct LpLayout {
  uint32_t G = 1, chunk = 0;
  size_t off_top = 0, bytes = 0;              // workspace (0: none)
};

LpLayout lp_layout(int64_t T, int64_t V, int64_t n, int num_cus);

struct LpCall {
  int dtype;
  int64_t T;
  LpArgs a;
  LpLayout L;
  uint8_t* ws;
  hipStream_t stream;
};

hipError_t launch_logprobs(LpCall c);

struct LpGradArgs {
  const void* x;
  uint64_t stride;
  uint32_t V, n;
  const int64_t* tokens;                      // null: no token has a gradient
  const float *lse, *lse_low, *entropy, *g_logprob, *g_entropy, *g_lse, *g_top;   // lse_low, g_..: may be null
  const int64_t* top_idx;
  void* out;
  uint64_t out_stride;
  uint32_t row, pieces;                       // first row of this launch; workgroups of a row
};

hipError_t launch_logprobs_grad(LpGradArgs a, int dtype, int64_t T, hipStream_t s);

}  // namespace profk
