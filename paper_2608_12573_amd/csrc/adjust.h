// Penalties, biases and masks on rows of logits, and their gradient
// (kernels_adjust.hip): what the C ABI needs of the kernels.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

namespace profk {

constexpr int64_t kAdjMaxList = (int64_t{1} << 30) - 1;   // entries of a list

struct AdjustArgs {
  const void* x;                    // logits
  const void* dy;                   // gradient of the adjusted logits (null: the forward call)
  void* out;
  uint64_t stride, dy_stride, out_stride;
  uint32_t V, row, pieces, piece;   // first row of this launch; pieces of a row, and their elements
  const int64_t *tokens, *offsets, *n_prompt;   // tokens null: no history
  int64_t n_tokens;
  const float *repetition, *presence, *frequency;
  const int64_t *bias_ids, *bias_offsets;       // bias_ids null: no biases
  const float* bias_values;
  int64_t n_bias;
  const uint32_t* allowed;          // null: all are
  uint64_t allowed_stride;          // words between the masks' starts
  int64_t n_masks;
  const int64_t* mask;              // null: row r takes mask r, or the only one
};

hipError_t launch_adjust(AdjustArgs a, int dtype, int64_t T, hipStream_t s);

}  // namespace profk
