// Microscaled 4-bit values and their product (kernels_mx4.hip): what the C ABI
// needs of the kernels.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

namespace profk {

// K is padded to whole steps of 128, 64 bytes of codes and 4 of scales each (of
// rows padded to groups of 32).
uint64_t mx_steps(int64_t K);
constexpr int64_t kMxMaxK = 1 << 20;
hipError_t launch_mx_quantize(int dtype, const void* x, uint64_t stride, int64_t R, int64_t K, uint8_t* codes,
                              uint8_t* scales, hipStream_t s);
hipError_t launch_mx_dequantize(int dtype, const uint8_t* codes, const uint8_t* scales, int64_t R, int64_t K,
                                void* out, hipStream_t s);

struct MxMatmulCall {
  const uint8_t *a, *as;      // codes and scales [M, ..]
  const uint8_t *b, *bs;      // ... [N, ..]
  int64_t M, N, K;
  int out_dtype;
  void* out;                  // [M, N]
  hipStream_t stream;
  const void* x;              // set: a is not quantised yet (mx_quantizes_x)
  uint64_t x_stride;
  int x_dtype;
};

// The product's kernel for this shape quantises a itself.
bool mx_quantizes_x(int64_t M, int64_t K);
hipError_t launch_mx_matmul(const MxMatmulCall& c);

}  // namespace profk
