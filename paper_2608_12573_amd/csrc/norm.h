// Layer norm of rows and its gradients (kernels_norm.hip): what the C ABI needs
// of the kernels.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

namespace profk {

constexpr int64_t kNormMaxD = 1 << 20;

struct NormArgs {
  const void* x;
  uint64_t stride, out_stride;      // elements between row starts
  uint32_t T, D;
  const void *w, *b;                // [D] each, or null
  int p_dtype;                      // ... their type
  float eps;
  void* out;
  float *mean, *rstd;               // [T]
};

struct NormGradArgs {
  const void *x, *dy;
  uint64_t stride, dy_stride, dx_stride;
  uint32_t T, D;
  const void* w;
  int p_dtype;
  const float *mean, *rstd;
  void *dx, *dw, *db;               // any may be null
  float* part;                      // [parts, 2, D]: sums of dy n and of dy over each part's rows
  uint32_t parts;
};

uint32_t norm_grad_parts(int64_t T, int64_t D, int num_cus);
hipError_t launch_norm(const NormArgs& a, int dtype, int out_dtype, hipStream_t s);
hipError_t launch_norm_grad(const NormGradArgs& a, int dtype, int dy_dtype, hipStream_t s);

}  // namespace profk
