// The dense product with its epilogue and its gradients (kernels_linear.hip):
// what the C ABI needs of the kernels.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

namespace profk {

constexpr int64_t kLinMaxK = 1 << 20;

struct LinCall {
  const void *x, *w;                // bf16 [M, K], [N, K]
  uint64_t x_stride, w_stride;      // elements between row starts
  int64_t M, N, K;
  const float* bias;                // [N], or null
  int act, out_dtype;
  const void* residual;             // [M, N] of out_dtype, or null
  uint64_t residual_stride;
  void *out, *pre;                  // contiguous [M, N]; pre may be null
  void* ws;
};

struct LinGradCall {
  const void *dy, *pre;             // [M, N] of dtype; pre null without an activation
  uint64_t dy_stride;
  int dtype, act;
  bool round_dz;                    // dz to one bf16 number for the products
  const void *x, *w;
  uint64_t x_stride, w_stride;
  int64_t M, N, K;
  void *dx, *dw;                    // contiguous bf16 [M, K], [N, K]; may be null
  float* db;                        // [N]; may be null
  void* ws;
};

size_t lin_workspace(int64_t M, int64_t N, int64_t K, int num_cus);
size_t lin_grad_workspace(int64_t M, int64_t N, int64_t K, int num_cus);
hipError_t launch_linear(const LinCall& c, hipStream_t s);
hipError_t launch_linear_grad(const LinGradCall& c, hipStream_t s);

}  // namespace profk
