// linear_few.cuh -- between linear.cu and linear_few.cu.
#pragma once

#include "linear.cuh"

namespace spec {

constexpr int kLinFewRows = 32;  // rows of a request, and rows times query heads per key-value head, at most

// Few rows of many heads: two states at least are in shared memory at a time, and
// every SM has a few to go through (fewer heads go to parts of states, linear.cu).
inline bool linear_few_serves(int B, int K, int q_heads, int kv_heads, int Dk, int Dv, int dtype, int sms) {
  if ((Dk != 64 && Dk != 128) || (Dv != 64 && Dv != 128)) return false;
  const int e = element_size(dtype), rows = (K + 1) * (q_heads / kv_heads);
  return rows <= kLinFewRows && (dtype == SPEC_BF16 || K + 1 <= kLinFewRows / 4) &&
         (long long)B * kv_heads >= 2LL * sms && 2 * (Dk * Dv * 4 + rows * Dk * e + (K + 1) * (Dk + Dv) * e) <= 200 * 1024;
}

cudaError_t launch_linear_few(const LinearLaunch& p, int dtype, cudaStream_t stream);

}  // namespace spec
