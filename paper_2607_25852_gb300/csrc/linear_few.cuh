// linear_few.cuh -- between linear.cu and linear_few.cu.
#pragma once

#include "linear.cuh"

namespace spec {

constexpr int kLinFewRows = 32;  // rows of a request, and rows times query heads per key-value head, at most

// Few rows of many heads: two states at least are in shared memory at a time, and
// every SM has a few to go through (fewer heads go by parts of states, linear.cu).
// By parts of states / here, 32 heads of 128 per request: 12 tokens without an update 11.7 / 7.4 us,
// 64 40.3 / 32.7, 128 with one 104 / 92; 64 requests of 8 rows 50.5 / 48.2, of 10 84 /
// 64, their commits 57.4 / 55.7 and 71.7 / 59.6.  Query heads in groups go one after
// another in both; 64 requests of 8 states, 2 / 4 / 8 query heads each: one row 18.0 / 15.3,
// 25.9 / 21.6, 41.5 / 34.6 us, two 18.5 / 16.7, 26.5 / 24.0, 42.7 / 39.2, four 19.2 / 20.6,
// 27.4 / 30.4, 43.9 / 50.1.
inline bool linear_few_serves(int B, int K, int q_heads, int kv_heads, int Dk, int Dv, int dtype, int sms) {
  if ((Dk != 64 && Dk != 128) || (Dv != 64 && Dv != 128)) return false;
  if (q_heads > kv_heads && K > 1) return false;
  const int e = element_size(dtype), rows = (K + 1) * (q_heads / kv_heads);
  return rows <= kLinFewRows && (dtype == SPEC_BF16 || K + 1 <= kLinFewRows / 4) &&
         (long long)B * kv_heads >= 2LL * sms && 2 * (Dk * Dv * 4 + rows * Dk * e + (K + 1) * (Dk + Dv) * e) <= 200 * 1024;
}

cudaError_t launch_linear_few(const LinearLaunch& p, int dtype, cudaStream_t stream);

}  // namespace spec
