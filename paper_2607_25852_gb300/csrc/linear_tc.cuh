// linear_tc.cuh -- between linear.cu and linear_tc.cu: which shapes the tensor
// cores serve, and how long calls are divided.
#pragma once

#include <algorithm>

#include "linear.cuh"

namespace spec {

constexpr int kLinChunk = 64;      // rows that a pass over the state takes
// Calls of more rows per request go to the tensor cores.  CUDA cores / tensor cores, 32 heads of 128: 64 requests of 10
// rows 65 / 60 us, of 12 72 / 60, of 17 114 / 61, commits of 12 62 / 61; 12 requests of 10 16.1 / 17.2, of 12 17.9 / 17.3,
// of 17 27.3 / 17.4, commits of 17 15.5 / 16.8; one of 12 6.5 / 9.7, of 17 9.2 / 9.8.  The rule goes by the rows alone,
// so that from 12 to about 17 rows calls of few heads take up to 3.2 us longer than they would on the CUDA cores, and 64
// requests of 10 rows 5 us longer than here.
constexpr int kLinTcRows = 11;
constexpr int kLinMaxSegments = 32;
constexpr int kLinSms = 152;       // the device that plans are made for (a workspace's size must not depend on the one it is asked on)

// Requests in segments of seg_rows rows, nseg at most; the sums of all but a
// request's last are made first, in parallel, into seg_state: each in the place of
// the next segment's first state, which a scan then makes of it.  `staged`: items
// take their first states from there, also where there is one segment but several
// query heads, of which one may store the new state in the old one's slot.
struct LinearPlan {
  int nseg, seg_rows;
  bool staged;
  float* seg_state;      // [B * H][nseg][Dk * Dv]
  long long* seg_steps;  // [B * H][nseg]
};

inline bool linear_tc_serves(int B, int K, int q_heads, int Dk, int Dv, int dtype) {
  return (long long)B * q_heads * kLinMaxSegments < (1LL << 31) && dtype == SPEC_BF16 && (Dk == 64 || Dk == 128) && (Dv == 64 || Dv == 128) && K + 1 > kLinTcRows;
}

// The number of segments with the least work on the busiest SM, in chunks: a
// segment's sums take about 0.6 of its outputs' time, another launch and the scan
// about 6 chunks.  Whole / in segments: two prompts of 16,384 rows of 32 heads of 128
// 602 / 523 us, one of 4,096 of 8 heads of 64 142 / 29.
inline LinearPlan linear_plan(int B, int K, int q_heads, int kv_heads, int max_segments) {
  LinearPlan best{};
  best.nseg = 1;
  const long long chunks = (K + kLinChunk) / kLinChunk;
  best.seg_rows = (int)(chunks * kLinChunk);
  double least = 0.0;
  for (int n = 1; n <= max_segments; ++n) {
    const long long per = (chunks + n - 1) / n;
    if (n > 1 && per < 4) break;
    const long long outs = ((long long)B * q_heads * n + kLinSms - 1) / kLinSms;
    const long long sums = ((long long)B * kv_heads * (n - 1) + kLinSms - 1) / kLinSms;
    const double cost = (double)(outs * per) + (n > 1 ? 0.6 * (double)(sums * per) + 6.0 : 0.0);
    if (n == 1 || cost < least) {
      least = cost;
      best.nseg = n;
      best.seg_rows = (int)(per * kLinChunk);
    }
  }
  return best;
}

// p.q null: states only.
cudaError_t launch_linear_tc(const LinearLaunch& p, const LinearPlan& plan, cudaStream_t stream);

// The segments' first states out of the sums of those before them and the request's own.
cudaError_t launch_linear_scan(const LinearLaunch& p, const LinearPlan& plan, cudaStream_t stream);

}  // namespace spec
