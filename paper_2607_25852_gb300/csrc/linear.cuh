// linear.cuh -- what the linear-attention kernels share: the launch parameters,
// a request's rows and states, and decays as whole numbers.
#pragma once

#include "paged.cuh"

namespace spec {

struct LinearLaunch {
  const void *q, *k, *v;          // q null: states only
  int64_t q_row, k_row, v_row;    // elements between rows
  int Hq, H, G;                   // query heads, key-value heads, queries per key-value head
  int Dk, Dv;
  const float* log_decay;
  int64_t decay_row;              // 0: one per head for all rows
  float* state;                   // of the layer: [slots][H][Dk][Dv]
  int64_t slot_stride;
  int slots;
  const int32_t *slots_in, *slots_out;  // slots_out null: states stay
  const int32_t* accepted;        // rows to take less one, or null: all
  RowLayout rows;
  float scale;
  void* out;
  int32_t* status;
};

// Request i's rows first .. last - 1 count (those before position 0 do not); its
// packed rows begin at row0; from, to: its states' slots, -1 for none.
struct LinearRequest {
  int row0, first, last, rows, from, to;
  bool ok;
};

__device__ __forceinline__ LinearRequest linear_request(const LinearLaunch& a, int i) {
  const int from = __ldg(a.slots_in + i), to = a.slots_out ? __ldg(a.slots_out + i) : -1;
  const RequestRows q = request_rows(a.rows, i);
  const int taken = a.accepted ? __ldg(a.accepted + i) + 1 : q.count;
  LinearRequest r;
  r.row0 = q.row0;
  r.rows = q.count;
  r.ok = q.ok && taken >= 1 && taken <= q.count && from >= -1 && from < a.slots && to >= -1 && to < a.slots;
  r.first = q.p >= 0 ? 0 : (int)(-q.p < taken ? -q.p : taken);
  r.last = taken;
  r.from = from;
  r.to = to;
  return r;
}

// log2 of a row's decay as a whole number of 2^-32: sums of any number of rows are
// exact, and so are their differences, which the weights are made of (sums in fp32
// lose them behind one strong decay).  Below 2^-200 a decay is as good as 0.
__device__ __forceinline__ long long decay_steps(float log_decay, int32_t* status) {
  if (!(log_decay <= 0.0f)) {
    report(status, SPEC_ERR_BAD_INPUT);  // growth, or NaN
    return 0;
  }
  return __double2ll_rn((double)fmaxf(log_decay, -138.62944f) * (1.4426950408889634 * 4294967296.0));
}
// Steps as a float.
__device__ __forceinline__ float steps_float(long long steps) { return __ll2float_rn(steps) * 2.3283064365386963e-10f; }

}  // namespace spec
