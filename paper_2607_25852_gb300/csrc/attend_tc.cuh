// attend_tc.cuh -- the tensor-core kernels of spec_attend (attend_tc.cu, attend_rows.cu).
#pragma once

#include "attend.cuh"

namespace spec {

// Columns per item: 17 rows of 8 heads, whose scores and two halves of the output
// fit TMEM; of the kernel for many rows, two sets of 128.
constexpr int kTcMaxCols = 144, kRowsMaxCols = 256;

// Whether the tensor-core kernels take a cache of this geometry (strides in bytes),
// and whether they take any of this dimension and type.
inline bool attend_tc_may_serve(int D, int dtype) { return dtype == SPEC_BF16 && (D == 64 || D == 128); }
bool attend_tc_serves(int D, int dtype, int page_size, int64_t head_b, int64_t token_b, int64_t page_b);

// Positions of one of their loads: the largest power of two that divides the page
// size, at most a tile.
int attend_tc_grain(int page_size);

// Columns per item for requests of up to `cols` columns.
int attend_tc_columns(int cols);

// CTAs of their grid per SM, for ct columns per item.
int attend_tc_ctas_per_sm(int D, int ct);

cudaError_t launch_attend_tc(const AttendLaunch& a, cudaStream_t stream);
cudaError_t launch_attend_rows(const AttendLaunch& a, cudaStream_t stream);  // more than kTcMaxCols columns

}  // namespace spec
