// attend_tc.cuh -- the tensor-core kernel of spec_attend (attend_tc.cu).
#pragma once

#include "attend.cuh"

namespace spec {

constexpr int kTcMaxCols = 144;  // columns per item: 17 rows of 8 heads; scores and two halves of the output fit TMEM

// Whether the tensor-core kernel takes a cache of this geometry (strides in bytes).
bool attend_tc_serves(int D, int dtype, int page_size, int64_t head_b, int64_t token_b, int64_t page_b);

// Positions of one of its loads: the largest power of two that divides the page
// size, at most a tile.
int attend_tc_grain(int page_size);

// Columns per item for requests of up to `cols` columns.
int attend_tc_columns(int cols);

// CTAs of its grid per SM, for ct columns per item.
int attend_tc_ctas_per_sm(int D, int ct);

cudaError_t launch_attend_tc(const AttendLaunch& a, cudaStream_t stream);

}  // namespace spec
