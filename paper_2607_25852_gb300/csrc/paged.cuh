// paged.cuh -- what the paged-cache kernels share: the cache's geometry and
// the row layout of a request.
#pragma once

#include "spec_internal.cuh"

namespace spec {

// One request's rows: count packed rows from row0, the first at position p.
struct RequestRows {
  int row0, count;
  int64_t p;
  bool ok;  // depth and offsets agree
};

struct RowLayout {
  const int32_t* row_offsets;  // [B + 1] or null
  const int32_t* depth;        // [B] or null
  const int64_t* pos_base;     // [B], or null: position 0
  int B, K;
};

__device__ __forceinline__ RequestRows request_rows(const RowLayout& a, int i) {
  RequestRows r;
  const int n = a.depth ? __ldg(a.depth + i) : a.K;
  int end;
  if (a.row_offsets) {
    r.row0 = __ldg(a.row_offsets + i);
    end = __ldg(a.row_offsets + i + 1);
  } else {
    r.row0 = i * (a.K + 1);
    end = r.row0 + a.K + 1;
  }
  // far past any table (and far below 0) is all the same: sums with p do not overflow
  const long long p = a.pos_base ? __ldg(reinterpret_cast<const long long*>(a.pos_base) + i) : 0, far = 1LL << 40;
  r.p = p > far ? far : p < -far ? -far : p;
  r.count = n + 1;
  r.ok = n >= 0 && n <= a.K && r.row0 >= 0 && end <= a.B * (a.K + 1) &&
         (a.row_offsets ? end - r.row0 == n + 1 : true);
  return r;
}

inline int element_size(int dtype) { return dtype == SPEC_F32 ? 4 : 2; }

// The contract of spec_cache: 16-byte aligned bases, strides and heads.
inline bool cache_ok(const spec_cache* c) {
  if (!c || !c->k || !c->v || (c->dtype != SPEC_BF16 && c->dtype != SPEC_F32)) return false;
  if (c->layers < 1 || c->pages < 1 || c->page_size < 1 || c->kv_heads < 1 || c->head_dim < 1 ||
      c->head_dim > SPEC_MAX_HEAD_DIM)
    return false;
  const int64_t e = element_size(c->dtype);
  if (((reinterpret_cast<uintptr_t>(c->k) | reinterpret_cast<uintptr_t>(c->v)) & 15u) != 0) return false;
  if (c->head_dim * e % 16 != 0) return false;
  const int64_t strides[4] = {c->layer_stride, c->page_stride, c->token_stride, c->head_stride};
  const int32_t extent[4] = {c->layers, c->pages, c->page_size, c->kv_heads};
  for (int k = 0; k < 4; ++k) {
    // the stride of an extent of one is never used
    if (extent[k] == 1) continue;
    if (strides[k] < c->head_dim || strides[k] > (INT64_MAX >> 4) / extent[k] || strides[k] * e % 16 != 0) return false;
  }
  return true;
}

inline bool rows_shape_ok(int B, int K) {
  return B >= 1 && K >= 0 && K <= SPEC_MAX_DRAFTS && (long long)B * (K + 1) <= (1LL << 28);
}

inline bool table_shape_ok(int B, int max_pages, int pages, int page_size) {
  return B >= 1 && max_pages >= 1 && pages >= 1 && page_size >= 1 && (long long)max_pages * page_size <= (1LL << 30) &&
         (long long)B * max_pages < (1LL << 31);
}

}  // namespace spec
