// pages.cu -- the pages of the key-value cache around a round: append, fork,
// reserve, release, compact, copy (see spec.h for what each computes).
//
// All of it is integer bookkeeping and copying, bound by launch latency at
// small sizes and by HBM in append and copy.  Nothing is ordered by an
// atomic: counts are added with integer atomics, whose order does not show,
// and every list and every choice of a page comes from a prefix sum in index
// order.
//
// GPU times below are of calls captured in a graph, one after another; a call
// costs the host 5 to 8 us, so all but the largest copies and appends are bound
// by the host that makes them, and the kernels are laid out for few launches and
// short chains of dependent loads rather than for bandwidth.
#include <cooperative_groups.h>

#include <algorithm>

#include "paged.cuh"
#include "tensor_core.cuh"

namespace spec {

namespace cg = cooperative_groups;

// ---------------------------------------------------------------------------
// append
// ---------------------------------------------------------------------------
struct AppendLaunch {
  char *k, *v;            // of the layer
  const char *k_new, *v_new;
  int64_t k_row, v_row;   // bytes between rows
  int64_t page_b, token_b, head_b;
  int kv_heads, vec_head; // 16-byte vectors per head
  int pages, page_size, max_pages;
  const int32_t* table;
  RowLayout rows;
  int32_t* status;
};

constexpr int kAppendWarps = 4;

// One warp per (request, row j): the row's vectors of K and V are loaded while
// the row's page is looked up, so that the two round trips overlap.  Bound by
// those round trips (578 rows of 8 heads of 128 in bf16, 4.7 MB: 2.6 us) and, for large
// calls, by HBM (1,536 rows of 12 heads of 96 in fp32, 28 MB: 4.7 us, 6.0 TB/s).
__global__ void __launch_bounds__(32 * kAppendWarps) append_kernel(const AppendLaunch p) {
  const int lane = threadIdx.x & 31;
  const long long r = (long long)blockIdx.x * kAppendWarps + (threadIdx.x >> 5);
  const int K1 = p.rows.K + 1;
  pdl_wait_prerequisites();
  pdl_launch_dependents();
  if (r >= (long long)p.rows.B * K1) return;
  const int i = (int)(r / K1), j = (int)(r - (long long)i * K1);
  const RequestRows q = request_rows(p.rows, i);
  if (!q.ok) {
    if (j == 0 && lane == 0) report(p.status, SPEC_ERR_BAD_INPUT);
    return;
  }
  if (j >= q.count) return;
  const int64_t pos = q.p + j;
  if (pos < 0) return;
  if (pos >= (int64_t)p.max_pages * p.page_size) {
    if (lane == 0) report(p.status, SPEC_ERR_BAD_INPUT);
    return;
  }
  const int slot = (int)pos / p.page_size;  // the table spans less than 2^31 positions
  const int page = p.table[(size_t)i * p.max_pages + slot];
  const int nvec = p.kv_heads * p.vec_head;
  const uint4* ks = reinterpret_cast<const uint4*>(p.k_new + (int64_t)(q.row0 + j) * p.k_row);
  const uint4* vs = reinterpret_cast<const uint4*>(p.v_new + (int64_t)(q.row0 + j) * p.v_row);
  constexpr int kU = 4;  // vectors of each in flight
  for (int x0 = lane; x0 < nvec; x0 += 32 * kU) {
    uint4 a[kU], b[kU];
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const int x = x0 + 32 * u;
      if (x < nvec) {
        a[u] = ldg_stream(ks + x);
        b[u] = ldg_stream(vs + x);
      }
    }
    if (page < 0 || page >= p.pages) {
      if (lane == 0) report(p.status, SPEC_ERR_BAD_INPUT);
      return;
    }
    const int64_t at = (int64_t)page * p.page_b + ((int)pos - slot * p.page_size) * p.token_b;
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const int x = x0 + 32 * u;
      if (x < nvec) {
        const int h = x / p.vec_head;
        const int64_t o = at + h * p.head_b + (int64_t)(x - h * p.vec_head) * 16;
        *reinterpret_cast<uint4*>(p.k + o) = a[u];
        *reinterpret_cast<uint4*>(p.v + o) = b[u];
      }
    }
  }
}

// ---------------------------------------------------------------------------
// copy
// ---------------------------------------------------------------------------
struct CopyLaunch {
  char *k, *v;
  int64_t layer_b, page_b, token_b, head_b;
  int layers, pages;
  int runs;       // contiguous runs of a page: 1 if the page is one block
  int heads;      // kv_heads where runs > 1
  int run_vec;    // 16-byte vectors per run
  const int32_t *src, *dst, *count;
  int max_count;
  int32_t* status;
};

// A warp takes (pair, layer, K or V, segment of kCopySeg vectors) units in
// turn; each lane has 8 loads in flight before its first store.  Bound by HBM: 5,282
// pages of 4 KB in two layers, K and V, 173 MB read and written: 27 us (6.4 TB/s);
// 12 to 244 such pages 2.3 to 2.8 us.
constexpr int kCopyWarps = 8;
constexpr int kCopyUnroll = 8;
constexpr int kCopySeg = 32 * kCopyUnroll;  // 4 KB

__global__ void __launch_bounds__(32 * kCopyWarps) copy_pages_kernel(const CopyLaunch p) {
  const int lane = threadIdx.x & 31;
  const long long warp = (long long)blockIdx.x * kCopyWarps + (threadIdx.x >> 5);
  const long long warps = (long long)gridDim.x * kCopyWarps;
  pdl_wait_prerequisites();
  pdl_launch_dependents();
  int n = *p.count;
  if (n < 0 || n > p.max_count) {
    if (warp == 0 && lane == 0) report(p.status, SPEC_ERR_BAD_INPUT);
    n = n < 0 ? 0 : p.max_count;
  }
  const int page_vec = p.runs * p.run_vec;
  const int segs = (page_vec + kCopySeg - 1) / kCopySeg;
  const long long units = (long long)n * p.layers * 2 * segs;
  for (long long u = warp; u < units; u += warps) {
    const int seg = (int)(u % segs);
    long long w = u / segs;
    const bool is_v = (w & 1) != 0;
    w >>= 1;
    const int layer = (int)(w % p.layers);
    const int x = (int)(w / p.layers);
    const int s = __ldg(p.src + x), d = __ldg(p.dst + x);
    if (s < 0 || s >= p.pages || d < 0 || d >= p.pages) {
      if (lane == 0) report(p.status, SPEC_ERR_BAD_INPUT);
      continue;
    }
    char* base = (is_v ? p.v : p.k) + layer * p.layer_b;
    const char* from = base + s * p.page_b;
    char* to = base + d * p.page_b;
    uint4 a[kCopyUnroll];
    int64_t off[kCopyUnroll];
#pragma unroll
    for (int k = 0; k < kCopyUnroll; ++k) {
      const int e = seg * kCopySeg + 32 * k + lane;
      if (p.runs == 1) {
        off[k] = (int64_t)e * 16;
      } else {
        const int run = e / p.run_vec, t = run / p.heads;
        off[k] = (int64_t)t * p.token_b + (int64_t)(run - t * p.heads) * p.head_b + (int64_t)(e - run * p.run_vec) * 16;
      }
      if (e < page_vec) a[k] = ldg_stream(from + off[k]);
    }
#pragma unroll
    for (int k = 0; k < kCopyUnroll; ++k)
      if (seg * kCopySeg + 32 * k + lane < page_vec) *reinterpret_cast<uint4*>(to + off[k]) = a[k];
  }
}

// ---------------------------------------------------------------------------
// fork
// ---------------------------------------------------------------------------
struct ForkLaunch {
  const int32_t *table, *refs, *parent;
  int B_in, B, max_pages, pages;
  int32_t *table_out, *refs_out;
  int32_t* status;
};

constexpr int kForkThreads = 256;
constexpr int kForkPer = 4;  // entries per thread
// The most entries (of tables and counts) and rows of a call that one cluster does.
constexpr int kForkHere = 1 << 15, kForkRows = 256;

// Counts that stay in place need nothing of the new rows: one launch.  Counts that
// go to a new array have to be copied there before they change: small calls do
// both in one cluster (fork_cluster_kernel), large ones in two launches.  12 rows
// of 128 slots: one cluster 5.9 us of the host and 3.5 of the GPU, two launches 7.4
// and 2.0; 256 rows of 320 in two launches 7.4 and 2.4.  Round trips to L2 bound
// the kernels.
// A block per (old row, segment): its entries' counts change by the row's
// children less one, so a row that one child takes over touches no count.  The
// inputs are read before `wait`.
template <typename Wait>
__device__ __forceinline__ void fork_counts(const ForkLaunch& p, int segs, long long block, Wait wait) {
  const int r = (int)(block / segs), seg = (int)(block - (long long)r * segs);
  int mine = 0;
  for (int i = threadIdx.x; i < p.B; i += kForkThreads) mine += __ldg(p.parent + i) == r ? 1 : 0;
  __shared__ int children;
  if (threadIdx.x == 0) children = 0;
  __syncthreads();
  mine = __reduce_add_sync(0xFFFFFFFFu, mine);
  if ((threadIdx.x & 31) == 0 && mine) atomicAdd(&children, mine);
  int e[kForkPer];
#pragma unroll
  for (int k = 0; k < kForkPer; ++k) {
    const int s = (seg * kForkPer + k) * kForkThreads + threadIdx.x;
    e[k] = s < p.max_pages ? __ldg(p.table + (size_t)r * p.max_pages + s) : -1;
  }
  __syncthreads();
  const int change = children - 1;
  wait();
  if (change == 0) return;
#pragma unroll
  for (int k = 0; k < kForkPer; ++k)
    if (e[k] >= 0 && e[k] < p.pages) atomicAdd(p.refs_out + e[k], change);
}

// Row i's entry at slot s.
__device__ __forceinline__ int fork_entry(const ForkLaunch& p, int par, int s) {
  const int e = par >= 0 && par < p.B_in && s < p.max_pages ? __ldg(p.table + (size_t)par * p.max_pages + s) : -1;
  if (e >= -1 && e < p.pages) return e;
  report(p.status, SPEC_ERR_BAD_INPUT);
  return -1;
}

// Blocks of kForkThreads threads: first the new rows, one per (row, segment of
// its slots), then `extra` that copy the counts when they go to a new array, then,
// where they stay in place, the counts' changes.
__global__ void __launch_bounds__(kForkThreads) fork_kernel(const ForkLaunch p, int segs, int extra) {
  pdl_wait_prerequisites();
  pdl_launch_dependents();  // only now: the next kernel reads this call's inputs before its own wait
  long long block = blockIdx.x;
  if (block >= (long long)p.B * segs) {
    block -= (long long)p.B * segs;
    if (block >= extra) {
      fork_counts(p, segs, block - extra, [] {});
      return;
    }
    const long long at = block * kForkThreads * kForkPer + threadIdx.x;
#pragma unroll
    for (int k = 0; k < kForkPer; ++k) {
      const long long e = at + k * kForkThreads;
      if (e < p.pages) p.refs_out[e] = p.refs[e];
    }
    return;
  }
  const int i = (int)(block / segs), seg = (int)(block - (long long)i * segs);
  const int par = __ldg(p.parent + i);
  if (par < -1 || par >= p.B_in) {
    if (seg == 0 && threadIdx.x == 0) report(p.status, SPEC_ERR_BAD_INPUT);
  }
  int e[kForkPer];
#pragma unroll
  for (int k = 0; k < kForkPer; ++k) e[k] = fork_entry(p, par, (seg * kForkPer + k) * kForkThreads + threadIdx.x);
#pragma unroll
  for (int k = 0; k < kForkPer; ++k) {
    const int s = (seg * kForkPer + k) * kForkThreads + threadIdx.x;
    if (s < p.max_pages) p.table_out[(size_t)i * p.max_pages + s] = e[k];
  }
}

// The counts' changes, past the copy of a larger call.
__global__ void __launch_bounds__(kForkThreads) fork_refs_kernel(const ForkLaunch p, int segs) {
  fork_counts(p, segs, blockIdx.x, [] {
    pdl_wait_prerequisites();  // the counts' copy
    pdl_launch_dependents();
  });
}

// ---------------------------------------------------------------------------
// Prefix sums in a CTA
// ---------------------------------------------------------------------------
constexpr int kPageThreads = 1024;
constexpr int kPageCluster = 8;

// Exclusive prefix sum of x over the CTA's threads; *total: the sum.  All
// threads call it; `sums` is 33 ints of shared memory, free again afterwards.
__device__ __forceinline__ int cta_exclusive(int x, int* sums, int* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int incl = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xFFFFFFFFu, incl, o);
    if (lane >= o) incl += y;
  }
  if (lane == 31) sums[warp] = incl;
  __syncthreads();
  if (warp == 0) {
    const int t = sums[lane];
    int ti = t;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xFFFFFFFFu, ti, o);
      if (lane >= o) ti += y;
    }
    sums[lane] = ti - t;
    if (lane == 31) sums[32] = ti;
  }
  __syncthreads();
  const int before = sums[warp];
  *total = sums[32];
  __syncthreads();
  return before + incl - x;
}

// A thread's run of pages, in index order over the cluster's threads: one prefix
// sum ranks them all.
struct PageRun {
  int begin, end;
};
__device__ __forceinline__ int pages_per_thread(int pages) {
  return (pages - 1) / (kPageCluster * kPageThreads) + 1;
}
__device__ __forceinline__ PageRun page_run(int pages) {
  const int run = pages_per_thread(pages);
  const long long at = (long long)((int)cg::this_cluster().block_rank() * kPageThreads + (int)threadIdx.x) * run;
  const int begin = (int)min((long long)pages, at);
  return PageRun{begin, begin + min(run, pages - begin)};
}

// Exclusive prefix sum of x over the cluster's threads; *total: the sum.  `slot` is
// an int of shared memory, which the CTA keeps until the cluster's next barrier.
__device__ __forceinline__ int cluster_exclusive(int x, int* sums, int* slot, int* total) {
  cg::cluster_group cluster = cg::this_cluster();
  int all;
  int before = cta_exclusive(x, sums, &all);
  if (threadIdx.x == 0) *slot = all;
  cluster.sync();
  *total = 0;
  for (int c = 0; c < kPageCluster; ++c) {
    const int y = *cluster.map_shared_rank(slot, c);
    *total += y;
    if (c < (int)cluster.block_rank()) before += y;
  }
  return before;
}

// A small call with counts in a new array: one cluster.
__global__ void __cluster_dims__(kPageCluster, 1, 1) __launch_bounds__(kPageThreads)
    fork_cluster_kernel(const ForkLaunch p) {
  cg::cluster_group cluster = cg::this_cluster();
  pdl_wait_prerequisites();
  pdl_launch_dependents();
  const int threads = kPageThreads * (int)cluster.num_blocks();
  const int at = (int)cluster.block_rank() * kPageThreads + (int)threadIdx.x;
  for (int e = at; e < p.pages; e += threads) p.refs_out[e] = p.refs[e];
  for (int x = at; x < p.B * p.max_pages; x += threads) {
    const int i = x / p.max_pages, s = x - i * p.max_pages, par = __ldg(p.parent + i);
    if (s == 0 && (par < -1 || par >= p.B_in)) report(p.status, SPEC_ERR_BAD_INPUT);
    p.table_out[x] = fork_entry(p, par, s);
  }
  __threadfence();
  cluster.sync();
  const int lane = threadIdx.x & 31;
  for (int r = at / 32; r < p.B_in; r += threads / 32) {  // a warp per old row
    int mine = 0;
    for (int i = lane; i < p.B; i += 32) mine += __ldg(p.parent + i) == r ? 1 : 0;
    const int change = __reduce_add_sync(0xFFFFFFFFu, mine) - 1;
    if (change == 0) continue;
    for (int s = lane; s < p.max_pages; s += 32) {
      const int e = __ldg(p.table + (size_t)r * p.max_pages + s);
      if (e >= 0 && e < p.pages) atomicAdd(p.refs_out + e, change);
    }
  }
}

// ---------------------------------------------------------------------------
// reserve
// ---------------------------------------------------------------------------
struct ReserveLaunch {
  int32_t *table, *refs;
  RowLayout rows;
  int max_pages, pages, page_size;
  int32_t *cow_src, *cow_dst, *counts, *granted;
  int cap;
  int32_t* free_list;  // workspace [cap]
  int32_t* status;
};

struct SlotSpan {
  int first, last;  // slots touched; first > last: none
  bool ok;
};

__device__ __forceinline__ SlotSpan slot_span(const ReserveLaunch& p, int i) {
  const RequestRows q = request_rows(p.rows, i);
  SlotSpan s{0, -1, q.ok};
  if (!q.ok || q.p + q.count <= 0) return s;
  const int64_t a = (q.p < 0 ? 0 : q.p) / p.page_size, b = (q.p + q.count - 1) / p.page_size;
  if (b >= p.max_pages) {
    s.ok = false;
    return s;
  }
  s.first = (int)a;
  s.last = (int)b;
  return s;
}

// 0: the slot's page is the request's own, 1: empty, 2: shared, -1: no page.
__device__ __forceinline__ int slot_need(const ReserveLaunch& p, int entry) {
  if (entry == -1) return 1;
  if (entry < 0 || entry >= p.pages) return -1;
  return p.refs[entry] > 1 ? 2 : 0;
}

// One cluster of 8 CTAs lists the free pages by rank (as far as the requests' need
// can reach); CTA 0 then walks the requests, a thread each: a prefix sum of the
// needs gives every needed slot its rank.  One cluster, because the ranks need
// every CTA's counts: a barrier of the cluster costs less than a second launch.
// 5.4 us (12 requests, 1,024 pages), 6.8 us (256 requests, 32,768 pages); barriers
// and round trips bound it.
__global__ void __cluster_dims__(kPageCluster, 1, 1) __launch_bounds__(kPageThreads)
    reserve_kernel(const ReserveLaunch p) {
  __shared__ int sums[33], slot;
  cg::cluster_group cluster = cg::this_cluster();
  pdl_wait_prerequisites();
  pdl_launch_dependents();
  const PageRun run = page_run(p.pages);
  int mine = 0, all_free;
  for (int e = run.begin; e < run.end; ++e) mine += p.refs[e] == 0 ? 1 : 0;
  int rank = cluster_exclusive(mine, sums, &slot, &all_free);
  for (int e = run.begin; e < run.end && rank < p.cap; ++e)
    if (p.refs[e] == 0) p.free_list[rank++] = e;
  __threadfence();
  cluster.sync();
  if (cluster.block_rank() != 0) return;

  int needed = 0, pairs = 0, taken = 0;  // of the requests before this round of threads
  for (int i0 = 0; i0 < p.rows.B; i0 += kPageThreads) {
    const int i = i0 + threadIdx.x;
    int need = 0, cow = 0;
    SlotSpan s{0, -1, true};
    if (i < p.rows.B) {
      s = slot_span(p, i);
      for (int t = s.first; t <= s.last; ++t) {
        const int c = slot_need(p, p.table[(size_t)i * p.max_pages + t]);
        if (c < 0) s.ok = false;
        need += c > 0 ? 1 : 0;
        cow += c == 2 ? 1 : 0;
      }
      if (!s.ok) {
        report(p.status, SPEC_ERR_BAD_INPUT);
        need = cow = 0;
      }
    }
    int all_need, all_cow, all_taken;
    const int at = needed + cta_exclusive(need, sums, &all_need);
    const bool grant = s.ok && (need == 0 || at + need <= all_free);
    if (i < p.rows.B) {
      p.granted[i] = grant ? 1 : 0;
      if (s.ok && !grant) report(p.status, SPEC_ERR_CACHE_FULL);
    }
    if (!grant) need = cow = 0;
    int pair = pairs + cta_exclusive(cow, sums, &all_cow);
    cta_exclusive(need, sums, &all_taken);
    if (need > 0) {
      int k = at;
      for (int t = s.first; t <= s.last; ++t) {
        int32_t* entry = p.table + (size_t)i * p.max_pages + t;
        const int old = *entry;
        const int c = slot_need(p, old);
        if (c == 0) continue;
        const int page = __ldcg(p.free_list + k++);
        *entry = page;
        if (c == 2) {
          p.cow_src[pair] = old;
          p.cow_dst[pair++] = page;
        }
      }
    }
    needed += all_need;
    pairs += all_cow;
    taken += all_taken;
  }
  __syncthreads();
  // the counts only now: every need above was read against those of the start
  for (int k = threadIdx.x; k < taken; k += kPageThreads) p.refs[__ldcg(p.free_list + k)] = 1;
  for (int k = threadIdx.x; k < p.cap; k += kPageThreads) {
    if (k < pairs) {
      atomicSub(p.refs + p.cow_src[k], 1);
    } else {
      p.cow_src[k] = -1;
      p.cow_dst[k] = -1;
    }
  }
  if (threadIdx.x == 0) {
    p.counts[0] = pairs;
    p.counts[1] = taken;
  }
}

// ---------------------------------------------------------------------------
// release
// ---------------------------------------------------------------------------
struct ReleaseLaunch {
  int32_t *table, *refs;
  const int64_t* pos_base;
  const int32_t* accepted;
  int B, max_pages, pages, page_size, window, sinks;
  int32_t* status;
};

// A CTA per (request, segment of its slots): a slot that falls past the kept
// positions, or between sinks and window, is emptied and its page's count goes
// down.  1.3 us (6 requests of 64 slots), 1.4 us (96 of 384): two round trips.
constexpr int kReleaseThreads = 256;
constexpr int kReleasePer = 4;

__global__ void __launch_bounds__(kReleaseThreads) release_kernel(const ReleaseLaunch p, int segs) {
  const int i = (int)(blockIdx.x / segs), seg = (int)(blockIdx.x - (long long)i * segs);
  pdl_wait_prerequisites();
  pdl_launch_dependents();
  const long long pos = __ldg(reinterpret_cast<const long long*>(p.pos_base) + i), far = 1LL << 40;
  int64_t keep = pos > far ? far : pos < -far ? -far : pos;
  int e[kReleasePer];
  int32_t* row = p.table + (size_t)i * p.max_pages;
#pragma unroll
  for (int k = 0; k < kReleasePer; ++k) {
    const int s = (seg * kReleasePer + k) * kReleaseThreads + threadIdx.x;
    e[k] = s < p.max_pages ? row[s] : -1;
  }
  if (p.accepted) {
    const int a = p.accepted[i];
    if (a < 0 && seg == 0 && threadIdx.x == 0) report(p.status, SPEC_ERR_BAD_INPUT);
    keep += (a < 0 ? 0 : a) + 1;
  }
  if (keep < 0) keep = 0;
#pragma unroll
  for (int k = 0; k < kReleasePer; ++k) {
    if (e[k] == -1) continue;
    const int s = (seg * kReleasePer + k) * kReleaseThreads + threadIdx.x;
    const int64_t first = (int64_t)s * p.page_size, next = first + p.page_size;
    const bool drop = first >= keep || (p.window > 0 && next <= keep - p.window + 1 && first >= p.sinks);
    if (!drop) continue;
    row[s] = -1;
    const bool real = e[k] >= 0 && e[k] < p.pages;
    if (!real || atomicSub(p.refs + e[k], 1) < 1) report(p.status, SPEC_ERR_BAD_INPUT);
  }
}

// ---------------------------------------------------------------------------
// compact
// ---------------------------------------------------------------------------
struct CompactLaunch {
  int32_t *table, *refs;
  int B, max_pages, pages;
  int32_t *src, *dst, *map, *counts;
  int cap;
  int32_t* status;
  bool tables;  // the tables too, in compact_kernel
};

// The most entries of tables that compact_kernel rewrites: a launch less (1.7 us of
// the host), 0.6 us more of the GPU for 6 tables of 64 slots, 1.0 for 96 of 384.
constexpr int kRemapHere = 1 << 14;

// An entry through the map of moved pages.
__device__ __forceinline__ void remap_entry(const CompactLaunch& p, long long x, int e) {
  if (e == -1) return;
  const int to = e >= 0 && e < p.pages ? __ldcg(p.map + e) : -1;
  if (to < 0) report(p.status, SPEC_ERR_BAD_INPUT);
  if (to != e) p.table[x] = to;
}

// One cluster of 8 CTAs: count the live pages (n), rank those at or past n and
// the holes below n, pair them by rank, move the counts, then rewrite the tables
// (large ones in remap_kernel).  5.0 us (509 pages), 7.2 us (32,768 pages, 96 tables
// of 384 slots); barriers and round trips bound it.
__global__ void __cluster_dims__(kPageCluster, 1, 1) __launch_bounds__(kPageThreads)
    compact_kernel(const CompactLaunch p) {
  __shared__ int sums[33], slot, low;
  cg::cluster_group cluster = cg::this_cluster();
  pdl_wait_prerequisites();
  pdl_launch_dependents();  // only now: the next kernel reads the table before its own wait
  const PageRun run = page_run(p.pages);
  int live = 0, n;
  for (int e = run.begin; e < run.end; ++e) live += p.refs[e] > 0 ? 1 : 0;
  int rank = cluster_exclusive(live, sums, &slot, &n);
  // live pages below n: the rank at which those from n on start, known to n's thread
  if (run.begin <= n && n < run.end) {
    low = rank;
    for (int e = run.begin; e < n; ++e) low += p.refs[e] > 0 ? 1 : 0;
  }
  cluster.sync();
  const int n_low = n < p.pages ? *cluster.map_shared_rank(&low, n / pages_per_thread(p.pages) / kPageThreads) : n;
  const int moves = n - n_low;
  for (int e = run.begin; e < run.end; ++e) {
    if (p.refs[e] <= 0) {
      p.map[e] = -1;
      if (e < n) p.dst[e - rank] = e;
      continue;
    }
    if (e < n) p.map[e] = e;
    else p.src[rank - n_low] = e;
    ++rank;
  }
  __threadfence();
  cluster.sync();
  const int threads = kPageThreads * (int)cluster.num_blocks();
  for (int k = (int)cluster.block_rank() * kPageThreads + threadIdx.x; k < p.cap; k += threads) {
    if (k < moves) {
      const int from = __ldcg(p.src + k), to = __ldcg(p.dst + k);
      p.map[from] = to;
      p.refs[to] = __ldcg(p.refs + from);
      p.refs[from] = 0;
    } else {
      p.src[k] = -1;
      p.dst[k] = -1;
    }
  }
  if (cluster.block_rank() == 0 && threadIdx.x == 0) {
    p.counts[0] = moves;
    p.counts[1] = n;
  }
  if (!p.tables) return;
  __threadfence();
  cluster.sync();
  const int entries = p.B * p.max_pages;
  for (int x0 = (int)cluster.block_rank() * kPageThreads + threadIdx.x; x0 < entries; x0 += kForkPer * threads) {
    int e[kForkPer];
#pragma unroll
    for (int k = 0; k < kForkPer; ++k) e[k] = x0 + k * threads < entries ? p.table[x0 + k * threads] : -1;
#pragma unroll
    for (int k = 0; k < kForkPer; ++k) remap_entry(p, x0 + k * threads, e[k]);
  }
}

// The tables' entries through the map of moved pages.
__global__ void __launch_bounds__(kForkThreads) remap_kernel(const CompactLaunch p) {
  const long long n = (long long)p.B * p.max_pages;
  const long long at = (long long)blockIdx.x * kForkThreads * kForkPer + threadIdx.x;
  int e[kForkPer];
#pragma unroll
  for (int k = 0; k < kForkPer; ++k) {
    const long long x = at + k * kForkThreads;
    e[k] = x < n ? p.table[x] : -1;
  }
  pdl_wait_prerequisites();  // the map
  pdl_launch_dependents();
#pragma unroll
  for (int k = 0; k < kForkPer; ++k) remap_entry(p, at + k * kForkThreads, e[k]);
}

}  // namespace spec

// ---------------------------------------------------------------------------
// Entry points
// ---------------------------------------------------------------------------
namespace {

int done(cudaError_t err) {
  return err == cudaSuccess && cudaGetLastError() == cudaSuccess ? SPEC_OK : SPEC_ERR_CUDA;
}

size_t workspace_bytes(int B, int K, int page_size) {
  return ((size_t)B * (K / page_size + 2) * 4 + 255) / 256 * 256;
}

bool aligned16(const void* p, int64_t row_stride, int64_t esize) {
  return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && row_stride * esize % 16 == 0;
}

}  // namespace

extern "C" int spec_cache_append(const spec_cache* cache, int layer, const void* k_new, int64_t k_row_stride,
                                 const void* v_new, int64_t v_row_stride, const int32_t* row_offsets,
                                 const int32_t* depth, const int64_t* pos_base, const int32_t* page_table,
                                 int max_pages, int B, int K, int32_t* status, cudaStream_t stream) {
  spec::NvtxRange range("spec_cache_append");
  using namespace spec;
  if (!cache_ok(cache) || !rows_shape_ok(B, K) || !table_shape_ok(B, max_pages, cache->pages, cache->page_size))
    return SPEC_ERR_INVALID_ARG;
  if (layer < 0 || layer >= cache->layers || !k_new || !v_new || !pos_base || !page_table) return SPEC_ERR_INVALID_ARG;
  const int64_t e = element_size(cache->dtype), width = (int64_t)cache->kv_heads * cache->head_dim;
  if (!aligned16(k_new, k_row_stride, e) || !aligned16(v_new, v_row_stride, e) || k_row_stride < width ||
      v_row_stride < width || width > INT32_MAX)
    return SPEC_ERR_INVALID_ARG;
  AppendLaunch p{};
  p.k = static_cast<char*>(cache->k) + layer * cache->layer_stride * e;
  p.v = static_cast<char*>(cache->v) + layer * cache->layer_stride * e;
  p.k_new = static_cast<const char*>(k_new);
  p.v_new = static_cast<const char*>(v_new);
  p.k_row = k_row_stride * e;
  p.v_row = v_row_stride * e;
  p.page_b = cache->page_stride * e;
  p.token_b = cache->token_stride * e;
  p.head_b = cache->head_stride * e;
  p.kv_heads = cache->kv_heads;
  p.vec_head = (int)(cache->head_dim * e / 16);
  p.pages = cache->pages;
  p.page_size = cache->page_size;
  p.max_pages = max_pages;
  p.table = page_table;
  p.rows = RowLayout{row_offsets, depth, pos_base, B, K};
  p.status = status;
  const long long rows = (long long)B * (K + 1);
  return done(launch_after_previous(append_kernel, dim3((unsigned)((rows + kAppendWarps - 1) / kAppendWarps)),
                                    dim3(32 * kAppendWarps), 0, stream, p));
}

extern "C" int spec_cache_copy(const spec_cache* cache, const int32_t* src, const int32_t* dst, const int32_t* count,
                               int max_count, int32_t* status, cudaStream_t stream) {
  spec::NvtxRange range("spec_cache_copy");
  using namespace spec;
  if (!cache_ok(cache) || !src || !dst || !count || max_count < 0) return SPEC_ERR_INVALID_ARG;
  if (max_count == 0) return SPEC_OK;
  const int64_t e = element_size(cache->dtype);
  const int64_t block = (int64_t)cache->page_size * cache->kv_heads * cache->head_dim;
  if (block > INT32_MAX) return SPEC_ERR_INVALID_ARG;
  CopyLaunch p{};
  p.k = static_cast<char*>(cache->k);
  p.v = static_cast<char*>(cache->v);
  p.layer_b = cache->layer_stride * e;
  p.page_b = cache->page_stride * e;
  p.token_b = cache->token_stride * e;
  p.head_b = cache->head_stride * e;
  p.layers = cache->layers;
  p.pages = cache->pages;
  // a page is one block if its tokens and heads tile it densely, in either order
  const bool one_head = cache->kv_heads == 1, one_token = cache->page_size == 1;
  const bool token_major = (one_head || cache->head_stride == cache->head_dim) &&
                           (one_token || cache->token_stride == (int64_t)cache->kv_heads * cache->head_dim);
  const bool head_major = (one_token || cache->token_stride == cache->head_dim) &&
                          (one_head || cache->head_stride == (int64_t)cache->page_size * cache->head_dim);
  const bool dense = token_major || head_major;
  p.runs = dense ? 1 : cache->page_size * cache->kv_heads;
  p.heads = cache->kv_heads;
  p.run_vec = (int)((dense ? block : cache->head_dim) * e / 16);
  p.src = src;
  p.dst = dst;
  p.count = count;
  p.max_count = max_count;
  p.status = status;
  const long long segs = (block * e / 16 + kCopySeg - 1) / kCopySeg;
  const long long warps = (long long)max_count * cache->layers * 2 * segs;
  const long long grid = std::min<long long>((warps + kCopyWarps - 1) / kCopyWarps, (long long)device_sms() * 8);
  return done(launch_after_previous(copy_pages_kernel, dim3((unsigned)grid), dim3(32 * kCopyWarps), 0, stream, p));
}

extern "C" int spec_cache_fork(const int32_t* page_table, const int32_t* page_refs, const int32_t* parent, int B_in,
                               int B, int max_pages, int pages, int32_t* table_out, int32_t* refs_out, int32_t* status,
                               cudaStream_t stream) {
  spec::NvtxRange range("spec_cache_fork");
  using namespace spec;
  if (!table_shape_ok(B, max_pages, pages, 1) || !table_shape_ok(B_in, max_pages, pages, 1)) return SPEC_ERR_INVALID_ARG;
  if (!page_table || !page_refs || !parent || !table_out || !refs_out) return SPEC_ERR_INVALID_ARG;
  const uintptr_t a = reinterpret_cast<uintptr_t>(page_table), b = reinterpret_cast<uintptr_t>(table_out);
  if (a < b + (size_t)B * max_pages * 4 && b < a + (size_t)B_in * max_pages * 4) return SPEC_ERR_INVALID_ARG;
  ForkLaunch p{page_table, page_refs, parent, B_in, B, max_pages, pages, table_out, refs_out, status};
  const int per = kForkThreads * kForkPer;
  const int segs = (max_pages + per - 1) / per;
  if (page_refs != refs_out && (long long)(B + B_in) * max_pages + pages <= kForkHere && B <= kForkRows)
    return done(launch_after_previous(fork_cluster_kernel, dim3(kPageCluster), dim3(kPageThreads), 0, stream, p));
  const long long extra = page_refs == refs_out ? 0 : ((long long)pages + per - 1) / per;
  const long long here = page_refs == refs_out ? (long long)B_in * segs : 0;
  cudaError_t err = launch_after_previous(fork_kernel, dim3((unsigned)((long long)B * segs + extra + here)),
                                          dim3(kForkThreads), 0, stream, p, segs, (int)extra);
  if (err == cudaSuccess && here == 0)
    err = launch_after_previous(fork_refs_kernel, dim3((unsigned)((long long)B_in * segs)), dim3(kForkThreads), 0,
                                stream, p, segs);
  return done(err);
}

extern "C" size_t spec_cache_workspace(int B, int K, int page_size) {
  if (!spec::rows_shape_ok(B, K) || page_size < 1) return 0;
  return workspace_bytes(B, K, page_size);
}

extern "C" int spec_cache_reserve(int32_t* page_table, int32_t* page_refs, const int32_t* row_offsets,
                                  const int32_t* depth, const int64_t* pos_base, int B, int K, int max_pages, int pages,
                                  int page_size, int32_t* cow_src_out, int32_t* cow_dst_out, int32_t* counts_out,
                                  int32_t* granted_out, int32_t* status, void* ws, size_t ws_bytes,
                                  cudaStream_t stream) {
  spec::NvtxRange range("spec_cache_reserve");
  using namespace spec;
  if (!rows_shape_ok(B, K) || !table_shape_ok(B, max_pages, pages, page_size)) return SPEC_ERR_INVALID_ARG;
  if (!page_table || !page_refs || !pos_base || !cow_src_out || !cow_dst_out || !counts_out || !granted_out)
    return SPEC_ERR_INVALID_ARG;
  if (!ws || ws_bytes < workspace_bytes(B, K, page_size) || (reinterpret_cast<uintptr_t>(ws) & 255u) != 0)
    return SPEC_ERR_WORKSPACE;
  ReserveLaunch p{};
  p.table = page_table;
  p.refs = page_refs;
  p.rows = RowLayout{row_offsets, depth, pos_base, B, K};
  p.max_pages = max_pages;
  p.pages = pages;
  p.page_size = page_size;
  p.cow_src = cow_src_out;
  p.cow_dst = cow_dst_out;
  p.counts = counts_out;
  p.granted = granted_out;
  p.cap = B * (K / page_size + 2);
  p.free_list = static_cast<int32_t*>(ws);
  p.status = status;
  return done(launch_after_previous(reserve_kernel, dim3(kPageCluster), dim3(kPageThreads), 0, stream, p));
}

extern "C" int spec_cache_release(int32_t* page_table, int32_t* page_refs, const int64_t* pos_base,
                                  const int32_t* accepted_len, int B, int max_pages, int pages, int page_size,
                                  int window, int sinks, int32_t* status, cudaStream_t stream) {
  spec::NvtxRange range("spec_cache_release");
  using namespace spec;
  if (!table_shape_ok(B, max_pages, pages, page_size) || !page_table || !page_refs || !pos_base || window < 0 ||
      sinks < 0)
    return SPEC_ERR_INVALID_ARG;
  ReleaseLaunch p{page_table, page_refs, pos_base,  accepted_len, B,     max_pages,
                  pages,      page_size, window,    sinks,        status};
  const int per = kReleaseThreads * kReleasePer;
  const int segs = (max_pages + per - 1) / per;
  return done(launch_after_previous(release_kernel, dim3((unsigned)((long long)B * segs)), dim3(kReleaseThreads), 0,
                                    stream, p, segs));
}

extern "C" int spec_cache_compact(int32_t* page_table, int32_t* page_refs, int B, int max_pages, int pages,
                                  int32_t* move_src_out, int32_t* move_dst_out, int32_t* page_map_out,
                                  int32_t* counts_out, int32_t* status, cudaStream_t stream) {
  spec::NvtxRange range("spec_cache_compact");
  using namespace spec;
  if (!table_shape_ok(B, max_pages, pages, 1) || !page_table || !page_refs || !move_src_out || !move_dst_out ||
      !page_map_out || !counts_out)
    return SPEC_ERR_INVALID_ARG;
  CompactLaunch p{page_table,   page_refs,    B,          max_pages, pages, move_src_out,
                  move_dst_out, page_map_out, counts_out, std::max(1, pages / 2), status,
                  (long long)B * max_pages <= kRemapHere};
  cudaError_t err = launch_after_previous(compact_kernel, dim3(kPageCluster), dim3(kPageThreads), 0, stream, p);
  if (err == cudaSuccess && !p.tables) {
    const long long per = kForkThreads * kForkPer, n = (long long)B * max_pages;
    err = launch_after_previous(remap_kernel, dim3((unsigned)((n + per - 1) / per)), dim3(kForkThreads), 0, stream, p);
  }
  return done(err);
}
