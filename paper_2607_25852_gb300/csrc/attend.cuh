// attend.cuh -- how spec_attend divides its work, and how a divided item is
// joined (shared by its kernels).
//
// An item is one key-value head of one request with up to ct of its (row,
// query head) columns; it is done in tiles of TT positions.  The lengths are
// on the device, so the division is too: the tiles of all items, one after
// another, are cut into equal ranges, one per CTA of a persistent grid.  A
// CTA's range covers whole items and at most two parts of items (its first
// and its last), so a fixed workspace of two partial results per CTA serves
// any batch, a single long request fills the GPU, and ragged batches balance.
// The last CTA to finish a part of an item adds the parts up, in CTA order.
// Two things bound how far items are divided, as a division costs the writing
// and the joining of parts: where there are no more items than CTAs, and the
// longest is little longer than an equal share, each CTA takes one item; and
// no more CTAs take part than make an item's share and its join together
// shortest.
//
// Lists.  Every key-value head has the same tiles, and the heads of a position
// lie side by side in the usual cache.  So where the CTAs divide evenly enough
// among the heads, each head is a list of its own: consecutive CTAs take
// different heads of the same positions at the same time, and the pieces they
// read make whole DRAM pages.  Otherwise one list holds the heads one after
// another.
#pragma once

#include "paged.cuh"

namespace spec {

constexpr int kAttendMaxSms = 160;  // SMs a grid uses at most; the workspace is sized for them

struct AttendLaunch {
  const void* q;
  int64_t q_row;  // elements between rows
  const char *k, *v;  // of the layer
  int64_t page_b, token_b, head_b;
  int pages, page_size, max_pages;
  int Hq, Hkv, G, D;
  uint32_t g_inverse;  // 2^32 / G, rounded up
  const int32_t* table;
  RowLayout rows;
  float c2;    // scale * log2(e)
  int window, sinks;
  int grain;          // positions of a load: a power of two that divides the page size
  void* out;
  float* lse;
  int32_t* status;
  int ct;             // columns per item
  float* part;        // [2 * ctas][ct][D] sums relative to the part's maximum
  float2* part_stat;  // [2 * ctas][ct] (maximum in log2 units, sum)
  uint32_t* arrived;  // [ctas], zero between calls
  int ctas;
  int lists;          // 1, or one per key-value head
  int part_cost, item_cost;  // tiles that dividing the items costs each CTA, and besides all CTAs per item
  float part_tiles;   // tiles in the time that the join of one more part takes
};

// The row of a column: column / G, exact for the fewer than 2^15 columns of a
// request and G <= 64 (the reciprocal is rounded up by less than G / 2^32).
__device__ __forceinline__ int group_row(const AttendLaunch& a, int column) {
  return a.G == 1 ? column : (int)__umulhi((uint32_t)column, a.g_inverse);
}

// What rows at positions p_first..p_last see, as one run of places: the sinks'
// positions 0 .. ns - 1, then the window's from w0, both in whole grains (what a
// load takes together), cut into tiles of TT.  A request that sees nothing has
// one (masked) tile, so that its rows are written.
struct ItemTiles {
  int ns, w0, count;
};
template <int TT>
__device__ __forceinline__ ItemTiles item_tiles(const AttendLaunch& a, int p_first, int p_last) {
  ItemTiles t{0, 0, 1};
  if (p_last < 0) return t;
  if (a.window > 0 && p_first >= a.window) {
    const int lo = p_first - a.window + 1;
    t.w0 = lo & -a.grain;
    t.ns = ((a.sinks < lo ? a.sinks : lo) + a.grain - 1) & -a.grain;
    if (t.ns >= t.w0) t.ns = t.w0 = 0;  // they meet: one run from 0
  }
  t.count = (t.ns + p_last - t.w0) / TT + 1;
  return t;
}
// The position at a place.
__device__ __forceinline__ int place_position(const ItemTiles& t, int place) {
  return place < t.ns ? place : place - t.ns + t.w0;
}

// And the place of a position, -1 if it has none.
__device__ __forceinline__ int position_place(const ItemTiles& t, int pos) {
  return pos < t.ns ? pos : pos < t.w0 ? -1 : pos - t.w0 + t.ns;
}

constexpr float kNoMax = -3.0e38f;  // the maximum of a column whose scores have none so far
constexpr int kNowhere = -(1 << 28);  // the position of rows that see nothing

// A request's rows as spec_attend takes them: p is kNowhere where its rows see
// nothing (idle, or positions past the table), count 0 where nothing of it
// is written.
struct AttendRows {
  int row0, count, p;
  bool bad;
};
__device__ __forceinline__ AttendRows attend_rows(const AttendLaunch& a, int i) {
  const RequestRows r = request_rows(a.rows, i);
  AttendRows o{r.row0, r.ok ? r.count : 0, kNowhere, !r.ok};
  if (r.ok && r.p > -(int64_t)(1 << 20)) {
    if (r.p + r.count > (int64_t)a.max_pages * a.page_size) o.bad = true;
    else o.p = (int)r.p;
  }
  return o;
}

// Tiles of one key-value head of a request, over its column tiles.  (2^30 positions
// make up to 2^24 tiles, 256 rows of 64 heads 512 column tiles.)
struct HeadUnits {
  long long all;       // tiles
  int items, longest;  // column tiles, tiles of the longest
};
template <int TT>
__device__ __forceinline__ int item_units(const AttendLaunch& a, const AttendRows& r, int c0) {
  const int c1 = min(r.count * a.G, c0 + a.ct) - 1;
  return item_tiles<TT>(a, r.p + group_row(a, c0), r.p + group_row(a, c1)).count;
}
template <int TT>
__device__ __forceinline__ HeadUnits head_units(const AttendLaunch& a, const AttendRows& r) {
  HeadUnits n{0, 0, 0};
  for (int c0 = 0; c0 < r.count * a.G; c0 += a.ct) {
    const int tiles = item_units<TT>(a, r, c0);
    n.all += tiles;
    n.longest = max(n.longest, tiles);
    ++n.items;
  }
  return n;
}

// A CTA's share: units [u0, u1) of its list's `units`, starting in request
// `request`, whose first unit is `base`.
struct Share {
  long long units, u0, u1, base;
  long long per;   // units of one head of the request
  int ctas, cta;   // of the list, and this one's place among them
  int request;
  AttendRows rows; // of the request
};

// x * y / z for 0 <= x < z, without a 64-bit division where 32 bits hold it.
__device__ __forceinline__ long long scale_floor(long long x, long long y, int z) {
  const long long p = x * y;
  return p < (1LL << 31) ? (long long)((uint32_t)p / (uint32_t)z) : p / z;
}

// Per warp, of its threads' requests.
struct ShareSums {
  long long units[32];
  int items[32], longest[32];
};

// All threads of the CTA (a multiple of 32, at most 1024).
template <int TT>
__device__ void find_share(const AttendLaunch& a, Share* sh, ShareSums* sums) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  const int B = a.rows.B, step = blockDim.x;
  const int heads = a.lists > 1 ? 1 : a.Hkv;  // of a list
  // pass 0: the total; pass 1: the request in which this CTA's range starts.
  // A batch of at most one request per thread does both with one scan.
  const int passes = B <= step ? 1 : 2;
  for (int pass = 0; pass < passes; ++pass) {
    long long carry = 0;
    for (int i0 = 0; i0 < B; i0 += step) {
      const int i = i0 + threadIdx.x;
      AttendRows r{0, 0, 0, false};
      HeadUnits per{0, 0, 0};
      if (i < B) {
        r = attend_rows(a, i);
        per = head_units<TT>(a, r);
        if (r.bad && pass == 0 && blockIdx.x == 0) report(a.status, SPEC_ERR_BAD_INPUT);
      }
      const long long mine = per.all * heads;
      // items are counted up to 4096 per request: exact where they are few
      const int my_items = min(per.items * heads, 4096);
      long long incl = mine;
      int incl_items = my_items;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const long long y = __shfl_up_sync(0xFFFFFFFFu, incl, o);
        const int z = __shfl_up_sync(0xFFFFFFFFu, incl_items, o);
        if (lane >= o) {
          incl += y;
          incl_items += z;
        }
      }
      const int longest_here = (int)__reduce_max_sync(0xFFFFFFFFu, (unsigned)per.longest);
      if (lane == 31) {
        sums->units[warp] = incl;
        sums->items[warp] = incl_items;
        sums->longest[warp] = longest_here;
      }
      __syncthreads();
      long long before = carry, total = carry;
      int items_before = 0, items = 0, longest = 0;
      for (int w = 0; w < warps; ++w) {
        if (w < warp) {
          before += sums->units[w];
          items_before += sums->items[w];
        }
        total += sums->units[w];
        items += sums->items[w];
        longest = max(longest, sums->longest[w]);
      }
      incl += before;
      incl_items += items_before;
      carry = total;
      if (passes == 2) __syncthreads();  // the sums may be written again
      if (pass < passes - 1) continue;
      if (passes == 2) total = sh->units;
      // this CTA's range: every thread that may hold its start works it out
      const int most = a.ctas / a.lists, c = (int)blockIdx.x / a.lists;
      int ctas = (int)(total < most ? total : most);
      long long u0 = 0, u1 = 0;
      if (passes == 1 && items > 0 && items <= most) {
        if ((longest - a.part_cost) * (long long)ctas <= total + (long long)a.item_cost * items) {
          ctas = items;  // an item each
          const int k = c - (incl_items - my_items);  // the item's place in this thread's request
          if (k >= 0 && k < my_items) {
            const int h = k / per.items;
            u0 = incl - mine + h * per.all;
            int c0 = 0;
            for (int x = h * per.items; x < k; ++x, c0 += a.ct) u0 += item_units<TT>(a, r, c0);
            sh->u0 = u0;
            sh->u1 = u0 + item_units<TT>(a, r, c0);
            sh->request = i;
            sh->base = incl - mine;
            sh->per = per.all;
            sh->rows = r;
          }
          if (threadIdx.x == 0) {
            sh->units = total;
            sh->ctas = ctas;
            sh->cta = c;
            if (c >= items) sh->u0 = sh->u1 = 0;
          }
          break;
        }
        // an item of W tiles in p parts takes W / p tiles and a join of p parts, so p
        // is at best the root of W part_tiles; then no more CTAs than the longest
        // share leaves work for
        const int few = (int)ceilf(sqrtf((float)total * (float)items * a.part_tiles));
        ctas = max(1, min(ctas, few));
        const long long share = (total + ctas - 1) / ctas;
        ctas = (int)((total + share - 1) / share);
      }
      if (c < ctas) {
        u0 = scale_floor(c, total, ctas);
        u1 = scale_floor(c + 1, total, ctas);
      }
      if (mine > 0 && incl - mine <= u0 && u0 < incl) {
        sh->request = i;
        sh->base = incl - mine;
        sh->per = per.all;
        sh->rows = r;
      }
      if (threadIdx.x == 0) {
        sh->units = total;
        sh->ctas = ctas;
        sh->cta = c;
        sh->u0 = u0;
        sh->u1 = u1;
      }
    }
    if (passes == 2 && pass == 0) {
      if (threadIdx.x == 0) sh->units = carry;
      __syncthreads();
    }
  }
  __syncthreads();
}

// A run of tiles of one item.
struct Segment {
  int request, head;   // key-value head
  int row0;            // packed row of the request's first row
  int col0, cols;      // columns (row, query head) of the item: col0 .. col0 + cols - 1
  int p;               // position of the request's first row
  ItemTiles tiles;
  int tile0, ntiles;   // the run
  int slot;            // where its partial result goes; -1: it is the whole item
  int first_cta, step, parts;  // the CTAs that share the item: first_cta, first_cta + step, ...
};

// Walks the segments of a CTA's share, one thread.
template <int TT>
struct Walk {
  const AttendLaunch& a;
  const Share& sh;
  long long u;        // next unit
  int i, h, c0, heads, list;
  AttendRows r;
  long long item;     // first unit of the item (i, h, c0)
  ItemTiles t;

  __device__ Walk(const AttendLaunch& a_, const Share& s_) : a(a_), sh(s_), u(s_.u0) {
    if (u >= sh.u1) return;
    heads = a.lists > 1 ? 1 : a.Hkv;
    list = a.lists > 1 ? (int)blockIdx.x % a.lists : 0;
    i = sh.request;
    r = sh.rows;
    h = 0;
    item = sh.base;
    while (item + sh.per <= u) {
      item += sh.per;
      ++h;
    }
    c0 = 0;
    set_tiles();
    while (item + t.count <= u) {
      item += t.count;
      c0 += a.ct;
      set_tiles();
    }
  }
  __device__ __forceinline__ void set_tiles() {
    const int cols = r.count * a.G;
    t = cols <= a.ct ? item_tiles<TT>(a, r.p, r.p + r.count - 1)
                     : item_tiles<TT>(a, r.p + group_row(a, c0), r.p + group_row(a, min(cols, c0 + a.ct) - 1));
  }
  // The CTA (of the list) whose range holds unit x.
  __device__ __forceinline__ int owner(long long x) const {
    const long long p = (x + 1) * sh.ctas - 1;
    return p < (1LL << 31) && sh.units < (1LL << 31) ? (int)((uint32_t)p / (uint32_t)sh.units) : (int)(p / sh.units);
  }

  __device__ bool next(Segment* s) {
    if (u >= sh.u1) return false;
    s->request = i;
    s->head = a.lists > 1 ? list : h;
    s->row0 = r.row0;
    s->col0 = c0;
    s->cols = min(r.count * a.G, c0 + a.ct) - c0;
    s->p = r.p;
    s->tiles = t;
    s->tile0 = (int)(u - item);
    const long long end = item + t.count;
    s->ntiles = (int)((end < sh.u1 ? end : sh.u1) - u);
    s->slot = -1;
    s->first_cta = blockIdx.x;
    s->step = a.lists;
    s->parts = 1;
    if (s->ntiles < t.count) {
      const int f = u > item ? owner(item) : sh.cta, l = end > sh.u1 ? owner(end - 1) : sh.cta;
      s->first_cta = f * a.lists + list;
      s->parts = l - f + 1;
      s->slot = 2 * (int)blockIdx.x + (sh.cta == f ? 1 : 0);
    }
    u += s->ntiles;
    return true;
  }

  // On to the next item, past a segment that `next` gave: apart from it, so that
  // the segment can be passed on before the next request's lengths are read.
  __device__ void advance() {
    if (u < sh.u1) {
      item += t.count;
      c0 += a.ct;
      if (c0 >= r.count * a.G) {
        c0 = 0;
        if (++h == heads) {
          h = 0;
          do {
            r = attend_rows(a, ++i);
          } while (r.count == 0);
        }
      }
      set_tiles();
    }
  }
};

// Slot of the x-th part of a divided item: the first CTA's part is the tail of
// its range, every other's the head.
__device__ __forceinline__ int part_slot(const Segment& s, int x) {
  return 2 * (s.first_cta + x * s.step) + (x == 0 ? 1 : 0);
}

// One thread, past the writing of a part: is it the item's last to arrive?  Then the
// counter is back at zero for the next call.
__device__ __forceinline__ bool arrive_part(const AttendLaunch& a, const Segment& s) {
  __threadfence();
  const bool last = atomicAdd(a.arrived + s.first_cta, 1u) == (uint32_t)s.parts - 1;
  if (last) a.arrived[s.first_cta] = 0;
  return last;
}

// One thread of a CTA whose wait gave up: the arrivals of the share's parts that it
// leaves out, from segment `done` on.  So every part arrives once in every call, and
// the counters are ready for the next one whatever became of this one.
template <int TT>
__device__ __noinline__ void arrive_for_rest(const AttendLaunch& a, const Share& share, int done) {
  Walk<TT> walk(a, share);
  Segment s;
  for (int n = 0; walk.next(&s); ++n) {
    if (n >= done && s.slot >= 0) arrive_part(a, s);
    walk.advance();
  }
}

// Where column c of a segment goes: packed row * Hq + query head.
__device__ __forceinline__ long long out_index(const AttendLaunch& a, const Segment& s, int c) {
  const int col = s.col0 + c, j = group_row(a, col);
  return (long long)(s.row0 + j) * a.Hq + s.head * a.G + (col - j * a.G);
}

constexpr float kLn2 = 0.69314718055994531f;

// A row's log-sum-exp from its maximum (log2 units) and sum; -inf where it saw
// nothing.
__device__ __forceinline__ float row_lse(float m2, float l) { return l == 0.0f ? -INFINITY : (m2 + log2f(l)) * kLn2; }

template <typename T>
__device__ __forceinline__ T from_float(float x);
template <>
__device__ __forceinline__ float from_float<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16(x); }

__device__ __forceinline__ void store4(float* p, float4 v) { *reinterpret_cast<float4*>(p) = v; }
__device__ __forceinline__ void store4(__nv_bfloat16* p, float4 v) {
  const __nv_bfloat162 lo = __floats2bfloat162_rn(v.x, v.y), hi = __floats2bfloat162_rn(v.z, v.w);
  *reinterpret_cast<uint2*>(p) =
      make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
}

// The weight of a part in its row's sum.
__device__ __forceinline__ float part_weight(float2 st, float m) {
  return st.x == -INFINITY ? 0.0f : exp2f(st.x - m);
}

// Adds the parts of a divided item up, in order: `threads` threads, `tid` of
// them, all of them past the arrival of the last part.  A thread takes four
// consecutive d of a column and eight parts at a time, whose loads are all in
// flight together: it is the latency of these loads that a join costs.
template <typename T>
__device__ void join_parts(const AttendLaunch& a, const Segment& s, int tid, int threads) {
  constexpr int kBatch = 8;
  const int dv = a.D / 4;
  for (int e = tid; e < s.cols * dv; e += threads) {
    const int c = e / dv, d = 4 * (e - c * dv);
    float m = -INFINITY, l = 0.0f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int x0 = 0; x0 < s.parts; x0 += kBatch) {
      float2 st[kBatch];
      float4 w[kBatch];
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        st[k] = make_float2(-INFINITY, 0.0f);
        if (x0 + k < s.parts) {
          const size_t at = (size_t)part_slot(s, x0 + k) * a.ct + c;
          st[k] = __ldcg(a.part_stat + at);
          w[k] = __ldcg(reinterpret_cast<const float4*>(a.part + at * a.D + d));
        }
      }
      float mb = m;
#pragma unroll
      for (int k = 0; k < kBatch; ++k) mb = fmaxf(mb, st[k].x);
      const float old = part_weight(make_float2(m, l), mb);
      l *= old;
      o = make_float4(o.x * old, o.y * old, o.z * old, o.w * old);
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        if (st[k].x == -INFINITY) continue;  // a part that saw nothing (or does not exist) adds nothing
        const float f = part_weight(st[k], mb);
        l = fmaf(st[k].y, f, l);
        o.x = fmaf(w[k].x, f, o.x);
        o.y = fmaf(w[k].y, f, o.y);
        o.z = fmaf(w[k].z, f, o.z);
        o.w = fmaf(w[k].w, f, o.w);
      }
      m = mb;
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    const long long at = out_index(a, s, c);
    store4(static_cast<T*>(a.out) + at * a.D + d, make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv));
    if (d == 0 && a.lse) a.lse[at] = row_lse(m, l);
  }
}

}  // namespace spec
