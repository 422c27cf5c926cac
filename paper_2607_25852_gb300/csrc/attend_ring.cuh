// attend_ring.cuh -- what the tensor-core kernels of spec_attend share: a ring of
// K and V tiles in shared memory that one warp fills by TMA, queries that
// another brings, the share's segments that a third lists, operand descriptors,
// and the join of divided items.
#pragma once

#include <algorithm>

#include "attend.cuh"
#include "attend_tc.cuh"
#include "tensor_core.cuh"

namespace spec {

constexpr int kTile = 128;        // positions per tile: the M of S^T
constexpr int kHalfBytes = kTile * 128;  // 64 elements of 128 positions
constexpr int kMaxSlots = 12;
constexpr int kSegRing = 4;
constexpr int kBadRing = 32;      // tiles between the loader and the softmax: fewer than 2 kMaxSlots
constexpr float kGrowth = 24.0f;  // log2 of how far weights may exceed 1

struct TcPlan {
  int chunk, nchunk;    // positions per TMA box, boxes per tile and half
  int slots;            // ring slots (a K or V tile each)
  int q_off, p_off;     // bytes from the start of shared memory
  int p_bytes;          // of one buffer of weights
};

// A place in a ring and the parity of its current use, stepped without a division.
struct RingPos {
  int slot;
  uint32_t use;
  __device__ __forceinline__ void step(int n, int slots) {
    slot += n;
    if (slot >= slots) {
      slot -= slots;
      use ^= 1u;
    }
  }
};

// ---- PTX ----
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, int w,
                                            uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], "
      "[%6];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(w), "r"(smem_u32(bar))
      : "memory");
}
// mbar_wait with its loop inline: a call would cost the softmax its registers
// around every wait.
__device__ __forceinline__ bool wait_phase(uint64_t* bar, uint32_t parity, int32_t* status) {
  if (mbar_try_wait(bar, parity)) return true;
  const uint64_t t0 = global_ns();
  for (uint32_t it = 1; !mbar_try_wait(bar, parity); ++it) {
    if ((it & 255u) == 0u && global_ns() - t0 > 1000000000ull) {
      report(status, SPEC_ERR_TIMEOUT);
      return false;
    }
  }
  return true;
}
__device__ __forceinline__ void proxy_fence() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
// One lane of a converged warp.  The compiler knows elect.sync: descriptors and
// coordinates under it go to the uniform registers that MMAs and TMA take (an
// MMA issued by `lane == 0` costs 138 cycles instead).
__device__ __forceinline__ bool elect_one() {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "elect.sync _|p, 0xffffffff;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(r));
  return r != 0;
}
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool real) {
  // nothing is read where `real` is false: 16 zero bytes are written
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(real ? 16 : 0) : "memory");
}
__device__ __forceinline__ void named_sync(int id, int threads) {
  asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
}
__device__ __forceinline__ bool named_or(int id, int threads, bool x) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.u32 p, %1, 0;\n\t"
      "bar.red.or.pred q, %2, %3, p;\n\t"
      "selp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(r)
      : "r"((uint32_t)x), "r"(id), "r"(threads)
      : "memory");
  return r != 0;
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Matrix descriptors: the address (in 16-byte units) in the low word, to which
// offsets are added, above it the strides and the swizzle.
constexpr uint32_t kDescVersion = 1u << 14;
__device__ __forceinline__ uint64_t desc(uint32_t lo, uint32_t hi) {
  uint64_t d;
  asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "r"(lo), "r"(hi));
  return d;
}
// K and Q: K-major, 128-byte swizzle, 1024 bytes to the next 8 rows.
constexpr uint32_t kHiKQ = (1024u >> 4) | kDescVersion | 2u << 29;
__device__ __forceinline__ uint32_t lo_kq(uint32_t saddr) { return (saddr >> 4) | 1u << 16; }
// V as the A operand, read transposed (its d is contiguous): 128-byte swizzled
// atoms of 64 d x 8 positions; `next` bytes to the next 64 d, 1024 to the next
// 8 positions.
constexpr uint32_t kHiV = (1024u >> 4) | kDescVersion | 2u << 29;
__device__ __forceinline__ uint32_t lo_v(uint32_t saddr, uint32_t next) { return (saddr >> 4) | (next >> 4) << 16; }
constexpr uint32_t kTransposeA = 1u << 15, kTransposeB = 1u << 16;

// Two fp32 numbers in one register pair, for the packed instructions.
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pair(float x, float y) {
  f32x2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
  return r;
}
__device__ __forceinline__ float2 unpair(f32x2 p) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(p));
  return r;
}
__device__ __forceinline__ f32x2 fma2(f32x2 x, f32x2 y, f32x2 z) {
  f32x2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(x), "l"(y), "l"(z));
  return r;
}
__device__ __forceinline__ f32x2 add2(f32x2 x, f32x2 y) {
  f32x2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(x), "l"(y));
  return r;
}
__device__ __forceinline__ f32x2 mul2(f32x2 x, f32x2 y) {
  f32x2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(x), "l"(y));
  return r;
}
__device__ __forceinline__ float max3(float x, float y, float z) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(x), "f"(y), "f"(z));
  return r;
}
// Two weights as pairs of bf16 numbers: their upper halves, and the rest rounded.
__device__ __forceinline__ void split_bf16(float x, float y, uint32_t* hi, uint32_t* lo) {
  const uint32_t xb = __float_as_uint(x), yb = __float_as_uint(y);
  *hi = __byte_perm(xb, yb, 0x7632);
  const f32x2 upper = pair(__uint_as_float(xb & 0xFFFF0000u), __uint_as_float(yb & 0xFFFF0000u));
  const float2 rest = unpair(fma2(upper, pair(-1.0f, -1.0f), pair(x, y)));
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(*lo) : "f"(rest.y), "f"(rest.x));
}
__device__ __forceinline__ bool bf16_not_finite(uint32_t h) { return (h & 0x7F80u) == 0x7F80u; }

// The values of position y of a tile at `tile` before the second product: cleared
// where no row sees them, and where some rows do and some do not what is not
// finite (noted in *poison).
template <int D>
__device__ __forceinline__ void hide_values(uint8_t* tile, int y, bool any, bool all, int* poison) {
  uint8_t* row = tile + y * 128;
  if (!any) {
#pragma unroll
    for (int k = 0; k < D / 8; ++k)
      *reinterpret_cast<uint4*>(row + (k >> 3) * kHalfBytes + (((k & 7) ^ (y & 7)) << 4)) = make_uint4(0u, 0u, 0u, 0u);
  } else if (!all) {
    for (int k = 0; k < D / 8; ++k) {
      uint4* at = reinterpret_cast<uint4*>(row + (k >> 3) * kHalfBytes + (((k & 7) ^ (y & 7)) << 4));
      uint4 w = *at;
      uint32_t e[4] = {w.x, w.y, w.z, w.w};
      bool found = false;
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const bool lo = bf16_not_finite(e[x]), hi = bf16_not_finite(e[x] >> 16);
        found |= lo || hi;
        e[x] &= (lo ? 0xFFFF0000u : 0xFFFFFFFFu) & (hi ? 0x0000FFFFu : 0xFFFFFFFFu);
      }
      if (found) {
        *poison = 1;
        *at = make_uint4(e[0], e[1], e[2], e[3]);
      }
    }
  }
}

// What was cleared in shared memory for the sake of rows that must not see it has
// to be given back to those that do: calls f(position, its values) for the
// positions of the segment that some of the item's rows see and some do not, in
// order.  Those are the positions past the first row's own and, with a window,
// those that it sees and the last row does not: at most twice as many as the item
// has rows, however long the segment is.  Rare, so a plain loop over the cache,
// which all threads walk alike.
template <typename F>
__device__ __forceinline__ void for_edge_values(const AttendLaunch& a, const Segment& s, F f) {
  const int p_first = s.p + group_row(a, s.col0), p_last = s.p + group_row(a, s.col0 + s.cols - 1);
  const int left = max(0, max(a.sinks, p_first - a.window + 1)), own = max(0, p_first + 1);
  const int leaving = a.window > 0 ? max(0, min(p_first, p_last - a.window) - left + 1) : 0;
  const int all = leaving + max(0, p_last - own + 1);
#pragma unroll 1
  for (int x = 0; x < all; ++x) {
    const int pos = x < leaving ? left + x : own + x - leaving;
    const int place = position_place(s.tiles, pos), tile = place / kTile - s.tile0;
    if (place < 0 || tile < 0 || tile >= s.ntiles) continue;  // another segment's
    const int page = a.table[(size_t)s.request * a.max_pages + pos / a.page_size];
    if (page < 0 || page >= a.pages) continue;
    f(pos, reinterpret_cast<const __nv_bfloat16*>(a.v + (int64_t)page * a.page_b +
                                                  (int64_t)(pos % a.page_size) * a.token_b + s.head * a.head_b));
  }
}
// Does a row at position r see position pos?
__device__ __forceinline__ bool row_sees(const AttendLaunch& a, int r, int pos) {
  return pos <= r && (a.window == 0 || pos > r - a.window || pos < a.sinks);
}

// An item's queries into shared memory, [64-element halves][column][128 bytes]
// (`columns` of them) with the 128-byte swizzle, up to the next multiple of 16 zero: `threads` threads (a
// multiple of 32), thread i a vector of every (threads / vectors)-th column.
// The column's row and head move along without divisions.
template <int D>
__device__ __forceinline__ void load_queries(const AttendLaunch& a, const Segment& s, uint32_t dst, int columns, int i, int threads) {
  constexpr int kVecs = D / 8;
  const int N = (s.cols + 15) / 16 * 16, step = threads / kVecs, v = i % kVecs;
  int c = i / kVecs, j = group_row(a, s.col0 + c), g = s.col0 + c - j * a.G;
  const __nv_bfloat16* row = static_cast<const __nv_bfloat16*>(a.q) + (int64_t)(s.row0 + j) * a.q_row +
                             (int64_t)s.head * a.G * D + v * 8;
  uint32_t at = dst + (v >> 3) * columns * 128 + c * 128;
  for (; c < N; c += step, at += step * 128) {
    const bool real = c < s.cols;
    cp_async16(at + (((v & 7) ^ (c & 7)) << 4), real ? row + g * D : static_cast<const __nv_bfloat16*>(a.q), real);
    g += step;
    while (g >= a.G) {
      g -= a.G;
      row += a.q_row;
    }
  }
  asm volatile("cp.async.commit_group;\n\tcp.async.wait_group 0;" ::: "memory");
  proxy_fence();
}

// Adds up E vectors of four consecutive d, X parts at a time, whose loads are all
// in flight together: what a join costs is the latency of its loads, and, as it
// runs once a CTA, of fetching its instructions, so its loops are short.
template <int D, int E, int X>
__device__ __forceinline__ void add_parts(const AttendLaunch& a, const Segment& s, const long long* where,
                                          const float* weights, int c0, int nc, int tid, int threads) {
  constexpr int kQ = D / 4;
#pragma unroll 1
  for (int e0 = tid; e0 < nc * kQ; e0 += threads * E) {
    float4 o[E];
#pragma unroll
    for (int k = 0; k < E; ++k) o[k] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
    for (int x0 = 0; x0 < s.parts; x0 += X) {
      float4 w[X][E];
      float f[X][E];
#pragma unroll
      for (int y = 0; y < X; ++y) {
        const int x = min(x0 + y, s.parts - 1);
        const float4* from = reinterpret_cast<const float4*>(a.part + ((size_t)part_slot(s, x) * a.ct + c0) * D);
#pragma unroll
        for (int k = 0; k < E; ++k) {
          const int e = min(e0 + k * threads, nc * kQ - 1);
          w[y][k] = __ldcg(from + e);
          f[y][k] = x0 + y < s.parts ? weights[x * nc + e / kQ] : 0.0f;
        }
      }
#pragma unroll
      for (int y = 0; y < X; ++y)
#pragma unroll
        for (int k = 0; k < E; ++k)
          if (f[y][k] != 0.0f) {  // a part that saw nothing adds nothing
            o[k].x = fmaf(w[y][k].x, f[y][k], o[k].x);
            o[k].y = fmaf(w[y][k].y, f[y][k], o[k].y);
            o[k].z = fmaf(w[y][k].z, f[y][k], o[k].z);
            o[k].w = fmaf(w[y][k].w, f[y][k], o[k].w);
          }
    }
#pragma unroll
    for (int k = 0; k < E; ++k) {
      const int e = e0 + k * threads, c = e / kQ;
      if (c < nc) store4(static_cast<__nv_bfloat16*>(a.out) + where[c0 + c] * D + 4 * (e % kQ), o[k]);
    }
  }
}

// Adds the parts of a divided item up, in order, with `threads` threads past the
// arrival of the last part.  Groups of lanes find the weights of a column's
// parts, a part per lane; they go to `weights` (`room` floats of shared memory),
// for as many columns at a time as fit.
template <int D>
__device__ __noinline__ void join_tc(const AttendLaunch& a, const Segment& s, const long long* where, float* weights,
                                     int room, int tid, int threads) {
  const int parts = s.parts, most = max(1, room / parts);
  int group = 2;  // lanes per column: a power of two
  while (group < parts && group < 32) group *= 2;
  const int first = tid & (group - 1);
#pragma unroll 1
  for (int c0 = 0; c0 < s.cols; c0 += most) {
    const int nc = min(most, s.cols - c0);
#pragma unroll 1
    for (int b = 0; b < nc; b += threads / group) {  // all lanes stay for the shuffles
      const int c = b + tid / group;
      float m = -INFINITY, l = 0.0f;
#pragma unroll 1
      for (int x0 = 0; x0 < parts; x0 += group) {  // one round but for more than 32 parts
        const int x = x0 + first;
        const bool mine = x < parts && c < nc;
        const float2 st = mine ? __ldcg(a.part_stat + (size_t)part_slot(s, x) * a.ct + c0 + c)
                               : make_float2(-INFINITY, 0.0f);
        float mn = fmaxf(m, st.x);
#pragma unroll 1
        for (int o = group / 2; o > 0; o >>= 1) mn = fmaxf(mn, __shfl_xor_sync(0xFFFFFFFFu, mn, o));
        float sum = st.y * part_weight(st, mn);
#pragma unroll 1
        for (int o = group / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
        l = fmaf(l, part_weight(make_float2(m, l), mn), sum);
        m = mn;
        if (mine) weights[x * nc + c] = st.x;
      }
      if (c >= nc) continue;
      const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll 1
      for (int x = first; x < parts; x += group)
        weights[x * nc + c] = part_weight(make_float2(weights[x * nc + c], 0.0f), m) * inv;
      if (first == 0 && a.lse) a.lse[where[c0 + c]] = row_lse(m, l);
    }
    named_sync(1, threads);
    if (nc * (D / 4) <= threads) add_parts<D, 1, 8>(a, s, where, weights, c0, nc, tid, threads);
    else if (parts <= 2) add_parts<D, 8, 2>(a, s, where, weights, c0, nc, tid, threads);
    else add_parts<D, 4, 4>(a, s, where, weights, c0, nc, tid, threads);
    named_sync(1, threads);
  }
}

// What the warps of a CTA share beside the ring itself.
struct Control {
  uint64_t full[kMaxSlots], empty[kMaxSlots], q_full[2], q_free[2], seg_full[kSegRing], seg_free[kSegRing], drained;
  volatile int aborted;
  volatile int loaded;     // tiles that the loader has come to
  int tile_bad[kBadRing];  // per tile: the boxes whose page is not one
  int2 page[2][16];        // a tile's boxes: page, first position in it
  Segment segs[kSegRing];
};
// One thread; `readers` warps read a segment.
__device__ __forceinline__ void init_control(Control& ctl, int slots, int readers) {
  for (int k = 0; k < slots; ++k) {
    mbar_init(&ctl.full[k], 1);
    mbar_init(&ctl.empty[k], 1);
  }
  for (int k = 0; k < 2; ++k) {
    mbar_init(&ctl.q_full[k], 1);
    mbar_init(&ctl.q_free[k], 1);
  }
  for (int k = 0; k < kSegRing; ++k) {
    mbar_init(&ctl.seg_full[k], 1);
    mbar_init(&ctl.seg_free[k], readers);
  }
  mbar_init(&ctl.drained, 1);
  ctl.aborted = 0;
  ctl.loaded = 0;
}

// wait_phase for what a segment's end gives back (a place in the list, the queries'
// buffer): a segment may take longer than any fixed time, so the wait gives up once
// the loader has come to no other tile for about a second, or the CTA has given up.
__device__ __forceinline__ bool wait_segment(Control& ctl, uint64_t* bar, uint32_t parity, int32_t* status) {
  if (mbar_try_wait(bar, parity)) return true;
  uint64_t t0 = global_ns();
  int loaded = ctl.loaded;
  for (uint32_t it = 1; !mbar_try_wait(bar, parity); ++it) {
    if ((it & 255u) != 0u) continue;
    if (ctl.aborted) return false;
    const uint64_t now = global_ns();
    if (ctl.loaded != loaded) {
      loaded = ctl.loaded;
      t0 = now;
    } else if (now - t0 > 1000000000ull) {
      report(status, SPEC_ERR_TIMEOUT);
      return false;
    }
  }
  return true;
}

// The n-th segment of the share, for a reading warp.
__device__ __forceinline__ bool take_segment(const AttendLaunch& a, Control& ctl, int n, int lane, Segment* s) {
  const int k = n % kSegRing;
  const bool ok = __all_sync(0xFFFFFFFFu, wait_phase(&ctl.seg_full[k], (uint32_t)((n / kSegRing) & 1), a.status));
  *s = ctl.segs[k];
  __syncwarp();
  if (lane == 0) mbar_arrive(&ctl.seg_free[k]);
  return ok;
}

// A warp: the share's pages into the ring.
template <int D>
__device__ __forceinline__ void load_pages(const AttendLaunch& a, const TcPlan& t, Control& ctl, const CUtensorMap* tmK,
                                           const CUtensorMap* tmV, uint32_t ring, int lane) {
  constexpr int kSlot = (D / 64) * kHalfBytes;
  const int c = lane;  // the box of this lane: positions c chunk .. of a tile
  const bool mine = c < t.nchunk;
  RingPos rp{0, 1u};          // the parity of the slot's previous use
  // The ring's order is K0 K1 V0 K2 V1 ...: a tile's keys are loaded a tile
  // ahead of its values, into the place of values that are done two tiles
  // before, so that with three places the scores do not wait for the output.
  int tiles = 0, issued = 0;  // tiles whose keys, places filled (by the lane that issues)
  int v_head = 0;             // head of the tile whose values are due
  auto fill = [&](const CUtensorMap* map, int head, const int2* pages) -> bool {
    if (issued >= t.slots && !wait_phase(&ctl.empty[rp.slot], rp.use, a.status)) return false;
    mbar_expect_tx(&ctl.full[rp.slot], kSlot);
    uint32_t dst = ring + rp.slot * kSlot;
    for (int b = 0; b < t.nchunk; ++b, dst += t.chunk * 128) {
      const int2 pt = pages[b];
      tma_load_4d(dst, map, 0, head, pt.y, pt.x, &ctl.full[rp.slot]);
      if (D == 128) tma_load_4d(dst + kHalfBytes, map, 64, head, pt.y, pt.x, &ctl.full[rp.slot]);
    }
    ++issued;
    rp.step(1, t.slots);
    return true;
  };
  bool ok = true;
  for (int n = 0; ok; ++n) {
    Segment s;
    ok = take_segment(a, ctl, n, lane, &s);
    if (!ok || s.request < 0) break;
    const int p_first = s.p + group_row(a, s.col0), p_last = s.p + group_row(a, s.col0 + s.cols - 1);
    const int32_t* row = a.table + (size_t)s.request * a.max_pages;
    // does some row see this lane's positions of tile x?
    auto seen = [&](int x) {
      const int pos = place_position(s.tiles, x * kTile + c * t.chunk);
      return mine && pos <= p_last && (a.window == 0 || pos + t.chunk - 1 > p_first - a.window || pos < a.sinks);
    };
    int tok_next = 0;  // its first position in the page
    auto lookup = [&](int x) {
      const int pos = place_position(s.tiles, x * kTile + c * t.chunk), slot = pos / a.page_size;
      tok_next = pos - slot * a.page_size;
      return __ldg(row + slot);
    };
    bool wanted_next = seen(s.tile0);
    int next = wanted_next ? lookup(s.tile0) : 0;
    for (int x = 0; x < s.ntiles && ok; ++x, ++tiles) {
      int page = next;
      const int tok = wanted_next ? tok_next : 0;
      const bool wanted = wanted_next;
      if (x + 1 < s.ntiles) {  // the next tile's page, a tile ahead
        wanted_next = seen(s.tile0 + x + 1);
        next = wanted_next ? lookup(s.tile0 + x + 1) : 0;
      }
      const bool bad = wanted && (page < 0 || page >= a.pages);
      const uint32_t bads = __ballot_sync(0xFFFFFFFFu, bad);
      if (bad) report(a.status, SPEC_ERR_BAD_INPUT);
      if (bad || !wanted) page = a.pages;  // past the map's last page: zeros are written, nothing is read
      if (lane == 0) {
        ctl.tile_bad[tiles % kBadRing] = (int)bads;
        ctl.loaded = tiles;
      }
      if (mine) ctl.page[tiles & 1][c] = make_int2(page, tok);
      __syncwarp();
      if (elect_one())
        ok = !ctl.aborted && fill(tmK, s.head, ctl.page[tiles & 1]) &&
             (tiles == 0 || fill(tmV, v_head, ctl.page[(tiles - 1) & 1]));
      v_head = s.head;
      ok = __all_sync(0xFFFFFFFFu, ok);
    }
  }
  if (ok && tiles > 0) {  // the last values; no keys go before them
    if (elect_one()) {
      ok = issued < t.slots || wait_phase(&ctl.empty[rp.slot], rp.use, a.status);
      ++issued;
      rp.step(1, t.slots);
      ok = ok && fill(tmV, v_head, ctl.page[(tiles - 1) & 1]);
    }
    ok = __all_sync(0xFFFFFFFFu, ok);
  }
  if (!ok) {
    ctl.aborted = 1;
    // what was issued has landed before the CTA ends
    issued = (int)__reduce_max_sync(0xFFFFFFFFu, (unsigned)issued);
    for (int u = max(0, issued - t.slots); u < issued; ++u)
      wait_phase(&ctl.full[u % t.slots], (uint32_t)((u / t.slots) & 1), a.status);
    __syncwarp();
  }
}

// A warp: the queries of the share's segments, [64-element halves][column][128
// bytes] with the 128-byte swizzle, in QB buffers of `columns` columns from `at`.
template <int D, int QB>
__device__ __forceinline__ void stage_queries(const AttendLaunch& a, Control& ctl, uint32_t at, int columns, int lane) {
  for (int n = 0;; ++n) {
    Segment s;
    if (!take_segment(a, ctl, n, lane, &s)) {
      ctl.aborted = 1;
      break;
    }
    if (s.request < 0 || __any_sync(0xFFFFFFFFu, ctl.aborted)) break;
    const int b = n % QB;
    if (n >= QB &&
        !__all_sync(0xFFFFFFFFu, wait_segment(ctl, &ctl.q_free[b], (uint32_t)(((n / QB) - 1) & 1), a.status))) {
      ctl.aborted = 1;
      break;
    }
    if (n == 0) continue;  // the softmax warps, idle then, load the first
    load_queries<D>(a, s, at + b * columns * D * 2, columns, lane, 32);
    __syncwarp();
    if (lane == 0) mbar_arrive(&ctl.q_full[b]);
  }
}

// A thread: the share's first segment.
__device__ __forceinline__ void list_first(const AttendLaunch& a, const Share& share, Control& ctl) {
  Walk<kTile> walk(a, share);
  if (!walk.next(&ctl.segs[0])) ctl.segs[0].request = -1;
  mbar_arrive(&ctl.seg_full[0]);
}
// A thread: the share's segments, from the first (N0 = 0) or past it (N0 = 1).
template <int N0>
__device__ __forceinline__ void list_segments(const AttendLaunch& a, const Share& share, Control& ctl) {
  Walk<kTile> walk(a, share);
  if (N0 == 1) {
    Segment first;
    if (!walk.next(&first)) return;
    walk.advance();
  }
  for (int n = N0; !ctl.aborted; ++n) {
    const int k = n % kSegRing;
    if (n >= kSegRing && !wait_segment(ctl, &ctl.seg_free[k], (uint32_t)(((n / kSegRing) - 1) & 1), a.status)) {
      ctl.aborted = 1;
      break;
    }
    const bool more = walk.next(&ctl.segs[k]);
    if (!more) ctl.segs[k].request = -1;
    mbar_arrive(&ctl.seg_full[k]);
    if (!more) break;
    walk.advance();
  }
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
// One layer of K or V as [page][token][head][d], in boxes of `chunk` tokens
// of 64 elements of one head.
inline bool make_cache_map(CUtensorMap* map, const char* base, const AttendLaunch& a, int chunk) {
  auto enc = tensor_map_encoder();
  if (!enc) return false;
  cuuint64_t dims[4] = {(cuuint64_t)a.D, (cuuint64_t)a.Hkv, (cuuint64_t)a.page_size, (cuuint64_t)a.pages};
  // the stride of an extent of one is never used: any valid one
  const cuuint64_t any = (cuuint64_t)a.D * 2;
  cuuint64_t strides[3] = {a.Hkv > 1 ? (cuuint64_t)a.head_b : any, a.page_size > 1 ? (cuuint64_t)a.token_b : any,
                           a.pages > 1 ? (cuuint64_t)a.page_b : any};
  cuuint32_t box[4] = {64u, 1u, (cuuint32_t)chunk, 1u};
  cuuint32_t estr[4] = {1u, 1u, 1u, 1u};
  return enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<char*>(base), dims, strides, box, estr,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
             // a head's row is 2 D bytes: fetching more would bring in another head's
             a.D == 64 ? CU_TENSOR_MAP_L2_PROMOTION_L2_128B : CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace spec
