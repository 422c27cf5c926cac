// attend_rows.cu -- spec_attend on the 5th-generation tensor cores for many rows:
// requests with more than 144 (row, query head) columns per key-value head, as a
// chunk of a prompt has.
//
// With enough columns to fill the 128 rows of the tensor cores, the products go
// the other way round than for few (attend_tc.cu):
//   S [128 columns x 128 positions] = Q K^T     Q and K from shared memory
//   O [128 columns x D]            += P V       P from TMEM, V as it lies
// A thread of the softmax holds one column's scores of a tile: its maximum and
// sum need no other thread, and the weights go back to TMEM in place of the
// scores instead of through shared memory, whose bandwidth bounds the other
// form (there a tile of 128 positions and columns reads V twice and moves the
// weights through it: 4,000 cycles, against the tensor cores' 1,536 for the
// three products of this one).
// An item is 256 columns: two sets of 128, each with its own scores and output
// in TMEM, which share the tiles of K and V and take turns at the tensor cores.
//
// As there, a column's reference maximum is replaced only when a score exceeds
// it by 24 binary orders (then the warp rescales its rows of O in TMEM), a
// weight is the sum of two bf16 numbers (two products), what rows must not see
// is cleared in shared memory, and every wait is bounded.
//
// What it measures: 4 requests of 256 rows, 32 query heads over 8, D = 128, over
// 4,096 positions 90 us (0.76 PFLOP/s of the two products), with a window of
// 2,048 55 us; one request of 256 rows of 64 heads over 8, 16,384 positions, 156 us
// (0.88).  The weights' two halves make three products of two, so the tensor
// cores bound it at 1.26 of the measured 1.89 PFLOP/s: a tile of both sets takes
// 4,000 cycles, of which the products take 3,072; the rest is the softmax's
// 1,700 cycles a set, which the other set's products do not hide altogether.
// Beginning the second product at half of the weights cost 5 % (its issue then
// waits inside the other set's turn); reading the scores twice, to hold half of
// them in registers, cost 7 %; finding the maximum along with the weights, which
// are done again where the reference does not serve, cost 15 % (all scores stay
// live, and registers spill).
//
// Warps: 0 loads pages, 1 issues the MMAs (a set's scores of tile t + 1 right
// behind its second product of tile t, while the other set is in its softmax),
// 2 loads queries, 3 lists segments, 4 to 11 are the softmax.
#include "attend_ring.cuh"

namespace spec {

namespace {

constexpr int kSets = 2, kSetRows = 128, kItemCols = kSets * kSetRows;
constexpr int kSoftThreads = kSets * 128;
constexpr int kJoinD = 64;         // elements of a row that a join takes at a time
constexpr int kTmemCols = 512;     // scores 128 per set, then outputs D per set

__device__ __forceinline__ void tmem_ld64(uint32_t addr, float* v) {
  uint32_t r[64];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x64.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32,%33,%34,%35,%36,%37,%38,%39,%40,%41,%42,%43,%44,%45,%46,%47,%48,%49,%50,%51,%52,%53,%54,%55,%56,%57,%58,%59,%60,%61,%62,%63}, [%64];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31]), "=r"(r[32]), "=r"(r[33]), "=r"(r[34]), "=r"(r[35]), "=r"(r[36]), "=r"(r[37]), "=r"(r[38]), "=r"(r[39]), "=r"(r[40]), "=r"(r[41]), "=r"(r[42]), "=r"(r[43]), "=r"(r[44]), "=r"(r[45]), "=r"(r[46]), "=r"(r[47]), "=r"(r[48]), "=r"(r[49]), "=r"(r[50]), "=r"(r[51]), "=r"(r[52]), "=r"(r[53]), "=r"(r[54]), "=r"(r[55]), "=r"(r[56]), "=r"(r[57]), "=r"(r[58]), "=r"(r[59]), "=r"(r[60]), "=r"(r[61]), "=r"(r[62]), "=r"(r[63])
      : "r"(addr)
      : "memory");
#pragma unroll
  for (int k = 0; k < 64; ++k) v[k] = __uint_as_float(r[k]);
}
__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint32_t (&r)[16]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t addr, const float (&v)[32]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(addr), "r"(__float_as_uint(v[0])), "r"(__float_as_uint(v[1])), "r"(__float_as_uint(v[2])), "r"(__float_as_uint(v[3])), "r"(__float_as_uint(v[4])), "r"(__float_as_uint(v[5])), "r"(__float_as_uint(v[6])), "r"(__float_as_uint(v[7])), "r"(__float_as_uint(v[8])), "r"(__float_as_uint(v[9])), "r"(__float_as_uint(v[10])), "r"(__float_as_uint(v[11])), "r"(__float_as_uint(v[12])), "r"(__float_as_uint(v[13])), "r"(__float_as_uint(v[14])), "r"(__float_as_uint(v[15])), "r"(__float_as_uint(v[16])), "r"(__float_as_uint(v[17])), "r"(__float_as_uint(v[18])), "r"(__float_as_uint(v[19])), "r"(__float_as_uint(v[20])), "r"(__float_as_uint(v[21])), "r"(__float_as_uint(v[22])), "r"(__float_as_uint(v[23])), "r"(__float_as_uint(v[24])), "r"(__float_as_uint(v[25])), "r"(__float_as_uint(v[26])), "r"(__float_as_uint(v[27])), "r"(__float_as_uint(v[28])), "r"(__float_as_uint(v[29])), "r"(__float_as_uint(v[30])), "r"(__float_as_uint(v[31])) : "memory");
}
// A from TMEM: a row per lane, two consecutive elements of K in a 32-bit column.
__device__ __forceinline__ void umma_bf16_tmem(uint32_t tmem_d, uint32_t tmem_a, uint64_t b, uint32_t idesc,
                                               uint32_t accum) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(tmem_d),
      "r"(tmem_a), "l"(b), "r"(idesc), "r"(accum)
      : "memory");
}
// Bits [lo, hi] of word w of a mask.
__device__ __forceinline__ uint32_t run_bits(int lo, int hi, int w) {
  const int x = min(max(lo - 32 * w, 0), 32), y = min(max(hi + 1 - 32 * w, 0), 32);
  const uint32_t below_y = (uint32_t)((1ull << y) - 1), below_x = (uint32_t)((1ull << x) - 1);
  return below_y & ~below_x;
}

// 32 consecutive d of a row of the output.
template <int D>
__device__ __forceinline__ void store_row32(const AttendLaunch& a, long long out, int d, const float* o, float by) {
  uint4* row = reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(a.out) + out * D + d);
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    uint32_t w[4];
#pragma unroll
    for (int y = 0; y < 4; ++y) {
      const __nv_bfloat162 two = __floats2bfloat162_rn(o[8 * k + 2 * y] * by, o[8 * k + 2 * y + 1] * by);
      w[y] = *reinterpret_cast<const uint32_t*>(&two);
    }
    row[k] = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// A part's sums here lie as [slot][d / 4][column][4], so that the columns of a
// warp's lanes are side by side: column c's first four d.
template <int D>
__device__ __forceinline__ float4* part_row(const AttendLaunch& a, int slot, int c) {
  return reinterpret_cast<float4*>(a.part) + (size_t)slot * (D / 4) * a.ct + c;
}

// Adds the parts of a divided item's column up, in order, past the arrival of
// the last part: a thread per column, the loads of kJoinD elements in flight
// together.
template <int D>
__device__ __forceinline__ void join_row(const AttendLaunch& a, const Segment& s, int c, long long out) {
  float m = -INFINITY, l = 0.0f;
#pragma unroll 1
  for (int x = 0; x < s.parts; ++x) m = fmaxf(m, __ldcg(a.part_stat + (size_t)part_slot(s, x) * a.ct + c).x);
#pragma unroll 1
  for (int x = 0; x < s.parts; ++x) {
    const float2 st = __ldcg(a.part_stat + (size_t)part_slot(s, x) * a.ct + c);
    l = fmaf(st.y, part_weight(st, m), l);
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll 1
  for (int d = 0; d < D; d += kJoinD) {
    float o[kJoinD];
#pragma unroll
    for (int k = 0; k < kJoinD; ++k) o[k] = 0.0f;
#pragma unroll 1
    for (int x = 0; x < s.parts; ++x) {
      const int slot = part_slot(s, x);
      const float4* from = part_row<D>(a, slot, c) + (size_t)(d / 4) * a.ct;
      float4 w[kJoinD / 4];
#pragma unroll
      for (int k = 0; k < kJoinD / 4; ++k) w[k] = __ldcg(from + (size_t)k * a.ct);
      const float f = part_weight(__ldcg(a.part_stat + (size_t)slot * a.ct + c), m);
      if (f == 0.0f) continue;  // a part that saw nothing adds nothing
#pragma unroll
      for (int k = 0; k < kJoinD / 4; ++k) {
        o[4 * k] = fmaf(w[k].x, f, o[4 * k]);
        o[4 * k + 1] = fmaf(w[k].y, f, o[4 * k + 1]);
        o[4 * k + 2] = fmaf(w[k].z, f, o[4 * k + 2]);
        o[4 * k + 3] = fmaf(w[k].w, f, o[4 * k + 3]);
      }
    }
#pragma unroll
    for (int k = 0; k < kJoinD; k += 32) store_row32<D>(a, out, d + k, o + k, inv);
  }
  if (a.lse) a.lse[out] = row_lse(m, l);
}

template <int D>
__global__ void __launch_bounds__((4 + 4 * kSets) * 32, 1)
    attend_rows_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                       const __grid_constant__ AttendLaunch a, const __grid_constant__ TcPlan t) {
  constexpr int kSlotBytes = (D / 64) * kHalfBytes;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  __shared__ Control ctl;
  __shared__ uint64_t s_full[kSets], p_full[kSets], o_full[kSets], o_free[kSets];
  __shared__ Share share;
  __shared__ ShareSums sums;
  __shared__ uint32_t tmem_sh;
  __shared__ int poison, last_sh;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  if (tid == 0) {
    init_control(ctl, t.slots, 3 + 4 * kSets);
    for (int h = 0; h < kSets; ++h) {
      mbar_init(&s_full[h], 1);
      mbar_init(&p_full[h], 4);
      mbar_init(&o_full[h], 1);
      mbar_init(&o_free[h], 4);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_sh)),
                 "r"(kTmemCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  if (warp == 0 && lane == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmK)) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmV)) : "memory");
  }
  pdl_wait_prerequisites();
  tc_fence_before();
  find_share<kTile>(a, &share, &sums);  // ends with a barrier
  tc_fence_after();
  const uint32_t tmem = tmem_sh, tO = tmem + kSets * kTile;
  const uint32_t ring = smem_u32(smem);

  // 4 warps x 32 x 72 + 8 x 32 x 216 = 64,512 = 384 x 168 registers: neither side
  // spills (4 requests of 256 rows, 4,096 positions: 90 us; with 88 and 208 95, with
  // 56 and 224 92)
  if (warp >= 4) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
    // ---- softmax ----
    const int quad = warp & 3, h = (warp - 4) >> 2;  // TMEM lanes 32 quad .. + 31; set
    const int st = tid - 128;
    const int tl = quad * 32 + lane;  // this thread's row of the set, and the position whose values it looks after
    const int c = h * kSetRows + tl;  // its column of the item
    const uint32_t lanes = (uint32_t)(32 * quad) << 16;
    const uint32_t my_s = tmem + h * kTile + lanes, my_o = tO + h * D + lanes;
    const f32x2 c2 = pair(a.c2, a.c2);
    bool failed = false;
    int T = 0;          // tiles
    int mine = 0;       // of them with this set
    int segments = 0;   // with this set
    RingPos vp{2, 0u};  // the place of a tile's values
    auto wait = [&](uint64_t* bar, uint32_t parity) {
      if (!failed) failed = !__all_sync(0xFFFFFFFFu, wait_phase(bar, parity & 1u, a.status));
    };
    for (int n = 0;; ++n) {
      const Segment& s = ctl.segs[n % kSegRing];  // given back at the segment's end
      wait(&ctl.seg_full[n % kSegRing], n / kSegRing);
      if (named_or(1, kSoftThreads, failed)) {  // no one has left the last segment's end behind
        ctl.aborted = 1;
        if (st == 0) arrive_for_rest<kTile>(a, share, n);
        __syncwarp();
        break;
      }
      if (s.request < 0) break;
      const int cols = s.cols, ntiles = s.ntiles, tile0 = s.tile0;
      const int p_first = s.p + group_row(a, s.col0), p_last = s.p + group_row(a, s.col0 + cols - 1);
      const ItemTiles tiles = s.tiles;
      const bool active = h * kSetRows < cols, real = c < cols;
      const int r = s.p + group_row(a, s.col0 + min(c, cols - 1));  // the position of this thread's row
      if (n == 0) load_queries<D>(a, s, ring + t.q_off, kItemCols, st, kSoftThreads);
      if (st == 0) poison = 0;
      named_sync(1, kSoftThreads);
      if (n == 0 && st == 0) mbar_arrive(&ctl.q_full[0]);
      float ref = kNoMax;
      f32x2 l[4] = {0ull, 0ull, 0ull, 0ull};
      if (!active) T += ntiles;

      for (int x = 0; active && x < ntiles; ++x, ++T, ++mine) {
        const int first = (tile0 + x) * kTile, t0 = place_position(tiles, first);
        wait(&s_full[h], mine);
        tc_fence_after();
        const int bads = ctl.tile_bad[T % kBadRing];
        // do all rows see all of the tile's positions (t0 .. t0 + kTile - 1, or some sinks and some others)?
        const bool edge = !(t0 + kTile - 1 <= p_first && (first >= tiles.ns || first + kTile <= tiles.ns) &&
                            (a.window == 0 || t0 > p_last - a.window || t0 + kTile <= a.sinks)) ||
                          bads != 0;
        uint32_t seen[4] = {~0u, ~0u, ~0u, ~0u};
        if (edge) {
          // place j of the tile is position first + j among the sinks (below ja), then first + j + shift; a row sees
          // positions to r from r - window + 1, and those below sinks
          const int ja = min(max(tiles.ns - first, 0), kTile), shift = tiles.w0 - tiles.ns;
          const int from = a.window == 0 ? 0 : r - a.window + 1, sink = min(r, a.sinks - 1);
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const uint32_t low = run_bits(0, ja - 1, w);
            const int ta = first, tb = first + shift;
            const uint32_t in_a = run_bits(from - ta, r - ta, w) | run_bits(0, sink - ta, w);
            const uint32_t in_b = run_bits(from - tb, r - tb, w) | run_bits(0, sink - tb, w);
            seen[w] = (low & in_a) | (~low & in_b);
          }
          for (int k = 0; bads >> k; ++k)
            if ((bads >> k) & 1) {
#pragma unroll
              for (int w = 0; w < 4; ++w) seen[w] &= ~run_bits(k * t.chunk, (k + 1) * t.chunk - 1, w);
            }
        }
        float v[128], top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          tmem_ld64(my_s + 64 * half, v + 64 * half);
          if (edge) {
#pragma unroll
            for (int j = 0; j < 64; ++j)
              if (!((seen[2 * half + (j >> 5)] >> (j & 31)) & 1u)) v[64 * half + j] = -INFINITY;
          }
#pragma unroll
          for (int k = 0; k < 32; ++k) top[k & 3] = max3(top[k & 3], v[64 * half + 2 * k], v[64 * half + 2 * k + 1]);
        }
        const float most = fmaxf(max3(top[0], top[1], top[2]), top[3]);
        if (x == 0) {
          ref = fmaxf(most * a.c2, kNoMax);
        } else {
          const bool grow = real && fmaf(most, a.c2, -ref) > kGrowth;
          if (__any_sync(0xFFFFFFFFu, grow)) {
            // the scores came after the last tile's product: O is complete up to it
            const float next = grow ? most * a.c2 : ref, f = ex2_approx(ref - next);
            ref = next;
            const f32x2 ff = pair(f, f);
#pragma unroll
            for (int k = 0; k < 4; ++k) l[k] = mul2(l[k], ff);
#pragma unroll 1
            for (int d = 0; d < D; d += 32) {
              float o[32];
              tmem_ld32(my_o + d, o);
#pragma unroll
              for (int k = 0; k < 32; ++k) o[k] *= f;
              tmem_st32(my_o + d, o);
            }
          }
        }
        // ---- weights, split in two: upper halves in the columns of the first 64
        // scores, rests in the others' ----
        const f32x2 m = pair(-ref, -ref);
        auto weigh = [&](int q, const float (&w)[32]) {
          uint32_t hi[16], lo[16];
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const float2 d = unpair(fma2(pair(w[2 * j], w[2 * j + 1]), c2, m));
            const float x0 = ex2_approx(d.x), x1 = ex2_approx(d.y);
            l[j & 3] = add2(l[j & 3], pair(x0, x1));
            split_bf16(x0, x1, &hi[j], &lo[j]);
          }
          tmem_st16(my_s + 16 * q, hi);
          tmem_st16(my_s + 64 + 16 * q, lo);
        };
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          float w[32];
#pragma unroll
          for (int j = 0; j < 32; ++j) w[j] = v[32 * q + j];
          weigh(q, w);
        }
        if (edge && h == 0) {
          // ---- values that rows must not see: this thread's position's ----
          const int pos = place_position(tiles, first + tl);
          const bool gone = (bads >> (tl / t.chunk)) & 1;
          const bool any = !gone && pos <= p_last && (a.window == 0 || pos > p_first - a.window || pos < a.sinks);
          const bool all = !gone && pos <= p_first && (a.window == 0 || pos > p_last - a.window || pos < a.sinks);
          if (!__all_sync(0xFFFFFFFFu, all)) {
            wait(&ctl.full[vp.slot], vp.use);
            hide_values<D>(smem + vp.slot * kSlotBytes, tl, any, all, &poison);
            proxy_fence();
            __syncwarp();
          }
        }
        vp.step(2, t.slots);
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&p_full[h]);
      }

      // ---- the item's result, or this part's ----
      const int slot = s.slot;
      const bool whole = slot < 0;
      const long long out = out_index(a, s, min(c, cols - 1));
      const float2 l01 = unpair(add2(l[0], l[1])), l23 = unpair(add2(l[2], l[3]));
      const float sum = (l01.x + l01.y) + (l23.x + l23.y);
      const float top = sum == 0.0f ? -INFINITY : ref;
      const float inv = !whole ? 1.0f : sum == 0.0f ? 0.0f : 1.0f / sum;
      if (real) {
        if (!whole) a.part_stat[(size_t)slot * a.ct + c] = make_float2(top, sum);
        else if (a.lse) a.lse[out] = row_lse(top, sum);
      }
      if (active) {
        wait(&o_full[h], segments);
        ++segments;
        tc_fence_after();
      }
      named_sync(1, kSoftThreads);
      const bool poisoned = poison != 0;
#pragma unroll 1
      for (int d = 0; active && d < D; d += 32) {
        float o[32];
        __syncwarp();  // lanes without a column have skipped the last round's rest
        tmem_ld32(my_o + d, o);
        if (!real) continue;
        if (poisoned) {
          for_edge_values(a, s, [&](int pos, const __nv_bfloat16* values) {
            if (!row_sees(a, r, pos)) return;
#pragma unroll
            for (int k = 0; k < 32; k += 8) {
              const uint4 w = __ldg(reinterpret_cast<const uint4*>(values + d + k));
              const uint32_t e[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
              for (int y = 0; y < 4; ++y) {
                if (bf16_not_finite(e[y])) o[k + 2 * y] += bf16_lo(e[y]);
                if (bf16_not_finite(e[y] >> 16)) o[k + 2 * y + 1] += bf16_hi(e[y]);
              }
            }
          });
        }
        if (whole) {
          store_row32<D>(a, out, d, o, inv);
        } else {
          float4* part = part_row<D>(a, slot, c) + (size_t)(d / 4) * a.ct;
#pragma unroll
          for (int k = 0; k < 8; ++k)
            part[(size_t)k * a.ct] = make_float4(o[4 * k], o[4 * k + 1], o[4 * k + 2], o[4 * k + 3]);
        }
      }
      __syncwarp();
      tc_fence_before();
      if (lane == 0 && active) mbar_arrive(&o_free[h]);
      if (!whole) {
        named_sync(1, kSoftThreads);
        if (st == 0) last_sh = arrive_part(a, s) ? 1 : 0;
        named_sync(1, kSoftThreads);
        if (last_sh) {
          __threadfence();
          if (real) join_row<D>(a, s, c, out);
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&ctl.seg_free[n % kSegRing]);
    }
  } else {
    // The first segment goes out before the registers move, for which the softmax
    // waits: 64 requests of 32 rows of 64 heads 3 % faster (in the kernel for few
    // columns the same cost 3 % at 17 rows).
    if (warp == 3 && lane == 0) list_first(a, share, ctl);
    __syncwarp();
    asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    if (warp == 0) {
      load_pages<D>(a, t, ctl, &tmK, &tmV, ring, lane);
    } else if (warp == 1) {
      // ---- MMAs ----
      if (elect_one()) {
        constexpr uint32_t kScores = umma_idesc_bf16(kSetRows, kTile);
        constexpr uint32_t kOutputs = umma_idesc_bf16(kSetRows, D) | kTransposeB;
        constexpr uint32_t kQHalf = (uint32_t)(kItemCols * 128) >> 4;
        const uint32_t q = lo_kq(ring + t.q_off);
        bool ok = true, first_keys = true;
        int done[kSets] = {0, 0}, segments[kSets] = {0, 0};  // a set's second products, segments
        RingPos kp{0, 0u}, vp{2, 0u};  // K0 K1 V0 K2 V1 ...
        auto wait = [&](uint64_t* bar, int use) { ok = ok && wait_phase(bar, (uint32_t)use & 1u, a.status); };
        // What is added to these stays beside its use: hoisted out of the loops, two
        // sets' addresses would take more registers than the warp has.
        auto recompute = [](uint32_t& x, uint32_t& y) { asm volatile("" : "+r"(x), "+r"(y)); };
        // the scores of set h of the tile at kp; `last`: no other set's follow
        auto scores = [&](int h, bool last, bool queries_done) {
          if (h == 0) wait(&ctl.full[kp.slot], (int)kp.use);
          if (!ok) return;
          tc_fence_after();
          const uint32_t key = lo_kq(ring + kp.slot * kSlotBytes);
          uint32_t mine = q + h * ((kSetRows * 128) >> 4), to = tmem + h * kTile;
          recompute(mine, to);
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk)
            umma_bf16(to, desc(mine + (kk >> 2) * kQHalf + (((kk & 3) * 32) >> 4), kHiKQ),
                      desc(key + (((kk >> 2) * kHalfBytes + (kk & 3) * 32) >> 4), kHiKQ), kScores, kk > 0 ? 1u : 0u);
          umma_commit(&s_full[h]);
          if (last) {
            umma_commit(&ctl.empty[kp.slot]);
            if (queries_done) umma_commit(&ctl.q_free[0]);
            kp.step(first_keys ? 1 : 2, t.slots);
            first_keys = false;
          }
        };
        for (int n = 0; ok; ++n) {
          const int k = n % kSegRing;
          ok = wait_phase(&ctl.seg_full[k], (uint32_t)((n / kSegRing) & 1), a.status);
          const int request = ctl.segs[k].request, cols = ctl.segs[k].cols, ntiles = ctl.segs[k].ntiles;
          mbar_arrive(&ctl.seg_free[k]);
          if (!ok || request < 0) break;
          const int sets = cols > kSetRows ? 2 : 1;
          wait(&ctl.q_full[0], n);
#pragma unroll
          for (int h = 0; h < kSets; ++h)
            if (h < sets) scores(h, h == sets - 1, ntiles == 1);
          for (int x = 0; x < ntiles && ok; ++x) {
#pragma unroll
            for (int h = 0; h < kSets; ++h) {
              if (h >= sets) break;
              if (h == 0) wait(&ctl.full[vp.slot], (int)vp.use);
              if (x == 0 && segments[h] > 0) wait(&o_free[h], segments[h] - 1);
              wait(&p_full[h], done[h]);
              ok = ok && !ctl.aborted;
              if (!ok) break;
              tc_fence_after();
              const uint32_t v = lo_v(ring + vp.slot * kSlotBytes, D == 128 ? kHalfBytes : 0);
              uint32_t from = tmem + h * kTile, to = tO + h * D;
              recompute(from, to);
#pragma unroll
              for (int kk = 0; kk < 2 * (kTile / 16); ++kk)  // the upper halves, then the rests
                umma_bf16_tmem(to, from + 8 * kk,
                               desc(v + (kk % (kTile / 16)) * (2048 >> 4), kHiV), kOutputs, kk > 0 || x > 0 ? 1u : 0u);
              ++done[h];
              if (x == ntiles - 1) {
                umma_commit(&o_full[h]);
                ++segments[h];
              }
              if (h == sets - 1) {
                umma_commit(&ctl.empty[vp.slot]);
                vp.step(2, t.slots);
              }
              if (x + 1 < ntiles) scores(h, h == sets - 1, x + 2 == ntiles);
            }
          }
        }
        if (!ok) ctl.aborted = 1;
        // everything issued has completed before the TMEM goes
        umma_commit(&ctl.drained);
        wait_phase(&ctl.drained, 0u, a.status);
      }
      __syncwarp();
    } else if (warp == 2) {
      stage_queries<D, 1>(a, ctl, ring + t.q_off, kItemCols, lane);
    } else {
      if (lane == 0) list_segments<1>(a, share, ctl);
      __syncwarp();
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
  }
}

template <int D>
cudaError_t launch(const AttendLaunch& a, cudaStream_t stream) {
  TcPlan t{};
  t.chunk = a.grain;
  t.nchunk = kTile / t.chunk;
  constexpr int kSlot = (D / 64) * kHalfBytes, kQueries = kItemCols * D * 2;
  static std::atomic<int> known;
  int fixed;  // bytes of static shared memory
  cudaError_t err = static_smem(attend_rows_kernel<D>, known, &fixed);
  if (err != cudaSuccess) return err;
  // dynamic shared memory starts behind the static one, on a 1024-byte boundary
  // (1 KB of an SM's 228 KB is reserved per CTA)
  const int limit = 227 * 1024, room = limit - (fixed + 1023) / 1024 * 1024;
  t.slots = std::min((room - kQueries) / kSlot, kMaxSlots);
  t.q_off = t.slots * kSlot;
  const int smem = t.q_off + kQueries + limit - room - fixed;  // and the gap before it
  CUtensorMap tmK, tmV;
  if (!make_cache_map(&tmK, a.k, a, t.chunk) || !make_cache_map(&tmV, a.v, a, t.chunk)) return cudaErrorInvalidValue;
  static std::atomic<size_t> raised[kMaxDevices];
  err = raise_smem(attend_rows_kernel<D>, (size_t)smem, raised);
  if (err != cudaSuccess) return err;
  return launch_after_previous(attend_rows_kernel<D>, dim3(a.ctas), dim3((4 + 4 * kSets) * 32), (size_t)smem, stream,
                               tmK, tmV, a, t);
}

}  // namespace

cudaError_t launch_attend_rows(const AttendLaunch& a, cudaStream_t stream) {
  return a.D == 64 ? launch<64>(a, stream) : launch<128>(a, stream);
}

}  // namespace spec
