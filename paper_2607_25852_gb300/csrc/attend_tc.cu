// attend_tc.cu -- spec_attend on the 5th-generation tensor cores: bf16 caches
// of head dimension 64 or 128 whose pages are a multiple of 8 positions, for up
// to 144 (row, query head) columns per key-value head (attend_rows.cu: more).
//
// The few columns (row, query head) that share a key-value head are the N
// dimension of both products, so their cost follows their number, and the
// positions of the cache fill the 128 rows of the tensor cores:
//   S^T [128 positions x N] = K Q^T        K from shared memory as it lies
//   O^T [D x N]            += V^T P^T      V as it lies, read transposed
// S^T and O^T live in TMEM, a position (or a d) per lane, a column per TMEM
// column.  A thread of the softmax holds one position's scores: the weights
// are elementwise, and the maximum over positions is looked at only for a
// bound: as long as no score exceeds its column's reference maximum by more
// than 24 binary orders, the old reference serves (weights stay below 2^24,
// far from any overflow and with the same relative precision), so most tiles
// need one vote and no reduction, no rescaling of O^T and no exchange between
// warps.
// The sum of the weights is kept per thread, in fp32, and reduced once per
// item.  For the second product a weight is the sum of two bf16 numbers, its
// upper 8 bits and the rounded rest (2^-16 relative: the rest is below 2^-7 of it,
// and keeps 8 bits): one bf16 number would
// put an error of the size of the result's own rounding on top of it.  The two
// are columns of one product of twice the width, whose two results the item's
// end adds: a product of 128 rows and 16 steps costs 65 cycles up to N = 32 and
// 79 at N = 144 (it is the reading of V that it costs), so the width is free
// where few columns share a head.
//
// Warps: 0 loads pages by TMA into a ring of K and V tiles; 1 issues the MMAs
// (the scores of tile t + 1 before the second product of tile t); 2 loads
// queries; 3 lists the CTA's share of the work; the rest are the softmax, one
// TMEM lane quarter per warp, in one set or in two that halve the columns and
// take turns at two buffers of the weights.
//
// Positions that no row sees must not reach the result whatever they hold: a
// weight of 0 does not cancel an infinite or NaN value, so in tiles at an edge
// of the mask such values are cleared in shared memory before the product
// (a value that some rows see and others do not is added back, row by row, in
// the item's epilogue: only if it is not finite).
//
// Every mbarrier wait is bounded (about a second; what a segment's end gives back,
// a second in which no tile was loaded): a wait that gives up sets SPEC_ERR_TIMEOUT
// and the kernel ends; the softmax warps, which meet at barriers, leave together by
// a vote and arrive for the parts that the CTA leaves out.
//
// What it measures, 64 requests of 64 query heads over 8, D = 128, 4,096
// positions each: 1 row 167 us (6.4 TB/s, 0.95 of the measured copy peak), 4 rows
// 171, 8 rows 184, 12 rows 195 (5.5 TB/s), 17 rows 249 us (4.3 TB/s).  Up to 12
// rows HBM bounds it; at 17 the chain from scores to weights to output: a tile
// takes 2.1 us where its bytes take 1.5, shared memory is 76 % busy (the MMAs'
// operands 33, the softmax 31, arriving tiles 12) and two softmax warps per
// scheduler issue 38 % of the time.  Short runs are bound by what comes before
// the first tile (8 us) and after the last (4 to 10 with a join).
#include "attend_ring.cuh"

namespace spec {

namespace {

// Items of few columns and small tiles go two CTAs to an SM: a CTA's chain from
// scores to weights to output is longer than the time its tile takes to arrive,
// and the ends of its items leave the loads idle.  (With D = 128 the tiles are
// twice as large: one CTA's chain keeps up, and two would not have three tiles'
// room each.)  Two / one, us: a token of 128 requests, 64 heads over 8, window of
// 1,024: 70 / 89; of 64 requests over 4,096 positions: 94 / 122.
constexpr bool two_per_sm(int D, int CG) { return D == 64 && CG == 2; }
__device__ __forceinline__ void tmem_ld8(uint32_t addr, float* v) {
  uint32_t r[8];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
      : "r"(addr)
      : "memory");
#pragma unroll
  for (int k = 0; k < 8; ++k) v[k] = __uint_as_float(r[k]);
}
__device__ __forceinline__ void tmem_ld16(uint32_t addr, float* v) {
  uint32_t r[16];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(addr)
      : "memory");
#pragma unroll
  for (int k = 0; k < 16; ++k) v[k] = __uint_as_float(r[k]);
}
__device__ __forceinline__ void tmem_ld48(uint32_t addr, float* v) {
  uint32_t r[48];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%48];\n\t"
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%32,%33,%34,%35,%36,%37,%38,%39,%40,%41,%42,%43,%44,%45,%46,%47}, [%49];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31]), "=r"(r[32]), "=r"(r[33]), "=r"(r[34]), "=r"(r[35]), "=r"(r[36]), "=r"(r[37]), "=r"(r[38]), "=r"(r[39]), "=r"(r[40]), "=r"(r[41]), "=r"(r[42]), "=r"(r[43]), "=r"(r[44]), "=r"(r[45]), "=r"(r[46]), "=r"(r[47])
      : "r"(addr), "r"(addr + 32)
      : "memory");
#pragma unroll
  for (int k = 0; k < 48; ++k) v[k] = __uint_as_float(r[k]);
}
__device__ __forceinline__ void tmem_ld72(uint32_t addr, float* v) {
  uint32_t r[72];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x64.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32,%33,%34,%35,%36,%37,%38,%39,%40,%41,%42,%43,%44,%45,%46,%47,%48,%49,%50,%51,%52,%53,%54,%55,%56,%57,%58,%59,%60,%61,%62,%63}, [%72];\n\t"
      "tcgen05.ld.sync.aligned.32x32b.x8.b32 {%64,%65,%66,%67,%68,%69,%70,%71}, [%73];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31]), "=r"(r[32]), "=r"(r[33]), "=r"(r[34]), "=r"(r[35]), "=r"(r[36]), "=r"(r[37]), "=r"(r[38]), "=r"(r[39]), "=r"(r[40]), "=r"(r[41]), "=r"(r[42]), "=r"(r[43]), "=r"(r[44]), "=r"(r[45]), "=r"(r[46]), "=r"(r[47]), "=r"(r[48]), "=r"(r[49]), "=r"(r[50]), "=r"(r[51]), "=r"(r[52]), "=r"(r[53]), "=r"(r[54]), "=r"(r[55]), "=r"(r[56]), "=r"(r[57]), "=r"(r[58]), "=r"(r[59]), "=r"(r[60]), "=r"(r[61]), "=r"(r[62]), "=r"(r[63]), "=r"(r[64]), "=r"(r[65]), "=r"(r[66]), "=r"(r[67]), "=r"(r[68]), "=r"(r[69]), "=r"(r[70]), "=r"(r[71])
      : "r"(addr), "r"(addr + 64)
      : "memory");
#pragma unroll
  for (int k = 0; k < 72; ++k) v[k] = __uint_as_float(r[k]);
}
__device__ __forceinline__ void tmem_st8(uint32_t addr, const float* v) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(addr),
               "r"(__float_as_uint(v[0])), "r"(__float_as_uint(v[1])), "r"(__float_as_uint(v[2])),
               "r"(__float_as_uint(v[3])), "r"(__float_as_uint(v[4])), "r"(__float_as_uint(v[5])),
               "r"(__float_as_uint(v[6])), "r"(__float_as_uint(v[7]))
               : "memory");
}
// P^T as the B operand, a position's columns contiguous: 32-byte swizzled atoms
// of 16 columns x 8 positions; 4096 bytes to the next 16 columns, 256 to the
// next 8 positions.
constexpr int kPChunkBytes = kTile * 32;
constexpr uint32_t kHiP = (256u >> 4) | kDescVersion | 6u << 29;
__device__ __forceinline__ uint32_t lo_p(uint32_t saddr) { return (saddr >> 4) | (uint32_t)(kPChunkBytes >> 4) << 16; }
// Four pairs of shared memory.
__device__ __forceinline__ void load_pairs(f32x2 (&p)[4], const float* at) {
  const ulonglong2 a = *reinterpret_cast<const ulonglong2*>(at), b = *reinterpret_cast<const ulonglong2*>(at + 4);
  p[0] = a.x; p[1] = a.y; p[2] = b.x; p[3] = b.y;
}
__device__ __forceinline__ void load_rows(int (&r)[8], const int* rows) {
  const int4 a = *reinterpret_cast<const int4*>(rows), b = *reinterpret_cast<const int4*>(rows + 4);
  r[0] = a.x; r[1] = a.y; r[2] = a.z; r[3] = a.w;
  r[4] = b.x; r[5] = b.y; r[6] = b.z; r[7] = b.w;
}
// Not ordered with loads from other places (nothing reads the weights' buffer
// back): only with other volatile statements, the fence among them.
__device__ __forceinline__ void st_shared16_if(bool yes, uint32_t at, const uint32_t (&w)[4]) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.u32 p, %0, 0;\n\t"
      "@p st.shared.v4.b32 [%1], {%2,%3,%4,%5};\n\t}" ::"r"((uint32_t)yes),
      "r"(at), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]));
}
// Columns of each softmax set, for an item of N (a multiple of 16).
template <int H>
__device__ __forceinline__ int set_cols(int N) {
  return N / H;
}
// Column sums over a warp's lanes of 8 values per lane: afterwards lanes 4k
// hold the sum of column k.
__device__ __forceinline__ float column_sum8(float (&v)[8], int lane) {
#pragma unroll
  for (int n = 8, o = 16; n > 1; n >>= 1, o >>= 1) {
    const bool hi = (lane & o) != 0;
#pragma unroll
    for (int j = 0; j < n / 2; ++j) {
      const float send = hi ? v[j] : v[j + n / 2];
      const float keep = hi ? v[j + n / 2] : v[j];
      v[j] = keep + __shfl_xor_sync(0xFFFFFFFFu, send, o);
    }
  }
  v[0] += __shfl_xor_sync(0xFFFFFFFFu, v[0], 2);
  v[0] += __shfl_xor_sync(0xFFFFFFFFu, v[0], 1);
  return v[0];  // column 4 * bit4 + 2 * bit3 + bit2 = lane / 4
}


// ---------------------------------------------------------------------------
// D: head dimension.  CG: groups of 8 columns per softmax thread.  H: sets of
// four softmax warps (they split the columns).
// ---------------------------------------------------------------------------
template <int D, int CG, int H>
__global__ void __launch_bounds__((4 + 4 * H) * 32, two_per_sm(D, CG) ? 2 : 1)
    attend_tc_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                     const __grid_constant__ AttendLaunch a, const __grid_constant__ TcPlan t) {
  constexpr int kSetCols = CG * 8;          // most columns of a set
  constexpr int kCols = H * kSetCols;       // and of an item
  constexpr int kSlotBytes = (D / 64) * kHalfBytes;
  // Two buffers of scores where they fit (else one: the scores are in registers
  // before the next tile's are due), two of weights.
  constexpr int SB = CG <= 6 ? 2 : 1, PB = 2, QB = H == 1 && !two_per_sm(D, CG) ? 2 : 1;
  constexpr int kScores = (kCols + 31) / 32 * 32, kOut = SB * kScores;  // TMEM columns; then per set 2 kSetCols of O^T
  constexpr int kTmemCols = H == 1 ? 128 : 512;
  static_assert(kOut + 2 * kCols <= kTmemCols, "scores and outputs fit TMEM");
  constexpr int kSoftThreads = 128 * H;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  __shared__ Control ctl;
  __shared__ uint64_t s_full[2], s_free[2], p_full[2], p_free[4], o_free;
  __shared__ Share share;
  __shared__ ShareSums sums;
  // per set and column: the reference's negative (-inf: no column), a factor, maxima and sums per warp
  __shared__ __align__(16) float sN[kCols], sF[kCols], red[4][kCols];
  __shared__ __align__(16) int sRow[kCols];        // position of the column's row
  __shared__ long long sOut[kCols];  // where the column goes
  __shared__ uint32_t tmem_sh;
  __shared__ int poison, last_sh;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  if (tid == 0) {
    init_control(ctl, t.slots, 3 + 4 * H);
    for (int k = 0; k < 2; ++k) {
      mbar_init(&s_full[k], 1);
      mbar_init(&s_free[k], 4 * H);
      mbar_init(&p_full[k], 4);
      mbar_init(&p_free[k], 1);
      mbar_init(&p_free[2 + k], 1);
    }
    mbar_init(&o_free, 4 * H);
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
  const uint32_t tmem = tmem_sh;
  const uint32_t tO = tmem + kOut;
  const uint32_t ring = smem_u32(smem);

  // Two softmax sets need more than the 168 registers a thread that 384 threads
  // get: 4 warps x 32 x 56 + 8 x 32 x 224 = 64,512 = 384 x 168.
  if (warp >= 4) {
    if constexpr (H == 2) asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");
    // ---- softmax ----
    const int quad = warp & 3, hf = (warp - 4) >> 2;  // TMEM lanes 32 quad .. + 31; column set
    const int st = tid - 128;                         // of kSoftThreads
    const int tl = quad * 32 + lane;                  // this thread's position in a tile, and its d of O^T
    const uint32_t lanes = (uint32_t)(32 * quad) << 16;
    const f32x2 c2 = pair(a.c2, a.c2);
    float *const ref = sN + hf * kSetCols, *const factor = sF + hf * kSetCols;  // this set's
    bool failed = false;
    int T = 0;
    int U = 0;       // units (tile, set) before this tile
    int mine_u = 0;  // this set's last unit
    float neg_lowest = 0.0f;  // the negative of this set's lowest reference
    RingPos vp{2, 0u};  // the place of a tile's values
    auto wait = [&](uint64_t* bar, uint32_t parity) {
      // by vote: the lanes leave their loops together, before what a whole warp has to execute as one
      if (!failed) failed = !__all_sync(0xFFFFFFFFu, wait_phase(bar, parity & 1u, a.status));
    };
    // The second product of unit u.  A wait by parity must not come two phases
    // early: with four barriers in turn that would be before unit u - 4 is done,
    // and who waits for u knows of u - 2 H or later.
    auto wait_unit = [&](int u) { wait(&p_free[u & 3], (uint32_t)u >> 2); };
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
      const int p_first = s.p + group_row(a, s.col0), p_last = s.p + group_row(a, s.col0 + s.cols - 1), ntiles = s.ntiles;
      const int cols = s.cols, N = (cols + 15) / 16 * 16, wide = set_cols<H>(N);
      const int cb = hf * wide, gc = wide / 8;  // this set's columns: gc groups of 8 from cb
      const ItemTiles tiles = s.tiles;
      const int tile0 = s.tile0;
      if (n == 0) load_queries<D>(a, s, ring + t.q_off, a.ct, st, kSoftThreads);
      for (int c = st; c < N; c += kSoftThreads) {
        const int cc = min(c, cols - 1);
        sRow[c + (c >= wide ? kSetCols - wide : 0)] = s.p + group_row(a, s.col0 + cc);
        sOut[c] = out_index(a, s, cc);
      }
      if (tl < kSetCols) ref[tl] = tl < gc * 8 ? -kNoMax : -INFINITY;
      if (st == 0) poison = 0;
      named_sync(1, kSoftThreads);
      if (n == 0 && st == 0) mbar_arrive(&ctl.q_full[0]);
      f32x2 l[CG * 4];
#pragma unroll
      for (int j = 0; j < CG * 4; ++j) l[j] = 0ull;

      for (int x = 0; x < ntiles; ++x, ++T) {
        const int b = T % SB, first = (tile0 + x) * kTile, t0 = place_position(tiles, first);
        wait(&s_full[b], T / SB);
        tc_fence_after();
        const int bads = ctl.tile_bad[T % kBadRing];
        // do all rows see all of the tile's positions (t0 .. t0 + kTile - 1, or some sinks and some others)?
        const bool edge = !(t0 + kTile - 1 <= p_first && (first >= tiles.ns || first + kTile <= tiles.ns) &&
                            (a.window == 0 || t0 > p_last - a.window || t0 + kTile <= a.sinks)) ||
                          bads != 0;
        const int pos = place_position(tiles, first + tl);
        const bool gone = edge && (bads >> (tl / t.chunk)) & 1;
        // scores; -inf where masked.  Columns past this set's are whatever TMEM
        // holds: their reference makes every weight of theirs 0 (or NaN), and
        // nothing of it is stored.
        float v[CG * 8];
        {
          const uint32_t at = tmem + b * kScores + lanes + cb;
          if constexpr (CG == 2) tmem_ld16(at, v);
          else if constexpr (CG == 4) tmem_ld32(at, v);
          else if constexpr (CG == 6) tmem_ld48(at, v);
          else tmem_ld72(at, v);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&s_free[b]);
        if (edge) {
#pragma unroll
          for (int g = 0; g < CG; ++g) {
            int r[8];
            load_rows(r, sRow + hf * kSetCols + g * 8);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const bool seen = pos <= r[j] && (a.window == 0 || pos > r[j] - a.window || pos < a.sinks) && !gone;
              if (!seen) v[8 * g + j] = -INFINITY;
            }
          }
        }
        // ---- does a score exceed its column's reference by too much?  First the
        // largest of the thread's scores against the lowest reference, which
        // nearly always says no; then each against its own ----
        bool grow = x == 0;
        if (x > 0) {
          float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int k = 0; k < CG * 4; ++k) top[k & 3] = max3(top[k & 3], v[2 * k], v[2 * k + 1]);
          const float most = fmaxf(max3(top[0], top[1], top[2]), top[3]);
          if (named_or(2 + hf, 128, fmaf(most, a.c2, neg_lowest) > kGrowth || failed)) {
            float far = -INFINITY;
#pragma unroll
            for (int g = 0; g < CG; ++g) {
              f32x2 m[4];
              load_pairs(m, ref + g * 8);
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const float2 d = unpair(fma2(pair(v[8 * g + 2 * j], v[8 * g + 2 * j + 1]), c2, m[j]));
                far = max3(far, d.x, d.y);
              }
            }
            grow = named_or(2 + hf, 128, far > kGrowth || failed);
          }
        }
        if (grow) {
          // new references: the columns' maxima so far
#pragma unroll
          for (int g = 0; g < CG; ++g) {
            float mine = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const float r = warp_max(v[8 * g + j]);
              if (lane == j) mine = r * a.c2;
            }
            if (lane < 8) red[quad][hf * kSetCols + g * 8 + lane] = mine;
          }
          named_sync(2 + hf, 128);
          if (tl < gc * 8) {
            const int c = hf * kSetCols + tl;
            const float old = -ref[tl];
            const float m = fmaxf(old, fmaxf(fmaxf(red[0][c], red[1][c]), fmaxf(red[2][c], red[3][c])));
            factor[tl] = ex2_approx(old - m);
            ref[tl] = -m;
          }
          if (x > 0) wait_unit(mine_u);  // O^T is complete up to the last tile
          failed = named_or(2 + hf, 128, failed);
          neg_lowest = -INFINITY;
          for (int c = 0; c < gc * 8; ++c) neg_lowest = fmaxf(neg_lowest, ref[c]);
          if (x > 0) {
            tc_fence_after();
#pragma unroll
            for (int g = 0; g < CG; ++g) {
              if (g >= gc) break;
              f32x2 f[4];
              float o[8];
              load_pairs(f, factor + g * 8);
#pragma unroll
              for (int j = 0; j < 4; ++j) l[4 * g + j] = mul2(l[4 * g + j], f[j]);
#pragma unroll
              for (int part = 0; part < 2; ++part) {
                const uint32_t at = tO + lanes + hf * 2 * kSetCols + part * gc * 8 + g * 8;
                tmem_ld8(at, o);
#pragma unroll
                for (int j = 0; j < 8; ++j) o[j] *= factor[g * 8 + j];
                tmem_st8(at, o);
              }
            }
            tmem_st_wait();
            tc_fence_before();
          }
        }
        // ---- weights, split in two, stored as they come.  Their buffer's last reader
        // is unit u - 2; with one set its product was issued before this tile's
        // scores, so those say that it is done.  (Keeping the weights in registers
        // until the buffer is free cost 6 % at 48 columns a thread.) ----
        const int u = U + hf;
        mine_u = u;
        if (H > 1 && u >= PB) wait_unit(u - PB);
        const uint32_t pw = ring + t.p_off + (u % PB) * t.p_bytes + tl * 32;
        const uint32_t swap = (uint32_t)((tl >> 2) & 1) << 4;
#pragma unroll
        for (int g = 0; g < CG; ++g) {
          f32x2 m[4];
          load_pairs(m, ref + g * 8);
          uint32_t hi[4], lo[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float2 d = unpair(fma2(pair(v[8 * g + 2 * j], v[8 * g + 2 * j + 1]), c2, m[j]));
            const float x0 = ex2_approx(d.x), x1 = ex2_approx(d.y);
            l[4 * g + j] = add2(l[4 * g + j], pair(x0, x1));
            split_bf16(x0, x1, &hi[j], &lo[j]);
          }
          const int r = gc + g;  // the rests' groups follow the upper halves'
          st_shared16_if(g < gc, pw + (g >> 1) * kPChunkBytes + (((uint32_t)(g & 1) << 4) ^ swap), hi);
          st_shared16_if(g < gc, pw + (r >> 1) * kPChunkBytes + (((uint32_t)(r & 1) << 4) ^ swap), lo);
        }
        U += H;
        if (edge && hf == 0) {
          // ---- values that rows must not see ----
          // seen by the last row alone or by the first alone: between the two
          const bool any = !gone && pos <= p_last && (a.window == 0 || pos > p_first - a.window || pos < a.sinks);
          const bool all = !gone && pos <= p_first && (a.window == 0 || pos > p_last - a.window || pos < a.sinks);
          if (!__all_sync(0xFFFFFFFFu, all)) {
            wait(&ctl.full[vp.slot], vp.use);
            hide_values<D>(smem + vp.slot * kSlotBytes, tl, any, all, &poison);
          }
        }
        vp.step(2, t.slots);
        proxy_fence();
        __syncwarp();
        if (lane == 0) mbar_arrive(&p_full[u & 1]);
      }

      // ---- the item's result, or this part's ----
#pragma unroll
      for (int g = 0; g < CG; ++g) {
        float mine[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 w = unpair(l[4 * g + j]);
          mine[2 * j] = w.x;
          mine[2 * j + 1] = w.y;
        }
        const float sum = column_sum8(mine, lane);
        if ((lane & 3) == 0) red[quad][hf * kSetCols + g * 8 + (lane >> 2)] = sum;
      }
      const int slot = s.slot;
      const bool whole = slot < 0;
      named_sync(2 + hf, 128);
      if (tl < gc * 8 && cb + tl < cols) {
        const int c = hf * kSetCols + tl;
        const float sum = (red[0][c] + red[1][c]) + (red[2][c] + red[3][c]);
        const float m = sum == 0.0f ? -INFINITY : -ref[tl];
        factor[tl] = whole ? (sum == 0.0f ? 0.0f : 1.0f / sum) : 1.0f;
        if (!whole) a.part_stat[(size_t)slot * a.ct + cb + tl] = make_float2(m, sum);
        else if (a.lse) a.lse[sOut[cb + tl]] = row_lse(m, sum);
      }
      wait_unit(mine_u);
      tc_fence_after();
      named_sync(1, kSoftThreads);
      const bool poisoned = poison != 0;
      // sixteen columns at a time, this thread's d = tl of each; a whole item's rows
      // go through the weights' buffer (every product of the segment is complete),
      // so that they are stored 16 bytes a thread
      __nv_bfloat16* staged = reinterpret_cast<__nv_bfloat16*>(smem + t.p_off + hf * t.p_bytes);
#pragma unroll 1
      for (int g = 0; g < gc; g += 2) {
        float o[16], rest[16];
        const uint32_t at = tO + lanes + hf * 2 * kSetCols + g * 8;
        tmem_ld16(at, o);
        tmem_ld16(at + gc * 8, rest);
        if (D < 128 && tl >= D) continue;
        const int c0 = cb + g * 8, nc = min(cols, cb + gc * 8) - c0;
#pragma unroll
        for (int j = 0; j < 16; ++j) o[j] += rest[j];
        if (poisoned) {
          const int* rows = sRow + hf * kSetCols + g * 8;
          for_edge_values(a, s, [&](int pos, const __nv_bfloat16* values) {
            const float add = load_elem(values + tl);
            if (isfinite(add)) return;
#pragma unroll
            for (int j = 0; j < 16; ++j)
              if (j < nc && row_sees(a, rows[j], pos)) o[j] += add;
          });
          __syncwarp();
        }
        if (whole) {
          __nv_bfloat16* row = staged + g * 8 * D + tl;
#pragma unroll
          for (int j = 0; j < 16; ++j)
            if (j < nc) row[j * D] = __float2bfloat16(o[j] * factor[g * 8 + j]);
        } else {
          float* part = a.part + ((size_t)slot * a.ct + c0) * D + tl;
#pragma unroll
          for (int j = 0; j < 16; ++j)
            if (j < nc) part[j * D] = o[j];
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&o_free);
      if (whole) {
        named_sync(2 + hf, 128);
        const int nv = max(0, min(cols - cb, gc * 8)) * (D / 8);
#pragma unroll 4
        for (int e = tl; e < nv; e += 128) {
          const int c = e / (D / 8);
          static_cast<uint4*>(a.out)[sOut[cb + c] * (D / 8) + e % (D / 8)] = reinterpret_cast<const uint4*>(staged)[e];
        }
      }
      if (!whole) {
        named_sync(1, kSoftThreads);
        if (st == 0) last_sh = arrive_part(a, s) ? 1 : 0;
        named_sync(1, kSoftThreads);
        if (last_sh) {
          __threadfence();
          // the weights' buffer is free: every product of the segment is complete
          join_tc<D>(a, s, sOut, reinterpret_cast<float*>(smem + t.p_off), PB * t.p_bytes / 4, st, kSoftThreads);
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&ctl.seg_free[n % kSegRing]);
    }
  } else {
    if constexpr (H == 2) asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
    if (warp == 0) {
      load_pages<D>(a, t, ctl, &tmK, &tmV, ring, lane);
    } else if (warp == 1) {
      // ---- MMAs ----
      if (elect_one()) {
        int T = 0, U = 0;  // tiles whose scores, units (tile, set) whose second product is issued
        int prev_n = 0, prev_N = 0;
        bool prev_first = false, ok = true;
        RingPos rp{0, 0u};  // K0 K1 V0 K2 V1 ...: the order of the products
        // O^T of a tile of width N, set by set; `first` of its segment n
        auto second = [&](bool first, int n, int N) -> bool {
          if (first && n > 0 && !wait_phase(&o_free, (uint32_t)((n - 1) & 1), a.status)) return false;
          if (!wait_phase(&ctl.full[rp.slot], rp.use, a.status)) return false;
          const uint32_t v = lo_v(ring + rp.slot * kSlotBytes, D == 128 ? kHalfBytes : 0);
          const int wide = set_cols<H>(N);
#pragma unroll
          for (int h = 0; h < H; ++h) {
            const int b = U % PB;
            if (!wait_phase(&p_full[U & 1], (uint32_t)((U >> 1) & 1), a.status)) return false;
            tc_fence_after();
            const uint32_t idesc = umma_idesc_bf16(kTile, 2 * wide) | kTransposeA | kTransposeB;
            const uint32_t w = lo_p(ring + t.p_off + b * t.p_bytes), tD = tO + h * 2 * kSetCols;
#pragma unroll
            for (int kk = 0; kk < kTile / 16; ++kk)
              umma_bf16(tD, desc(v + kk * (2048 >> 4), kHiV), desc(w + kk * (512 >> 4), kHiP), idesc,
                        kk > 0 || !first ? 1u : 0u);
            umma_commit(&p_free[U & 3]);
            ++U;
          }
          umma_commit(&ctl.empty[rp.slot]);
          rp.step(1, t.slots);
          return true;
        };
        for (int n = 0; ok; ++n) {
          const int k = n % kSegRing;
          ok = wait_phase(&ctl.seg_full[k], (uint32_t)((n / kSegRing) & 1), a.status);
          const int request = ctl.segs[k].request, cols = ctl.segs[k].cols, ntiles = ctl.segs[k].ntiles;
          mbar_arrive(&ctl.seg_free[k]);
          if (!ok || request < 0) break;
          const int N = (cols + 15) / 16 * 16, qb = n % QB;
          const uint32_t idesc = umma_idesc_bf16(kTile, N);
          ok = wait_phase(&ctl.q_full[qb], (uint32_t)((n / QB) & 1), a.status);
          const uint32_t q = lo_kq(ring + t.q_off + qb * a.ct * D * 2), q_half = (uint32_t)(a.ct * 128) >> 4;
          for (int x = 0; x < ntiles && ok; ++x, ++T) {
            const int b = T % SB;
            ok = !ctl.aborted && wait_phase(&ctl.full[rp.slot], rp.use, a.status);
            if (ok && T >= SB) ok = wait_phase(&s_free[b], (uint32_t)((T / SB - 1) & 1), a.status);
            if (!ok) break;
            tc_fence_after();
            const uint32_t key = lo_kq(ring + rp.slot * kSlotBytes), tD = tmem + b * kScores;
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk)
              umma_bf16(tD, desc(key + (((kk >> 2) * kHalfBytes + (kk & 3) * 32) >> 4), kHiKQ),
                        desc(q + (kk >> 2) * q_half + (((kk & 3) * 32) >> 4), kHiKQ), idesc, kk > 0 ? 1u : 0u);
            umma_commit(&s_full[b]);
            umma_commit(&ctl.empty[rp.slot]);
            rp.step(1, t.slots);
            if (x == ntiles - 1) umma_commit(&ctl.q_free[qb]);
            if (T > 0) ok = second(prev_first, prev_n, prev_N);
            prev_first = x == 0;
            prev_n = n;
            prev_N = N;
          }
        }
        rp.step(1, t.slots);  // the place of keys that do not come
        if (ok && T > 0) ok = second(prev_first, prev_n, prev_N);
        if (!ok) ctl.aborted = 1;
        // everything issued has completed before the TMEM goes
        umma_commit(&ctl.drained);
        wait_phase(&ctl.drained, 0u, a.status);
      }
      __syncwarp();
    } else if (warp == 2) {
      stage_queries<D, QB>(a, ctl, ring + t.q_off, a.ct, lane);
    } else if (warp == 3) {
      if (lane == 0) list_segments<0>(a, share, ctl);
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

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
template <int D, int CG, int H>
cudaError_t launch_variant(const AttendLaunch& a, cudaStream_t stream) {
  TcPlan t{};
  t.chunk = a.grain;
  t.nchunk = kTile / t.chunk;
  constexpr int QB = H == 1 && !two_per_sm(D, CG) ? 2 : 1, PB = 2;
  constexpr int kPerSm = two_per_sm(D, CG) ? 2 : 1;
  const int q_bytes = a.ct * D * 2, p_bytes = a.ct / 8 / H * kPChunkBytes, slot = (D / 64) * kHalfBytes;
  t.p_bytes = p_bytes;
  static std::atomic<int> known;
  int fixed;  // bytes of static shared memory
  cudaError_t err = static_smem(attend_tc_kernel<D, CG, H>, known, &fixed);
  if (err != cudaSuccess) return err;
  // dynamic shared memory starts behind the static one, on a 1024-byte boundary
  // (1 KB of an SM's 228 KB is reserved per CTA)
  const int limit = 228 * 1024 / kPerSm - 1024;
  const int room = limit - (fixed + 1023) / 1024 * 1024;
  t.slots = (room - QB * q_bytes - PB * p_bytes) / slot;
  if (t.slots > kMaxSlots) t.slots = kMaxSlots;
  t.q_off = t.slots * slot;
  t.p_off = t.q_off + QB * q_bytes;
  const int smem = t.p_off + PB * p_bytes + limit - room - fixed;  // and the gap before it
  CUtensorMap tmK, tmV;
  if (!make_cache_map(&tmK, a.k, a, t.chunk) || !make_cache_map(&tmV, a.v, a, t.chunk)) return cudaErrorInvalidValue;
  static std::atomic<size_t> raised[kMaxDevices];
  err = raise_smem(attend_tc_kernel<D, CG, H>, (size_t)smem, raised);
  if (err != cudaSuccess) return err;
  return launch_after_previous(attend_tc_kernel<D, CG, H>, dim3(a.ctas), dim3((4 + 4 * H) * 32), (size_t)smem, stream,
                               tmK, tmV, a, t);
}

}  // namespace

bool attend_tc_serves(int D, int dtype, int page_size, int64_t head_b, int64_t token_b, int64_t page_b) {
  const int64_t far = 1LL << 40;  // a tensor map's strides end there
  return attend_tc_may_serve(D, dtype) && page_size % 8 == 0 && head_b < far && token_b < far && page_b < far;
}

int attend_tc_grain(int page_size) { return std::min(page_size & -page_size, kTile); }

int attend_tc_ctas_per_sm(int D, int ct) { return two_per_sm(D, ct <= 16 ? 2 : 4) ? 2 : 1; }

int attend_tc_columns(int cols) {
  if (cols <= kTcMaxCols) return (cols + 15) / 16 * 16;
  const int n = (cols + kRowsMaxCols - 1) / kRowsMaxCols;  // column tiles, of equal width
  return std::max(kTcMaxCols + 16, ((cols + n - 1) / n + 15) / 16 * 16);
}

// The narrowest variant that holds an item: wider ones spend their softmax on
// columns that are not there.  64 requests of 64 heads over 8, 4,096 positions, us
// in the variants of 16 / 32 / 96 / 144 columns: a token, D = 128: 166 / 165 / 168 /
// 213; D = 64: 94 / 122 / 151 / 194; 8 rows, D = 128: - / - / 181 / 224.  17 rows (136
// columns): 250 here, 328 in the kernel for many rows, whose second set holds 8
// columns; 21 rows: 362 here as two items of 84, 305 there.
cudaError_t launch_attend_tc(const AttendLaunch& a, cudaStream_t stream) {
  if (a.ct > kTcMaxCols) return launch_attend_rows(a, stream);
  if (a.ct <= 16) return a.D == 64 ? launch_variant<64, 2, 1>(a, stream) : launch_variant<128, 2, 1>(a, stream);
  if (a.ct <= 32) return a.D == 64 ? launch_variant<64, 4, 1>(a, stream) : launch_variant<128, 4, 1>(a, stream);
  if (a.ct <= 96) return a.D == 64 ? launch_variant<64, 6, 2>(a, stream) : launch_variant<128, 6, 2>(a, stream);
  return a.D == 64 ? launch_variant<64, 9, 2>(a, stream) : launch_variant<128, 9, 2>(a, stream);
}

}  // namespace spec
