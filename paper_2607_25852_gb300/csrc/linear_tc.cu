// linear_tc.cu -- linear attention of many rows per request on the 5th-generation
// tensor cores: bf16 rows, key and value sizes of 64 or 128.
//
// A request's rows go by chunks of 64.  With the chunk's decays summed up to row
// i, L_i, and S the head's state before it,
//   O = diag(exp L) Q S + P V,     P_ij = exp(L_i - L_j) (q_i k_j) for j <= i, else 0
//   S' = exp(L_64) S + K^T V',     v'_j = exp(L_64 - L_j) v_j.
// All products are made with the value index along the 128 lanes of tensor
// memory, i.e. transposed, so that each operand is where it arises:
//   scores [i x j]   = Q K^T        Q and K as they lie in shared memory
//   O2^T   [v x i]   = S^T Q^T      S^T from tensor memory
//   U^T    [v x k]   = V'^T K       V'^T from tensor memory, K as it lies
//   O1^T   [v x i]   = V^T P^T      V as it lies, P from shared memory
// The state itself stays in fp32 registers: thread (v, half of k) adds U to it and
// stores it as operand for the next chunk in two bf16 numbers (2^-16 relative);
// so are the entries of P.  V' is stored in three (2^-24), as the state must not
// lose what fp32 holds.  The products of the pieces are 1.75 times those of the
// formula, which leaves the tensor cores 2,000 cycles a chunk of heads of 128,
// against the 2,800 in which its 64 KB come and go at the HBM's rate.
//
// Rows past a request's last are zeros in shared memory.  A value that is not
// finite must not reach earlier rows of its chunk through a product with 0: its
// finder clears it for that product and notes its row and column, whose outputs
// from the row on become NaN.
//
// Few heads: the rows are divided into segments (linear_tc.cuh).  The sums of all
// segments but the last are made first (one product of the four), a small kernel
// carries the state over them in order, and the segments' outputs then start from
// their own states.
//
// Warps: 0 to 3 load (a chunk each in turn), 4 issues the MMAs, 5 sums the decays,
// 8 to 11 make V', 12 to 19 keep the state, 20 to 27 make P and store O.
#include "attend_ring.cuh"
#include "linear_tc.cuh"

namespace spec {

namespace {

constexpr int kHalf = kLinChunk * 128;  // 64 elements of a chunk's rows
constexpr int kGRing = 4;               // chunks of decays
constexpr int kTS = 0, kTV = 128, kTU = 224, kTX = 352, kTO = 416;  // columns: S, V', U, scores and O1, O2
constexpr int kLinTmem = 512;
constexpr int kOutThreads = 28 * 32, kSumThreads = 20 * 32;

enum LinPhase { kSegmentSums, kLastSegment, kAllSegments };

struct LinTcLaunch {
  LinearLaunch p;
  LinearPlan plan;
  int phase, heads;  // heads: items per request and segment
  long long items;
  int stages;
};

struct alignas(16) DecayChunk {
  float hi[kLinChunk], lo[kLinChunk];      // L_i as a sum of two
  float weight[kLinChunk], first[kLinChunk];  // exp(L_64 - L_j), exp(L_i)
  float all;
};

struct LinControl {
  uint64_t full[4], empty[4], g_full[kGRing], g_empty[kGRing];
  uint64_t state_ready, weighted, sums, sums_read, scores, p_ready, out_ready, out_read, drained;
  DecayChunk g[kGRing];
  int bad_row[2][128];
  int aborted;
  uint32_t tmem;
};

// What a CTA works on at a time: rows of a request and head.
struct LinItem {
  const float* from;  // null: zeros
  float* to;          // null: not stored
  long long* steps;
  int row0, n, h, hq;
  int early;          // rows before position 0, right before row0
};

__device__ __forceinline__ bool lin_item(const LinTcLaunch& a, long long x, bool tell, LinItem* t) {
  const LinearLaunch& p = a.p;
  const int nseg = a.plan.nseg, seg = (int)(x % nseg), i = (int)(x / nseg / a.heads);
  const LinearRequest r = linear_request(p, i);
  if (!r.ok) {
    if (tell && x == (long long)i * a.heads * nseg) report(p.status, SPEC_ERR_BAD_INPUT);
    return false;
  }
  const int rows = r.last - r.first, segs = max(1, (rows + a.plan.seg_rows - 1) / a.plan.seg_rows);
  if (seg >= segs || (a.phase == kSegmentSums && seg == segs - 1) || (a.phase == kLastSegment && seg != segs - 1))
    return false;
  const int per = a.heads / p.H;  // 1 where states alone are made
  t->hq = (int)(x / nseg - (long long)i * a.heads);
  t->h = t->hq / per;
  const int first = r.first + seg * a.plan.seg_rows;
  t->row0 = r.row0 + first;
  t->n = min(a.plan.seg_rows, r.last - first);
  t->early = seg == 0 ? r.first : 0;
  const int64_t size = (int64_t)p.Dk * p.Dv, head = (int64_t)(i * (int64_t)p.H + t->h) * nseg;
  t->steps = nullptr;
  if (a.phase == kSegmentSums) {
    t->from = nullptr;
    t->to = a.plan.seg_state + (head + seg + 1) * size;
    t->steps = a.plan.seg_steps + head + seg;
    return true;
  }
  t->from = a.plan.staged ? a.plan.seg_state + (head + seg) * size
            : r.from >= 0 ? p.state + r.from * p.slot_stride + t->h * size
                          : nullptr;
  t->to = seg == segs - 1 && r.to >= 0 && t->hq % per == 0 ? p.state + r.to * p.slot_stride + t->h * size : nullptr;
  return true;
}

__device__ __forceinline__ void tmem_ld16(uint32_t addr, float (&v)[16]) {
  uint32_t r[16];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(addr)
      : "memory");
#pragma unroll
  for (int k = 0; k < 16; ++k) v[k] = __uint_as_float(r[k]);
}

// Two numbers as bf16, rounded, and what is left of them.
__device__ __forceinline__ uint32_t round_pair(float& x, float& y) {
  uint32_t b;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(b) : "f"(y), "f"(x));
  const float2 rest = unpair(fma2(pair(bf16_lo(b), bf16_hi(b)), pair(-1.0f, -1.0f), pair(x, y)));
  x = rest.x;
  y = rest.y;
  return b;
}
__device__ __forceinline__ uint32_t last_pair(float x, float y) {
  uint32_t b;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(b) : "f"(y), "f"(x));
  return b;
}

template <int DK, int DV, bool kOut>
__global__ void __launch_bounds__(kOut ? kOutThreads : kSumThreads, 1) linear_tc_kernel(const __grid_constant__ LinTcLaunch a) {
  constexpr int kKeyBytes = kLinChunk * DK * 2, kValueBytes = kLinChunk * DV * 2;
  constexpr int kKeyAt = kOut ? kKeyBytes : 0, kValueAt = kKeyAt + kKeyBytes, kStage = kValueAt + kValueBytes;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  __shared__ LinControl ctl;
  const LinearLaunch& p = a.p;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t ring = smem_u32(smem), pbuf = ring + a.stages * kStage;
  uint8_t* pmem = smem + a.stages * kStage;

  if (tid == 0) {
    for (int s = 0; s < a.stages; ++s) {
      mbar_init(&ctl.full[s], 1);
      mbar_init(&ctl.empty[s], 1 + 4);
    }
    for (int s = 0; s < kGRing; ++s) {
      mbar_init(&ctl.g_full[s], 1);
      mbar_init(&ctl.g_empty[s], 4 + 8 + (kOut ? 8 : 0));
    }
    mbar_init(&ctl.state_ready, 8);
    mbar_init(&ctl.weighted, 4);
    mbar_init(&ctl.sums, 1);
    mbar_init(&ctl.sums_read, 8);
    mbar_init(&ctl.scores, 1);
    mbar_init(&ctl.p_ready, 4);
    mbar_init(&ctl.out_ready, 1);
    mbar_init(&ctl.out_read, 8);
    mbar_init(&ctl.drained, 1);
    ctl.aborted = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 4) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ctl.tmem)),
                 "r"(kLinTmem)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  pdl_wait_prerequisites();
  pdl_launch_dependents();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = ctl.tmem;

  // Waits end after a second without progress, or when another role has given up.
  auto wait_one = [&](uint64_t* bar, uint32_t parity) {
    if (mbar_try_wait(bar, parity & 1u)) return true;
    const uint64_t t0 = global_ns();
    for (uint32_t it = 1; !mbar_try_wait(bar, parity & 1u); ++it) {
      if ((it & 63u) == 0u) {
        if (*(volatile int*)&ctl.aborted) return false;
        if (global_ns() - t0 > 1000000000ull) {
          report(p.status, SPEC_ERR_TIMEOUT);
          *(volatile int*)&ctl.aborted = 1;
          return false;
        }
      }
    }
    return true;
  };
  bool ok = true;
  auto wait = [&](uint64_t* bar, uint32_t parity) { ok = __all_sync(0xFFFFFFFFu, ok && wait_one(bar, parity)); };
  // calls f(item) for the CTA's items in turn
  auto items = [&](bool tell, auto f) {
    LinItem t;
    for (long long x = blockIdx.x; ok && x < a.items; x += gridDim.x)
      if (lin_item(a, x, tell, &t)) f(t);
  };
  uint32_t c = 0;  // chunks so far, of all items

  if (warp < 4) {
    // ---- loads: chunk c by warp c % stages ----
    auto bring = [&](const __nv_bfloat16* from, int64_t stride, auto dim, uint32_t to, int rows) {
      constexpr int kVecs = decltype(dim)::value / 8;
#pragma unroll 4
      for (int x = lane; x < kLinChunk * kVecs; x += 32) {
        const int r = x / kVecs, v = x % kVecs;
        const bool real = r < rows;
        cp_async16(to + (v >> 3) * kHalf + r * 128 + (((v & 7) ^ (r & 7)) << 4), real ? from + r * stride + v * 8 : from, real);
      }
    };
    if (warp < a.stages)
      items(false, [&](const LinItem& t) {
        const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(p.q) + t.row0 * p.q_row + (int64_t)t.hq * DK;
        const __nv_bfloat16* k = static_cast<const __nv_bfloat16*>(p.k) + t.row0 * p.k_row + (int64_t)t.h * DK;
        const __nv_bfloat16* v = static_cast<const __nv_bfloat16*>(p.v) + t.row0 * p.v_row + (int64_t)t.h * DV;
        for (int x = 0; x < t.n && ok; x += kLinChunk, ++c) {
          const int s = c % a.stages;
          if (s != warp) continue;
          const uint32_t use = c / a.stages;
          if (use > 0) wait(&ctl.empty[s], use - 1);
          if (!ok) break;
          const uint32_t at = ring + s * kStage;
          const int rows = t.n - x;
          if (kOut) bring(q + x * p.q_row, p.q_row, std::integral_constant<int, DK>{}, at, rows);
          bring(k + x * p.k_row, p.k_row, std::integral_constant<int, DK>{}, at + kKeyAt, rows);
          bring(v + x * p.v_row, p.v_row, std::integral_constant<int, DV>{}, at + kValueAt, rows);
          asm volatile("cp.async.commit_group;\n\tcp.async.wait_group 0;" ::: "memory");
          proxy_fence();
          __syncwarp();
          if (lane == 0) mbar_arrive(&ctl.full[s]);
        }
      });
  } else if (warp == 4) {
    // ---- MMAs ----
    if (elect_one()) {
      constexpr uint32_t kScores = umma_idesc_bf16(128, kLinChunk);
      constexpr uint32_t kOut1 = umma_idesc_bf16(128, kLinChunk) | kTransposeA;
      constexpr uint32_t kSums = umma_idesc_bf16(128, DK) | kTransposeB;
      auto need = [&](uint64_t* bar, uint32_t parity) { ok = ok && wait_one(bar, parity); };
      LinItem t;
      for (long long it = blockIdx.x; ok && it < a.items; it += gridDim.x) {
        if (!lin_item(a, it, false, &t)) continue;
        for (int x = 0; x < t.n && ok; x += kLinChunk, ++c) {
          const int s = c % a.stages;
          const uint32_t q = ring + s * kStage, k = q + kKeyAt, v = q + kValueAt;
          need(&ctl.full[s], c / a.stages);
          if (kOut) {
            if (c > 0) need(&ctl.out_read, c - 1);
            if (!ok) break;
            tc_fence_after();
            // rows 64 to 127 of the scores are of what lies behind Q, and are not read
#pragma unroll
            for (int kk = 0; kk < DK / 16; ++kk)
              umma_bf16(tmem + kTX, desc(lo_kq(q) + (((kk >> 2) * kHalf + (kk & 3) * 32) >> 4), kHiKQ),
                        desc(lo_kq(k) + (((kk >> 2) * kHalf + (kk & 3) * 32) >> 4), kHiKQ), kScores, kk > 0 ? 1u : 0u);
            umma_commit(&ctl.scores);
            need(&ctl.state_ready, c);
            if (!ok) break;
            tc_fence_after();
#pragma unroll
            for (int kk = 0; kk < 2 * (DK / 16); ++kk) {  // the upper parts, then the rests
              const int y = kk % (DK / 16);
              umma_bf16_tmem(tmem + kTO, tmem + kTS + 8 * kk, desc(lo_kq(q) + (((y >> 2) * kHalf + (y & 3) * 32) >> 4), kHiKQ),
                             kScores, kk > 0 ? 1u : 0u);
            }
          }
          need(&ctl.weighted, c);
          if (c > 0) need(&ctl.sums_read, c - 1);
          if (!ok) break;
          tc_fence_after();
#pragma unroll
          for (int kk = 0; kk < 3 * (kLinChunk / 16); ++kk)
            umma_bf16_tmem(tmem + kTU, tmem + kTV + 8 * kk, desc(lo_v(k, kHalf) + (kk % (kLinChunk / 16)) * (2048 >> 4), kHiV),
                           kSums, kk > 0 ? 1u : 0u);
          umma_commit(&ctl.sums);
          if (kOut) {
            need(&ctl.p_ready, c);
            if (!ok) break;
            tc_fence_after();
#pragma unroll
            for (int kk = 0; kk < 2 * (kLinChunk / 16); ++kk) {
              const int y = kk % (kLinChunk / 16);
              umma_bf16(tmem + kTX, desc(lo_v(v, kHalf) + y * (2048 >> 4), kHiV),
                        desc(lo_kq(pbuf + (kk / (kLinChunk / 16)) * kHalf) + ((y * 32) >> 4), kHiKQ), kOut1, kk > 0 ? 1u : 0u);
            }
            umma_commit(&ctl.out_ready);
          }
          umma_commit(&ctl.empty[s]);
        }
      }
      // everything issued has completed before the tensor memory goes
      umma_commit(&ctl.drained);
      wait_phase(&ctl.drained, 0u, p.status);
    }
    __syncwarp();
  } else if (warp == 5) {
    // ---- decays: rows 2 lane and 2 lane + 1 of the chunk ----
    items(true, [&](const LinItem& t) {
      long long total = 0;
      const float* from = p.log_decay + t.row0 * p.decay_row + t.h;
      auto row = [&](int r) { return r < t.n ? __ldg(from + r * p.decay_row) : 0.0f; };
      float n0 = row(2 * lane), n1 = row(2 * lane + 1);
      for (int x = 0; x < t.n && ok; x += kLinChunk, ++c) {
        const long long d0 = decay_steps(n0, p.status), d1 = decay_steps(n1, p.status);
        n0 = row(x + kLinChunk + 2 * lane), n1 = row(x + kLinChunk + 2 * lane + 1);
        long long sum = d0 + d1;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const long long y = __shfl_up_sync(0xFFFFFFFFu, sum, o);
          if (lane >= o) sum += y;
        }
        const long long all = __shfl_sync(0xFFFFFFFFu, sum, 31);
        total += all;
        const int s = c % kGRing;
        if (c >= kGRing) wait(&ctl.g_empty[s], c / kGRing - 1);
        if (!ok) break;
        DecayChunk& g = ctl.g[s];
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const long long l = y ? sum : sum - d1;
          const float hi = steps_float(l);
          g.hi[2 * lane + y] = hi;
          g.lo[2 * lane + y] = steps_float(l - __float2ll_rn(hi * 4294967296.0f));
          g.weight[2 * lane + y] = exp2f(steps_float(all - l));
          g.first[2 * lane + y] = exp2f(hi);
        }
        if (lane == 0) g.all = exp2f(steps_float(all));
        __syncwarp();
        if (lane == 0) mbar_arrive(&ctl.g_full[s]);
      }
      if (t.steps && lane == 0) *t.steps = total;
    });
  } else if (warp >= 8 && warp < 12) {
    // ---- V': value `d` of the rows, weighted, in three parts ----
    const int d = (warp & 3) * 32 + lane;
    const bool mine = (warp & 3) * 32 < DV;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16, to = tmem + kTV + lanes;
    items(false, [&](const LinItem& t) {
      for (int x = 0; x < t.n && ok; x += kLinChunk, ++c) {
        const int s = c % a.stages;
        wait(&ctl.full[s], c / a.stages);
        wait(&ctl.g_full[c % kGRing], c / kGRing);
        if (c > 0) wait(&ctl.sums, c - 1);
        if (!ok) break;
        if (mine) {
          uint8_t* at = smem + s * kStage + kValueAt + (d >> 6) * kHalf + (d & 7) * 2;
          const int v8 = (d & 63) >> 3;
          const DecayChunk& g = ctl.g[c % kGRing];
          float check = 0.0f;
          tc_fence_after();
#pragma unroll 1
          for (int half = 0; half < 2; ++half) {
            uint32_t part[3][16];
#pragma unroll
            for (int y = 0; y < 16; ++y) {
              const int r = half * 32 + 2 * y;
              const float2 w = *reinterpret_cast<const float2*>(&g.weight[r]);
              const uint16_t b0 = *reinterpret_cast<const uint16_t*>(at + r * 128 + ((v8 ^ (2 * y & 7)) << 4));
              const uint16_t b1 = *reinterpret_cast<const uint16_t*>(at + (r + 1) * 128 + ((v8 ^ ((2 * y + 1) & 7)) << 4));
              const float x0 = __uint_as_float((uint32_t)b0 << 16), x1 = __uint_as_float((uint32_t)b1 << 16);
              check = fmaf(x0, 0.0f, fmaf(x1, 0.0f, check));
              float y0 = x0 * w.x, y1 = x1 * w.y;
              part[0][y] = round_pair(y0, y1);
              part[1][y] = round_pair(y0, y1);
              part[2][y] = last_pair(y0, y1);
            }
#pragma unroll
            for (int k = 0; k < 3; ++k) tmem_st16(to + 32 * k + 16 * half, part[k]);
          }
          if (kOut) {
            int bad = kLinChunk;
            if (check != check) {  // rare: what is not finite goes, its first row is noted
              for (int r = kLinChunk - 1; r >= 0; --r) {
                uint16_t* e = reinterpret_cast<uint16_t*>(at + r * 128 + ((v8 ^ (r & 7)) << 4));
                if (!bf16_not_finite(*e)) continue;
                *e = 0;
                bad = r;
              }
              proxy_fence();
            }
            ctl.bad_row[c & 1][d] = bad;
          }
          tmem_st_wait();
          tc_fence_before();
        }
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&ctl.weighted);
          mbar_arrive(&ctl.empty[s]);
          mbar_arrive(&ctl.g_empty[c % kGRing]);
        }
      }
    });
  } else if (warp >= 12 && warp < 20) {
    // ---- the state: value d, keys of half kh ----
    constexpr int kKeys = DK / 2;
    const int d = (warp & 3) * 32 + lane, kh = (warp - 12) >> 2;
    const bool mine = (warp & 3) * 32 < DV;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t u = tmem + kTU + lanes + kh * kKeys, to = tmem + kTS + lanes + kh * (kKeys / 2);
    float st[kKeys];
    auto operand = [&]() {  // the state for the next chunk's product
      if (mine) {
#pragma unroll
        for (int k = 0; k < kKeys; k += 32) {
          uint32_t hi[16], lo[16];
#pragma unroll
          for (int y = 0; y < 16; ++y) {
            float y0 = st[k + 2 * y], y1 = st[k + 2 * y + 1];
            hi[y] = round_pair(y0, y1);
            lo[y] = last_pair(y0, y1);
          }
          tmem_st16(to + k / 2, hi);
          tmem_st16(to + DK / 2 + k / 2, lo);
        }
        tmem_st_wait();
        tc_fence_before();
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&ctl.state_ready);
    };
    items(false, [&](const LinItem& t) {
#pragma unroll
      for (int k = 0; k < kKeys; ++k) st[k] = t.from && mine ? __ldcg(t.from + (int64_t)(kh * kKeys + k) * DV + d) : 0.0f;
      if (kOut && t.n > 0) operand();
      for (int x = 0; x < t.n && ok; x += kLinChunk, ++c) {
        wait(&ctl.g_full[c % kGRing], c / kGRing);
        const float f = ctl.g[c % kGRing].all;
        wait(&ctl.sums, c);  // O2 of the chunk, issued before, has read the operand as well
        if (!ok) break;
        tc_fence_after();
        if (mine) {
#pragma unroll
          for (int k = 0; k < kKeys; k += 16) {
            float w[16];
            tmem_ld16(u + k, w);
#pragma unroll
            for (int y = 0; y < 16; ++y) st[k + y] = fmaf(f, st[k + y], w[y]);
          }
          tc_fence_before();
        }
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&ctl.sums_read);
          mbar_arrive(&ctl.g_empty[c % kGRing]);
        }
        if (kOut && x + kLinChunk < t.n) operand();
      }
      if (t.to && mine && ok) {
#pragma unroll
        for (int k = 0; k < kKeys; ++k) t.to[(int64_t)(kh * kKeys + k) * DV + d] = st[k];
      }
    });
  } else if (kOut && warp >= 20) {
    // ---- P, then O: half `set` of the columns ----
    const int quad = warp & 3, set = (warp - 20) >> 2, d = quad * 32 + lane;
    const uint32_t lanes = (uint32_t)(quad * 32) << 16;
    items(false, [&](const LinItem& t) {
      __nv_bfloat16* out = static_cast<__nv_bfloat16*>(p.out) + ((int64_t)t.row0 * p.Hq + t.hq) * DV;
      const int64_t out_row = (int64_t)p.Hq * DV;
      for (long long x = tid - 20 * 32; x < (long long)t.early * (DV / 8); x += 256) {
        const int r = (int)(x / (DV / 8)), v = (int)(x % (DV / 8));
        *reinterpret_cast<uint4*>(out - (r + 1) * out_row + v * 8) = make_uint4(0u, 0u, 0u, 0u);
      }
      for (int x = 0; x < t.n && ok; x += kLinChunk, ++c) {
        wait(&ctl.g_full[c % kGRing], c / kGRing);
        const DecayChunk& g = ctl.g[c % kGRing];
        wait(&ctl.scores, c);
        if (!ok) break;
        if (quad < 2) {  // row d of P
          tc_fence_after();
          uint32_t hi[16], lo[16];
          if (quad >= set) {
            float w[32];
            tmem_ld32(tmem + kTX + lanes + 32 * set, w);
            const float gh = g.hi[d], gl = g.lo[d];
#pragma unroll
            for (int y = 0; y < 16; ++y) {
              const int j = 32 * set + 2 * y;
              const float2 h = *reinterpret_cast<const float2*>(&g.hi[j]), l = *reinterpret_cast<const float2*>(&g.lo[j]);
              float y0 = j <= d ? w[2 * y] * ex2_approx((gh - h.x) + (gl - l.x)) : 0.0f;
              float y1 = j + 1 <= d ? w[2 * y + 1] * ex2_approx((gh - h.y) + (gl - l.y)) : 0.0f;
              hi[y] = round_pair(y0, y1);
              lo[y] = last_pair(y0, y1);
            }
          } else {
#pragma unroll
            for (int y = 0; y < 16; ++y) hi[y] = lo[y] = 0u;
          }
          tc_fence_before();
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            uint8_t* at = pmem + d * 128 + (((4 * set + y) ^ (d & 7)) << 4);
            *reinterpret_cast<uint4*>(at) = make_uint4(hi[4 * y], hi[4 * y + 1], hi[4 * y + 2], hi[4 * y + 3]);
            *reinterpret_cast<uint4*>(at + kHalf) = make_uint4(lo[4 * y], lo[4 * y + 1], lo[4 * y + 2], lo[4 * y + 3]);
          }
          proxy_fence();
          __syncwarp();
          if (lane == 0) mbar_arrive(&ctl.p_ready);
        }
        wait(&ctl.weighted, c);  // whose finders note rows that are not finite
        wait(&ctl.out_ready, c);
        if (!ok) break;
        if (quad * 32 < DV) {
          tc_fence_after();
          const int bad = ctl.bad_row[c & 1][d];
#pragma unroll
          for (int y = 0; y < 32; y += 16) {
            float o1[16], o2[16];
            tmem_ld16(tmem + kTX + lanes + 32 * set + y, o1);
            tmem_ld16(tmem + kTO + lanes + 32 * set + y, o2);
#pragma unroll
            for (int k = 0; k < 16; ++k) {
              const int r = 32 * set + y + k;
              const float o = p.scale * fmaf(g.first[r], o2[k], o1[k]);
              if (x + r < t.n) out[(x + r) * out_row + d] = __float2bfloat16_rn(r >= bad ? __int_as_float(0x7FC00000) : o);
            }
          }
          tc_fence_before();
        }
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&ctl.out_read);
          mbar_arrive(&ctl.g_empty[c % kGRing]);
        }
      }
    });
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == 4) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kLinTmem) : "memory");
  }
}

// The state before each segment, the segments' sums (each in its next one's place) added up in order: four elements
// per thread.
__global__ void __launch_bounds__(256) linear_scan_kernel(const LinearLaunch p, const LinearPlan plan) {
  const int head = blockIdx.x, i = head / p.H, h = head - i * p.H;
  pdl_wait_prerequisites();
  pdl_launch_dependents();
  const LinearRequest r = linear_request(p, i);
  const int segs = (r.last - r.first + plan.seg_rows - 1) / plan.seg_rows;
  const int64_t size = (int64_t)p.Dk * p.Dv, e = ((int64_t)blockIdx.y * 256 + threadIdx.x) * 4;
  if (!r.ok || e >= size) return;
  float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  if (r.from >= 0) s = *reinterpret_cast<const float4*>(p.state + r.from * p.slot_stride + h * size + e);
  float* seg = plan.seg_state + (int64_t)head * plan.nseg * size + e;
  const long long* steps = plan.seg_steps + (int64_t)head * plan.nseg;
  *reinterpret_cast<float4*>(seg) = s;
  constexpr int kU = 8;  // segments in flight
  for (int x0 = 1; x0 < segs; x0 += kU) {
    float4 z[kU];
    long long d[kU];
#pragma unroll
    for (int u = 0; u < kU; ++u)
      if (x0 + u < segs) {
        z[u] = *reinterpret_cast<const float4*>(seg + (x0 + u) * size);
        d[u] = steps[x0 + u - 1];
      }
#pragma unroll
    for (int u = 0; u < kU; ++u)
      if (x0 + u < segs) {
        const float f = exp2f(steps_float(d[u]));
        s.x = fmaf(f, s.x, z[u].x), s.y = fmaf(f, s.y, z[u].y);
        s.z = fmaf(f, s.z, z[u].z), s.w = fmaf(f, s.w, z[u].w);
        *reinterpret_cast<float4*>(seg + (x0 + u) * size) = s;
      }
  }
}

template <int DK, int DV, bool kOut>
cudaError_t launch_tc(const LinearLaunch& p, const LinearPlan& plan, int phase, cudaStream_t stream) {
  LinTcLaunch a{};
  a.p = p;
  a.plan = plan;
  a.phase = phase;
  a.heads = kOut ? p.Hq : p.H;
  a.items = (long long)p.rows.B * a.heads * plan.nseg;
  constexpr int kStage = kLinChunk * 2 * ((kOut ? 2 : 1) * DK + DV), kP = kOut ? 2 * kHalf : 0;
  static std::atomic<int> known;
  int fixed;
  cudaError_t err = static_smem(linear_tc_kernel<DK, DV, kOut>, known, &fixed);
  if (err != cudaSuccess) return err;
  // dynamic shared memory from a 1024-byte boundary; 8 KB behind the last stage may be read (and not used)
  const int room = 227 * 1024 - (fixed + 1023) / 1024 * 1024 - 1024 - kP - kHalf;
  a.stages = std::min(4, room / kStage);
  const size_t smem = (size_t)a.stages * kStage + kP + kHalf + 1024;
  static std::atomic<size_t> raised[kMaxDevices];
  err = raise_smem(linear_tc_kernel<DK, DV, kOut>, smem, raised);
  if (err != cudaSuccess) return err;
  return launch_after_previous(linear_tc_kernel<DK, DV, kOut>, dim3((unsigned)std::min<long long>(a.items, device_sms())),
                               dim3(kOut ? kOutThreads : kSumThreads), smem, stream, a);
}

template <int DK, int DV>
cudaError_t launch_phases(const LinearLaunch& p, const LinearPlan& plan, cudaStream_t stream) {
  if (plan.nseg > 1) {
    const cudaError_t err = launch_tc<DK, DV, false>(p, plan, kSegmentSums, stream);
    if (err != cudaSuccess) return err;
  }
  if (plan.staged) {
    const cudaError_t err = launch_after_previous(linear_scan_kernel, dim3((unsigned)(p.rows.B * p.H), (unsigned)(DK * DV / 1024)), dim3(256),
                                0, stream, p, plan);
    if (err != cudaSuccess) return err;
  }
  return p.q ? launch_tc<DK, DV, true>(p, plan, kAllSegments, stream)
             : launch_tc<DK, DV, false>(p, plan, kLastSegment, stream);
}

}  // namespace

cudaError_t launch_linear_tc(const LinearLaunch& p, const LinearPlan& plan, cudaStream_t stream) {
  if (p.Dk == 64) return p.Dv == 64 ? launch_phases<64, 64>(p, plan, stream) : launch_phases<64, 128>(p, plan, stream);
  return p.Dv == 64 ? launch_phases<128, 64>(p, plan, stream) : launch_phases<128, 128>(p, plan, stream);
}

}  // namespace spec
