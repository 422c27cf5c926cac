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
//   U^T    [v x k]   = V'^T K       V' from shared memory, K as it lies
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
// Warp 7 lists the chunks, with their decays summed up, in a ring of records that
// all others go by.  2 and 3 load, 6 issues the MMAs, 8 to 11 and 28 to 31 (20 to 23
// where only states are made) make V', 12 to 19 keep the state, 0, 1, 4 and 5 (their
// lanes hold the scores) make P, 20 to 27 read O and store it by way of shared memory.
// U is made in two halves, which the state's two groups of warps take as they come, and
// before O2, whose operand they write behind it.
//
// What bounds it: of the 4,800 cycles of a chunk of heads of 128 the tensor cores work
// 1,850.  The MMAs' thread is never idle: their issue takes those, and what is between
// them as much, as every role's code is fetched again and again (62 KB together, 81 % of
// requests hit the instruction cache).  So loops stay rolled where registers allow: a
// variant with other code in the loops, but no more work, hit 68 % and took 198 us for
// 169.  Two threads that issue MMAs took 206, a table of steps in place of the code 314.
// Measured: 4 requests of 4,096 rows of 38 heads of 128 164 us (4.0 TB/s), 2 of 16,384 of
// 32 heads 523 (in segments), 64 of 256 of 32 heads 180 (4.5 TB/s), 64 of 64 73 (5.5).
// (With V' by four warps by way of tensor memory 185, 542, 197 and 95.)  Registers
// end at 64 and 80 a thread: five of the eight instances keep 8 to 16 bytes on the stack.
#include "attend_ring.cuh"
#include "linear_tc.cuh"

namespace spec {

namespace {

constexpr int kHalf = kLinChunk * 128;  // 64 elements of a chunk's rows
constexpr int kRecords = 8;             // chunks listed ahead
constexpr int kTS = 0, kTU = 128;       // columns: S, U
constexpr int kTX = 256, kTO = 320;     // scores and then O1, O2, of even chunks; those of odd ones 128 on
constexpr int kLinTmem = 512;
constexpr int kOutThreads = 32 * 32, kSumThreads = 24 * 32;
constexpr int kWeighers = 8;            // warps that make V'

enum LinPhase { kSegmentSums, kLastSegment, kAllSegments };

struct LinTcLaunch {
  LinearLaunch p;
  LinearPlan plan;
  int phase;
  uint32_t heads, items;  // heads: items per request and segment
  bool tma;  // the tensor maps are there
};

// A chunk: up to 64 rows of a request and head.  One without rows moves a state.
struct alignas(16) Record {
  float hi[kLinChunk], lo[kLinChunk];         // L_i as a sum of two
  float weight[kLinChunk], first[kLinChunk];  // exp(L_64 - L_j), scale exp(L_i)
  float all;                                  // exp(L_64)
  int rows, row0, h, hq;
  int early;          // rows before position 0, right before row0
  bool begins, ends;  // the item's first and last chunk
  bool none;          // the list is over
  const float* from;  // the item's first state; null: zeros
  float* to;          // where its last goes; null: nowhere
};

struct LinControl {
  uint64_t full[4], empty[4], q_empty[4], listed[kRecords], used[kRecords];
  uint64_t state_ready, operand_read, scores, p_ready, drained;
  uint64_t sums[2], sums_read[2];  // U of half of the keys there, and read
  // of even and odd chunks, as some warps may be a chunk ahead of others: V' there; where only states are made V'
  // read; O there and read.  Of every fourth: bad_row there
  uint64_t weighted[2], read[2], out_ready[2], out_read[2], noted[4];
  uint64_t staged, stored;  // O in shared memory, and out of it
  Record records[kRecords];
  unsigned long long bad_row[4][128];  // chunk << 8 | 255 - the first row that is not finite, of every fourth chunk
  uint32_t sent[2];  // one past each loading warp's last chunk
  int aborted;
  uint32_t tmem;
};

// In shared memory: the chunks' K and V (V' is not the only reader of V), their Q, which
// are free again earlier, V' (twice where only states are made), P's two parts, and O.
constexpr int lin_q_stages(int DK) { return DK == 64 ? 4 : 2; }
constexpr int lin_smem(int DK, int DV, bool out, int stages) {
  // (a product over 128 values of 64 reads what lies behind them: P, or nothing)
  return kLinChunk * 2 * (stages * (DK + DV) + (out ? lin_q_stages(DK) * DK + 4 * DV + 128 : 6 * DV + 64)) + 1024;
}
constexpr int lin_stages(int DK, int DV, bool out) { return lin_smem(DK, DV, out, 4) <= 213 * 1024 ? 4 : 3; }

// What a CTA works on at a time: rows of a request and head.
struct LinItem {
  const float* from;
  float* to;
  long long* steps;
  int row0, n, h, hq, early;
};

__device__ __forceinline__ bool lin_item(const LinTcLaunch& a, uint32_t x, LinItem* t) {
  const LinearLaunch& p = a.p;
  const uint32_t nseg = a.plan.nseg, y = x / nseg, i = y / a.heads;
  const int seg = (int)(x - y * nseg);
  const LinearRequest r = linear_request(p, i);
  if (!r.ok) {
    if (x == i * a.heads * nseg) report(p.status, SPEC_ERR_BAD_INPUT);
    return false;
  }
  const int rows = r.last - r.first, segs = max(1, (rows + a.plan.seg_rows - 1) / a.plan.seg_rows);
  if (seg >= segs || (a.phase == kSegmentSums && seg == segs - 1) || (a.phase == kLastSegment && seg != segs - 1))
    return false;
  const int per = a.heads / p.H;  // 1 where states alone are made
  t->hq = (int)(y - i * a.heads);
  t->h = t->hq / per;
  const int first = r.first + seg * a.plan.seg_rows;
  t->row0 = r.row0 + first;
  t->n = min(a.plan.seg_rows, r.last - first);
  t->early = seg == 0 ? r.first : 0;
  const int64_t size = (int64_t)p.Dk * p.Dv, head = ((int64_t)i * p.H + t->h) * nseg;
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

// 16 columns; not there before wait_ld().
__device__ __forceinline__ void tmem_ld16(uint32_t addr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(addr)
      : "memory");
}
__device__ __forceinline__ void tmem_ld8(uint32_t addr, uint32_t (&r)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(addr)
               : "memory");
}
template <int N>
__device__ __forceinline__ void wait_ld(uint32_t (&r)[N]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int k = 0; k < N; ++k) asm volatile("" : "+r"(r[k]));  // no use of them moves up
}
__device__ __forceinline__ void tmem_st8(uint32_t addr, const uint32_t (&r)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(addr), "r"(r[0]), "r"(r[1]),
               "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}
// Two numbers as bf16, rounded, and what is left of them.
__device__ __forceinline__ uint32_t round_pair(f32x2& x) {
  const uint32_t b = last_pair(x);
  x = fma2(pair(bf16_lo(b), bf16_hi(b)), pair(-1.0f, -1.0f), x);
  return b;
}
__device__ __forceinline__ f32x2 pair_of(uint32_t x, uint32_t y) { return pair(__uint_as_float(x), __uint_as_float(y)); }

template <int DK, int DV, bool kOut>
__global__ void __launch_bounds__(kOut ? kOutThreads : kSumThreads, 1)
    linear_tc_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                     const __grid_constant__ CUtensorMap tmV, const __grid_constant__ LinTcLaunch a) {
  constexpr int kKeyBytes = kLinChunk * DK * 2, kValueBytes = kLinChunk * DV * 2;
  constexpr int kValueAt = kKeyBytes, kStage = kKeyBytes + kValueBytes;
  constexpr int kStages = lin_stages(DK, DV, kOut), kQueries = kOut ? lin_q_stages(DK) : 1;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  __shared__ LinControl ctl;
  const LinearLaunch& p = a.p;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t ring = smem_u32(smem);
  constexpr int kQueryAt = kStages * kStage, kWeightedAt = kQueryAt + (kOut ? kQueries * kKeyBytes : 0);
  uint8_t* pmem = smem + kWeightedAt + 3 * kValueBytes;  // P's two parts
  uint8_t* omem = pmem + 2 * kHalf;                       // O, row by row

  for (int x = tid; x < 4 * 128; x += blockDim.x) ctl.bad_row[x >> 7][x & 127] = 0;
  if (tid == 0) {
    for (int s = 0; s < kQueries; ++s) mbar_init(&ctl.q_empty[s], 1);
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&ctl.full[s], 1);
      mbar_init(&ctl.empty[s], 1 + kWeighers);
    }
    for (int s = 0; s < kRecords; ++s) {
      mbar_init(&ctl.listed[s], 1);
      mbar_init(&ctl.used[s], 3 + kWeighers + 8 + (kOut ? 4 + 8 : 0));  // all that read it
    }
    mbar_init(&ctl.state_ready, 8);
    mbar_init(&ctl.operand_read, 1);
    mbar_init(&ctl.scores, 1);
    mbar_init(&ctl.p_ready, 4);
    mbar_init(&ctl.drained, 1);
    for (int s = 0; s < 2; ++s) {
      mbar_init(&ctl.weighted[s], kWeighers);
      mbar_init(&ctl.sums[s], 1);
      mbar_init(&ctl.sums_read[s], 4);
      mbar_init(&ctl.read[s], 1);
      mbar_init(&ctl.out_ready[s], 1);
      mbar_init(&ctl.out_read[s], 8);
    }
    for (int s = 0; s < 4; ++s) mbar_init(&ctl.noted[s], kWeighers);
    mbar_init(&ctl.staged, 8);
    mbar_init(&ctl.stored, 8);
    ctl.aborted = 0;
    ctl.sent[0] = ctl.sent[1] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 6) {
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
    uint32_t began = 0;
    for (uint32_t it = 0; !mbar_try_wait(bar, parity & 1u); ++it) {
      if ((it & 63u) != 63u) continue;
      uint32_t now;
      asm volatile("mov.u32 %0, %%globaltimer_lo;" : "=r"(now));  // in ns
      if (it == 63u) began = now;
      if (now - began > 1000000000u) *(volatile int*)&ctl.aborted = 1;
      if (*(volatile int*)&ctl.aborted) return false;
    }
    return true;
  };
  bool ok = true;
  auto wait = [&](uint64_t* bar, uint32_t parity) { ok = __all_sync(0xFFFFFFFFu, ok && wait_one(bar, parity)); };
  // Record c, or null at the list's end; n counts those with rows, and a phase of
  // most barriers is one of them.
  uint32_t c = 0, n = 0;
  auto next = [&]() -> const Record* {
    wait(&ctl.listed[c % kRecords], c / kRecords);
    const Record* r = &ctl.records[c % kRecords];
    return ok && !r->none ? r : nullptr;
  };
  auto done = [&]() {  // with record c, by the whole warp
    __syncwarp();
    if (lane == 0) mbar_arrive(&ctl.used[c % kRecords]);
    __syncwarp();
    ++c;
  };
  // registers: 32 warps of 64 are split as 56, 56, 48, 104 twice, 48 three times per 4 warps; 24 of 80 as 40, 64, 80,
  // 104 twice, 80
  const bool scorer = kOut && warp < 8 && (warp & 3) < 2;
  if (warp < 8) {
    if (kOut) asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
    else if (warp >= 4) asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    else asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
    if (scorer) {
      // ---- P: row d, half `set` of the columns ----
      const int set = warp >> 2, quad = warp & 1, d = quad * 32 + lane;
      const uint32_t from = tmem + kTX + ((uint32_t)(quad * 32) << 16) + 32 * set;
      while (const Record* r = next()) {
        if (r->rows > 0) {
          wait(&ctl.scores, n);  // the last chunk's product has read P
          if (!ok) break;
          tc_fence_after();
          const f32x2 minus = pair(-1.0f, -1.0f);
          const f32x2 gh = pair(r->hi[d], r->hi[d]), gl = pair(r->lo[d], r->lo[d]);
#pragma unroll 1
          for (int part = 0; part < 4; ++part) {  // eight columns
            const int j0 = 32 * set + 8 * part;
            uint32_t w[8], hi[4] = {0u, 0u, 0u, 0u}, lo[4] = {0u, 0u, 0u, 0u};
            if (quad >= set) {  // (columns 32 to 63 are behind rows 0 to 31)
              tmem_ld8(from + 128 * (n & 1) + 8 * part, w);
              wait_ld(w);
#pragma unroll
              for (int y = 0; y < 4; y += 2) {
                const int j = j0 + 2 * y;
                const float4 h = *reinterpret_cast<const float4*>(&r->hi[j]), l = *reinterpret_cast<const float4*>(&r->lo[j]);
#pragma unroll
                for (int z = 0; z < 2; ++z) {
                  const float2 e = unpair(add2(fma2(z ? pair(h.z, h.w) : pair(h.x, h.y), minus, gh),
                                               fma2(z ? pair(l.z, l.w) : pair(l.x, l.y), minus, gl)));
                  const float s0 = __uint_as_float(w[2 * (y + z)]), s1 = __uint_as_float(w[2 * (y + z) + 1]);
                  f32x2 x = pair(j + 2 * z <= d ? s0 * ex2_approx(e.x) : 0.0f, j + 2 * z + 1 <= d ? s1 * ex2_approx(e.y) : 0.0f);
                  hi[y + z] = round_pair(x), lo[y + z] = last_pair(x);
                }
              }
            }
            uint8_t* at = pmem + d * 128 + (((4 * set + part) ^ (d & 7)) << 4);
            *reinterpret_cast<uint4*>(at) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
            *reinterpret_cast<uint4*>(at + kHalf) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
          }
          tc_fence_before();
          proxy_fence();
          __syncwarp();
          if (lane == 0) mbar_arrive(&ctl.p_ready);
          ++n;
        }
        done();
      }
    } else if (warp == 2 || warp == 3) {
      // ---- loads, every second chunk each: whole chunks by TMA, a request's last rows by plain copies, which read nothing
      // behind them and put zeros there (but for Q, whose rows are separate): 64 requests of 32 rows of 32 heads of 128
      // take 76 us, 92 with a division per vector and Q's zeros ----
      auto copy = [&](const __nv_bfloat16* from, int64_t stride, int width, uint32_t to, int rows, int end) {
        const int vecs = width / 8, v = lane % vecs, step = 32 / vecs;
#pragma unroll 2
        for (int r = lane / vecs; r < end; r += step) {
          const bool real = r < rows;
          cp_async16(to + (v >> 3) * kHalf + r * 128 + (((v & 7) ^ (r & 7)) << 4), real ? from + r * stride + v * 8 : from, real);
        }
      };
      auto bring = [&](const CUtensorMap* map, int width, int column, int row, int to, uint64_t* bar) {
        for (int k = 0; k < width / 64; ++k) tma_load_2d(smem + to + k * kHalf, map, column + 64 * k, row, bar);
      };
      while (const Record* r = next()) {
        const int rows = r->rows, row = r->row0, h = r->h, hq = r->hq;
        done();  // both read every record, to count the chunks
        if (rows == 0) continue;
        const uint32_t chunk = n++;
        if ((chunk & 1) != (uint32_t)(warp & 1)) continue;
        const int s = chunk % kStages;
        const uint32_t use = chunk / kStages;
        if (use > 0) wait(&ctl.empty[s], use - 1);
        const int to_q = kQueryAt + (kOut ? (int)(chunk % kQueries) * kKeyBytes : 0);
        if (kOut && chunk >= kQueries) wait(&ctl.q_empty[chunk % kQueries], chunk / kQueries - 1);
        if (!ok) break;
        if (lane == 0) ctl.sent[warp & 1] = chunk + 1;
        if (a.tma && rows == kLinChunk) {
          if (lane == 0) {
            mbar_expect_tx(&ctl.full[s], kStage + (kOut ? kKeyBytes : 0));
            if (kOut) bring(&tmQ, DK, hq * DK, row, to_q, &ctl.full[s]);
            bring(&tmK, DK, h * DK, row, s * kStage, &ctl.full[s]);
            bring(&tmV, DV, h * DV, row, s * kStage + kValueAt, &ctl.full[s]);
          }
          __syncwarp();
          continue;
        }
        const uint32_t at = ring + s * kStage;
#pragma unroll 1
        for (int x = kOut ? 0 : 1; x < 3; ++x) {
          const void* base = x == 0 ? p.q : x == 1 ? p.k : p.v;
          const int64_t stride = x == 0 ? p.q_row : x == 1 ? p.k_row : p.v_row;
          const int width = x == 2 ? DV : DK, head = x == 0 ? hq : h;
          copy(static_cast<const __nv_bfloat16*>(base) + row * stride + (int64_t)head * width, stride, width,
               x == 0 ? ring + to_q : x == 1 ? at : at + kValueAt, rows, x == 0 ? rows : kLinChunk);
        }
        asm volatile("cp.async.commit_group;\n\tcp.async.wait_group 0;" ::: "memory");
        proxy_fence();
        __syncwarp();
        if (lane == 0) mbar_arrive(&ctl.full[s]);
      }
    } else if (warp == 6) {
      // ---- MMAs ----
      if (elect_one()) {
        constexpr uint32_t kScores = umma_idesc_bf16(128, kLinChunk);
        constexpr uint32_t kOut1 = umma_idesc_bf16(128, kLinChunk) | kTransposeA;
        constexpr uint32_t kSums = umma_idesc_bf16(128, 64) | kTransposeA | kTransposeB;
        auto need = [&](uint64_t* bar, uint32_t parity) { ok = ok && wait_one(bar, parity); };
        // four products over 16 each: A and B in shared memory so many bytes apart, or A in tensor memory
        auto four = [&](int to, uint32_t x, int x_step, uint32_t y, int y_step, uint32_t kind, bool fresh) {
          const uint32_t x0 = x_step == 2048 ? lo_v(x, kHalf) : lo_kq(x), y0 = lo_kq(y);
#pragma unroll
          for (int m = 0; m < 4; ++m)
            umma_bf16(tmem + to, desc(x0 + (m * x_step >> 4), x_step == 2048 ? kHiV : kHiKQ), desc(y0 + (m * y_step >> 4), kHiKQ),
                      kind, m > 0 || !fresh ? 1u : 0u);
        };
        auto four_tmem = [&](int to, int x, uint32_t y, uint32_t kind, bool fresh) {
#pragma unroll
          for (int m = 0; m < 4; ++m)
            umma_bf16_tmem(tmem + to, tmem + x + 8 * m, desc(lo_kq(y) + (m * 32 >> 4), kHiKQ), kind, m > 0 || !fresh ? 1u : 0u);
        };
        auto four_rows = [&](int to, uint32_t x, uint32_t y, uint32_t kind, bool fresh) {  // both transposed
#pragma unroll
          for (int m = 0; m < 4; ++m)
            umma_bf16(tmem + to, desc(lo_v(x, kHalf) + (m * 2048 >> 4), kHiV), desc(lo_v(y, kHalf) + (m * 2048 >> 4), kHiV), kind,
                      m > 0 || !fresh ? 1u : 0u);
        };
        for (; ok; ++c) {
          need(&ctl.listed[c % kRecords], c / kRecords);
          if (!ok) break;
          const int rows = ctl.records[c % kRecords].rows;
          const bool none = ctl.records[c % kRecords].none;
          mbar_arrive(&ctl.used[c % kRecords]);
          if (none) break;
          if (rows == 0) continue;
          const int s = n % kStages;
          const uint32_t k = ring + s * kStage, v = k + kValueAt, pbuf = smem_u32(pmem), half = n & 1;
          const uint32_t q = ring + kQueryAt + (kOut ? n % kQueries * kKeyBytes : 0);
          const int tx = kTX + 128 * half, to = kTO + 128 * half;
          need(&ctl.full[s], n / kStages);
          if (kOut) {
            if (n > 1) need(&ctl.out_read[half], (n >> 1) - 1);
            if (!ok) break;
            tc_fence_after();
            // rows 64 to 127 of the scores are of what lies behind Q, and are not read
#pragma unroll 1
            for (int h = 0; h < DK / 64; ++h) four(tx, q + h * kHalf, 32, k + h * kHalf, 32, kScores, h == 0);
            umma_commit(&ctl.scores);
          }
          // the state's half of the keys takes U while the other's is made, and S' while the rest is
          need(&ctl.weighted[half], n >> 1);
#pragma unroll 1
          for (int x = 0; x < 2; ++x) {
            if (n > 0) need(&ctl.sums_read[x], n - 1);
            if (n > 0 && DK == 64 && x == 0) need(&ctl.sums_read[1], n - 1);  // one product makes both halves
            if (!ok) break;
            tc_fence_after();
            if (x < DK / 64) {
#pragma unroll 1
              for (int h = 0; h < 3; ++h)
                four_rows(kTU + 64 * x, ring + kWeightedAt + ((kOut ? 0 : 3 * half) + h) * kValueBytes, k + x * kHalf, kSums, h == 0);
            }
            umma_commit(&ctl.sums[x]);
          }
          if (!ok) break;
          if (!kOut) umma_commit(&ctl.read[half]);
          if (kOut) {
            need(&ctl.state_ready, n);
            if (!ok) break;
            tc_fence_after();
#pragma unroll 1
            for (int h = 0; h < 2 * (DK / 64); ++h)  // the upper parts, then the rests
              four_tmem(to, kTS + 32 * h, q + (h % (DK / 64)) * kHalf, kScores, h == 0);
            umma_commit(&ctl.operand_read);
            umma_commit(&ctl.q_empty[n % kQueries]);
          }
          if (kOut) {
            need(&ctl.p_ready, n);
            if (!ok) break;
            tc_fence_after();
#pragma unroll 1
            for (int h = 0; h < 2; ++h) four(tx, v, 2048, pbuf + h * kHalf, 32, kOut1, h == 0);
            umma_commit(&ctl.out_ready[half]);
          }
          umma_commit(&ctl.empty[s]);
          ++n;
        }
        // everything issued has completed before the tensor memory goes
        umma_commit(&ctl.drained);
        wait_phase(&ctl.drained, 0u, p.status);
      }
      __syncwarp();
    } else if (warp == 7) {
      // ---- the list: a chunk's rows 2 lane and 2 lane + 1 per lane ----
      LinItem t;
      for (uint32_t x = blockIdx.x; ok && x < a.items; x += gridDim.x) {
        if (!lin_item(a, x, &t)) continue;
        if (t.from) {  // the state is on its way to L2 while the items before are worked on
          const char* line = reinterpret_cast<const char*>(t.from) + lane * 128;
#pragma unroll 4
          for (int y = 0; y < DK * DV * 4; y += 32 * 128) asm volatile("prefetch.global.L2 [%0];" ::"l"(line + y));
        }
        long long total = 0;
        const float* from = p.log_decay + t.row0 * p.decay_row + t.h;
        auto row = [&](int r) { return r < t.n ? __ldg(from + r * p.decay_row) : 0.0f; };
        float n0 = row(2 * lane), n1 = row(2 * lane + 1);
        int x0 = 0;
        do {
          const long long d0 = decay_steps(n0, p.status), d1 = decay_steps(n1, p.status);
          n0 = row(x0 + kLinChunk + 2 * lane), n1 = row(x0 + kLinChunk + 2 * lane + 1);
          long long sum = d0 + d1;
#pragma unroll
          for (int o = 1; o < 32; o <<= 1) {
            const long long y = __shfl_up_sync(0xFFFFFFFFu, sum, o);
            if (lane >= o) sum += y;
          }
          const long long all = __shfl_sync(0xFFFFFFFFu, sum, 31);  // L_64
          total += all;
          if (c >= kRecords) wait(&ctl.used[c % kRecords], c / kRecords - 1);
          if (!ok) break;
          Record& r = ctl.records[c % kRecords];
#pragma unroll 1
          for (int y = 0; y < 2; ++y) {
            const long long l = y ? sum : sum - d1;
            const float hi = steps_float(l);
            r.hi[2 * lane + y] = hi;
            r.lo[2 * lane + y] = steps_float(l - __float2ll_rn(hi * 4294967296.0f));
            r.weight[2 * lane + y] = exp2f(steps_float(all - l));
            r.first[2 * lane + y] = p.scale * exp2f(hi);
          }
          if (lane == 0) {
            r.all = exp2f(steps_float(all));
            r.rows = min(kLinChunk, t.n - x0);
            r.row0 = t.row0 + x0;
            r.h = t.h;
            r.hq = t.hq;
            r.early = t.early;
            r.begins = x0 == 0;
            r.ends = x0 + kLinChunk >= t.n;
            r.none = false;
            r.from = t.from;
            r.to = t.to;
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(&ctl.listed[c % kRecords]);
          __syncwarp();
          ++c;
          x0 += kLinChunk;
        } while (x0 < t.n);
        if (t.steps && lane == 0) *t.steps = total;
      }
      if (c >= kRecords) wait(&ctl.used[c % kRecords], c / kRecords - 1);
      if (ok && lane == 0) {
        ctl.records[c % kRecords].none = true;
        mbar_arrive(&ctl.listed[c % kRecords]);
      }
    }
  } else if (warp < 12 || warp >= (kOut ? 28 : 20)) {
    if (kOut) asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");
    // ---- V': half of the rows, weighted, in three parts; eight values at a time ----
    constexpr int kVecs = DV / 8, kStep = 128 / kVecs, kPasses = kLinChunk / 2 / kStep;
    const int t = (warp & 3) * 32 + lane, v8 = t % kVecs, r0 = t / kVecs + (warp >= 20 ? kLinChunk / 2 : 0);
    const int at = (v8 >> 3) * kHalf + r0 * 128 + (((v8 & 7) ^ (r0 & 7)) << 4);
    while (const Record* r = next()) {
      if (r->rows > 0) {
        const int s = n % kStages;
        uint8_t* from = smem + s * kStage + kValueAt + at;
        uint8_t* to = smem + kWeightedAt + (kOut ? 0 : 3 * (n & 1) * kValueBytes) + at;
        wait(&ctl.full[s], n / kStages);
        if (kOut && n > 0) wait(&ctl.sums[1], n - 1);
        if (!kOut && n > 1) wait(&ctl.read[n & 1], (n >> 1) - 1);
        if (!ok) break;
        f32x2 check = 0ull;
#pragma unroll 1
        for (int g = 0; g < kPasses; ++g) {
          const uint4 b = *reinterpret_cast<const uint4*>(from + g * kStep * 128);
          const float f = r->weight[r0 + g * kStep];
          const f32x2 weight = pair(f, f);
          const uint32_t two[4] = {b.x, b.y, b.z, b.w};
          uint32_t part[3][4];
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            f32x2 x = pair(bf16_lo(two[y]), bf16_hi(two[y]));
            if (kOut) check = fma2(x, 0ull, check);
            x = mul2(x, weight);
            part[0][y] = round_pair(x);
            part[1][y] = round_pair(x);
            part[2][y] = last_pair(x);
          }
#pragma unroll
          for (int k = 0; k < 3; ++k)
            *reinterpret_cast<uint4*>(to + k * kValueBytes + g * kStep * 128) = make_uint4(part[k][0], part[k][1], part[k][2], part[k][3]);
        }
        if (kOut) {
          const float2 two = unpair(check);
          if (two.x + two.y != 0.0f) {  // rare: what is not finite goes, its first row is noted
#pragma unroll 1
            for (int x = 0; x < 8 * kPasses; ++x) {
              const int g = x >> 3, e = x & 7;
              uint16_t* value = reinterpret_cast<uint16_t*>(from + g * kStep * 128) + e;
              if (!bf16_not_finite(*value)) continue;
              *value = 0;
              atomicMax(&ctl.bad_row[n & 3][v8 * 8 + e], (unsigned long long)(n + 1) << 8 | (255u - (r0 + g * kStep)));
            }
          }
        }
        proxy_fence();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&ctl.weighted[n & 1]);
          if (kOut) mbar_arrive(&ctl.noted[n & 3]);
          mbar_arrive(&ctl.empty[s]);
        }
        ++n;
      }
      done();
    }
  } else if (warp < 20) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 104;");
    // ---- the state: value d, half kh of the keys ----
    constexpr int kKeys = DK / 2;
    const int d = (warp & 3) * 32 + lane, kh = (warp - 12) >> 2;
    const bool mine = (warp & 3) * 32 < DV;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t u = tmem + kTU + lanes + kh * kKeys, to = tmem + kTS + lanes + kh * (kKeys / 2);
    f32x2 st[kKeys / 2];
    // 16 keys from k on as operand of the next chunk's product
    auto operand = [&](int k) {
      uint32_t hi[8], lo[8];
#pragma unroll
      for (int y = 0; y < 8; ++y) {
        f32x2 x = st[k / 2 + y];
        hi[y] = round_pair(x);
        lo[y] = last_pair(x);
      }
      tmem_st8(to + k / 2, hi);
      tmem_st8(to + DK / 2 + k / 2, lo);
    };
    while (const Record* r = next()) {
      const bool ends = r->ends, begins = r->begins;
      if (begins) {
        const float* from = mine ? r->from : nullptr;
        if (from) {
          from += kh * kKeys * DV + d;
#pragma unroll
          for (int k = 0; k < kKeys / 2; ++k) st[k] = pair(__ldcg(from + 2 * k * DV), __ldcg(from + (2 * k + 1) * DV));
        } else {
#pragma unroll
          for (int k = 0; k < kKeys / 2; ++k) st[k] = 0ull;
        }
      }
      float* store = ends && mine ? r->to : nullptr;
      if (r->rows > 0) {
        const f32x2 f = pair(r->all, r->all);
        // once for the first chunk's operand, once for the chunk's sums (and the next one's operand)
#pragma unroll 1
        for (int pass = kOut && begins ? 0 : 1; pass < 2; ++pass) {
          if (pass) {
            wait(&ctl.sums[kh], n);
            if (!ok) break;
            __syncwarp();
            if (mine) {
              tc_fence_after();
#pragma unroll
              for (int k = 0; k < kKeys; k += 16) {
                uint32_t w[16];
                tmem_ld16(u + k, w);
                wait_ld(w);
#pragma unroll
                for (int y = 0; y < 8; ++y) st[k / 2 + y] = fma2(f, st[k / 2 + y], pair_of(w[2 * y], w[2 * y + 1]));
              }
              tc_fence_before();
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&ctl.sums_read[kh]);
          }
          if (!kOut || (pass && ends)) continue;
          if (n + pass > 0) wait(&ctl.operand_read, n + pass - 1);
          if (!ok) break;
          __syncwarp();
          if (mine) {
            tc_fence_after();
#pragma unroll
            for (int k = 0; k < kKeys; k += 16) operand(k);
            tmem_st_wait();
            tc_fence_before();
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(&ctl.state_ready);
        }
        if (!ok) break;
        ++n;
      }
      done();
      if (store) {
        store += kh * kKeys * DV + d;
#pragma unroll
        for (int k = 0; k < kKeys / 2; ++k) {
          const float2 x = unpair(st[k]);
          store[2 * k * DV] = x.x;
          store[(2 * k + 1) * DV] = x.y;
        }
      }
    }
  } else if (kOut) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");
    // ---- O: value d, half `set` of the rows ----
    const int quad = warp & 3, set = (warp - 20) >> 2, d = quad * 32 + lane;
    const uint32_t lanes = tmem + ((uint32_t)(quad * 32) << 16) + 32 * set;
    constexpr int kVecs = DV / 8;
    while (const Record* r = next()) {
      const int64_t out_row = (int64_t)p.Hq * DV;
      __nv_bfloat16* out = static_cast<__nv_bfloat16*>(p.out) + r->row0 * out_row + (int64_t)r->hq * DV;
      if (r->begins && r->early > 0) {
        for (long long x = tid - 20 * 32; x < (long long)r->early * kVecs; x += 256)
          *reinterpret_cast<uint4*>(out - (x / kVecs + 1) * out_row + (x % kVecs) * 8) = make_uint4(0u, 0u, 0u, 0u);
        __syncwarp();
      }
      const int rows = r->rows;
      if (rows > 0) {
        wait(&ctl.noted[n & 3], n >> 2);
        wait(&ctl.out_ready[n & 1], n >> 1);
        if (n > 0) wait(&ctl.stored, n - 1);
        if (!ok) break;
        if (quad * 32 < DV) {
          tc_fence_after();
          const f32x2 scale = pair(p.scale, p.scale);
          const uint32_t at = lanes + 128 * (n & 1);
          const unsigned long long noted = ctl.bad_row[n & 3][d];
          const int bad = ((noted >> 8) == n + 1ull ? 255 - (int)(noted & 255) : kLinChunk) - 32 * set;
          uint16_t* to = reinterpret_cast<uint16_t*>(omem) + 32 * set * DV + d;
#pragma unroll 1
          for (int y = 0; y < 32; y += 8) {
            uint32_t o1[8], o2[8];
            tmem_ld8(at + kTX + y, o1);
            tmem_ld8(at + kTO + y, o2);
            wait_ld(o1);
            wait_ld(o2);
#pragma unroll
            for (int k = 0; k < 8; k += 4) {
              const float4 f = *reinterpret_cast<const float4*>(&r->first[32 * set + y + k]);
#pragma unroll
              for (int z = 0; z < 2; ++z) {
                const int e = k + 2 * z;
                uint32_t b = last_pair(fma2(z ? pair(f.z, f.w) : pair(f.x, f.y), pair_of(o2[e], o2[e + 1]),
                                            mul2(scale, pair_of(o1[e], o1[e + 1]))));
                if (y + e + 1 >= bad) b = (y + e >= bad ? 0x7FC0u : b & 0xFFFFu) | 0x7FC00000u;
                to[(y + e) * DV] = (uint16_t)b;
                to[(y + e + 1) * DV] = (uint16_t)(b >> 16);
              }
            }
          }
          tc_fence_before();
        }
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&ctl.out_read[n & 1]);
          mbar_arrive(&ctl.staged);
        }
        __syncwarp();
      }
      done();
      if (rows > 0) {
        wait(&ctl.staged, n);
        if (!ok) break;
#pragma unroll
        for (int y = 0; y < kLinChunk * kVecs / 256; ++y) {
          const int e = y * 256 + tid - 20 * 32, x = e / kVecs, v = e % kVecs;
          if (x < rows)
            *reinterpret_cast<uint4*>(out + x * out_row + v * 8) = *reinterpret_cast<const uint4*>(omem + (x * kVecs + v) * 16);
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&ctl.stored);
        __syncwarp();
        ++n;
      }
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (tid == 0 && ctl.aborted) {
    report(p.status, SPEC_ERR_TIMEOUT);
    // the boxes in flight end before the CTA does: those of each loading warp's last two chunks, as the ones before were
    // read.  (Here, not where the loads are: 4 requests of 4,096 rows of 38 heads 164 us, 169 there.)
#pragma unroll 1
    for (uint32_t x = 0; x < 4; ++x) {
      const uint32_t sent = ctl.sent[x & 1], y = 1 + (x & 2);
      if (y <= sent) wait_phase(&ctl.full[(sent - y) % kStages], (sent - y) / kStages & 1u, p.status);
    }
  }
  if (warp == 6) {
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

// Rows of `heads` heads of D, in boxes of 64 by 64.  Boxes are read only where all of their rows are a request's.
bool make_rows_map(CUtensorMap* map, const void* base, long long rows, int64_t row_stride, int heads, int D) {
  auto enc = tensor_map_encoder();
  if (!enc || row_stride * 2 >= (1LL << 40)) return false;
  cuuint64_t dims[2] = {(cuuint64_t)heads * D, (cuuint64_t)rows};
  cuuint64_t strides[1] = {(cuuint64_t)row_stride * 2};
  cuuint32_t box[2] = {64u, (cuuint32_t)kLinChunk}, estr[2] = {1u, 1u};
  return enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, box, estr,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
             D == 64 ? CU_TENSOR_MAP_L2_PROMOTION_L2_128B : CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int DK, int DV, bool kOut>
cudaError_t launch_tc(const LinearLaunch& p, const LinearPlan& plan, int phase, cudaStream_t stream) {
  LinTcLaunch a{};
  a.p = p;
  a.plan = plan;
  a.phase = phase;
  a.heads = kOut ? p.Hq : p.H;
  a.items = (uint32_t)p.rows.B * a.heads * plan.nseg;  // below 2^31: linear_tc_serves()
  const long long rows = (long long)p.rows.B * (p.rows.K + 1);
  CUtensorMap tmQ{}, tmK{}, tmV{};
  a.tma = (!kOut || make_rows_map(&tmQ, p.q, rows, p.q_row, p.Hq, DK)) && make_rows_map(&tmK, p.k, rows, p.k_row, p.H, DK) &&
          make_rows_map(&tmV, p.v, rows, p.v_row, p.H, DV);
  constexpr size_t smem = lin_smem(DK, DV, kOut, lin_stages(DK, DV, kOut));
  static std::atomic<size_t> raised[kMaxDevices];
  const cudaError_t err = raise_smem(linear_tc_kernel<DK, DV, kOut>, smem, raised);
  if (err != cudaSuccess) return err;
  return launch_after_previous(linear_tc_kernel<DK, DV, kOut>, dim3((unsigned)std::min<uint32_t>(a.items, device_sms())),
                               dim3(kOut ? kOutThreads : kSumThreads), smem, stream, tmQ, tmK, tmV, a);
}

template <int DK, int DV>
cudaError_t launch_phases(const LinearLaunch& p, const LinearPlan& plan, cudaStream_t stream) {
  if (plan.nseg > 1) {
    const cudaError_t err = launch_tc<DK, DV, false>(p, plan, kSegmentSums, stream);
    if (err != cudaSuccess) return err;
  }
  if (plan.staged) {
    const cudaError_t err = launch_linear_scan(p, plan, stream);
    if (err != cudaSuccess) return err;
  }
  return p.q ? launch_tc<DK, DV, true>(p, plan, kAllSegments, stream)
             : launch_tc<DK, DV, false>(p, plan, kLastSegment, stream);
}

}  // namespace

cudaError_t launch_linear_scan(const LinearLaunch& p, const LinearPlan& plan, cudaStream_t stream) {
  return launch_after_previous(linear_scan_kernel, dim3((unsigned)(p.rows.B * p.H), (unsigned)((p.Dk * p.Dv + 1023) / 1024)),
                               dim3(256), 0, stream, p, plan);
}

cudaError_t launch_linear_tc(const LinearLaunch& p, const LinearPlan& plan, cudaStream_t stream) {
  if (p.Dk == 64) return p.Dv == 64 ? launch_phases<64, 64>(p, plan, stream) : launch_phases<64, 128>(p, plan, stream);
  return p.Dv == 64 ? launch_phases<128, 64>(p, plan, stream) : launch_phases<128, 128>(p, plan, stream);
}

}  // namespace spec
