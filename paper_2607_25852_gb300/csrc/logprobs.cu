// logprobs.cu -- log probabilities of given tokens, their ranks, the entropy and
// the most likely alternatives, from logits rows [rows, V] in one pass.
//
// With c2 = log2(e) / t, a reference M = fl(c2 m), m the largest logit so far, and
// d_v = c2 l_v - M with one rounding,
//   s = sum_v 2^d_v,  e = sum_v d_v 2^d_v,
//   ln p_v = ln 2 (c2 l_v - M - log2 s),  H = ln 2 (log2 s - e / s),
// whose terms are non-negative but for M's rounding, so nothing cancels.  (Where M
// is beyond thousands of binary orders d_v is c2 (l_v - m), whose first step is exact near m;
// sums of both kinds are joined with M's rounding.)
// A token's rank counts the entries that come before it (greater, or equal with a
// lower index); its logit is read first, so the count goes along, and only through
// the vectors whose largest element reaches it.
//
// The alternatives come along too.  Each thread notes the largest element of each of
// its 16-byte vectors.  After at most 8 rounds (of 512 vectors; a span), the n-th
// largest of the threads' maxima is a bound that the n-th best cannot be below; the
// few vectors that reach it are looked through again, and what reaches it goes to a
// list as a 64-bit key that orders by value and then by lower index.  A list that
// overflows, as many equal logits make it, is replaced by n searches for the next
// best key.  So the order in which lanes append does not show.
//
// The rows that are asked for, which only the device knows (of 64 requests of up to
// 17 rows a third may be), are laid end to end and cut into equal shares, one per
// CTA: a CTA has the end of a row, whole rows and the beginning of one.  So all
// are busy to the end, and their pieces end at different times.  Four warps go
// through the rounds and do nothing else; one brings them by bulk copies into a
// ring in shared memory; one looks for the best of a span and ends a piece while
// the four are at the next: done by the four themselves, with barriers, that took
// as long as the rounds did.  The last CTA to arrive at a row joins its pieces, in
// order.  No unit bounds many rows: of a round's 54 us the issue of about 14 instructions
// an entry takes 23, HBM 18, the exponentials 14; what is left are waits, for the vectors
// of a round and along each thread's two chains of sums, and the calls' begin and end
// (issue active 59 % of the SMs' active cycles, 44 % of all).  Few rows are bound by a
// chain of round trips.  587 rows of 201,088 with 8 alternatives 89 us after an L2 flush, 76 without
// alternatives (3.1 TB/s); one row 19 us then.
#include <cfloat>
#include <cmath>

#include <algorithm>

#include "attend_ring.cuh"
#include "paged.cuh"

namespace spec {

namespace {

// Measured at 64 requests of up to 17 rows of 201,088, a third asked for, with 8 alternatives / 1,024 rows of 50,021 in
// fp32 with 20: four CTAs of four warps 53.7 / 78.7 us, two of eight 51.6 / 82.7, three of four 58 / 91; eight vectors a
// thread 61 / 92; spans of four rounds 53.3 / 86.4.
constexpr int kLogWarps = 4, kLogThreads = kLogWarps * 32;  // that go through the rounds
constexpr int kVecs = 4;             // 16-byte vectors per thread and round
constexpr int kRoundVecs = kLogThreads * kVecs;
constexpr int kLogStages = 3;        // rounds in shared memory
constexpr int kCtasPerSm = 4;
constexpr int kMaxPieces = 22;       // of a row
// Vectors per CTA at least, so that short rows are not cut into more pieces than their join is worth: shares of 64 / 256 /
// 1,024 make no difference of 3 % but for 1,024 in 8 rows of 1,000 (25 / 27 / 41 us after an L2 flush).
constexpr int kMinShare = 256;
constexpr int kListCap = kMaxPieces * SPEC_MAX_TOP;  // keys that are looked at together: of all pieces, or of a span
constexpr int kFoundCap = 256;       // vectors of a span
// Requests up to which only the rows asked for are gone through (their list is 2 KB of shared memory); beyond, all rows
// have places, and those not asked for are passed over, which leaves CTAs idle: 142 us for 89 where a third is asked for.
constexpr int kMaxListed = 512;
constexpr int kSpan = 8;             // rounds whose best are looked for together
constexpr float kHuge = 8192.0f;     // of |M|: below it M's rounding, and so the largest d, is at most 2^-11
constexpr float kLowest = -3.0e38f;  // rounds to a finite number in both types
typedef unsigned long long Key;      // 0: none

struct alignas(16) LogPartial {
  float m, s, e;
  int32_t before;  // entries that come before the token; -1 where a logit is NaN or +inf
};

struct LogLaunch {
  const void* logits;
  const int32_t *tokens, *accepted;
  RowLayout rows;
  int V, n;
  float c2, inv_c2;
  float *logprob, *entropy, *top_logprobs;
  int32_t *rank, *top_tokens, *status;
  LogPartial* part;    // [row + CTA]: a row's pieces are consecutive CTAs', so no two are alike
  Key* part_keys;      // [row + CTA][n]
  uint32_t* arrived;   // [B (K + 1)]
};

__device__ __forceinline__ Key make_key(float x, int idx) {
  const uint32_t b = __float_as_uint(x + 0.0f);  // one zero
  const uint32_t o = b ^ ((b >> 31) ? 0xFFFFFFFFu : 0x80000000u);
  return ((Key)o << 32) | (uint32_t)~idx;
}
__device__ __forceinline__ float key_value(Key k) {
  const uint32_t o = (uint32_t)(k >> 32);
  return __uint_as_float(o ^ ((o >> 31) ? 0x80000000u : 0xFFFFFFFFu));
}
__device__ __forceinline__ int key_index(Key k) { return (int)~(uint32_t)k; }

// Element e (a constant) of a vector.
template <typename T>
__device__ __forceinline__ float element(const uint4& v, int e);
template <>
__device__ __forceinline__ float element<float>(const uint4& v, int e) {
  return __uint_as_float(e == 0 ? v.x : e == 1 ? v.y : e == 2 ? v.z : v.w);
}
template <>
__device__ __forceinline__ float element<__nv_bfloat16>(const uint4& v, int e) {
  const uint32_t w = e < 2 ? v.x : e < 4 ? v.y : e < 6 ? v.z : v.w;
  return (e & 1) ? bf16_hi(w) : bf16_lo(w);
}

// The largest element of a vector, NaN if one is.
template <typename T>
__device__ __forceinline__ float largest(const uint4& v);
template <>
__device__ __forceinline__ float largest<float>(const uint4& v) {
  return fmax_nan(fmax_nan(__uint_as_float(v.x), __uint_as_float(v.y)), fmax_nan(__uint_as_float(v.z), __uint_as_float(v.w)));
}
__device__ __forceinline__ uint32_t max_pair_nan(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
template <>
__device__ __forceinline__ float largest<__nv_bfloat16>(const uint4& v) {
  const uint32_t m = max_pair_nan(max_pair_nan(v.x, v.y), max_pair_nan(v.z, v.w));
  return fmax_nan(bf16_lo(m), bf16_hi(m));
}
// Elements 2 k and 2 k + 1, not below `least` (in both types; a NaN becomes that too).
template <typename T>
__device__ __forceinline__ f32x2 pair_from(const uint4& v, int k, float least, uint32_t);
template <>
__device__ __forceinline__ f32x2 pair_from<float>(const uint4& v, int k, float least, uint32_t) {
  return pair(fmaxf(element<float>(v, 2 * k), least), fmaxf(element<float>(v, 2 * k + 1), least));
}
template <>
__device__ __forceinline__ f32x2 pair_from<__nv_bfloat16>(const uint4& v, int k, float, uint32_t least) {
  uint32_t r;
  asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(k == 0 ? v.x : k == 1 ? v.y : k == 2 ? v.z : v.w), "r"(least));
  return pair(bf16_lo(r), bf16_hi(r));
}
// How many elements of a vector are at least `least`, a value of T.
template <typename T>
__device__ __forceinline__ int count_from(const uint4& v, float least);
template <>
__device__ __forceinline__ int count_from<float>(const uint4& v, float least) {
  int n = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) n += element<float>(v, k) >= least ? 1 : 0;
  return n;
}
template <>
__device__ __forceinline__ int count_from<__nv_bfloat16>(const uint4& v, float least) {
  const __nv_bfloat162 b = __float2bfloat162_rn(least);
  auto two = [&](uint32_t w) { return __hge2(*reinterpret_cast<const __nv_bfloat162*>(&w), b); };  // 1 or 0 each
  const __nv_bfloat162 n = __hadd2(__hadd2(two(v.x), two(v.y)), __hadd2(two(v.z), two(v.w)));
  return (int)(__low2float(n) + __high2float(n));
}
// The next number of T above x (a number of T).
template <typename T>
__device__ __forceinline__ float next_above(float x) {
  constexpr int kStep = sizeof(T) == 4 ? 1 : 0x10000;
  const int b = __float_as_int(x);
  return __int_as_float(x == 0.0f ? kStep : x > 0.0f ? min(b + kStep, 0x7F800000) : b - kStep);
}

// The difference of the references of the sums of a and of b, a at most b.  Below kHuge a reference is the rounded
// product with c2, beyond it the exact one: where one is of each kind, the rounding of the first counts.
__device__ __forceinline__ float reference_step(float a, float b, float c2) {
  const float x = __fmul_rn(a, c2), y = __fmul_rn(b, c2);
  const bool small_a = fabsf(x) < kHuge, small_b = fabsf(y) < kHuge;
  float d = a == b ? 0.0f : (a - b) * c2;
  if (small_a && small_b) d = x - y;
  else if (small_a) d += fmaf(-a, c2, x);
  else if (small_b) d += fmaf(b, c2, -y);
  return fmaxf(d, -1000.0f);  // -inf, and NaN of two that are -inf
}
// c2 l_v - M for the reference of m.
__device__ __forceinline__ float above_reference(float l, float m, float c2) {
  const float M = __fmul_rn(m, c2);
  return fabsf(M) < kHuge ? fmaf(l, c2, -M) : (l - m) * c2;
}
// Sums (m, s, e) brought to the reference of m' = top.
__device__ __forceinline__ void move_sums(float top, float m, float& s, float& e, float c2) {
  const float d = reference_step(m, top, c2), f = exp2f(d);
  e = f * fmaf(d, s, e);
  s = f * s;
}
// Adds up a value of each lane, in an order of its own.
__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
  return x;
}

// The n best of `count` keys in `list` to out[0 .. n), the best first; one warp, which has written them.
__device__ __forceinline__ void select_keys(const Key* list, int count, int n, Key* out) {
  const int lane = threadIdx.x & 31;
  __syncwarp();
  if (lane < n) out[lane] = 0;
  __syncwarp();
#pragma unroll 1
  for (int x = lane; x < count; x += 32) {
    const Key k = list[x];
    int before = 0;
#pragma unroll 4
    for (int y = 0; y < count; ++y) before += list[y] > k ? 1 : 0;
    if (before < n) out[before] = k;
  }
  __syncwarp();
}

struct LogShared {
  alignas(128) uint4 ring[kLogStages][kRoundVecs];
  // two spans' vectors' largest, as bf16 rounded up, and threads' largest
  alignas(16) uint16_t tops[2][kSpan * kVecs][kLogThreads];
  float most[2][kLogThreads];
  Key list[kListCap];
  Key best[SPEC_MAX_TOP];
  uint64_t full[kLogStages], empty[kLogStages], span_full[2], span_empty[2];
  int asked[kMaxListed + 1];  // rows asked for of the requests before
  int found[kFoundCap];
  float m[2][kLogWarps], s[2][kLogWarps], e[2][kLogWarps];  // of a piece that ends with the span
  int before[2][kLogWarps], sums[kLogWarps];
  int count, vectors, aborted;
};

// Rows of request i that are asked for; -1 where its arrays do not fit together.
__device__ __forceinline__ int asked_rows(const LogLaunch& p, int i) {
  const RequestRows q = request_rows(p.rows, i);
  const int accepted = p.accepted ? __ldg(p.accepted + i) : q.count - 1;
  return q.ok && accepted >= 0 && accepted < q.count ? accepted + 1 : -1;
}

// Element x of the outputs of a row that is not asked for, or cannot be answered.
__device__ __forceinline__ void write_nothing(const LogLaunch& p, long long r, int x) {
  if (x < p.n) {
    if (p.top_tokens) p.top_tokens[r * p.n + x] = -1;
    if (p.top_logprobs) p.top_logprobs[r * p.n + x] = -INFINITY;
  }
  if (x == 0) {
    p.logprob[r] = -INFINITY;
    if (p.rank) p.rank[r] = 0;
    if (p.entropy) p.entropy[r] = 0.0f;
  }
}

// The row's outputs from its sums and its best keys, by one warp.
__device__ __forceinline__ void write_row(const LogLaunch& p, long long r, float m, float s, float e, int before,
                                          int token, float given, const Key* best) {
  const int lane = threadIdx.x & 31;
  if (before < 0 || m == -INFINITY) {
    if (lane == 0) report(p.status, SPEC_ERR_BAD_INPUT);
    write_nothing(p, r, lane);
    return;
  }
  constexpr float kLn2 = 0.693147180559945309f;
  const float norm = log2f(s), c2 = p.c2, M = __fmul_rn(m, c2);
  // above_reference less log2 s, in halves: of a logit near the type's lowest value ln p is in fp32's range where log2 p is
  // not.  Roundings of a probability near 1 stay on this side of it (a NaN would stay one).
  auto log_of = [&](float l) {
    const float half = fabsf(M) < kHuge ? fmaf(0.5f * l, c2, -0.5f * M) : (0.5f * l - 0.5f * m) * c2;
    const float x = 2.0f * (kLn2 * (half - 0.5f * norm));
    return x > 0.0f ? 0.0f : x;
  };
  for (int x = lane; x < p.n; x += 32) {
    const Key k = best[x];
    if (p.top_tokens) p.top_tokens[r * p.n + x] = k ? key_index(k) : -1;
    if (p.top_logprobs) p.top_logprobs[r * p.n + x] = k ? log_of(key_value(k)) : -INFINITY;
  }
  if (lane == 0) {
    p.logprob[r] = token >= 0 ? log_of(given) : -INFINITY;
    if (p.rank) p.rank[r] = token >= 0 ? before + 1 : 0;
    const float x = kLn2 * (norm - e / s);
    if (p.entropy) p.entropy[r] = x < 0.0f ? 0.0f : x;
  }
}

// The vector whose first element is element `first` of a row, where the row ends in it: -inf for what is not the row's.
template <typename T>
__device__ __noinline__ uint4 row_end(const T* row, int first, int V) {
  constexpr int W = 16 / (int)sizeof(T);
  uint32_t y[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    uint32_t b[2] = {0xFF800000u, 0xFF800000u};
#pragma unroll
    for (int z = 0; z < W / 4; ++z) {
      const int e = first + k * (W / 4) + z;
      if (e >= 0 && e < V) b[z] = __float_as_uint(load_elem(row + e));
    }
    y[k] = sizeof(T) == 4 ? b[0] : b[0] >> 16 | (b[1] & 0xFFFF0000u);
  }
  return make_uint4(y[0], y[1], y[2], y[3]);
}
// The upper half of the least bf16 number that is not below x (a NaN stays above all bounds' reach).
__device__ __forceinline__ uint16_t rounded_up(float x) {
  const uint32_t b = __float_as_uint(x);
  return (uint16_t)((b + ((b >> 31) ? 0u : 0xFFFFu)) >> 16);
}

// A piece of a row.
template <typename T>
struct LogPiece {
  const T* row;
  int r, a;        // place in the outputs; place among the rows that are gone through
  int skip;        // elements of other rows in the row's first vector
  int begin, end;  // vectors; none where the row is not asked for
  bool asked;
  long long next;  // the next piece's position
};

template <typename T>
__global__ void __launch_bounds__(kLogThreads + 64, kCtasPerSm) logprobs_kernel(const LogLaunch p) {
  constexpr int W = 16 / (int)sizeof(T);
  extern __shared__ uint4 smem_raw[];
  LogShared& sh = *reinterpret_cast<LogShared*>((reinterpret_cast<uintptr_t>(smem_raw) + 127) & ~(uintptr_t)127);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, K1 = p.rows.K + 1, B = p.rows.B;
  if (tid == 0) {
    for (int s = 0; s < kLogStages; ++s) {
      mbar_init(&sh.full[s], 1);
      mbar_init(&sh.empty[s], kLogWarps);
    }
    for (int s = 0; s < 2; ++s) {
      mbar_init(&sh.span_full[s], kLogWarps);
      mbar_init(&sh.span_empty[s], 1);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    sh.aborted = 0;
    sh.asked[0] = 0;
    sh.count = 0;
    sh.vectors = 0;
  }
  pdl_wait_prerequisites();
  pdl_launch_dependents();

  // ---- the rows that are asked for (all, unsorted, where there are too many requests to list) ----
  const bool listed = B <= kMaxListed;
  int rows = B * K1;
  if (listed) {
    rows = 0;
    for (int i0 = 0; i0 < B; i0 += kLogThreads) {
      const int i = i0 + tid, mine = i < B && tid < kLogThreads ? asked_rows(p, i) : 0;
      if (mine < 0 && blockIdx.x == 0) report(p.status, SPEC_ERR_BAD_INPUT);
      int sum = max(mine, 0);
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xFFFFFFFFu, sum, o);
        if (lane >= o) sum += y;
      }
      if (lane == 31 && warp < kLogWarps) sh.sums[warp] = sum;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < kLogWarps; ++w) {
        if (w < warp) sum += sh.sums[w];
      }
      if (i < B && tid < kLogThreads) sh.asked[i + 1] = rows + sum;
#pragma unroll
      for (int w = 0; w < kLogWarps; ++w) rows += sh.sums[w];
      __syncthreads();
    }
  } else {
    __syncthreads();
  }
  // request and place of row a
  auto place = [&](int a, int& i, int& j) {
    if (listed) {
      int lo = 0, hi = B - 1;
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (sh.asked[mid + 1] <= a) lo = mid + 1;
        else hi = mid;
      }
      i = lo;
      j = a - sh.asked[lo];
    } else {
      i = a / K1;
      j = a - i * K1;
    }
  };

  // ---- this CTA's share: vectors at .. share_end - 1 of the rows laid end to end ----
  const int nv = (int)(((long long)p.V + 2 * W - 2) / W);  // a row's, its ends as misaligned as can be
  const long long total = (long long)rows * nv;
  auto divide = [&](long long x, long long by) {  // (few pieces need 64 bits)
    return total < (1LL << 31) ? (int)((uint32_t)x / (uint32_t)by) : (int)(x / by);
  };
  const long long share = max(max((total + gridDim.x - 1) / gridDim.x, (long long)(nv / (kMaxPieces - 2) + 1)), (long long)kMinShare);
  const long long share_begin = blockIdx.x * share, share_end = min(share_begin + share, total);
  // the piece at `pos`; false past the share
  auto piece_at = [&](long long pos, LogPiece<T>& t) {
    if (pos >= share_end) return false;
    t.a = divide(pos, nv);
    int i, j;
    place(t.a, i, j);
    t.r = i * K1 + j;
    t.begin = (int)(pos - (long long)t.a * nv);
    t.next = pos + min((long long)(nv - t.begin), share_end - pos);
    t.asked = listed || j < asked_rows(p, i);
    const int row0 = p.rows.row_offsets ? __ldg(p.rows.row_offsets + i) : i * K1;
    t.row = static_cast<const T*>(p.logits) + (t.asked ? (long long)(row0 + j) * p.V : 0);
    t.skip = (int)((reinterpret_cast<uintptr_t>(t.row) & 15u) / sizeof(T));
    // a row may have one vector fewer than nv
    t.end = t.asked ? min(t.begin + (int)(t.next - pos), (int)(((long long)p.V + t.skip + W - 1) / W)) : t.begin;
    return true;
  };
  LogPiece<T> t;

  if (warp == kLogWarps) {
    // ---- brings the rounds, ahead of the others ----
    if (lane == 0) {
      uint32_t brought = 0;
      bool ok = true;
      for (long long pos = share_begin; ok && piece_at(pos, t); pos = t.next) {
        // whole vectors of the row; its ends are read where they are used
        const int inner = t.skip ? 1 : 0, outer = (int)(((long long)p.V + t.skip) / W);
        for (int at = t.begin; at < t.end; at += kRoundVecs, ++brought) {
          const int lo = max(at, inner), hi = min(min(at + kRoundVecs, t.end), outer), s = brought % kLogStages;
          ok = brought < kLogStages || wait_phase(&sh.empty[s], (brought / kLogStages - 1) & 1u, p.status);
          if (!ok) break;
          const uint32_t bytes = hi > lo ? (uint32_t)(hi - lo) * 16u : 0u;
          mbar_expect_tx(&sh.full[s], bytes);
          if (bytes)
            asm volatile(
                "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                    smem_u32(&sh.ring[s][lo - at])),
                "l"(t.row - t.skip + (long long)lo * W), "r"(bytes), "r"(smem_u32(&sh.full[s]))
                : "memory");
        }
      }
      if (!ok) {
        *(volatile int*)&sh.aborted = 1;
        // the copies in flight end before the CTA does
        for (uint32_t y = brought - kLogStages; y < brought; ++y) wait_phase(&sh.full[y % kLogStages], (y / kLogStages) & 1u, p.status);
      }
    }
    return;
  }

  // Waits by a whole warp; false, for all of the CTA soon, where one gave up.
  auto wait = [&](uint64_t* bar, uint32_t parity) {
    if (__all_sync(0xFFFFFFFFu, mbar_try_wait(bar, parity & 1u))) return true;
    const bool there = !*(volatile int*)&sh.aborted && mbar_wait_slow(bar, parity & 1u, p.status);
    if (__all_sync(0xFFFFFFFFu, there)) return true;
    *(volatile int*)&sh.aborted = 1;
    return false;
  };
  uint32_t spans = 0;

  if (warp < kLogWarps) {
    // ---- goes through the rounds ----
    uint32_t used = 0;
    for (long long pos = share_begin; piece_at(pos, t); pos = t.next) {
      if (!t.asked) continue;
      int token = __ldg(p.tokens + t.r);
      if (token < -1 || token >= p.V) {
        if (t.begin == 0 && tid == 0) report(p.status, SPEC_ERR_BAD_INPUT);
        token = -1;
      }
      const float given = token >= 0 ? load_elem(t.row + token) : INFINITY;
      const float above = next_above<T>(given);
      float m = -INFINITY;
      f32x2 s2 = 0ull, e2 = 0ull;
      int before = 0;
      bool bad = false;
      const f32x2 c2 = pair(p.c2, p.c2);
      int v0 = t.begin;
      do {  // a span
        const int buffer = spans & 1;
        if (spans >= 2 && !wait(&sh.span_empty[buffer], (spans >> 1) - 1)) return;
        float most_of_span = -INFINITY;
        int round = 0;
#pragma unroll 1
        for (; round < kSpan && v0 < t.end; ++round, v0 += kRoundVecs, ++used) {
          // ---- a round's vectors ----
          uint4 w[kVecs];
          const int st = used % kLogStages;
          if (!wait(&sh.full[st], used / kLogStages)) return;
          const bool plain = v0 + kRoundVecs <= t.end && v0 * W >= t.skip && (v0 + kRoundVecs) * W - t.skip <= p.V;
#pragma unroll
          for (int u = 0; u < kVecs; ++u) {
            w[u] = sh.ring[st][u * kLogThreads + tid];
            if (!plain) {
              const int v = v0 + u * kLogThreads + tid, first = v * W - t.skip;
              if (v >= t.end || first < 0 || first + W > p.V) w[u] = row_end<T>(t.row, v < t.end ? first : p.V, p.V);
            }
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(&sh.empty[st]);
          float top[kVecs], most = -INFINITY;
#pragma unroll
          for (int u = 0; u < kVecs; ++u) {
            top[u] = largest<T>(w[u]);
            bad |= !(top[u] < INFINITY);
            most = fmaxf(most, top[u]);
          }
          // ---- sums ----
          if (most > m) {
            const float d = reference_step(m, most, p.c2), f = exp2f(d);
            e2 = mul2(pair(f, f), fma2(pair(d, d), s2, e2));
            s2 = mul2(pair(f, f), s2);
            m = most;
          }
          const float M = __fmul_rn(m, p.c2);
          // what is 1,000 binary orders below the largest, and -inf, counts as that: 0 times a number
          const float low = m - 1000.0f * p.inv_c2;
          if (fabsf(M) < kHuge && low > kLowest) {
            const f32x2 minus_M = pair(-M, -M);
            const uint32_t low2 = last_pair(pair(low, low));
#pragma unroll
            for (int u = 0; u < kVecs; ++u)
#pragma unroll
              for (int k = 0; k < W / 2; ++k) {
                const f32x2 d = fma2(pair_from<T>(w[u], k, low, low2), c2, minus_M);
                const float2 x = unpair(d);
                const f32x2 y = pair(ex2_approx(x.x), ex2_approx(x.y));
                s2 = add2(s2, y);
                e2 = fma2(d, y, e2);
              }
          } else if (m > -INFINITY) {  // M is huge, or temperatures put those orders outside the type
#pragma unroll
            for (int u = 0; u < kVecs; ++u)
#pragma unroll
              for (int k = 0; k < W; ++k) {
                const float x = fmaxf(above_reference(element<T>(w[u], k), m, p.c2), -1000.0f);
                const f32x2 y = pair(ex2_approx(x), 0.0f);
                s2 = add2(s2, y);
                e2 = fma2(pair(x, 0.0f), y, e2);
              }
          }
          // ---- entries before the token: of `given` and more, behind the token of more than that ----
          if (token >= 0) {
#pragma unroll
            for (int u = 0; u < kVecs; ++u) {
              const int v = v0 + u * kLogThreads + tid, first = v * W - t.skip;
              if (!(top[u] >= given) || v >= t.end) continue;
              before += count_from<T>(w[u], first + W <= token ? given : above);
              if (first <= token && first + W > token) {  // its own vector: those equal to it before it
#pragma unroll
                for (int k = 0; k < W; ++k) before += element<T>(w[u], k) == given && first + k < token ? 1 : 0;
              }
              // what is not the row's is -inf, before its first entry as well
              if (first < 0 && given == -INFINITY) before += first;
            }
          }
          if (p.n > 0) {
#pragma unroll
            for (int u = 0; u < kVecs; ++u) sh.tops[buffer][round * kVecs + u][tid] = rounded_up(top[u]);
            most_of_span = fmaxf(most_of_span, most);
          }
        }
        sh.most[buffer][tid] = most_of_span;
        if (v0 >= t.end) {  // the piece's sums
          const float top = warp_max(m);
          float2 half = unpair(s2);
          float s = half.x + half.y;
          half = unpair(e2);
          float e = half.x + half.y;
          move_sums(top, m, s, e, p.c2);
          s = warp_sum(s);
          e = warp_sum(e);
          before = __reduce_add_sync(0xFFFFFFFFu, before);
          bad = __any_sync(0xFFFFFFFFu, bad);
          if (lane == 0) {
            sh.m[buffer][warp] = top;
            sh.s[buffer][warp] = s;
            sh.e[buffer][warp] = e;
            sh.before[buffer][warp] = bad ? -1 : before;
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.span_full[buffer]);
        ++spans;
      } while (v0 < t.end);
    }
    return;
  }

  // ---- the last warp: outputs of rows that are not asked for, the best of spans, the ends of pieces ----
  const int cells = max(p.n, 1);
  for (long long x = (long long)blockIdx.x * 32 + lane; x < (long long)B * K1 * cells; x += (long long)gridDim.x * 32) {
    const int r = (int)(x / cells), i = r / K1, j = r - i * K1;
    const int n = listed ? sh.asked[i + 1] - sh.asked[i] : asked_rows(p, i);
    if (n < 0 && j == 0) report(p.status, SPEC_ERR_BAD_INPUT);
    if (j >= n) write_nothing(p, r, (int)(x - (long long)r * cells));
  }
  for (long long pos = share_begin; piece_at(pos, t); pos = t.next) {
    if (!t.asked) continue;
    int token = __ldg(p.tokens + t.r);
    if (token < -1 || token >= p.V) token = -1;
    const float given = token >= 0 ? load_elem(t.row + token) : INFINITY;
    float bound = -FLT_MAX;
    int kept = 0;  // keys in the list: the best so far
    int v0 = t.begin, buffer;
    for (;;) {
      buffer = spans & 1;
      const int span = v0, rounds = min(kSpan, (t.end - v0 + kRoundVecs - 1) / kRoundVecs);
      v0 += kSpan * kRoundVecs;
      if (!wait(&sh.span_full[buffer], spans >> 1)) return;
      ++spans;
      if (p.n > 0 && rounds > 0) {
        // ---- a bound: the n-th best of the spans before, or the n-th largest of the threads' maxima ----
        float most[kLogWarps], reached = -FLT_MAX;
#pragma unroll
        for (int y = 0; y < kLogWarps; ++y) most[y] = sh.most[buffer][y * 32 + lane];
#pragma unroll 1
        for (int k = kept < p.n ? 0 : p.n; k < p.n; ++k) {
          float mine = most[0];
#pragma unroll
          for (int y = 1; y < kLogWarps; ++y) mine = fmaxf(mine, most[y]);
          reached = warp_max(mine);
          const uint32_t has = __ballot_sync(0xFFFFFFFFu, mine == reached);
          if (lane == __ffs((int)has) - 1) {
            bool gone = false;
#pragma unroll
            for (int y = 0; y < kLogWarps; ++y)
              if (!gone && most[y] == reached) most[y] = -INFINITY, gone = true;
          }
        }
        bound = fmaxf(bound, reached);
        // ---- the vectors that reach it ----
        auto vectors = [&](auto f) {  // calls f(vector of the span)
#pragma unroll 1
          for (int slot = 0; slot < rounds * kVecs; slot += 2) {
            // 8 of 128 threads per lane, two slots at a time
            const uint4 v = *reinterpret_cast<const uint4*>(&sh.tops[buffer][slot + (lane >> 4)][(lane & 15) * 8]);
            if (!(largest<__nv_bfloat16>(v) >= bound)) continue;
#pragma unroll
            for (int k = 0; k < 8; ++k)
              if (element<__nv_bfloat16>(v, k) >= bound) f((slot + (lane >> 4)) * kLogThreads + (lane & 15) * 8 + k);
          }
          __syncwarp();
        };
        auto entries = [&](int x, auto f) {  // calls f(key) for what reaches the bound in vector x
          const int first = (span + x) * W - t.skip;
          const uint4 v = first >= 0 && first + W <= p.V ? __ldg(reinterpret_cast<const uint4*>(t.row + first))
                                                         : row_end<T>(t.row, first, p.V);
#pragma unroll
          for (int k = 0; k < W; ++k)
            if (element<T>(v, k) >= bound) f(make_key(element<T>(v, k), first + k));
        };
        vectors([&](int x) {
          const int at = atomicAdd(&sh.vectors, 1);
          if (at < kFoundCap) sh.found[at] = x;
        });
        const int found = sh.vectors;
        __syncwarp();
        if (lane == 0) sh.vectors = 0, sh.count = kept;
        __syncwarp();
        int keys = kListCap + 1;
        if (found <= kFoundCap) {
#pragma unroll 1
          for (int x = lane; x < found; x += 32)
            entries(sh.found[x], [&](Key k) {
              const int at = atomicAdd(&sh.count, 1);
              if (at < kListCap) sh.list[at] = k;
            });
          __syncwarp();
          keys = sh.count;
        }
        if (keys > kListCap) {
          // ---- too many: this span's n best one after another, behind those of the spans before ----
          Key last = ~(Key)0;
          keys = kept;
#pragma unroll 1
          for (int y = 0; y < p.n; ++y) {
            Key next = 0;
            vectors([&](int x) {
              entries(x, [&](Key k) {
                if (k < last && k > next) next = k;
              });
            });
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) next = max(next, __shfl_xor_sync(0xFFFFFFFFu, next, o));
            if (next == 0) break;
            last = next;
            if (lane == 0) sh.list[keys] = next;
            ++keys;
          }
        }
        select_keys(sh.list, keys, p.n, sh.best);
        kept = min(keys, p.n);
        if (lane < kept) sh.list[lane] = sh.best[lane];
        if (kept == p.n) bound = fmaxf(bound, key_value(sh.best[p.n - 1]));
        __syncwarp();
      }
      if (v0 >= t.end) break;
      if (lane == 0) mbar_arrive(&sh.span_empty[buffer]);
    }

    // ---- the piece's sums and best ----
    if (p.n > 0 && kept < p.n) {
      if (lane >= kept && lane < p.n) sh.best[lane] = 0;
      __syncwarp();
    }
    float m = lane < kLogWarps ? sh.m[buffer][lane] : -INFINITY, s = 0.0f, e = 0.0f;
    int before = 0;
    if (lane < kLogWarps) s = sh.s[buffer][lane], e = sh.e[buffer][lane], before = sh.before[buffer][lane];
    __syncwarp();
    if (lane == 0) mbar_arrive(&sh.span_empty[buffer]);
    auto join = [&]() {  // the lanes' sums
      const float top = warp_max(m);
      move_sums(top, m, s, e, p.c2);
      m = top;
      s = warp_sum(s);
      e = warp_sum(e);
      const bool bad = __any_sync(0xFFFFFFFFu, before < 0);
      before = __reduce_add_sync(0xFFFFFFFFu, before);
      if (bad) before = -1;
    };
    join();
    // the CTAs that have a piece of the row
    const int b0 = divide((long long)t.a * nv, share), b1 = divide((long long)(t.a + 1) * nv - 1, share), pieces = b1 - b0 + 1;
    if (pieces > 1) {
      const size_t x = (size_t)t.a + blockIdx.x;
      if (lane < p.n) p.part_keys[x * p.n + lane] = sh.best[lane];
      if (lane == 0) p.part[x] = LogPartial{m, s, e, before};
      __threadfence();
      __syncwarp();
      int last = 0;
      if (lane == 0) last = atomicAdd(p.arrived + t.a, 1u) == (uint32_t)pieces - 1;
      if (!__shfl_sync(0xFFFFFFFFu, last, 0)) continue;
      // ---- the last CTA of the row joins the pieces, one per lane ----
      __threadfence();
      if (lane == 0) p.arrived[t.a] = 0;
      const uint4 v = lane < pieces ? __ldcg(reinterpret_cast<const uint4*>(p.part + t.a + b0 + lane))
                                    : make_uint4(0xFF800000u, 0u, 0u, 0u);
      const Key* keys = p.part_keys + ((size_t)t.a + b0) * p.n;
      if (p.n) {
        // what is below some piece's n-th best is not among the n best
        Key least = lane < pieces ? __ldcg(keys + (size_t)lane * p.n + p.n - 1) : 0;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) least = max(least, __shfl_xor_sync(0xFFFFFFFFu, least, o));
        if (lane == 0) sh.count = 0;
        __syncwarp();
#pragma unroll 4
        for (int y = lane; y < pieces * p.n; y += 32) {
          const Key k = __ldcg(keys + y);
          if (k != 0 && k >= least) sh.list[atomicAdd(&sh.count, 1)] = k;
        }
        __syncwarp();
        const int count = sh.count;
        select_keys(sh.list, count, p.n, sh.best);
      }
      m = __uint_as_float(v.x), s = __uint_as_float(v.y), e = __uint_as_float(v.z), before = (int)v.w;
      join();
    }
    write_row(p, t.r, m, s, e, before, token, given, sh.best);
    __syncwarp();
  }
}

struct LogGeometry {
  int ctas;
  size_t part_off, keys_off, bytes;
};

bool logprobs_shape_ok(int B, int K, int V, int n) {
  return rows_shape_ok(B, K) && V >= 1 && V < SPEC_MAX_VOCAB && n >= 0 && n <= SPEC_MAX_TOP;
}

LogGeometry logprobs_geometry(int B, int K, int V, int n) {
  LogGeometry g{};
  const long long R = (long long)B * (K + 1);
  // the device that plans are made for: a workspace's size must not depend on the one it is asked on
  g.ctas = (int)std::min<long long>(152 * kCtasPerSm, R * (V / (8 * kMinShare) + 1));
  const size_t pieces = (size_t)R + g.ctas;
  g.part_off = ((size_t)R * 4 + 255) / 256 * 256;
  g.keys_off = g.part_off + (pieces * sizeof(LogPartial) + 255) / 256 * 256;
  g.bytes = g.keys_off + (pieces * n * sizeof(Key) + 255) / 256 * 256;
  return g;
}

template <typename T>
cudaError_t launch_logprobs(const LogLaunch& p, int ctas, cudaStream_t stream) {
  constexpr size_t smem = sizeof(LogShared) + 128;
  static std::atomic<size_t> raised[kMaxDevices];
  const cudaError_t err = raise_smem(logprobs_kernel<T>, smem, raised);
  if (err != cudaSuccess) return err;
  return launch_after_previous(logprobs_kernel<T>, dim3((unsigned)ctas), dim3(kLogThreads + 64), smem, stream, p);
}

}  // namespace

}  // namespace spec

extern "C" size_t spec_logprobs_workspace(int B, int K, int V, int top_n) {
  if (!spec::logprobs_shape_ok(B, K, V, top_n)) return 0;
  return spec::logprobs_geometry(B, K, V, top_n).bytes;
}

extern "C" int spec_logprobs(const void* logits, int logits_dtype, const int32_t* row_offsets, const int32_t* depth,
                             const int32_t* tokens, const int32_t* accepted_len, int B, int K, int V, float temperature,
                             int top_n, float* logprob_out, int32_t* rank_out, float* entropy_out,
                             int32_t* top_tokens_out, float* top_logprobs_out, int32_t* status, void* ws,
                             size_t ws_bytes, cudaStream_t stream) {
  spec::NvtxRange range("spec_logprobs");
  using namespace spec;
  if (!logprobs_shape_ok(B, K, V, top_n) || (logits_dtype != SPEC_BF16 && logits_dtype != SPEC_F32))
    return SPEC_ERR_INVALID_ARG;
  if (!logits || !tokens || !logprob_out || (top_n > 0 && !top_tokens_out && !top_logprobs_out))
    return SPEC_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(logits) % element_size(logits_dtype) != 0 || !(temperature >= 0.0f) ||
      std::isinf(temperature) || (temperature > 0.0f && temperature < FLT_MIN))  // log2(e) / t is finite
    return SPEC_ERR_INVALID_ARG;
  const LogGeometry g = logprobs_geometry(B, K, V, top_n);
  if (!ws || ws_bytes < g.bytes || (reinterpret_cast<uintptr_t>(ws) & 255u) != 0) return SPEC_ERR_WORKSPACE;
  LogLaunch p{};
  p.logits = logits;
  p.tokens = tokens;
  p.accepted = accepted_len;
  p.rows = RowLayout{row_offsets, depth, nullptr, B, K};
  p.V = V;
  p.n = top_n;
  p.c2 = (float)(1.4426950408889634 / (temperature > 0.0f ? (double)temperature : 1.0));
  p.inv_c2 = 1.0f / p.c2;
  p.logprob = logprob_out;
  p.entropy = entropy_out;
  p.top_logprobs = top_logprobs_out;
  p.rank = rank_out;
  p.top_tokens = top_tokens_out;
  p.status = status;
  char* base = static_cast<char*>(ws);
  p.arrived = reinterpret_cast<uint32_t*>(base);
  p.part = reinterpret_cast<LogPartial*>(base + g.part_off);
  p.part_keys = reinterpret_cast<Key*>(base + g.keys_off);
  const cudaError_t err = logits_dtype == SPEC_F32 ? launch_logprobs<float>(p, g.ctas, stream)
                                                   : launch_logprobs<__nv_bfloat16>(p, g.ctas, stream);
  return err == cudaSuccess && cudaGetLastError() == cudaSuccess ? SPEC_OK : SPEC_ERR_CUDA;
}
