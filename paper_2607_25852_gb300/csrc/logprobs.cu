// logprobs.cu -- log probabilities of given tokens, their ranks, the entropy and
// the most likely alternatives, from logits rows [rows, V] in one pass.
//
// With c2 = log2(e) / t, a reference M = fl(c2 m), m the largest logit so far, and
// d_v = c2 l_v - M with one rounding,
//   s = sum_v 2^d_v,  e = sum_v d_v 2^d_v,
//   ln p_v = ln 2 (c2 l_v - M - log2 s),  H = ln 2 (log2 s - e / s),
// whose terms are non-negative but for M's rounding, so nothing cancels.  (Where M
// is so large that the logits' own spacing is tens of binary orders, d_v is c2 (l_v - m).)
// A token's rank counts the entries that come before it (greater, or equal with a
// lower index); its logit is read first, so the count goes along, and only through
// the vectors whose largest element reaches it.
//
// The alternatives come along too.  Each thread notes the largest element of each of
// its 16-byte vectors.  After at most 16 rounds of 1,024 vectors, n values that are
// known to be there (the four largest of each warp's lanes' maxima) give a bound
// that the n-th best cannot be below; the few vectors that reach it are looked
// through again, and what reaches it goes to a list as a 64-bit key that orders by
// value and then by lower index.  A list that overflows, as many equal logits make
// it, is replaced by n searches for the next best key.  So the order in which
// threads append does not show.
//
// The rows that are asked for, which only the device knows (of 64 requests of up to
// 17 rows a third may be), are laid end to end and cut into equal shares, one per
// CTA: a CTA has the end of a row, whole rows and the beginning of one.  So all
// are busy to the end, and their pieces end at different times.  A warp of
// its own brings the rounds by bulk copies into a ring in shared memory, ahead
// across pieces.  The last
// CTA to arrive at a row joins its pieces, in order.  Bound by HBM for many rows,
// by the launch and three round trips for few.
#include <cfloat>
#include <cmath>

#include <algorithm>

#include "attend_ring.cuh"
#include "paged.cuh"

namespace spec {

namespace {

constexpr int kLogThreads = 256, kLogWarps = kLogThreads / 32;
constexpr int kVecs = 4;             // 16-byte vectors per thread and round
constexpr int kRoundVecs = kLogThreads * kVecs;
constexpr int kLogStages = 4;        // rounds in shared memory
constexpr int kCtasPerSm = 2;
constexpr int kMaxPieces = 64;       // of a row
constexpr int kMinShare = 256;       // vectors per CTA
constexpr int kMaxListed = 1024;     // requests up to which only the rows asked for are gone through
constexpr int kSpan = 16;            // rounds whose best are looked for together
constexpr float kHuge = 1073741824.0f;  // 2^30: of |M|
constexpr int kListCap = kMaxPieces * SPEC_MAX_TOP;  // what a join may have to look at
constexpr int kListFull = 512;       // what a round may append to
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
  float c2;
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
// The difference of the references of two sums, at most 0 for b the larger.
__device__ __forceinline__ float reference_step(float a, float b, float c2) {
  const float x = __fmul_rn(a, c2), y = __fmul_rn(b, c2);
  const float d = fabsf(x) < kHuge && fabsf(y) < kHuge ? x - y : a == b ? 0.0f : (a - b) * c2;
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

// The n best of `count` keys in `list` to out[0 .. n), the best first.
static __device__ __noinline__ void select_keys(const Key* list, int count, int n, Key* out) {
  for (int x = threadIdx.x; x < n; x += kLogThreads)
    if (x >= count) out[x] = 0;
  for (int x = threadIdx.x; x < count; x += kLogThreads) {
    const Key k = list[x];
    int before = 0;
#pragma unroll 4
    for (int y = 0; y < count; ++y) before += list[y] > k ? 1 : 0;
    if (before < n) out[before] = k;
  }
}

struct LogShared {
  alignas(128) uint4 ring[kLogStages][kRoundVecs];
  union {
    uint16_t tops[kSpan * kVecs][kLogThreads];  // each thread's vectors' largest, as bf16, rounded up
    Key joined[kListCap];
  };
  Key list[kListFull];
  Key best[SPEC_MAX_TOP];
  Key warp_key[kLogWarps];
  uint64_t full[kLogStages], empty[kLogStages];
  int asked[kMaxListed + 1];  // rows asked for of the requests before
  float warp_top[kLogWarps * 4];
  float m[kLogWarps], s[kLogWarps], e[kLogWarps];
  int before[kLogWarps], sums[kLogWarps];
  int count, last, aborted;
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

// The row's outputs from its sums and its best keys (in shared memory).
__device__ __forceinline__ void write_row(const LogLaunch& p, long long r, float m, float s, float e, int before,
                                          int token, float given, const Key* best) {
  if (before < 0 || m == -INFINITY) {
    if (threadIdx.x == 0) report(p.status, SPEC_ERR_BAD_INPUT);
    if (threadIdx.x < 32) write_nothing(p, r, threadIdx.x);
    return;
  }
  constexpr float kLn2 = 0.693147180559945309f;
  const float norm = log2f(s), c2 = p.c2;
  for (int x = threadIdx.x; x < p.n; x += kLogThreads) {
    const Key k = best[x];
    if (p.top_tokens) p.top_tokens[r * p.n + x] = k ? key_index(k) : -1;
    if (p.top_logprobs) p.top_logprobs[r * p.n + x] = k ? kLn2 * (above_reference(key_value(k), m, c2) - norm) : -INFINITY;
  }
  if (threadIdx.x == 0) {
    p.logprob[r] = token >= 0 ? kLn2 * (above_reference(given, m, c2) - norm) : -INFINITY;
    if (p.rank) p.rank[r] = token >= 0 ? before + 1 : 0;
    if (p.entropy) p.entropy[r] = kLn2 * (norm - e / s);
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
  int begin, end;  // vectors; nothing where the row is not asked for
  bool asked;
};

template <typename T>
__global__ void __launch_bounds__(kLogThreads + 32, kCtasPerSm) logprobs_kernel(const LogLaunch p) {
  constexpr int W = 16 / (int)sizeof(T);
  extern __shared__ uint4 smem_raw[];
  LogShared& sh = *reinterpret_cast<LogShared*>((reinterpret_cast<uintptr_t>(smem_raw) + 127) & ~(uintptr_t)127);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, K1 = p.rows.K + 1, B = p.rows.B;
  if (tid == 0) {
    for (int s = 0; s < kLogStages; ++s) {
      mbar_init(&sh.full[s], 1);
      mbar_init(&sh.empty[s], kLogWarps);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    sh.aborted = 0;
    sh.asked[0] = 0;
    sh.count = 0;
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
      int all = 0;
#pragma unroll
      for (int w = 0; w < kLogWarps; ++w) all += sh.sums[w];
      rows += all;
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
  // ---- the others' outputs ----
  const int cells = max(p.n, 1);
  for (long long x = (long long)blockIdx.x * kLogThreads + tid; tid < kLogThreads && x < (long long)B * K1 * cells; x += (long long)gridDim.x * kLogThreads) {
    const int r = (int)(x / cells), i = r / K1, j = r - i * K1;
    const int n = listed ? sh.asked[i + 1] - sh.asked[i] : asked_rows(p, i);
    if (n < 0 && j == 0) report(p.status, SPEC_ERR_BAD_INPUT);
    if (j >= n) write_nothing(p, r, (int)(x - (long long)r * cells));
  }
  // ---- this CTA's share: vectors at .. share_end - 1 of the rows laid end to end ----
  const int nv = (int)(((long long)p.V + 2 * W - 2) / W);  // a row's, its ends as misaligned as can be
  const long long total = (long long)rows * nv;
  const long long share = max(max((total + gridDim.x - 1) / gridDim.x, (long long)(nv / (kMaxPieces - 2) + 1)), (long long)kMinShare);
  const long long share_end = min((blockIdx.x + 1) * share, total);
  // the piece at `pos`; false past the share
  auto piece_at = [&](long long pos, LogPiece<T>& t) {
    if (pos >= share_end) return false;
    t.a = (int)(pos / nv);
    int i, j;
    place(t.a, i, j);
    t.r = i * K1 + j;
    t.begin = (int)(pos - (long long)t.a * nv);
    t.end = (int)min((long long)nv, t.begin + (share_end - pos));
    t.asked = listed || j < asked_rows(p, i);
    const int row0 = p.rows.row_offsets ? __ldg(p.rows.row_offsets + i) : i * K1;
    t.row = static_cast<const T*>(p.logits) + (t.asked ? (long long)(row0 + j) * p.V : 0);
    t.skip = (int)((reinterpret_cast<uintptr_t>(t.row) & 15u) / sizeof(T));
    return true;
  };
  // its last vector: a row may have one fewer than nv
  auto piece_end = [&](const LogPiece<T>& t) {
    return t.asked ? min(t.end, (int)(((long long)p.V + t.skip + W - 1) / W)) : t.begin;
  };

  if (warp == kLogWarps) {
    // ---- rounds, ahead of the others ----
    if (lane == 0) {
      LogPiece<T> t;
      uint32_t brought = 0;
      bool ok = true;
      for (long long pos = blockIdx.x * share; ok && piece_at(pos, t); pos += t.end - t.begin) {
        // whole vectors of the row; its ends are read where they are used
        const int end = piece_end(t), inner = t.skip ? 1 : 0, outer = (int)(((long long)p.V + t.skip) / W);
        for (int at = t.begin; at < end; at += kRoundVecs, ++brought) {
          const int lo = max(at, inner), hi = min(min(at + kRoundVecs, end), outer), s = brought % kLogStages;
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
        sh.aborted = 1;
        // the copies in flight end before the CTA does
        for (uint32_t y = brought - kLogStages; y < brought; ++y) wait_phase(&sh.full[y % kLogStages], (y / kLogStages) & 1u, p.status);
      }
    }
    return;
  }

  uint32_t used = 0;
  bool gone = false;
  LogPiece<T> t, next{};
  long long pos = blockIdx.x * share;
  bool more = piece_at(pos, next);
  // the next piece's token, and its logit, are loaded ahead
  int next_token = more ? __ldg(p.tokens + next.r) : -1;
  auto logit_of = [&](int token) { return next.asked && token >= 0 && token < p.V ? load_elem(next.row + token) : INFINITY; };
  float next_given = more ? logit_of(next_token) : 0.0f;
  while (more) {
    t = next;
    pos += t.end - t.begin;
    t.end = piece_end(t);
    int token = next_token;
    const float given = next_given;
    more = piece_at(pos, next);
    if (more) next_token = __ldg(p.tokens + next.r);
    bool logit_next = more;
    if (!t.asked) {
      if (logit_next) next_given = logit_of(next_token);
      continue;
    }
    if (token < -1 || token >= p.V) {
      if (t.begin == 0 && tid == 0) report(p.status, SPEC_ERR_BAD_INPUT);
      token = -1;
    }
    const float above = __int_as_float(given == 0.0f  ? 1
                                       : given > 0.0f ? min(__float_as_int(given) + 1, 0x7F800000)
                                                      : __float_as_int(given) - 1);  // the next fp32 number
    float m = -INFINITY, bound = -FLT_MAX, most_of_span = -INFINITY;
    f32x2 s2 = 0ull, e2 = 0ull;
    int before = 0;
    bool bad = false;
    const f32x2 c2 = pair(p.c2, p.c2);

    int span = t.begin, round = 0;  // the span's first vector, rounds of it done
    for (int v0 = t.begin; v0 < t.end; v0 += kRoundVecs, ++used) {
      // ---- a round's vectors ----
      uint4 w[kVecs];
      const int st = used % kLogStages;
      bool there = !*(volatile int*)&sh.aborted && wait_phase(&sh.full[st], (used / kLogStages) & 1u, p.status);
      const bool plain = v0 + kRoundVecs <= t.end && v0 * W >= t.skip && (v0 + kRoundVecs) * W - t.skip <= p.V;
#pragma unroll
      for (int u = 0; u < kVecs; ++u) {
        w[u] = sh.ring[st][u * kLogThreads + tid];
        if (!plain) {
          const int v = v0 + u * kLogThreads + tid, first = v * W - t.skip;
          if (v >= t.end || first < 0 || first + W > p.V) w[u] = row_end<T>(t.row, v < t.end ? first : p.V, p.V);
        }
      }
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
      const bool huge = !(fabsf(M) < kHuge);  // or nothing above -inf
      const f32x2 minus_M = pair(-M, -M);
      auto add = [&](f32x2 x) {
        float2 d = unpair(x);
        d.x = fmaxf(d.x, -1000.0f), d.y = fmaxf(d.y, -1000.0f);  // -inf, and NaN where nothing is finite
        const f32x2 y = pair(ex2_approx(d.x), ex2_approx(d.y));
        s2 = add2(s2, y);
        e2 = fma2(pair(d.x, d.y), y, e2);
      };
      if (!huge) {
#pragma unroll
        for (int u = 0; u < kVecs; ++u)
#pragma unroll
          for (int k = 0; k < W; k += 2) {
            const float l0 = element<T>(w[u], k), l1 = element<T>(w[u], k + 1);
            add(fma2(pair(l0, l1), c2, minus_M));
          }
      } else {
#pragma unroll
        for (int u = 0; u < kVecs; ++u)
#pragma unroll
          for (int k = 0; k < W; k += 2) {
            const float l0 = element<T>(w[u], k), l1 = element<T>(w[u], k + 1);
            add(pair((l0 - m) * p.c2, (l1 - m) * p.c2));
          }
      }
      // ---- entries before the token: of `given` and more, behind the token of more than that ----
      if (token >= 0) {
#pragma unroll
        for (int u = 0; u < kVecs; ++u) {
          const int v = v0 + u * kLogThreads + tid, first = v * W - t.skip;
          if (!(top[u] >= given) || v >= t.end) continue;
          const float least = first + W <= token ? given : above;
#pragma unroll
          for (int k = 0; k < W; ++k) before += element<T>(w[u], k) >= least ? 1 : 0;
          if (first <= token && first + W > token) {  // its own vector: those equal to it before it
#pragma unroll
            for (int k = 0; k < W; ++k) before += element<T>(w[u], k) == given && first + k < token ? 1 : 0;
          }
          // what is not the row's is -inf, before its first entry as well
          if (first < 0 && given == -INFINITY) before += first;
        }
      }
      if (logit_next) next_given = logit_of(next_token), logit_next = false;
      if (p.n > 0) {
#pragma unroll
        for (int u = 0; u < kVecs; ++u) sh.tops[round * kVecs + u][tid] = rounded_up(top[u]);
        most_of_span = fmaxf(most_of_span, most);
      }
      // the round's place in the ring is free
      there = __all_sync(0xFFFFFFFFu, there);
      if (lane == 0) mbar_arrive(&sh.empty[st]);
      if (!there) sh.aborted = 1;
      __syncwarp();
      if (p.n == 0 || (++round < kSpan && v0 + kRoundVecs < t.end)) continue;

      // ---- the span's candidates: a bound, and what reaches it ----
      float lanes = most_of_span;
      for (int k = 0; k < 4; ++k) {
        const float y = warp_max(lanes);
        if (lane == 0) sh.warp_top[warp * 4 + k] = y;
        const uint32_t has = __ballot_sync(0xFFFFFFFFu, lanes == y);
        if (lane == __ffs((int)has) - 1) lanes = -INFINITY;
      }
      named_sync(1, kLogThreads);
      const float mine = sh.warp_top[lane];
      int rank = 0;
#pragma unroll 8
      for (int o = 0; o < 32; ++o) {
        const float y = sh.warp_top[o];
        rank += y > mine || (y == mine && o < lane) ? 1 : 0;
      }
      const uint32_t nth = __ballot_sync(0xFFFFFFFFu, rank == p.n - 1);
      bound = fmaxf(bound, __shfl_sync(0xFFFFFFFFu, mine, __ffs((int)nth) - 1));
      // calls f(value, index) for this thread's elements of the span that reach the bound
      auto candidates = [&](auto f) {
#pragma unroll 1
        for (int y0 = 0; y0 < round * kVecs; y0 += 4) {
          uint32_t reach = 0;
#pragma unroll
          for (int y = 0; y < 4; ++y)
            reach |= __uint_as_float((uint32_t)sh.tops[y0 + y][tid] << 16) >= bound ? 1u << y : 0u;
#pragma unroll 1
          for (; reach; reach &= reach - 1) {
            const int first = (span + (y0 + __ffs((int)reach) - 1) * kLogThreads + tid) * W - t.skip;
            const uint4 v = first >= 0 && first + W <= p.V ? __ldg(reinterpret_cast<const uint4*>(t.row + first))
                                                           : row_end<T>(t.row, first, p.V);
#pragma unroll
            for (int k = 0; k < W; ++k)
              if (element<T>(v, k) >= bound) f(element<T>(v, k), first + k);
          }
        }
      };
      bool full = false;
      candidates([&](float l, int k) {
        const int slot = atomicAdd(&sh.count, 1);
        if (slot < kListFull) sh.list[slot] = make_key(l, k);
        else full = true;
      });
      if (named_or(1, kLogThreads, full)) {
        // too many: the n best of the spans before (by their indices), and the n best of this one, one after another
        const int start = span * W - t.skip;
        Key old[kListFull / kLogThreads];
#pragma unroll
        for (int y = 0; y < kListFull / kLogThreads; ++y) {
          old[y] = sh.list[y * kLogThreads + tid];
          if (key_index(old[y]) >= start) old[y] = 0;
        }
        named_sync(1, kLogThreads);
        if (tid == 0) sh.count = 0;
        named_sync(1, kLogThreads);
#pragma unroll
        for (int y = 0; y < kListFull / kLogThreads; ++y)
          if (old[y]) sh.list[atomicAdd(&sh.count, 1)] = old[y];
        named_sync(1, kLogThreads);
        int kept = sh.count;  // at most n, from the span before
        Key last = ~(Key)0;
        for (int y = 0; y < p.n; ++y) {
          Key next = 0;
          candidates([&](float l, int k) {
            const Key key = make_key(l, k);
            if (key < last && key > next) next = key;
          });
#pragma unroll 1
          for (int o = 16; o > 0; o >>= 1) next = max(next, __shfl_xor_sync(0xFFFFFFFFu, next, o));
          if (lane == 0) sh.warp_key[warp] = next;
          named_sync(1, kLogThreads);
#pragma unroll 1
          for (int w = 0; w < kLogWarps; ++w) next = max(next, sh.warp_key[w]);
          named_sync(1, kLogThreads);
          last = next;
          if (last == 0) break;
          if (tid == 0) sh.list[kept] = last;
          ++kept;
        }
        if (tid == 0) sh.count = kept;
        named_sync(1, kLogThreads);
      }
      const int listed_now = sh.count, kept = min(listed_now, p.n);
      select_keys(sh.list, listed_now, p.n, sh.best);
      named_sync(1, kLogThreads);
      if (tid < kept) sh.list[tid] = sh.best[tid];
      if (tid == 0) sh.count = kept;
      if (kept == p.n) bound = fmaxf(bound, key_value(sh.best[p.n - 1]));
      named_sync(1, kLogThreads);
      span = v0 + kRoundVecs;
      round = 0;
      most_of_span = -INFINITY;
    }
    if (sh.aborted) gone = true;
    if (logit_next) next_given = logit_of(next_token);
    // the CTAs that have a piece of the row
    const int b0 = (int)((long long)t.a * nv / share), b1 = (int)(((long long)(t.a + 1) * nv - 1) / share), pieces = b1 - b0 + 1;

    // ---- the piece's sums and best ----
    const float warp_m = warp_max(m);
    if (lane == 0) sh.m[warp] = warp_m;
    // a span's end has left the best there, in order
    const int found = sh.count;
    const size_t x = (size_t)t.a + blockIdx.x;
    if (tid < p.n) (pieces > 1 ? p.part_keys + x * p.n : sh.best)[tid] = tid < found ? sh.list[tid] : 0;
    if (named_or(1, kLogThreads, gone)) break;
    if (tid == 0) sh.count = 0;  // for the next piece, whose appends come after another barrier
    float all_m = sh.m[0];
#pragma unroll
    for (int w = 1; w < kLogWarps; ++w) all_m = fmaxf(all_m, sh.m[w]);
    float2 half = unpair(s2);
    float s = half.x + half.y;
    half = unpair(e2);
    float e = half.x + half.y;
    move_sums(all_m, m, s, e, p.c2);
    m = all_m;
    s = warp_sum(s);
    e = warp_sum(e);
    before = __reduce_add_sync(0xFFFFFFFFu, before);
    bad = __any_sync(0xFFFFFFFFu, bad);
    if (lane == 0) {
      sh.s[warp] = s;
      sh.e[warp] = e;
      sh.before[warp] = bad ? -1 : before;
    }
    named_sync(1, kLogThreads);
    s = sh.s[0], e = sh.e[0], before = sh.before[0];
#pragma unroll
    for (int w = 1; w < kLogWarps; ++w) {
      s += sh.s[w];
      e += sh.e[w];
      before = before < 0 || sh.before[w] < 0 ? -1 : before + sh.before[w];
    }
    if (pieces > 1) {
      if (tid == 0) {
        p.part[x] = LogPartial{m, s, e, before};
        __threadfence();  // and what the others wrote before the barrier
        sh.last = atomicAdd(p.arrived + t.a, 1u) == (uint32_t)pieces - 1;
        __threadfence();
      }
      named_sync(1, kLogThreads);
      if (!sh.last) continue;

      // ---- the last CTA of the row joins the pieces: one or two per lane, every warp the same ----
      if (tid == 0) p.arrived[t.a] = 0;
      const LogPartial* parts = p.part + t.a + b0;
      uint4 v[2];
#pragma unroll
      for (int y = 0; y < 2; ++y)
        v[y] = lane + 32 * y < pieces ? __ldcg(reinterpret_cast<const uint4*>(parts + lane + 32 * y))
                                      : make_uint4(0xFF800000u, 0u, 0u, 0u);
      Key least = 0;
      const Key* keys = p.part_keys + ((size_t)t.a + b0) * p.n;
      if (p.n) {
        // what is below some piece's n-th best is not among the n best
        for (int y = lane; y < pieces; y += 32) least = max(least, __ldcg(keys + (size_t)y * p.n + p.n - 1));
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) least = max(least, __shfl_xor_sync(0xFFFFFFFFu, least, o));
        for (int y = tid; y < pieces * p.n; y += kLogThreads) {
          const Key k = __ldcg(keys + y);
          if (k != 0 && k >= least) sh.joined[atomicAdd(&sh.count, 1)] = k;
        }
      }
      m = warp_max(fmaxf(__uint_as_float(v[0].x), __uint_as_float(v[1].x)));
      float part_s[2], part_e[2];
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        part_s[y] = __uint_as_float(v[y].y), part_e[y] = __uint_as_float(v[y].z);
        move_sums(m, __uint_as_float(v[y].x), part_s[y], part_e[y], p.c2);
      }
      s = warp_sum(part_s[0] + part_s[1]);
      e = warp_sum(part_e[0] + part_e[1]);
      bad = __any_sync(0xFFFFFFFFu, (int)v[0].w < 0 || (int)v[1].w < 0);
      before = __reduce_add_sync(0xFFFFFFFFu, (int)v[0].w + (int)v[1].w);
      if (bad) before = -1;
      if (p.n) {
        named_sync(1, kLogThreads);
        select_keys(sh.joined, sh.count, p.n, sh.best);
        named_sync(1, kLogThreads);
        if (tid == 0) sh.count = 0;
      }
    }
    write_row(p, t.r, m, s, e, before, token, given, sh.best);
    named_sync(1, kLogThreads);
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
  return launch_after_previous(logprobs_kernel<T>, dim3((unsigned)ctas), dim3(kLogThreads + 32), smem, stream, p);
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
      std::isinf(temperature))
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
