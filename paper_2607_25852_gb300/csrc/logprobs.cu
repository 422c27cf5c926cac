// logprobs.cu -- log probabilities of given tokens, their ranks, the entropy and
// the most likely alternatives, from logits rows [rows, V] in one pass.
//
// With c2 = log2(e) / t, m = max_v l_v and d_v = c2 (l_v - m) in fp32 (differences
// first: at the maximum nothing is left, however large the logits),
//   s = sum_v 2^d_v,  e = sum_v d_v 2^d_v,
//   ln p_v = ln 2 (d_v - log2 s),  H = ln 2 (log2 s - e / s),
// all terms of H non-negative, so nothing cancels.  A token's rank counts the
// entries that come before it (greater, or equal with a lower index); its logit
// is read first, so the count goes along.
//
// The alternatives come along too.  A CTA holds a round of its chunk in
// registers; n values that are known to be there (the four largest of its warps'
// lanes' maxima) give a bound that the n-th best cannot be below, and only
// what reaches the bound (some dozens of 16,384) goes to a list in shared
// memory, as a 64-bit key that orders by value and then by lower index.  A list
// that overflows, as many equal logits make it, is replaced by n searches for
// the next best key.  So the order in which threads append does not show.
//
// Chunks of a row are joined by the last CTA to arrive, in order of the chunks.
// Bound by HBM for many rows, by the launch and three round trips for few.
#include <cfloat>
#include <cmath>

#include <algorithm>

#include "paged.cuh"

namespace spec {

namespace {

constexpr int kLogThreads = 256, kLogWarps = kLogThreads / 32;
constexpr int kVecs = 8;             // 16-byte vectors per thread and round
constexpr int kMaxChunks = 64;       // per row
constexpr int kListCap = kMaxChunks * SPEC_MAX_TOP;
typedef unsigned long long Key;      // 0: none

struct alignas(16) LogPartial {
  float m, s, e;
  int32_t before;  // entries that come before the token; -1 where a logit is NaN or +inf
};

struct LogLaunch {
  const void* logits;
  const int32_t *tokens, *accepted;
  RowLayout rows;
  int V, n, NC, chunk_vecs;
  float c2;
  float *logprob, *entropy, *top_logprobs;
  int32_t *rank, *top_tokens, *status;
  LogPartial* part;    // [B (K + 1)][NC]
  Key* part_keys;      // [B (K + 1)][NC][n]
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

// Adds the sums (ms, ss, es) to (m, s, e); differences of 2^-1000 and less count as that.
__device__ __forceinline__ void join_sums(float& m, float& s, float& e, float m2, float s2, float e2, float c2) {
  const float top = fmaxf(m, m2);
  const float da = fmaxf((m - top) * c2, -1000.0f), db = fmaxf((m2 - top) * c2, -1000.0f);
  const float fa = exp2f(da), fb = exp2f(db);
  e = fa * fmaf(da, s, e) + fb * fmaf(db, s2, e2);
  s = fa * s + fb * s2;
  m = top;
}

// The n best of `count` keys in `list` to out[0 .. n), the best first.
__device__ __forceinline__ void select_keys(const Key* list, int count, int n, Key* out) {
  for (int x = threadIdx.x; x < n; x += kLogThreads)
    if (x >= count) out[x] = 0;
  for (int x = threadIdx.x; x < count; x += kLogThreads) {
    const Key k = list[x];
    int before = 0;
    for (int y = 0; y < count; ++y) before += list[y] > k ? 1 : 0;
    if (before < n) out[before] = k;
  }
}

struct LogShared {
  Key list[kListCap];
  Key best[SPEC_MAX_TOP];
  Key warp_key[kLogWarps];
  float warp_top[kLogWarps * 4];
  float m[kLogWarps], s[kLogWarps], e[kLogWarps];
  int before[kLogWarps];
  int count, last;
};

// A row that is not asked for, or cannot be answered.
__device__ __forceinline__ void write_nothing(const LogLaunch& p, long long r) {
  for (int x = threadIdx.x; x < p.n; x += kLogThreads) {
    if (p.top_tokens) p.top_tokens[r * p.n + x] = -1;
    if (p.top_logprobs) p.top_logprobs[r * p.n + x] = -INFINITY;
  }
  if (threadIdx.x == 0) {
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
    write_nothing(p, r);
    return;
  }
  constexpr float kLn2 = 0.693147180559945309f;
  const float norm = log2f(s);
  for (int x = threadIdx.x; x < p.n; x += kLogThreads) {
    const Key k = best[x];
    if (p.top_tokens) p.top_tokens[r * p.n + x] = k ? key_index(k) : -1;
    if (p.top_logprobs) p.top_logprobs[r * p.n + x] = k ? kLn2 * ((key_value(k) - m) * p.c2 - norm) : -INFINITY;
  }
  if (threadIdx.x == 0) {
    p.logprob[r] = token >= 0 ? kLn2 * ((given - m) * p.c2 - norm) : -INFINITY;
    if (p.rank) p.rank[r] = token >= 0 ? before + 1 : 0;
    if (p.entropy) p.entropy[r] = kLn2 * (norm - e / s);
  }
}

template <typename T>
__global__ void __launch_bounds__(kLogThreads) logprobs_kernel(const LogLaunch p) {
  constexpr int W = 16 / (int)sizeof(T);
  __shared__ LogShared sh;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, K1 = p.rows.K + 1;
  const int r = (int)(blockIdx.x / (unsigned)p.NC), c = (int)(blockIdx.x - (unsigned)r * (unsigned)p.NC);
  const int i = r / K1, j = r - i * K1;
  pdl_wait_prerequisites();
  pdl_launch_dependents();
  const RequestRows q = request_rows(p.rows, i);
  const int accepted = p.accepted ? __ldg(p.accepted + i) : q.count - 1;
  int token = __ldg(p.tokens + r);
  const bool ok = q.ok && accepted >= 0 && accepted < q.count;
  if (!ok || j > accepted) {
    if (c == 0) {
      if (!ok && j == 0 && tid == 0) report(p.status, SPEC_ERR_BAD_INPUT);
      write_nothing(p, r);
    }
    return;
  }
  const T* row = static_cast<const T*>(p.logits) + (long long)(q.row0 + j) * p.V;
  if (token < -1 || token >= p.V) {
    if (c == 0 && tid == 0) report(p.status, SPEC_ERR_BAD_INPUT);
    token = -1;
  }
  const float given = token >= 0 ? load_elem(row + token) : INFINITY;
  const float above = __int_as_float(given == 0.0f  ? 1
                                     : given > 0.0f ? min(__float_as_int(given) + 1, 0x7F800000)
                                                    : __float_as_int(given) - 1);  // the next fp32 number
  // 16-byte vectors of memory; the first and the last may hold elements of other rows
  const int skip = (int)((reinterpret_cast<uintptr_t>(row) & 15u) / sizeof(T));
  const T* base = row - skip;
  const int v_end = (int)(((long long)p.V + skip + W - 1) / W);
  const int begin = c * p.chunk_vecs, end = min(begin + p.chunk_vecs, v_end);
  float m = -INFINITY, s = 0.0f, e = 0.0f, bound = -FLT_MAX;
  int before = 0, count = 0;
  bool bad = false;
  if (tid == 0) sh.count = 0;
  __syncthreads();

  for (int v0 = begin; v0 < end; v0 += kLogThreads * kVecs) {
    // ---- a round's vectors ----
    uint4 x[kVecs];
#pragma unroll
    for (int u = 0; u < kVecs; ++u) {
      const int v = v0 + u * kLogThreads + tid;
      constexpr uint32_t kNone = sizeof(T) == 4 ? 0xFF800000u : 0xFF80FF80u;
      x[u] = make_uint4(kNone, kNone, kNone, kNone);
      if (v >= end) continue;
      const long long at = (long long)v * W - skip;
      if (at >= 0 && at + W <= p.V) {
        x[u] = ldg_stream(base + (long long)v * W);
      } else {
        uint32_t w[4] = {kNone, kNone, kNone, kNone};
#pragma unroll
        for (int k = 0; k < W; ++k) {
          if (at + k < 0 || at + k >= p.V) continue;
          const uint32_t b = __float_as_uint(load_elem(row + at + k));
          if (sizeof(T) == 4) w[k] = b;
          else w[k / 2] = (k & 1) ? (w[k / 2] & 0xFFFFu) | b : (w[k / 2] & 0xFFFF0000u) | b >> 16;
        }
        x[u] = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
    float top[kVecs], most = -INFINITY;
#pragma unroll
    for (int u = 0; u < kVecs; ++u) {
      top[u] = element<T>(x[u], 0);
#pragma unroll
      for (int k = 1; k < W; ++k) top[u] = fmax_nan(top[u], element<T>(x[u], k));
      bad |= !(top[u] < INFINITY);
      most = fmaxf(most, top[u]);
    }
    // ---- sums ----
    if (most > m) {
      const float d = fmaxf((m - most) * p.c2, -1000.0f), f = exp2f(d);
      e = f * fmaf(d, s, e);
      s *= f;
      m = most;
    }
    float s1 = 0.0f, e1 = 0.0f;
#pragma unroll
    for (int u = 0; u < kVecs; ++u) {
      const int at = (v0 + u * kLogThreads + tid) * W - skip;  // an index, below 2^30
      // an entry before the token counts from `given` on, one behind it from `above`, what is no entry not at all
      const bool real = v0 + u * kLogThreads + tid < end;
      float least = !real ? INFINITY : at >= token ? above : given;
      const bool cut = real && ((at < token && at + W > token) || at < 0 || at + W > p.V);
#pragma unroll
      for (int k = 0; k < W; ++k) {
        const float l = element<T>(x[u], k);
        const float d = fmaxf((l - m) * p.c2, -1000.0f);  // -inf, and NaN where nothing is finite
        const float y = ex2_approx(d);
        if (k & 1) {
          s1 += y;
          e1 = fmaf(d, y, e1);
        } else {
          s += y;
          e = fmaf(d, y, e);
        }
        if (cut) least = at + k < 0 || at + k >= p.V ? INFINITY : at + k >= token ? above : given;
        before += l >= least ? 1 : 0;
      }
    }
    s += s1;
    e += e1;
    if (p.n == 0) continue;

    // ---- what may be among the n best ----
    if (v0 == begin) {
      float lanes = most == most ? most : -INFINITY;
      for (int k = 0; k < 4; ++k) {
        float y = lanes;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) y = fmaxf(y, __shfl_xor_sync(0xFFFFFFFFu, y, o));
        if (lane == 0) sh.warp_top[warp * 4 + k] = y;
        const uint32_t has = __ballot_sync(0xFFFFFFFFu, lanes == y);
        if (lane == __ffs((int)has) - 1) lanes = -INFINITY;
      }
      __syncthreads();
      const float mine = sh.warp_top[lane];
      int rank = 0;
#pragma unroll
      for (int o = 0; o < 32; ++o) {
        const float y = sh.warp_top[o];
        rank += y > mine || (y == mine && o < lane) ? 1 : 0;
      }
      const uint32_t nth = __ballot_sync(0xFFFFFFFFu, rank == p.n - 1);
      bound = fmaxf(__shfl_sync(0xFFFFFFFFu, mine, __ffs((int)nth) - 1), -FLT_MAX);
    }
#pragma unroll
    for (int u = 0; u < kVecs; ++u) {
      if (!(top[u] >= bound)) continue;
      const int at = (v0 + u * kLogThreads + tid) * W - skip;
#pragma unroll
      for (int k = 0; k < W; ++k) {
        const float l = element<T>(x[u], k);
        if (l >= bound) {
          const int slot = atomicAdd(&sh.count, 1);
          if (slot < kListCap) sh.list[slot] = make_key(l, at + k);
        }
      }
    }
    __syncthreads();
    const int now = sh.count;
    __syncthreads();
    if (now > kListCap - SPEC_MAX_TOP) {
      Key last = ~(Key)0;
      if (now > kListCap) {
        // ---- too many: the n best of this round one after another ----
        for (int y = 0; y < p.n; ++y) {
          Key next = 0;
#pragma unroll
          for (int u = 0; u < kVecs; ++u) {
            const int at = (v0 + u * kLogThreads + tid) * W - skip;
            if (!(top[u] >= bound)) continue;
#pragma unroll
            for (int k = 0; k < W; ++k) {
              const float l = element<T>(x[u], k);
              const Key key = make_key(l, at + k);
              if (l >= bound && key < last && key > next) next = key;
            }
          }
#pragma unroll
          for (int o = 16; o > 0; o >>= 1) next = max(next, __shfl_xor_sync(0xFFFFFFFFu, next, o));
          if (lane == 0) sh.warp_key[warp] = next;
          __syncthreads();
#pragma unroll
          for (int w = 0; w < kLogWarps; ++w) next = max(next, sh.warp_key[w]);
          __syncthreads();
          last = next;
          if (last == 0) break;
          if (tid == 0) sh.list[count + y] = last;  // count + n <= kListCap
          if (tid == 0) sh.count = count + y + 1;
        }
        __syncthreads();
      }
      // ---- room for the next round: the n best of all so far ----
      select_keys(sh.list, sh.count, p.n, sh.best);
      __syncthreads();
      const int kept = min(sh.count, p.n);
      if (tid < kept) sh.list[tid] = sh.best[tid];
      __syncthreads();
      if (tid == 0) sh.count = kept;
      if (kept == p.n) bound = fmaxf(bound, key_value(sh.best[p.n - 1]));
      __syncthreads();
    }
    count = sh.count;
    __syncthreads();
  }

  // ---- the chunk's sums and best ----
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    join_sums(m, s, e, __shfl_xor_sync(0xFFFFFFFFu, m, o), __shfl_xor_sync(0xFFFFFFFFu, s, o),
              __shfl_xor_sync(0xFFFFFFFFu, e, o), p.c2);
    before += __shfl_xor_sync(0xFFFFFFFFu, before, o);
  }
  bad = __any_sync(0xFFFFFFFFu, bad);
  if (lane == 0) {
    sh.m[warp] = m;
    sh.s[warp] = s;
    sh.e[warp] = e;
    sh.before[warp] = bad ? -1 : before;
  }
  __syncthreads();
  m = sh.m[0], s = sh.s[0], e = sh.e[0], before = sh.before[0];
#pragma unroll
  for (int w = 1; w < kLogWarps; ++w) {
    join_sums(m, s, e, sh.m[w], sh.s[w], sh.e[w], p.c2);
    before = before < 0 || sh.before[w] < 0 ? -1 : before + sh.before[w];
  }
  Key* mine = p.NC == 1 ? sh.best : p.part_keys + ((size_t)r * p.NC + c) * p.n;
  if (p.n) select_keys(sh.list, sh.count, p.n, mine);
  if (p.NC == 1) {
    __syncthreads();
    write_row(p, r, m, s, e, before, token, given, sh.best);
    return;
  }
  if (tid == 0) p.part[(size_t)r * p.NC + c] = LogPartial{m, s, e, before};
  __threadfence();
  __syncthreads();
  if (tid == 0) sh.last = atomicAdd(p.arrived + r, 1u) == (uint32_t)p.NC - 1;
  __syncthreads();
  if (!sh.last) return;

  // ---- the last CTA of the row joins the chunks, in order ----
  __threadfence();
  if (tid == 0) {
    p.arrived[r] = 0;
    sh.count = 0;
  }
  m = -INFINITY, s = 0.0f, e = 0.0f, before = 0;
  for (int y = lane; y < p.NC; y += 32) {  // a chunk or two per lane, every warp the same
    const uint4 v = __ldcg(reinterpret_cast<const uint4*>(p.part + (size_t)r * p.NC + y));
    join_sums(m, s, e, __uint_as_float(v.x), __uint_as_float(v.y), __uint_as_float(v.z), p.c2);
    before = before < 0 || (int)v.w < 0 ? -1 : before + (int)v.w;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    join_sums(m, s, e, __shfl_xor_sync(0xFFFFFFFFu, m, o), __shfl_xor_sync(0xFFFFFFFFu, s, o),
              __shfl_xor_sync(0xFFFFFFFFu, e, o), p.c2);
    const int other = __shfl_xor_sync(0xFFFFFFFFu, before, o);
    before = before < 0 || other < 0 ? -1 : before + other;
  }
  if (p.n) {
    // what is below some chunk's n-th best is not among the n best
    const Key* keys = p.part_keys + (size_t)r * p.NC * p.n;
    Key least = 0;
    for (int y = lane; y < p.NC; y += 32) least = max(least, __ldcg(keys + (size_t)y * p.n + p.n - 1));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) least = max(least, __shfl_xor_sync(0xFFFFFFFFu, least, o));
    __syncthreads();
    for (int y = tid; y < p.NC * p.n; y += kLogThreads) {
      const Key k = __ldcg(keys + y);
      if (k != 0 && k >= least) sh.list[atomicAdd(&sh.count, 1)] = k;
    }
    __syncthreads();
    select_keys(sh.list, sh.count, p.n, sh.best);
    __syncthreads();
  }
  write_row(p, r, m, s, e, before, token, given, sh.best);
}

struct LogGeometry {
  int NC, chunk_vecs;  // vectors of 8 elements in bf16, of 4 in fp32: set for the wider
  size_t part_off, keys_off, bytes;
};

bool logprobs_shape_ok(int B, int K, int V, int n) {
  return rows_shape_ok(B, K) && V >= 1 && V < SPEC_MAX_VOCAB && n >= 0 && n <= SPEC_MAX_TOP;
}

// Chunks per row: about 4,096 CTAs if all rows are asked, of at least 4,096 entries.
LogGeometry logprobs_geometry(int B, int K, int V, int n) {
  LogGeometry g{};
  const long long R = (long long)B * (K + 1);
  long long nc = std::min<long long>({kMaxChunks, std::max(1LL, 4096 / R), std::max(1, V / 4096)});
  g.NC = (int)nc;
  g.part_off = ((size_t)R * 4 + 255) / 256 * 256;
  g.keys_off = g.part_off + ((size_t)R * nc * sizeof(LogPartial) + 255) / 256 * 256;
  g.bytes = g.keys_off + ((size_t)R * nc * n * sizeof(Key) + 255) / 256 * 256;
  return g;
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
  p.NC = g.NC;
  const int W = 16 / element_size(logits_dtype);
  p.chunk_vecs = (V / W + 2 + g.NC - 1) / g.NC;  // V and the misaligned ends of a row
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
  const dim3 grid((unsigned)((long long)B * (K + 1) * g.NC)), block(kLogThreads);
  const cudaError_t err = logits_dtype == SPEC_F32
                              ? launch_after_previous(logprobs_kernel<float>, grid, block, 0, stream, p)
                              : launch_after_previous(logprobs_kernel<__nv_bfloat16>, grid, block, 0, stream, p);
  return err == cudaSuccess && cudaGetLastError() == cudaSuccess ? SPEC_OK : SPEC_ERR_CUDA;
}
