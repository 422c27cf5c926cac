// linear.cu -- linear attention with a decay per head over the requests' states,
// on the CUDA cores: single tokens, verification rounds, fp32 and odd sizes.
//
// For a head with state S [Dk x Dv], row j's decay l_j = exp(g_j):
//   S_j = l_j S_{j-1} + k_j v_j^T,   o_j = scale q_j S_j.
// With L_j = g_1 + .. + g_j over a block of rows this is, without a pass over the
// state per row,
//   o_i = scale (exp(L_i) q_i S_0 + sum_{j <= i} exp(L_i - L_j) (q_i k_j) v_j)
//   S_n = exp(L_n) S_0 + sum_j exp(L_n - L_j) k_j v_j^T,
// two multiply-adds per element of the state and row (one where the states stay).
//
// A CTA holds the state of a head, or some of its columns, in registers: 16-byte
// loads, all in flight together, read once and written once.  8 rows at a time, the
// next 8 on their way meanwhile (201 us without that and without segments, 141 with
// it, 3 requests of up to 201 rows of 12 query heads, 4 states of 72 x 96 each, fp32);
// long calls of few heads in segments: sums of all but the last from zero, a scan, and
// all segments' outputs, a query head to a CTA (32 us there; 1 request of 2,001 rows of
// 8 heads of 128 668 -> 82 us).  One token of 16 heads of 128 3.8 us, 64 requests of 8
// rows of 8 heads of 256 77 us (3.6 TB/s).  Few rows are bound by HBM's latency, many by
// the issue of FMAs and of the loads from shared memory that feed them: 64 requests of
// 256 rows of 16 heads of 64 take 411 us, 24 TFLOP/s.  (Two instances with 16 rows of
// the state per thread keep 8 and 24 bytes on the stack.)
#include <cmath>

#include <algorithm>

#include "linear_few.cuh"
#include "linear_tc.cuh"
#include "tensor_core.cuh"

namespace spec {

namespace {

constexpr int kLinThreads = 256, kLinWarps = kLinThreads / 32;
constexpr int kBlockRows = 8, kPassRows = 4;  // a block's rows; those whose products with the state are made at a time

template <typename T>
__device__ __forceinline__ void unpack16(const uint4& w, float* f);
template <>
__device__ __forceinline__ void unpack16<float>(const uint4& w, float* f) {
  f[0] = __uint_as_float(w.x), f[1] = __uint_as_float(w.y), f[2] = __uint_as_float(w.z), f[3] = __uint_as_float(w.w);
}
template <>
__device__ __forceinline__ void unpack16<__nv_bfloat16>(const uint4& w, float* f) {
  f[0] = bf16_lo(w.x), f[1] = bf16_hi(w.x), f[2] = bf16_lo(w.y), f[3] = bf16_hi(w.y);
  f[4] = bf16_lo(w.z), f[5] = bf16_hi(w.z), f[6] = bf16_lo(w.w), f[7] = bf16_hi(w.w);
}

// A thread's part of a block of rows, a warp per row, on its way to shared memory as
// floats: rows of the block from n on and elements from `width` on are 0.
template <typename T, int NV>
struct RowPart {
  static constexpr int W = 16 / (int)sizeof(T);
  uint4 w[NV];
  __device__ __forceinline__ void fetch(const T* from, int64_t row_stride, int n, int width) {
    const int r = threadIdx.x >> 5, d = (threadIdx.x & 31) * W;
#pragma unroll
    for (int y = 0; y < NV; ++y) {
      w[y] = make_uint4(0u, 0u, 0u, 0u);
      if (r < n && d + y * 32 * W < width) w[y] = ldg_stream(from + r * row_stride + d + y * 32 * W);
    }
  }
  __device__ __forceinline__ void put(float* to, int pitch, int padded) const {
    const int r = threadIdx.x >> 5, d = (threadIdx.x & 31) * W;
#pragma unroll
    for (int y = 0; y < NV; ++y) {
      if (d + y * 32 * W >= padded) break;
      float f[W];
      unpack16<T>(w[y], f);
#pragma unroll
      for (int z = 0; z < W; z += 4)
        *reinterpret_cast<float4*>(to + r * pitch + d + y * 32 * W + z) = make_float4(f[z], f[z + 1], f[z + 2], f[z + 3]);
    }
  }
};
static_assert(kBlockRows == kLinWarps, "a warp per row");

__device__ __forceinline__ void store4(float* to, const float4& x) { *reinterpret_cast<float4*>(to) = x; }
__device__ __forceinline__ void store4(__nv_bfloat16* to, const float4& x) {
  const __nv_bfloat162 a = __floats2bfloat162_rn(x.x, x.y), b = __floats2bfloat162_rn(x.z, x.w);
  *reinterpret_cast<uint2*>(to) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}

inline __host__ __device__ int key_pitch(int Dk) { return (Dk + 31) / 32 * 32 + 16; }  // rows 16 banks apart

template <int S>
inline size_t linear_smem(int Dk) {
  return sizeof(float) * (2 * (size_t)kBlockRows * key_pitch(Dk) + (size_t)kBlockRows * S * (1 + kLinWarps));
}

// What a launch of the rows' kernel does: requests from their slots to their slots, the
// sums of their segments but the last, or all segments from the first states that a scan
// made of these (of states alone: the last segment).
enum LinearPhase { kWholeRows, kRowSums, kRowSegments };

// S columns of the state, KR of its rows per thread.
template <typename T, int S, int KR>
__global__ void __launch_bounds__(kLinThreads) linear_rows_kernel(const LinearLaunch p, const LinearPlan plan, int phase,
                                                                  int slices) {
  constexpr int L = S / 4;  // threads across columns
  constexpr int NV = (KR * (kLinThreads / L) * (int)sizeof(T) + 511) / 512;  // a key's vectors of a warp's lane
  extern __shared__ float4 smem4[];
  __shared__ long long steps[kBlockRows];
  __shared__ float score[kBlockRows][kBlockRows], weight[kBlockRows], first_weight[kBlockRows], all_weight;
  const int pitch = key_pitch(p.Dk);
  float* kb = reinterpret_cast<float*>(smem4);
  float* qb = kb + kBlockRows * pitch;
  float* vb = qb + kBlockRows * pitch;
  float* red = vb + kBlockRows * S;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  // ---- block: part of the columns, fastest, then head, segment, request ----
  const bool outs = p.q && phase != kRowSums, one = outs && phase == kRowSegments;  // one query head, or its group's
  const int heads = one ? p.Hq : p.H, segments = phase == kRowSegments && !p.q ? 1 : phase == kRowSums ? plan.nseg - 1 : plan.nseg;
  unsigned x0 = blockIdx.x;
  const int c0 = (int)(x0 % (unsigned)slices) * S;
  x0 /= (unsigned)slices;
  const int hx = (int)(x0 % (unsigned)heads), h = one ? hx / p.G : hx;
  x0 /= (unsigned)heads;
  int seg = (int)(x0 % (unsigned)segments);
  const int i = (int)(x0 / (unsigned)segments);
  const int col = (tid % L) * 4, kr0 = (tid / L) * KR;
  const int columns = min(S, p.Dv - c0);
  pdl_wait_prerequisites();
  pdl_launch_dependents();
  const LinearRequest r = linear_request(p, i);
  if (!r.ok) {
    if (blockIdx.x % (unsigned)(slices * heads * segments) == 0 && tid == 0) report(p.status, SPEC_ERR_BAD_INPUT);
    return;
  }
  const int segs = phase == kWholeRows ? 1 : max(1, (r.last - r.first + plan.seg_rows - 1) / plan.seg_rows);
  if (phase == kRowSegments && !p.q) seg = segs - 1;
  if (seg >= segs - (phase == kRowSums)) return;
  const int first = phase == kWholeRows ? r.first : r.first + seg * plan.seg_rows;
  const int last = seg == segs - 1 ? r.last : first + plan.seg_rows;
  // ---- the state's part ----
  const bool mine = col < columns;
  const int64_t size = (int64_t)p.Dk * p.Dv, at = (int64_t)kr0 * p.Dv + c0 + col;
  float* seg_state = plan.seg_state + ((int64_t)i * p.H + h) * plan.nseg * size;
  const float* from = phase == kRowSegments ? seg_state + seg * size
                      : phase == kWholeRows && r.from >= 0 ? p.state + r.from * p.slot_stride + h * size : nullptr;
  float* to = phase == kRowSums                                               ? seg_state + (seg + 1) * size
              : r.to >= 0 && seg == segs - 1 && (!one || hx == h * p.G) ? p.state + r.to * p.slot_stride + h * size
                                                                        : nullptr;
  float4 s[KR];
#pragma unroll
  for (int x = 0; x < KR; ++x) {
    s[x] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (from && mine && kr0 + x < p.Dk) s[x] = *reinterpret_cast<const float4*>(from + at + (int64_t)x * p.Dv);
  }
  const T* k = static_cast<const T*>(p.k) + (int64_t)h * p.Dk;
  const T* v = static_cast<const T*>(p.v) + (int64_t)h * p.Dv + c0;
  T* out = static_cast<T*>(p.out);
  const int g0 = one ? hx : h * p.G, groups = one ? 1 : p.G;
  if (outs && seg == 0) {  // rows before position 0
#pragma unroll 1
    for (long long x = tid; x < (long long)r.first * groups * (columns / 4); x += kLinThreads) {
      const int c = (int)(x % (columns / 4)), y = (int)(x / (columns / 4));
      store4(out + ((int64_t)(r.row0 + y / groups) * p.Hq + g0 + y % groups) * p.Dv + c0 + 4 * c,
             make_float4(0.0f, 0.0f, 0.0f, 0.0f));
    }
  }

  // Each block's rows are on their way while the one before is worked on.
  RowPart<T, NV> next_k, next_q;
  RowPart<T, 1> next_v;
  auto fetch_kv = [&](int b) {
    const int64_t row = r.row0 + b;
    next_k.fetch(k + row * p.k_row, p.k_row, min(kBlockRows, last - b), p.Dk);
    next_v.fetch(v + row * p.v_row, p.v_row, min(kBlockRows, last - b), columns);
  };
  auto fetch_q = [&](int b, int g) {
    const T* q = static_cast<const T*>(p.q) + (int64_t)(r.row0 + b) * p.q_row + (int64_t)(g0 + g) * p.Dk;
    next_q.fetch(q, p.q_row, min(kBlockRows, last - b), p.Dk);
  };
  if (first < last) {
    fetch_kv(first);
    if (outs) fetch_q(first, 0);
  }
  long long seg_steps = 0;
  for (int b0 = first; b0 < last; b0 += kBlockRows) {
    const int n = min(kBlockRows, last - b0);
    const int64_t row = r.row0 + b0;
    __syncthreads();
    next_k.put(kb, pitch, pitch - 16);
    next_v.put(vb, S, S);
    if (b0 + kBlockRows < last) fetch_kv(b0 + kBlockRows);
    if (warp == 0) {
      long long g = 0;
      if (lane < n) g = decay_steps(__ldg(p.log_decay + (row + lane) * p.decay_row + h), p.status);
#pragma unroll
      for (int o = 1; o < kBlockRows; o <<= 1) {
        const long long y = __shfl_up_sync(0xFFFFFFFFu, g, o);
        if (lane >= o) g += y;
      }
      const long long all = __shfl_sync(0xFFFFFFFFu, g, kBlockRows - 1);  // rows past n add 0
      seg_steps += all;
      if (lane < kBlockRows) {
        steps[lane] = g;
        weight[lane] = exp2f(steps_float(all - g));
        first_weight[lane] = exp2f(steps_float(g));
      }
      if (lane == 0) all_weight = exp2f(steps_float(all));
    }
    if (outs) {
      for (int g = 0; g < groups; ++g) {
        if (g) __syncthreads();
        next_q.put(qb, pitch, pitch - 16);
        if (g + 1 < groups)
          fetch_q(b0, g + 1);
        else if (b0 + kBlockRows < last)
          fetch_q(b0 + kBlockRows, 0);
        __syncthreads();
        // ---- exp(L_i - L_j) (q_i k_j): four threads per pair ----
        {
          const int pair = tid >> 2, a = pair / kBlockRows, b = pair % kBlockRows;
          float x = 0.0f;
#pragma unroll 2
          for (int d = (tid & 3) * 4; d < pitch - 16; d += 16) {
            const float4 y = *reinterpret_cast<const float4*>(qb + a * pitch + d);
            const float4 z = *reinterpret_cast<const float4*>(kb + b * pitch + d);
            x = fmaf(y.x, z.x, fmaf(y.y, z.y, fmaf(y.z, z.z, fmaf(y.w, z.w, x))));
          }
          x += __shfl_xor_sync(0xFFFFFFFFu, x, 1);
          x += __shfl_xor_sync(0xFFFFFFFFu, x, 2);
          if ((tid & 3) == 0) score[a][b] = b <= a ? x * exp2f(steps_float(steps[a] - steps[b])) : 0.0f;
        }
        // ---- q_i S_0: this thread's rows of the state, then all ----
#pragma unroll 1
        for (int y0 = 0; y0 < n; y0 += kPassRows) {
          float4 o[kPassRows];
#pragma unroll
          for (int y = 0; y < kPassRows; ++y) o[y] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
          for (int x = 0; x < KR; x += 4) {
            if (kr0 + x >= pitch - 16) break;
#pragma unroll
            for (int y = 0; y < kPassRows; ++y) {
              const float4 z = *reinterpret_cast<const float4*>(qb + (y0 + y) * pitch + kr0 + x);
              const float f[4] = {z.x, z.y, z.z, z.w};
#pragma unroll
              for (int t = 0; t < 4; ++t) {
                o[y].x = fmaf(f[t], s[x + t].x, o[y].x);
                o[y].y = fmaf(f[t], s[x + t].y, o[y].y);
                o[y].z = fmaf(f[t], s[x + t].z, o[y].z);
                o[y].w = fmaf(f[t], s[x + t].w, o[y].w);
              }
            }
          }
#pragma unroll
          for (int y = 0; y < kPassRows; ++y) {
#pragma unroll
            for (int w = L; w < 32; w <<= 1) {
              o[y].x += __shfl_xor_sync(0xFFFFFFFFu, o[y].x, w);
              o[y].y += __shfl_xor_sync(0xFFFFFFFFu, o[y].y, w);
              o[y].z += __shfl_xor_sync(0xFFFFFFFFu, o[y].z, w);
              o[y].w += __shfl_xor_sync(0xFFFFFFFFu, o[y].w, w);
            }
            if (lane < L) *reinterpret_cast<float4*>(red + (warp * kBlockRows + y0 + y) * S + col) = o[y];
          }
        }
        __syncthreads();
#pragma unroll 1
        for (int x = tid; x < n * L; x += kLinThreads) {
          const int y = x / L, c = (x - y * L) * 4;
          if (c >= columns) continue;
          float4 a = make_float4(0.0f, 0.0f, 0.0f, 0.0f), b = a;
#pragma unroll
          for (int w = 0; w < kLinWarps; ++w) {
            const float4 z = *reinterpret_cast<const float4*>(red + (w * kBlockRows + y) * S + c);
            a.x += z.x, a.y += z.y, a.z += z.z, a.w += z.w;
          }
#pragma unroll 2
          for (int j = 0; j <= y; ++j) {  // no later row's value, whatever it holds
            const float4 z = *reinterpret_cast<const float4*>(vb + j * S + c);
            const float f = score[y][j];
            b.x = fmaf(f, z.x, b.x), b.y = fmaf(f, z.y, b.y), b.z = fmaf(f, z.z, b.z), b.w = fmaf(f, z.w, b.w);
          }
          const float f = first_weight[y];
          a.x = p.scale * fmaf(f, a.x, b.x), a.y = p.scale * fmaf(f, a.y, b.y);
          a.z = p.scale * fmaf(f, a.z, b.z), a.w = p.scale * fmaf(f, a.w, b.w);
          store4(out + ((row + y) * p.Hq + g0 + g) * p.Dv + c0 + c, a);
        }
      }
    } else {
      __syncthreads();
    }
    // ---- the state past the block ----
    if (!to && b0 + kBlockRows >= last) break;
    const float f = all_weight;
#pragma unroll
    for (int x = 0; x < KR; ++x) s[x].x *= f, s[x].y *= f, s[x].z *= f, s[x].w *= f;
#pragma unroll(KR <= 4 ? 2 : 1)
    for (int j = 0; j < n; ++j) {
      float4 z = *reinterpret_cast<const float4*>(vb + j * S + col);
      const float w = weight[j];
      z.x *= w, z.y *= w, z.z *= w, z.w *= w;
#pragma unroll
      for (int x = 0; x < KR; x += 4) {
        if (kr0 + x >= pitch - 16) break;
        const float4 y = *reinterpret_cast<const float4*>(kb + j * pitch + kr0 + x);
        const float t[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          s[x + u].x = fmaf(t[u], z.x, s[x + u].x);
          s[x + u].y = fmaf(t[u], z.y, s[x + u].y);
          s[x + u].z = fmaf(t[u], z.z, s[x + u].z);
          s[x + u].w = fmaf(t[u], z.w, s[x + u].w);
        }
      }
    }
  }
  if (to && mine) {
#pragma unroll
    for (int x = 0; x < KR; ++x)
      if (kr0 + x < p.Dk) *reinterpret_cast<float4*>(to + at + (int64_t)x * p.Dv) = s[x];
  }
  if (phase == kRowSums && c0 == 0 && tid == 0) plan.seg_steps[((int64_t)i * p.H + h) * plan.nseg + seg] = seg_steps;
}

template <typename T, int S, int KR>
cudaError_t launch_rows(const LinearLaunch& p, const LinearPlan& plan, int phase, long long items, cudaStream_t stream) {
  const int slices = (p.Dv + S - 1) / S;
  const size_t smem = linear_smem<S>(p.Dk);
  static std::atomic<size_t> raised[kMaxDevices];
  const cudaError_t err = raise_smem(linear_rows_kernel<T, S, KR>, smem, raised);
  if (err != cudaSuccess) return err;
  return launch_after_previous(linear_rows_kernel<T, S, KR>, dim3((unsigned)(items * slices)), dim3(kLinThreads), smem, stream,
                               p, plan, phase, slices);
}

// The columns of a CTA's part and what `items` states take with them: rounds of two CTAs
// per SM, times a round's cost.  Wide parts share their work among more products: with 32
// / 64 / 128 columns 8 requests of 8 rows of 16 heads of 128 take 10.7 / 7.1 / 7.3 us, 64
// single tokens of 4 states of 72 x 96 19.1 / 14.2 / 9.5, 3 tokens of 32 heads of 128 7.5 /
// 5.8 / 5.4, 64 requests of 256 rows of 16 heads of 64 x 64 in fp32 699 / 406 / 532.
struct RowsCost {
  int columns;
  double cost;
};
inline RowsCost rows_cost(long long items, int Dk, int Dv, int sms) {
  constexpr double weights[3] = {1.0, 1.5, 2.4};
  RowsCost best{};
  for (int c = 0; c < 3; ++c) {
    const int columns = 32 << c;
    if (columns == 128 && Dk > 128) break;  // more rows than a thread's registers take
    const long long ctas = items * ((Dv + columns - 1) / columns);
    const double cost = (double)((ctas + 2 * sms - 1) / (2 * sms)) * weights[c];
    if (c == 0 || cost < best.cost) best = RowsCost{columns, cost};
  }
  return best;
}

template <typename T>
cudaError_t launch_phase(const LinearLaunch& p, const LinearPlan& plan, int phase, cudaStream_t stream) {
  const long long items = (long long)p.rows.B * (phase == kRowSegments && p.q ? p.Hq : p.H) *
                          (phase == kRowSums ? plan.nseg - 1 : p.q ? plan.nseg : 1);
  const int columns = rows_cost(items, p.Dk, p.Dv, device_sms()).columns;
  if (columns == 128)
    return p.Dk <= 64 ? launch_rows<T, 128, 8>(p, plan, phase, items, stream)
                      : launch_rows<T, 128, 16>(p, plan, phase, items, stream);
  if (columns == 64)
    return p.Dk <= 64    ? launch_rows<T, 64, 4>(p, plan, phase, items, stream)
           : p.Dk <= 128 ? launch_rows<T, 64, 8>(p, plan, phase, items, stream)
                         : launch_rows<T, 64, 16>(p, plan, phase, items, stream);
  return p.Dk <= 128 ? launch_rows<T, 32, 4>(p, plan, phase, items, stream)
                     : launch_rows<T, 32, 8>(p, plan, phase, items, stream);
}

template <typename T>
cudaError_t launch_rows(const LinearLaunch& p, const LinearPlan& plan, cudaStream_t stream) {
  if (plan.nseg == 1) return launch_phase<T>(p, plan, kWholeRows, stream);
  cudaError_t err = launch_phase<T>(p, plan, kRowSums, stream);
  if (err == cudaSuccess) err = launch_linear_scan(p, plan, stream);
  return err == cudaSuccess ? launch_phase<T>(p, plan, kRowSegments, stream) : err;
}

// Segments for the rows' kernel: the number with the least work on the busiest SM, in
// blocks of 8 rows of a query head; the sums take half of that, two more launches about
// 6 of them.  1 / 3 / 8 / 16 segments: 3 requests of 201 rows of 32 heads of 128 in fp32
// 111 / 94 / 101 / 118 us (3 taken), one of 501 169 / 129 / 80 / 84 (73 with 10, taken),
// 16 requests of 256 rows of 16 heads of 64 106 / 152 / 159 / 186 (1 taken).
LinearPlan linear_rows_plan(int B, int K, int q_heads, int kv_heads, int Dk, int Dv, int max_segments) {
  LinearPlan best{};
  best.nseg = 1;
  const long long blocks = (K + kBlockRows) / kBlockRows, heads = (long long)B * kv_heads, queries = (long long)B * q_heads;
  best.seg_rows = (int)(blocks * kBlockRows);
  double least = rows_cost(heads, Dk, Dv, kLinSms).cost * (double)blocks * (q_heads / kv_heads + 0.5);
  for (int n = 2; n <= max_segments && queries * n <= 64 * kLinSms; ++n) {
    const long long per = (blocks + n - 1) / n;
    if (per < 2) break;
    const double cost = (rows_cost(queries * n, Dk, Dv, kLinSms).cost * 1.5 +
                         rows_cost(heads * (n - 1), Dk, Dv, kLinSms).cost * 0.5) * (double)per + 6.0;
    if (cost < least) {
      least = cost;
      best.nseg = n;
      best.seg_rows = (int)(per * kBlockRows);
    }
  }
  return best;
}

bool linear_shape_ok(int B, int K, int q_heads, int kv_heads, int Dk, int Dv, int dtype) {
  if (B < 1 || K < 0 || K >= SPEC_MAX_LINEAR_ROWS || (long long)B * (K + 1) > (1LL << 28)) return false;
  if (dtype != SPEC_BF16 && dtype != SPEC_F32) return false;
  const int e = element_size(dtype);
  return kv_heads >= 1 && q_heads >= kv_heads && q_heads % kv_heads == 0 && q_heads / kv_heads <= SPEC_MAX_GROUP &&
         Dk >= 1 && Dv >= 1 && Dk <= SPEC_MAX_HEAD_DIM && Dv <= SPEC_MAX_HEAD_DIM && Dk * e % 16 == 0 &&
         Dv * e % 16 == 0 && (long long)B * kv_heads <= (1LL << 26) && q_heads <= (1 << 20);
}

bool states_ok(const spec_states* s) {
  if (!s || !s->state || (reinterpret_cast<uintptr_t>(s->state) & 15u) != 0) return false;
  if (s->layers < 1 || s->slots < 1 || s->kv_heads < 1 || s->kv_heads > (1 << 20) || s->key_dim < 1 ||
      s->key_dim > SPEC_MAX_HEAD_DIM || s->value_dim < 1 || s->value_dim > SPEC_MAX_HEAD_DIM)
    return false;
  const int64_t size = (int64_t)s->kv_heads * s->key_dim * s->value_dim;
  const int64_t strides[2] = {s->layer_stride, s->slot_stride};
  const int32_t extent[2] = {s->layers, s->slots};
  for (int k = 0; k < 2; ++k) {
    if (extent[k] == 1) continue;  // never used
    if (strides[k] < size || strides[k] > (INT64_MAX >> 4) / extent[k] || strides[k] % 4 != 0) return false;
  }
  return true;
}

bool linear_rows_ok(const void* p, int64_t stride, int64_t width, int64_t e) {
  return p && (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && stride * e % 16 == 0 && stride >= width &&
         stride <= (INT64_MAX >> 36);
}

// Segments' first states, and behind them their decays; at least 256 bytes.  The best plan for a length may want more
// than that for a longer one: a workspace for the longer one serves as well, with the best plan of those that fit.
struct LinearGeometry {
  LinearPlan plan;
  size_t steps_off, bytes;
};

LinearGeometry linear_geometry(int B, int K, int q_heads, int kv_heads, int Dk, int Dv, int dtype, size_t limit = SIZE_MAX) {
  LinearGeometry g{};
  const auto bytes = [&](size_t heads) {
    return std::max<size_t>(256, heads * Dk * Dv * sizeof(float) + (heads * sizeof(long long) + 255) / 256 * 256);
  };
  int most = kLinMaxSegments;
  while (most > 1 && bytes((size_t)B * kv_heads * most) > limit) --most;
  const bool tc = linear_tc_serves(B, K, q_heads, Dk, Dv, dtype);
  g.plan = tc ? linear_plan(B, K, q_heads, kv_heads, most) : linear_rows_plan(B, K, q_heads, kv_heads, Dk, Dv, most);
  g.plan.staged = g.plan.nseg > 1 || (tc && q_heads > kv_heads);
  const size_t heads = g.plan.staged ? (size_t)B * kv_heads * g.plan.nseg : 0;
  g.steps_off = heads * Dk * Dv * sizeof(float);
  g.bytes = bytes(heads);
  return g;
}

int run_linear(const LinearLaunch& p, int dtype, void* ws, size_t ws_bytes, cudaStream_t stream) {
  LinearGeometry g = linear_geometry(p.rows.B, p.rows.K, p.Hq, p.H, p.Dk, p.Dv, dtype, ws_bytes);
  if (!ws || ws_bytes < g.bytes || (reinterpret_cast<uintptr_t>(ws) & 255u) != 0) return SPEC_ERR_WORKSPACE;
  g.plan.seg_state = static_cast<float*>(ws);
  g.plan.seg_steps = reinterpret_cast<long long*>(static_cast<char*>(ws) + g.steps_off);
  const cudaError_t err = linear_tc_serves(p.rows.B, p.rows.K, p.Hq, p.Dk, p.Dv, dtype) ? launch_linear_tc(p, g.plan, stream)
                          : linear_few_serves(p.rows.B, p.rows.K, p.Hq, p.H, p.Dk, p.Dv, dtype, device_sms())
                              ? launch_linear_few(p, dtype, stream)
                          : dtype == SPEC_F32 ? launch_rows<float>(p, g.plan, stream)
                                              : launch_rows<__nv_bfloat16>(p, g.plan, stream);
  return err == cudaSuccess && cudaGetLastError() == cudaSuccess ? SPEC_OK : SPEC_ERR_CUDA;
}

// What both calls have in common; false where an argument is refused.
bool linear_common(LinearLaunch* p, const void* k, int64_t k_row_stride, const void* v, int64_t v_row_stride, int dtype,
                   const float* log_decay, int64_t decay_row_stride, const spec_states* states, int layer,
                   const int32_t* slots_in, const int32_t* row_offsets, const int32_t* depth, const int64_t* pos_base,
                   int B, int K) {
  const int64_t e = element_size(dtype);
  if (layer < 0 || layer >= states->layers || !slots_in || !log_decay ||
      (reinterpret_cast<uintptr_t>(log_decay) & 3u) != 0 ||
      (decay_row_stride != 0 && (decay_row_stride < states->kv_heads || decay_row_stride > (INT64_MAX >> 36))))
    return false;
  if (!linear_rows_ok(k, k_row_stride, (int64_t)states->kv_heads * states->key_dim, e) ||
      !linear_rows_ok(v, v_row_stride, (int64_t)states->kv_heads * states->value_dim, e))
    return false;
  p->k = k;
  p->v = v;
  p->k_row = k_row_stride;
  p->v_row = v_row_stride;
  p->H = p->Hq = states->kv_heads;
  p->G = 1;
  p->Dk = states->key_dim;
  p->Dv = states->value_dim;
  p->log_decay = log_decay;
  p->decay_row = decay_row_stride;
  p->state = states->state + (states->layers > 1 ? layer * states->layer_stride : 0);
  p->slot_stride = states->slots > 1 ? states->slot_stride : 0;
  p->slots = states->slots;
  p->slots_in = slots_in;
  p->rows = RowLayout{row_offsets, depth, pos_base, B, K};
  return true;
}

}  // namespace

}  // namespace spec

extern "C" size_t spec_linear_workspace(int B, int K, int q_heads, int kv_heads, int key_dim, int value_dim,
                                        int dtype) {
  if (!spec::linear_shape_ok(B, K, q_heads, kv_heads, key_dim, value_dim, dtype)) return 0;
  // a commit's plan goes by the key-value heads
  return std::max(spec::linear_geometry(B, K, q_heads, kv_heads, key_dim, value_dim, dtype).bytes,
                  spec::linear_geometry(B, K, kv_heads, kv_heads, key_dim, value_dim, dtype).bytes);
}

extern "C" int spec_linear_attend(const void* q, int64_t q_row_stride, int q_heads, const void* k, int64_t k_row_stride,
                                  const void* v, int64_t v_row_stride, int dtype, const float* log_decay,
                                  int64_t decay_row_stride, const spec_states* states, int layer,
                                  const int32_t* slots_in, const int32_t* slots_out, const int32_t* row_offsets,
                                  const int32_t* depth, const int64_t* pos_base, int B, int K, float scale, void* out,
                                  int32_t* status, void* ws, size_t ws_bytes, cudaStream_t stream) {
  spec::NvtxRange range("spec_linear_attend");
  using namespace spec;
  if (!states_ok(states) ||
      !linear_shape_ok(B, K, q_heads, states->kv_heads, states->key_dim, states->value_dim, dtype))
    return SPEC_ERR_INVALID_ARG;
  LinearLaunch p{};
  if (!linear_common(&p, k, k_row_stride, v, v_row_stride, dtype, log_decay, decay_row_stride, states, layer, slots_in,
                     row_offsets, depth, pos_base, B, K))
    return SPEC_ERR_INVALID_ARG;
  if (!linear_rows_ok(q, q_row_stride, (int64_t)q_heads * p.Dk, element_size(dtype)) || !out ||
      (reinterpret_cast<uintptr_t>(out) & 15u) != 0 || !std::isfinite(scale))
    return SPEC_ERR_INVALID_ARG;
  p.q = q;
  p.q_row = q_row_stride;
  p.Hq = q_heads;
  p.G = q_heads / p.H;
  p.slots_out = slots_out;
  p.scale = scale;
  p.out = out;
  p.status = status;
  return run_linear(p, dtype, ws, ws_bytes, stream);
}

extern "C" int spec_linear_commit(const void* k, int64_t k_row_stride, const void* v, int64_t v_row_stride, int dtype,
                                  const float* log_decay, int64_t decay_row_stride, const spec_states* states, int layer,
                                  const int32_t* slots_in, const int32_t* slots_out, const int32_t* accepted_len,
                                  const int32_t* row_offsets, const int32_t* depth, const int64_t* pos_base, int B,
                                  int K, int32_t* status, void* ws, size_t ws_bytes, cudaStream_t stream) {
  spec::NvtxRange range("spec_linear_commit");
  using namespace spec;
  if (!states_ok(states) ||
      !linear_shape_ok(B, K, states->kv_heads, states->kv_heads, states->key_dim, states->value_dim, dtype))
    return SPEC_ERR_INVALID_ARG;
  LinearLaunch p{};
  if (!slots_out ||
      !linear_common(&p, k, k_row_stride, v, v_row_stride, dtype, log_decay, decay_row_stride, states, layer, slots_in,
                     row_offsets, depth, pos_base, B, K))
    return SPEC_ERR_INVALID_ARG;
  p.slots_out = slots_out;
  p.accepted = accepted_len;
  p.status = status;
  return run_linear(p, dtype, ws, ws_bytes, stream);
}
