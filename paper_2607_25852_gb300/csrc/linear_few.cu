// linear_few.cu -- linear attention of few rows per request (single tokens,
// verification rounds) where there are many heads: what counts is that the states
// come and go at the HBM's rate.
//
// The formulas are linear.cu's.  A head's state is one block of memory, so
// persistent CTAs take head after head through a ring in shared memory: a warp
// lists the heads with their rows' decays, brings states, queries, keys and values
// by bulk copies, and sends the new states back the same way; eight warps compute,
// 16 keys by four values of the state per thread (heads of 128), in registers for
// all rows of the head.  Up to three states are in flight per SM while one is
// worked on.  The rows' products with the state are summed over the warps through
// shared memory, four or eight rows at a time.
//
// Bound by HBM for up to about eight rows, by the rows' passes beyond: 128 tokens of 32
// heads of 128 with their states 92 us (5.9 TB/s), 64 requests of up to 8 rows 48 us
// (the states alone 2.8 TB/s) and their commit 55 (5.1 TB/s).
#include "attend_ring.cuh"
#include "linear_few.cuh"

namespace spec {

namespace {

constexpr int kFewThreads = 256, kFewWarps = kFewThreads / 32;  // and a warp that brings
constexpr int kMaxStages = 4;

struct FewLaunch {
  LinearLaunch p;
  uint32_t heads;       // B * H
  int stages, rows_off, stage_bytes;  // of shared memory: where the rows begin in a stage
  int k_off, v_off;     // from the rows' begin
};

// A head and its rows.
struct alignas(16) FewItem {
  long long steps[kLinFewRows];
  float weight[kLinFewRows], first[kLinFewRows];  // exp(L_n - L_j), scale exp(L_i)
  float all;
  int n, h, early;
  long long row0;
  bool fresh, none;  // begins from zeros; the list is over
  float* to;
};

struct FewShared {
  uint64_t full[kMaxStages], empty[kMaxStages];
  FewItem items[kMaxStages];
  float score[kLinFewRows][kLinFewRows + 1];
  int aborted;
};

__device__ __forceinline__ void bulk_load(uint32_t to, const void* from, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(to), "l"(from),
               "r"(bytes), "r"(smem_u32(bar))
               : "memory");
}
__device__ __forceinline__ void bulk_store(void* to, uint32_t from, uint32_t bytes) {
  asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(to), "r"(from), "r"(bytes) : "memory");
}

// Eight (bf16) or four elements of a row in shared memory.
template <typename T>
__device__ __forceinline__ void row_vec(const T* row, float (&f)[16 / sizeof(T)]) {
  const uint4 w = *reinterpret_cast<const uint4*>(row);
  if (sizeof(T) == 4) {
    f[0] = __uint_as_float(w.x), f[1] = __uint_as_float(w.y), f[2] = __uint_as_float(w.z), f[3] = __uint_as_float(w.w);
  } else {
    f[0] = bf16_lo(w.x), f[1] = bf16_hi(w.x), f[2] = bf16_lo(w.y), f[3] = bf16_hi(w.y);
    f[16 / sizeof(T) - 4] = bf16_lo(w.z), f[16 / sizeof(T) - 3] = bf16_hi(w.z);
    f[16 / sizeof(T) - 2] = bf16_lo(w.w), f[16 / sizeof(T) - 1] = bf16_hi(w.w);
  }
}
// Four elements of a row in shared memory, as pairs.
__device__ __forceinline__ void row_four(const float* row, f32x2 (&f)[2]) {
  const float4 w = *reinterpret_cast<const float4*>(row);
  f[0] = pair(w.x, w.y), f[1] = pair(w.z, w.w);
}
__device__ __forceinline__ void row_four(const __nv_bfloat16* row, f32x2 (&f)[2]) {
  const uint2 w = *reinterpret_cast<const uint2*>(row);
  f[0] = pair(bf16_lo(w.x), bf16_hi(w.x)), f[1] = pair(bf16_lo(w.y), bf16_hi(w.y));
}
__device__ __forceinline__ void store_four(float* to, f32x2 a, f32x2 b) {
  const float2 x = unpair(a), y = unpair(b);
  *reinterpret_cast<float4*>(to) = make_float4(x.x, x.y, y.x, y.y);
}
__device__ __forceinline__ void store_four(__nv_bfloat16* to, f32x2 a, f32x2 b) {
  *reinterpret_cast<uint2*>(to) = make_uint2(last_pair(a), last_pair(b));
}

template <typename T, int DK, int DV, int kPass>
__global__ void __launch_bounds__(kFewThreads + 32, 1) linear_few_kernel(const __grid_constant__ FewLaunch a) {
  constexpr int L = DV / 4, KG = kFewThreads / L, KR = DK / KG;  // threads across values, groups of KR keys
  constexpr int W = 16 / (int)sizeof(T);
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 127) & ~(uintptr_t)127);
  __shared__ FewShared sh;
  __shared__ alignas(16) float red[kFewWarps][kPass][DV];
  const LinearLaunch& p = a.p;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (tid == 0) {
    for (int s = 0; s < a.stages; ++s) {
      mbar_init(&sh.full[s], 1);
      mbar_init(&sh.empty[s], kFewWarps);
    }
    sh.aborted = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  pdl_wait_prerequisites();
  pdl_launch_dependents();
  __syncthreads();
  constexpr uint32_t kStateBytes = DK * DV * 4;

  if (warp == kFewWarps) {
    // ---- lists, brings, and sends back ----
    uint32_t c = 0;  // items so far
    bool ok = true;
    // the stage of item c - stages is free, and its state on its way
    auto wait_free = [&](uint32_t c) {
      if (c < (uint32_t)a.stages) return;
      const int s = c % a.stages;
      bool there = mbar_try_wait(&sh.empty[s], (c / a.stages - 1) & 1u);
      if (!there) there = mbar_wait_slow(&sh.empty[s], (c / a.stages - 1) & 1u, p.status);
      ok = __all_sync(0xFFFFFFFFu, there);
      if (!ok) return;
      float* to = sh.items[s].to;
      if (lane == 0) {
        if (to) bulk_store(to, smem_u32(smem + s * a.stage_bytes), kStateBytes);
        asm volatile("cp.async.bulk.commit_group;\n\tcp.async.bulk.wait_group.read 0;" ::: "memory");
      }
      __syncwarp();
    };
    LinearRequest r{};
    int known = -1;
    for (uint32_t x = blockIdx.x; ok && x < a.heads; x += gridDim.x) {
      const int i = (int)(x / (uint32_t)p.H), h = (int)(x - (uint32_t)i * (uint32_t)p.H);
      if (i != known) r = linear_request(p, i), known = i;
      if (!r.ok) {
        if (h == 0 && lane == 0) report(p.status, SPEC_ERR_BAD_INPUT);
        continue;
      }
      const int n = r.last - r.first;
      const long long row0 = r.row0 + r.first;
      long long g = 0;
      if (lane < n) g = decay_steps(__ldg(p.log_decay + (row0 + lane) * p.decay_row + h), p.status);
#pragma unroll
      for (int o = 1; o < kLinFewRows; o <<= 1) {
        const long long y = __shfl_up_sync(0xFFFFFFFFu, g, o);
        if (lane >= o) g += y;
      }
      const long long all = __shfl_sync(0xFFFFFFFFu, g, kLinFewRows - 1);  // rows past n add 0
      wait_free(c);
      if (!ok) break;
      const int s = c % a.stages;
      FewItem& t = sh.items[s];
      t.steps[lane] = g;
      t.weight[lane] = exp2f(steps_float(all - g));
      t.first[lane] = p.scale * exp2f(steps_float(g));
      uint8_t* stage = smem + s * a.stage_bytes;
      if (lane == 0) {
        t.all = exp2f(steps_float(all));
        t.n = n;
        t.h = h;
        t.early = r.first;
        t.row0 = row0;
        t.fresh = r.from < 0;
        t.none = false;
        t.to = r.to >= 0 ? p.state + r.to * p.slot_stride + (int64_t)h * DK * DV : nullptr;
        const uint32_t rows = (uint32_t)n * (DK + DV + (p.q ? p.G * DK : 0)) * sizeof(T);
        mbar_expect_tx(&sh.full[s], rows + (r.from >= 0 ? kStateBytes : 0u));
        if (r.from >= 0)
          bulk_load(smem_u32(stage), p.state + r.from * p.slot_stride + (int64_t)h * DK * DV, kStateBytes, &sh.full[s]);
      }
      __syncwarp();
      if (lane < n) {
        const uint32_t to = smem_u32(stage) + a.rows_off;
        const int64_t row = row0 + lane;
        if (p.q)
          for (int y = 0; y < p.G; ++y)
            bulk_load(to + (y * (p.rows.K + 1) + lane) * DK * (int)sizeof(T),
                      static_cast<const T*>(p.q) + row * p.q_row + (int64_t)(h * p.G + y) * DK, DK * sizeof(T), &sh.full[s]);
        bulk_load(to + a.k_off + lane * DK * (int)sizeof(T), static_cast<const T*>(p.k) + row * p.k_row + (int64_t)h * DK,
                  DK * sizeof(T), &sh.full[s]);
        bulk_load(to + a.v_off + lane * DV * (int)sizeof(T), static_cast<const T*>(p.v) + row * p.v_row + (int64_t)h * DV,
                  DV * sizeof(T), &sh.full[s]);
      }
      __syncwarp();
      ++c;
    }
    // the list's end, and the last items' states
    wait_free(c);
    if (ok && lane == 0) {
      sh.items[c % a.stages].none = true;
      sh.items[c % a.stages].to = nullptr;
      mbar_arrive(&sh.full[c % a.stages]);
    }
    __syncwarp();
    for (int y = 1; ok && y < a.stages; ++y) wait_free(c + y);
    if (!ok) {
      if (lane == 0) *(volatile int*)&sh.aborted = 1;
      // the copies in flight end before the CTA does
      for (int y = 0; y < a.stages; ++y) {
        const uint32_t z = c - 1 - y;
        if (lane == 0 && z < c) mbar_wait_slow(&sh.full[z % a.stages], (z / a.stages) & 1u, p.status);
      }
    }
    if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    return;
  }

  // ---- eight warps compute: this thread's keys kr0 .. + KR - 1, values col .. + 3 ----
  const int col = (tid % L) * 4, kr0 = (tid / L) * KR;
  T* out = static_cast<T*>(p.out);
  for (uint32_t c = 0;; ++c) {
    const int s = c % a.stages;
    bool there = mbar_try_wait(&sh.full[s], (c / a.stages) & 1u);
    if (!there) there = !*(volatile int*)&sh.aborted && mbar_wait_slow(&sh.full[s], (c / a.stages) & 1u, p.status);
    if (named_or(1, kFewThreads, !there)) break;  // (also: the last item's shared arrays are free)
    const FewItem& t = sh.items[s];
    if (t.none) break;
    const int n = t.n, h = t.h;
    float* state = reinterpret_cast<float*>(smem + s * a.stage_bytes);
    const T* qs = reinterpret_cast<const T*>(smem + s * a.stage_bytes + a.rows_off);
    const T* ks = reinterpret_cast<const T*>(smem + s * a.stage_bytes + a.rows_off + a.k_off);
    const T* vs = reinterpret_cast<const T*>(smem + s * a.stage_bytes + a.rows_off + a.v_off);
    f32x2 st[KR / 2][4];  // pairs of keys
#pragma unroll
    for (int x = 0; x < KR; x += 2) {
      float4 w = make_float4(0.0f, 0.0f, 0.0f, 0.0f), y = w;
      if (!t.fresh) {
        w = *reinterpret_cast<const float4*>(state + (kr0 + x) * DV + col);
        y = *reinterpret_cast<const float4*>(state + (kr0 + x + 1) * DV + col);
      }
      st[x / 2][0] = pair(w.x, y.x), st[x / 2][1] = pair(w.y, y.y);
      st[x / 2][2] = pair(w.z, y.z), st[x / 2][3] = pair(w.w, y.w);
    }
    if (p.q) {
      for (int x = tid; x < t.early * p.G * L; x += kFewThreads) {  // rows before position 0
        const int y = x / L;
        store_four(out + ((t.row0 - 1 - y / p.G) * p.Hq + h * p.G + y % p.G) * DV + (x % L) * 4, 0ull, 0ull);
      }
#pragma unroll 1
      for (int g = 0; g < p.G; ++g) {
        const T* q = qs + g * (p.rows.K + 1) * DK;
        // ---- exp(L_i - L_j) (q_i k_j): eight threads per pair ----
        if (g) named_sync(1, kFewThreads);
        for (int x = tid >> 3; x < n * n; x += kFewThreads / 8) {
          const int i = x / n, j = x - i * n;
          float sum = 0.0f;
          if (j <= i) {
            for (int d = (tid & 7) * W; d < DK; d += 8 * W) {
              float y[W], z[W];
              row_vec<T>(q + i * DK + d, y);
              row_vec<T>(ks + j * DK + d, z);
#pragma unroll
              for (int e = 0; e < W; ++e) sum = fmaf(y[e], z[e], sum);
            }
          }
          const uint32_t mask = 0xFFu << (lane & 24);
          sum += __shfl_xor_sync(mask, sum, 1);
          sum += __shfl_xor_sync(mask, sum, 2);
          sum += __shfl_xor_sync(mask, sum, 4);
          if ((tid & 7) == 0 && j <= i) sh.score[i][j] = p.scale * (sum * exp2f(steps_float(t.steps[i] - t.steps[j])));
        }
#pragma unroll 1
        for (int y0 = 0; y0 < n; y0 += kPass) {
          // ---- rows y0 .. y0 + 3 times the state, this thread's keys ----
#pragma unroll
          for (int y = 0; y < kPass; ++y) {
            if (y0 + y >= n) break;
            f32x2 o[4] = {0ull, 0ull, 0ull, 0ull};  // of even and odd keys
#pragma unroll
            for (int x = 0; x < KR; x += 4) {
              f32x2 f[2];
              row_four(q + (y0 + y) * DK + kr0 + x, f);
#pragma unroll
              for (int z = 0; z < 4; ++z) o[z] = fma2(f[1], st[x / 2 + 1][z], fma2(f[0], st[x / 2][z], o[z]));
            }
            float v[4];
#pragma unroll
            for (int z = 0; z < 4; ++z) {
              const float2 two = unpair(o[z]);
              v[z] = two.x + two.y;
              if (L < 32) v[z] += __shfl_xor_sync(0xFFFFFFFFu, v[z], 16);
            }
            if (lane < L) *reinterpret_cast<float4*>(&red[warp][y][col]) = make_float4(v[0], v[1], v[2], v[3]);
          }
          named_sync(1, kFewThreads);
          // ---- all of the state, and the block's own rows ----
          for (int x = tid; x < min(kPass, n - y0) * L; x += kFewThreads) {
            const int y = x / L, v = (x - y * L) * 4, i = y0 + y;
            f32x2 b[2] = {0ull, 0ull}, w[2];
#pragma unroll
            for (int z = 0; z < kFewWarps; ++z) {
              row_four(&red[z][y][v], w);
              b[0] = add2(b[0], w[0]), b[1] = add2(b[1], w[1]);
            }
            const f32x2 f = pair(t.first[i], t.first[i]);
            b[0] = mul2(f, b[0]), b[1] = mul2(f, b[1]);
            for (int j = 0; j <= i; ++j) {  // no later row's value, whatever it holds
              const f32x2 m = pair(sh.score[i][j], sh.score[i][j]);
              row_four(vs + j * DV + v, w);
              b[0] = fma2(m, w[0], b[0]), b[1] = fma2(m, w[1], b[1]);
            }
            store_four(out + ((t.row0 + i) * p.Hq + h * p.G + g) * DV + v, b[0], b[1]);
          }
          if (y0 + kPass < n) named_sync(1, kFewThreads);
        }
      }
    }
    // ---- the state past the rows, in its place ----
    if (t.to) {
      const f32x2 f = pair(t.all, t.all);
#pragma unroll
      for (int x = 0; x < KR / 2; ++x)
#pragma unroll
        for (int z = 0; z < 4; ++z) st[x][z] = mul2(st[x][z], f);
#pragma unroll 1
      for (int j = 0; j < n; ++j) {
        f32x2 w[2];
        row_four(vs + j * DV + col, w);
        const float2 w0 = unpair(w[0]), w1 = unpair(w[1]);
        const float m = t.weight[j], v[4] = {m * w0.x, m * w0.y, m * w1.x, m * w1.y};
#pragma unroll
        for (int x = 0; x < KR; x += 4) {
          f32x2 k[2];
          row_four(ks + j * DK + kr0 + x, k);
#pragma unroll
          for (int z = 0; z < 4; ++z) {
            st[x / 2][z] = fma2(k[0], pair(v[z], v[z]), st[x / 2][z]);
            st[x / 2 + 1][z] = fma2(k[1], pair(v[z], v[z]), st[x / 2 + 1][z]);
          }
        }
      }
#pragma unroll
      for (int x = 0; x < KR; x += 2) {
        float2 w[4];
#pragma unroll
        for (int z = 0; z < 4; ++z) w[z] = unpair(st[x / 2][z]);
        *reinterpret_cast<float4*>(state + (kr0 + x) * DV + col) = make_float4(w[0].x, w[1].x, w[2].x, w[3].x);
        *reinterpret_cast<float4*>(state + (kr0 + x + 1) * DV + col) = make_float4(w[0].y, w[1].y, w[2].y, w[3].y);
      }
      proxy_fence();
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(&sh.empty[s]);
  }
}

template <typename T, int DK, int DV, int kPass>
cudaError_t launch_pass(const LinearLaunch& p, cudaStream_t stream) {
  FewLaunch a{};
  a.p = p;
  a.heads = (uint32_t)p.rows.B * (uint32_t)p.H;
  const int q_bytes = p.q ? p.G * (p.rows.K + 1) * DK * (int)sizeof(T) : 0, k_bytes = (p.rows.K + 1) * DK * (int)sizeof(T);
  a.rows_off = DK * DV * 4;
  a.k_off = q_bytes;
  a.v_off = a.k_off + k_bytes;
  a.stage_bytes = (a.rows_off + a.v_off + (p.rows.K + 1) * DV * (int)sizeof(T) + 127) / 128 * 128;
  static std::atomic<int> known;
  int fixed;
  cudaError_t err = static_smem(linear_few_kernel<T, DK, DV, kPass>, known, &fixed);
  if (err != cudaSuccess) return err;
  const int room = 227 * 1024 - (fixed + 1023) / 1024 * 1024 - 128;
  a.stages = std::min(kMaxStages, room / a.stage_bytes);
  const size_t smem = (size_t)a.stages * a.stage_bytes + 128;
  static std::atomic<size_t> raised[kMaxDevices];
  err = raise_smem(linear_few_kernel<T, DK, DV, kPass>, smem, raised);
  if (err != cudaSuccess) return err;
  return launch_after_previous(linear_few_kernel<T, DK, DV, kPass>, dim3(std::min<uint32_t>(a.heads, device_sms())),
                               dim3(kFewThreads + 32), smem, stream, a);
}

// Up to four rows leave room for a third state of 64 KB.
template <typename T, int DK, int DV>
cudaError_t launch_few(const LinearLaunch& p, cudaStream_t stream) {
  return p.rows.K < 4 || !p.q ? launch_pass<T, DK, DV, 4>(p, stream) : launch_pass<T, DK, DV, 8>(p, stream);
}

template <typename T>
cudaError_t launch_few(const LinearLaunch& p, cudaStream_t stream) {
  if (p.Dk == 64) return p.Dv == 64 ? launch_few<T, 64, 64>(p, stream) : launch_few<T, 64, 128>(p, stream);
  return p.Dv == 64 ? launch_few<T, 128, 64>(p, stream) : launch_few<T, 128, 128>(p, stream);
}

}  // namespace

cudaError_t launch_linear_few(const LinearLaunch& p, int dtype, cudaStream_t stream) {
  return dtype == SPEC_F32 ? launch_few<float>(p, stream) : launch_few<__nv_bfloat16>(p, stream);
}

}  // namespace spec
