// attend.cu -- attention of the packed verification rows over the paged
// key-value cache (spec_attend).
//
//   x_t = scale <q, k_t>,  out = sum_t e^(x_t - m) v_t / sum_t e^(x_t - m)
//
// over the positions a row sees, in one pass over the keys and values with a
// running maximum m and sum per (row, query head).  All the columns (row,
// query head) that share a key-value head are done together, so each key and
// value is read once for them.  attend.cuh says how the work is divided.
//
// attend_general_kernel serves every layout of the contract on the CUDA
// cores: fp32 caches, head dimensions and page sizes that the tensor-core
// kernel does not take.
#include <algorithm>

#include "attend.cuh"
#include "attend_tc.cuh"
#include "tensor_core.cuh"

namespace spec {

// ---------------------------------------------------------------------------
// The general kernel
// ---------------------------------------------------------------------------
constexpr int kGenThreads = 256;
constexpr int kGenCols = 16;   // columns per item
constexpr int kGenTile = 64;   // positions per tile
constexpr int kGenPitchS = kGenTile + 4;

__device__ __forceinline__ void cp_async16(void* dst, const void* src, bool real) {
  // nothing is read where `real` is false: 16 zero bytes are written
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(real ? 16 : 0)
               : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// 4 consecutive elements of shared memory as fp32.
__device__ __forceinline__ float4 load4(const float* p) { return *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ float4 load4(const __nv_bfloat16* p) {
  const uint2 w = *reinterpret_cast<const uint2*>(p);
  return make_float4(bf16_lo(w.x), bf16_hi(w.x), bf16_lo(w.y), bf16_hi(w.y));
}

// Bytes of shared memory: `stages` tiles of K and V (rows padded by 16 bytes,
// so that eight rows' 16-byte loads fall into different banks), Q in fp32,
// the scores.
static size_t general_smem(int D, int esize, int stages) {
  return (size_t)stages * 2 * kGenTile * (D * esize + 16) + (size_t)kGenCols * D * 4 + (size_t)kGenCols * kGenPitchS * 4;
}

template <typename T>
__global__ void __launch_bounds__(kGenThreads, 1) attend_general_kernel(const AttendLaunch a, int stages) {
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ Share share;
  __shared__ Segment seg;
  __shared__ long long sums[32];
  __shared__ float sh_alpha[kGenCols], sh_l[kGenCols], sh_m[kGenCols];
  __shared__ int sh_tok[2][kGenTile];  // position of a loaded token, -1: none or without a page
  __shared__ int more, last;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int pitch = a.D * (int)sizeof(T) + 16;  // bytes
  uint8_t* sK = smem;
  uint8_t* sV = sK + (size_t)stages * kGenTile * pitch;
  float* sQ = reinterpret_cast<float*>(sV + (size_t)stages * kGenTile * pitch);
  float* sS = sQ + kGenCols * a.D;  // [col][token]

  pdl_wait_prerequisites();
  find_share<kGenTile>(a, &share, sums);
  Walk<kGenTile> walk(a, share);
  const int vecs = a.D * (int)sizeof(T) / 16;
  // outputs of a thread: 4 consecutive d of up to 4 columns
  const int dv = a.D / 4;
  const int groups = kGenThreads / dv;  // >= 4 (D <= 256)
  const int cpg = (kGenCols + groups - 1) / groups;
  const int my_d = (tid % dv) * 4, my_c = (tid / dv) * cpg;
  const bool pv_active = tid / dv < groups && my_c < kGenCols;

  for (;;) {
    if (tid == 0) more = walk.next(&seg) ? 1 : 0;
    __syncthreads();
    if (!more) break;
    const Segment s = seg;
    // ---- Q, in fp32; unused columns zero ----
    for (int x = tid; x < kGenCols * dv; x += kGenThreads) {
      const int c = x / dv, d = (x - c * dv) * 4;
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      if (c < s.cols) {
        const int col = s.col0 + c, j = col / a.G;
        const T* src = static_cast<const T*>(a.q) + (int64_t)(s.row0 + j) * a.q_row +
                       (int64_t)(s.head * a.G + col - j * a.G) * a.D + d;
        if (sizeof(T) == 4) {
          v = __ldg(reinterpret_cast<const float4*>(src));
        } else {
          const uint2 w = __ldg(reinterpret_cast<const uint2*>(src));
          v = make_float4(bf16_lo(w.x), bf16_hi(w.x), bf16_lo(w.y), bf16_hi(w.y));
        }
      }
      *reinterpret_cast<float4*>(sQ + c * a.D + d) = v;
    }
    const int p_first = s.p + s.col0 / a.G, p_last = s.p + (s.col0 + s.cols - 1) / a.G;
    // four threads per token
    auto load_tile = [&](int x, int stage) {
      const int tok = tid >> 2, pos = tile_start<kGenTile>(s.tiles, x) + tok;
      const bool wanted =
          pos <= p_last && (a.window == 0 || pos > p_first - a.window || pos < a.sinks);  // some row sees it
      int page = -1;
      if (wanted) {
        page = __ldg(a.table + (size_t)s.request * a.max_pages + pos / a.page_size);
        if (page < 0 || page >= a.pages) {
          page = -1;
          if ((tid & 3) == 0) report(a.status, SPEC_ERR_BAD_INPUT);
        }
      }
      if ((tid & 3) == 0) sh_tok[stage][tok] = page >= 0 ? pos : -1;
      const int64_t off = (page >= 0 ? (int64_t)page * a.page_b + (int64_t)(pos % a.page_size) * a.token_b : 0) +
                          s.head * a.head_b;
      uint8_t* dk = sK + ((size_t)stage * kGenTile + tok) * pitch;
      uint8_t* dvv = sV + ((size_t)stage * kGenTile + tok) * pitch;
      for (int w = tid & 3; w < vecs; w += 4) {
        cp_async16(dk + w * 16, a.k + off + w * 16, page >= 0);
        cp_async16(dvv + w * 16, a.v + off + w * 16, page >= 0);
      }
      cp_async_commit();
    };
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.0f, 0.0f};  // columns 2 warp, 2 warp + 1 (all lanes alike)
    float acc[4][4];
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int d = 0; d < 4; ++d) acc[k][d] = 0.0f;
    load_tile(s.tile0, 0);
    for (int x = 0; x < s.ntiles; ++x) {
      const int stage = stages == 2 ? x & 1 : 0;
      if (stages == 2 && x + 1 < s.ntiles) {
        load_tile(s.tile0 + x + 1, stage ^ 1);
        cp_async_wait<1>();
      } else {
        cp_async_wait<0>();
      }
      __syncthreads();
      {  // ---- scores: a token and 4 columns per thread ----
        const int tok = tid & (kGenTile - 1), c0 = (tid / kGenTile) * 4;
        if (c0 < s.cols) {
          const T* kr = reinterpret_cast<const T*>(sK + ((size_t)stage * kGenTile + tok) * pitch);
          float dot[4] = {0.f, 0.f, 0.f, 0.f};
          for (int d = 0; d < a.D; d += 4) {
            const float4 k4 = load4(kr + d);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              const float4 q4 = load4(sQ + (c0 + c) * a.D + d);
              dot[c] = fmaf(k4.x, q4.x, dot[c]);
              dot[c] = fmaf(k4.y, q4.y, dot[c]);
              dot[c] = fmaf(k4.z, q4.z, dot[c]);
              dot[c] = fmaf(k4.w, q4.w, dot[c]);
            }
          }
          const int pos = sh_tok[stage][tok];
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const int row = s.p + (s.col0 + c0 + c) / a.G;
            const bool seen = pos >= 0 && pos <= row && (a.window == 0 || pos > row - a.window || pos < a.sinks);
            sS[(c0 + c) * kGenPitchS + tok] = seen ? dot[c] * a.c2 : -INFINITY;
          }
        }
      }
      __syncthreads();
      // ---- the running maximum and sum: two columns per warp ----
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int c = 2 * warp + k;
        if (c >= s.cols) continue;
        float* row = sS + c * kGenPitchS;
        const float x0 = row[lane], x1 = row[lane + 32];
        float t = fmaxf(x0, x1);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) t = fmaxf(t, __shfl_xor_sync(0xFFFFFFFFu, t, o));
        const float mn = fmaxf(m[k], t);
        const float alpha = m[k] == -INFINITY ? 0.0f : exp2f(m[k] - mn);
        // a masked score is -inf and weighs 0; a NaN score stays NaN
        const float p0 = x0 == -INFINITY ? 0.0f : exp2f(x0 - mn), p1 = x1 == -INFINITY ? 0.0f : exp2f(x1 - mn);
        row[lane] = p0;
        row[lane + 32] = p1;
        float sum = p0 + p1;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
        l[k] = fmaf(l[k], alpha, sum);
        m[k] = mn;
        if (lane == 0) sh_alpha[c] = alpha;
      }
      __syncthreads();
      // ---- out += P V ----
      if (pv_active && my_c < s.cols) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          if (k >= cpg) break;
          const float alpha = sh_alpha[min(my_c + k, s.cols - 1)];
#pragma unroll
          for (int d = 0; d < 4; ++d) acc[k][d] *= alpha;
        }
        const uint8_t* vr = sV + (size_t)stage * kGenTile * pitch + my_d * sizeof(T);
        for (int tok = 0; tok < kGenTile; ++tok) {
          const float4 v4 = load4(reinterpret_cast<const T*>(vr + (size_t)tok * pitch));
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            if (k >= cpg) break;
            const float w = my_c + k < s.cols ? sS[(my_c + k) * kGenPitchS + tok] : 0.0f;
            if (w != 0.0f) {  // what a masked token holds does not reach the sum
              acc[k][0] = fmaf(w, v4.x, acc[k][0]);
              acc[k][1] = fmaf(w, v4.y, acc[k][1]);
              acc[k][2] = fmaf(w, v4.z, acc[k][2]);
              acc[k][3] = fmaf(w, v4.w, acc[k][3]);
            }
          }
        }
      }
      __syncthreads();
      if (stages == 1 && x + 1 < s.ntiles) load_tile(s.tile0 + x + 1, 0);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int c = 2 * warp + k;
      if (lane == 0 && c < s.cols) {
        sh_l[c] = l[k];
        sh_m[c] = m[k];
      }
    }
    __syncthreads();
    // ---- the item's result, or this part's ----
    if (pv_active) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int c = my_c + k;
        if (k >= cpg || c >= s.cols) break;
        if (s.slot < 0) {
          const float inv = sh_l[c] == 0.0f ? 0.0f : 1.0f / sh_l[c];
          T* o = static_cast<T*>(a.out) + out_index(a, s, c) * a.D + my_d;
#pragma unroll
          for (int d = 0; d < 4; ++d) o[d] = from_float<T>(acc[k][d] * inv);
        } else {
          *reinterpret_cast<float4*>(a.part + ((size_t)s.slot * kGenCols + c) * a.D + my_d) =
              make_float4(acc[k][0], acc[k][1], acc[k][2], acc[k][3]);
        }
      }
    }
    if (tid < s.cols) {
      if (s.slot < 0) {
        if (a.lse) a.lse[out_index(a, s, tid)] = row_lse(sh_m[tid], sh_l[tid]);
      } else {
        a.part_stat[(size_t)s.slot * kGenCols + tid] = make_float2(sh_m[tid], sh_l[tid]);
      }
    }
    if (s.slot >= 0) {
      __threadfence();
      __syncthreads();
      if (tid == 0) {
        last = atomicAdd(a.arrived + s.first_cta, 1u) == (uint32_t)s.parts - 1 ? 1 : 0;
        if (last) a.arrived[s.first_cta] = 0;
      }
      __syncthreads();
      if (last) {
        __threadfence();
        join_parts<T>(a, s, tid, kGenThreads);
      }
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
struct AttendGeometry {
  int ct;  // columns per item, the most of the kernels that may serve the shape
  int ctas;  // most CTAs: two parts each
  size_t part_off, stat_off, bytes;
};

// The counters come first, so that their place does not depend on the kernel.
static AttendGeometry attend_geometry(int cols, int D, int dtype) {
  AttendGeometry g{};
  g.ct = dtype == SPEC_BF16 ? std::max(kGenCols, attend_tc_columns(cols)) : kGenCols;
  g.ctas = kAttendMaxSms * (dtype == SPEC_BF16 ? attend_tc_ctas_per_sm(D, g.ct) : 1);
  const size_t slots = 2 * (size_t)g.ctas;
  g.part_off = ((size_t)g.ctas * 4 + 255) / 256 * 256;
  g.stat_off = g.part_off + (slots * g.ct * D * 4 + 255) / 256 * 256;
  g.bytes = g.stat_off + (slots * g.ct * 8 + 255) / 256 * 256;
  return g;
}

static bool attend_shape_ok(int B, int K, int q_heads, int kv_heads, int D, int dtype) {
  return rows_shape_ok(B, K) && kv_heads >= 1 && q_heads >= kv_heads && q_heads % kv_heads == 0 &&
         q_heads / kv_heads <= SPEC_MAX_GROUP && D >= 1 && D <= SPEC_MAX_HEAD_DIM &&
         (dtype == SPEC_BF16 || dtype == SPEC_F32) && D * element_size(dtype) % 16 == 0;
}

template <typename T>
static cudaError_t launch_general(const AttendLaunch& a, cudaStream_t stream) {
  const int esize = (int)sizeof(T);
  // two stages where they fit (228 KB an SM, 1 KB of it reserved per CTA)
  const int stages = general_smem(a.D, esize, 2) <= 220 * 1024 ? 2 : 1;
  const size_t smem = general_smem(a.D, esize, stages);
  static std::atomic<size_t> raised[kMaxDevices];
  const cudaError_t err = raise_smem(attend_general_kernel<T>, smem, raised);
  if (err != cudaSuccess) return err;
  return launch_after_previous(attend_general_kernel<T>, dim3(a.ctas), dim3(kGenThreads), smem, stream, a, stages);
}

}  // namespace spec

extern "C" size_t spec_attend_workspace(int B, int K, int q_heads, int kv_heads, int head_dim, int dtype) {
  if (!spec::attend_shape_ok(B, K, q_heads, kv_heads, head_dim, dtype)) return 0;
  return spec::attend_geometry((K + 1) * (q_heads / kv_heads), head_dim, dtype).bytes;
}

extern "C" int spec_attend(const void* q, int64_t q_row_stride, int q_heads, const spec_cache* cache, int layer,
                           const int32_t* row_offsets, const int32_t* depth, const int64_t* pos_base,
                           const int32_t* page_table, int max_pages, int B, int K, float scale, int window, int sinks,
                           void* out, float* lse_out, int32_t* status, void* ws, size_t ws_bytes,
                           cudaStream_t stream) {
  spec::NvtxRange range("spec_attend");
  using namespace spec;
  if (!cache_ok(cache) || !attend_shape_ok(B, K, q_heads, cache->kv_heads, cache->head_dim, cache->dtype) ||
      !table_shape_ok(B, max_pages, cache->pages, cache->page_size))
    return SPEC_ERR_INVALID_ARG;
  if (layer < 0 || layer >= cache->layers || !q || !pos_base || !page_table || !out) return SPEC_ERR_INVALID_ARG;
  if (!(scale > 0.0f) || isinf(scale) || window < 0 || sinks < 0) return SPEC_ERR_INVALID_ARG;
  const int64_t e = element_size(cache->dtype);
  if (((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(out)) & 15u) != 0 || q_row_stride * e % 16 != 0 ||
      q_row_stride < (int64_t)q_heads * cache->head_dim)
    return SPEC_ERR_INVALID_ARG;
  const AttendGeometry g = attend_geometry((K + 1) * (q_heads / cache->kv_heads), cache->head_dim, cache->dtype);
  if (!ws || ws_bytes < g.bytes || (reinterpret_cast<uintptr_t>(ws) & 255u) != 0) return SPEC_ERR_WORKSPACE;
  AttendLaunch a{};
  a.q = q;
  a.q_row = q_row_stride;
  a.k = static_cast<const char*>(cache->k) + layer * cache->layer_stride * e;
  a.v = static_cast<const char*>(cache->v) + layer * cache->layer_stride * e;
  a.page_b = cache->page_stride * e;
  a.token_b = cache->token_stride * e;
  a.head_b = cache->head_stride * e;
  a.pages = cache->pages;
  a.page_size = cache->page_size;
  a.max_pages = max_pages;
  a.Hq = q_heads;
  a.Hkv = cache->kv_heads;
  a.G = q_heads / cache->kv_heads;
  a.D = cache->head_dim;
  a.table = page_table;
  a.rows = RowLayout{row_offsets, depth, pos_base, B, K};
  a.c2 = (float)(1.4426950408889634 * (double)scale);
  // a window longer than the table hides nothing
  a.window = (long long)window > (long long)max_pages * cache->page_size ? 0 : window;
  a.sinks = sinks;
  a.out = out;
  a.lse = lse_out;
  a.status = status;
  char* base = static_cast<char*>(ws);
  a.arrived = reinterpret_cast<uint32_t*>(base);
  a.part = reinterpret_cast<float*>(base + g.part_off);
  a.part_stat = reinterpret_cast<float2*>(base + g.stat_off);
  const int sms = std::min(device_sms(), kAttendMaxSms);
  a.min_tiles = 1;
  a.lists = 1;
  cudaError_t err;
  if (attend_tc_serves(a.D, cache->dtype, a.page_size, a.head_b, a.token_b, a.page_b)) {
    a.ct = attend_tc_columns((K + 1) * a.G);
    a.ctas = sms * attend_tc_ctas_per_sm(a.D, a.ct);
    // a list per head, if that leaves no more than one CTA in sixteen idle
    if (a.ctas % a.Hkv <= a.ctas / 16) {
      a.lists = a.Hkv;
      a.ctas -= a.ctas % a.Hkv;
    }
    err = launch_attend_tc(a, stream);
  } else {
    a.ct = kGenCols;
    a.ctas = sms;
    err = cache->dtype == SPEC_F32 ? launch_general<float>(a, stream) : launch_general<__nv_bfloat16>(a, stream);
  }
  return err == cudaSuccess && cudaGetLastError() == cudaSuccess ? SPEC_OK : SPEC_ERR_CUDA;
}
