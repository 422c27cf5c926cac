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
// kernels (attend_tc.cu, attend_rows.cu) do not take.
#include <algorithm>

#include "attend.cuh"
#include "attend_tc.cuh"
#include "tensor_core.cuh"

namespace spec {

// ---------------------------------------------------------------------------
// The general kernel
// ---------------------------------------------------------------------------
constexpr int kGenThreads = 256;
constexpr int kGenCols = 32;   // columns per item
constexpr int kGenTile = 64;   // positions per tile
constexpr int kGenPitchS = kGenTile + 4;
constexpr int kGenQuarter = kGenCols / 4;  // columns of a thread's scores, and of a warp's softmax x 2

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

// C: columns of a thread's outputs (4 consecutive d of each).
//
// Scores: a token and eight columns per thread, from a K row of its own and Q
// rows that the warp shares (12 shared-memory wavefronts for 32 products a
// lane).  Weights: up to four columns per warp, the sums kept per lane.  Output:
// four d of C columns per thread.  Threads that few columns leave over split the
// sums: the scores' over d (the weights add their parts up), the output's over the
// tile's tokens (added up, in order, at the item's end).  The running time is that of
// shared memory and of the four barriers a tile, not of the cache's bytes; two
// CTAs share an SM where two fit.  Measured in fp32: 8 requests of 5 rows, 16 heads
// over 4, D = 64, 1,500 positions each 29 us (0.4 TB/s); 4 requests of 8 rows, 8
// heads over 2, 3,000 positions 30 us; one of 256 rows of 8 heads over 1, D = 128,
// 4,096 positions 218 us (19.7 TFLOP/s); 64 of one row, 32 heads over 8, 4,096
// positions 668 us (3.2 TB/s; 1,013 without the split sums, at 4 columns of 32).
// bf16, D = 96, 16 of one row, 16 heads over 4, 4,000 positions 74 us (without 108).
// Bringing the tiles by a bulk copy per row instead of 16-byte copies of all
// threads made it a quarter slower.
template <typename T, int C>
__global__ void __launch_bounds__(kGenThreads, C <= 2 ? 2 : 1) attend_general_kernel(const AttendLaunch a, int stages) {
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ Share share;
  __shared__ Segment seg;
  __shared__ ShareSums sums;
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
  find_share<kGenTile>(a, &share, &sums);
  Walk<kGenTile> walk(a, share);
  const int vecs = a.D * (int)sizeof(T) / 16;
  const int dv = a.D / 4;
  const int my_d = (tid % dv) * 4;

  for (;;) {
    if (tid == 0) more = walk.next(&seg) ? 1 : 0;
    __syncthreads();
    if (!more) break;
    const Segment s = seg;
    // scores: quarters of columns, and how many ways d is split; output: groups of C
    // columns, and how many ways the tokens are (a power of two)
    const int quarters = (s.cols + kGenQuarter - 1) / kGenQuarter, d_ways = 4 / quarters;
    const int part = tid / kGenTile / quarters, c0 = (tid / kGenTile - part * quarters) * kGenQuarter;
    const int groups = (s.cols + C - 1) / C;
    int t_ways = 1;
    while (t_ways < kGenTile / 4 && 2 * t_ways * groups <= kGenThreads / dv) t_ways *= 2;
    const int my_part = tid / dv / groups, my_c = (tid / dv - my_part * groups) * C;
    const bool pv_active = my_part < t_ways;
    const int p_first = s.p + group_row(a, s.col0), p_last = s.p + group_row(a, s.col0 + s.cols - 1);
    // four threads per token
    auto load_tile = [&](int x, int stage) {
      const int tok = tid >> 2, pos = place_position(s.tiles, x * kGenTile + tok);
      const bool wanted =
          pos <= p_last && (a.window == 0 || pos > p_first - a.window || pos < a.sinks);  // some row sees it
      int page = -1, in_page = 0;
      if (wanted) {
        const int slot = pos / a.page_size;
        in_page = pos - slot * a.page_size;
        page = __ldg(a.table + (size_t)s.request * a.max_pages + slot);
        if (page < 0 || page >= a.pages) {
          page = -1;
          if ((tid & 3) == 0) report(a.status, SPEC_ERR_BAD_INPUT);
        }
      }
      if ((tid & 3) == 0) sh_tok[stage][tok] = page >= 0 ? pos : -1;
      const int64_t off = (page >= 0 ? (int64_t)page * a.page_b + (int64_t)in_page * a.token_b : 0) + s.head * a.head_b;
      uint8_t* dk = sK + ((size_t)stage * kGenTile + tok) * pitch;
      uint8_t* dvv = sV + ((size_t)stage * kGenTile + tok) * pitch;
      for (int w = tid & 3; w < vecs; w += 4) {
        cp_async16(dk + w * 16, a.k + off + w * 16, page >= 0);
        cp_async16(dvv + w * 16, a.v + off + w * 16, page >= 0);
      }
      cp_async_commit();
    };
    load_tile(s.tile0, 0);
    if (tid == 0) walk.advance();
    // ---- Q, in fp32; unused columns zero ----
    for (int x = tid; x < kGenCols * dv; x += kGenThreads) {
      const int c = x / dv, d = (x - c * dv) * 4;
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      if (c < s.cols) {
        const int col = s.col0 + c, j = group_row(a, col);
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
    // columns warp, warp + 8, ..: the maximum (all lanes alike), a lane's part of the sum
    float m[4], l[4], acc[C][4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      m[k] = -INFINITY;
      l[k] = 0.0f;
    }
#pragma unroll
    for (int k = 0; k < C; ++k)
#pragma unroll
      for (int d = 0; d < 4; ++d) acc[k][d] = 0.0f;
    for (int x = 0; x < s.ntiles; ++x) {
      const int stage = stages == 2 ? x & 1 : 0;
      if (stages == 2 && x + 1 < s.ntiles) {
        load_tile(s.tile0 + x + 1, stage ^ 1);
        cp_async_wait<1>();
      } else {
        cp_async_wait<0>();
      }
      __syncthreads();
      // ---- scores ----
      bool masked = false;
      {
        const int tok = tid & (kGenTile - 1);
        const int pos = sh_tok[stage][tok];
        if (part < d_ways) {
          const T* kr = reinterpret_cast<const T*>(sK + ((size_t)stage * kGenTile + tok) * pitch);
          float dot[kGenQuarter];
#pragma unroll
          for (int c = 0; c < kGenQuarter; ++c) dot[c] = 0.0f;
          auto add = [&](int first, int step) {
#pragma unroll 2
            for (int d = first; d < a.D; d += step) {
              const float4 k4 = load4(kr + d);
#pragma unroll
              for (int c = 0; c < kGenQuarter; ++c) {
                const float4 q4 = load4(sQ + (c0 + c) * a.D + d);
                dot[c] = fmaf(k4.x, q4.x, dot[c]);
                dot[c] = fmaf(k4.y, q4.y, dot[c]);
                dot[c] = fmaf(k4.z, q4.z, dot[c]);
                dot[c] = fmaf(k4.w, q4.w, dot[c]);
              }
            }
          };
          if (d_ways == 1) add(0, 4);  // apart, for its addresses without arithmetic
          else add(4 * part, 4 * d_ways);
#pragma unroll
          for (int c = 0; c < kGenQuarter; ++c) {
            const int row = s.p + group_row(a, s.col0 + min(c0 + c, s.cols - 1));
            const bool seen = pos >= 0 && pos <= row && (a.window == 0 || pos > row - a.window || pos < a.sinks);
            masked |= !seen;
            sS[(part * quarters * kGenQuarter + c0 + c) * kGenPitchS + tok] = seen ? dot[c] * a.c2 : -INFINITY;
          }
        }
      }
      const bool edge = __syncthreads_or(masked);
      // ---- weights ----
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int c = warp + kGenThreads / 32 * k;
        if (c >= s.cols) break;
        float* row = sS + c * kGenPitchS;
        float x0 = row[lane], x1 = row[lane + 32];
        for (int y = 1; y < d_ways; ++y) {
          const float* more_d = row + y * quarters * kGenQuarter * kGenPitchS;
          x0 += more_d[lane];
          x1 += more_d[lane + 32];
        }
        const float mn = fmaxf(m[k], warp_max(fmaxf(x0, x1)));
        const float alpha = m[k] == -INFINITY ? 0.0f : exp2f(m[k] - mn);
        // a masked score is -inf and weighs 0; a NaN score stays NaN
        const float p0 = x0 == -INFINITY ? 0.0f : exp2f(x0 - mn), p1 = x1 == -INFINITY ? 0.0f : exp2f(x1 - mn);
        row[lane] = p0;
        row[lane + 32] = p1;
        l[k] = fmaf(l[k], alpha, p0 + p1);
        m[k] = mn;
        if (lane == 0) sh_alpha[c] = alpha;
      }
      __syncthreads();
      // ---- output ----
      if (pv_active) {
#pragma unroll
        for (int k = 0; k < C; ++k) {
          const float alpha = sh_alpha[min(my_c + k, s.cols - 1)];
#pragma unroll
          for (int d = 0; d < 4; ++d) acc[k][d] *= alpha;
        }
        const uint8_t* vr = sV + (size_t)stage * kGenTile * pitch + my_d * sizeof(T);
        const float* wr = sS + my_c * kGenPitchS;
        auto add = [&](int begin, int end) {
#pragma unroll 2
          for (int tok = begin; tok < end; tok += 4) {
            float4 v4[4];
#pragma unroll
            for (int y = 0; y < 4; ++y) v4[y] = load4(reinterpret_cast<const T*>(vr + (size_t)(tok + y) * pitch));
#pragma unroll
            for (int k = 0; k < C; ++k) {
              // (columns past the item's hold old weights: their sums are not written)
              const float4 w4 = load4(wr + k * kGenPitchS + tok);
              const float w[4] = {w4.x, w4.y, w4.z, w4.w};
#pragma unroll
              for (int y = 0; y < 4; ++y) {
                if (edge && w[y] == 0.0f) continue;  // what a masked token holds does not reach the sum
                acc[k][0] = fmaf(w[y], v4[y].x, acc[k][0]);
                acc[k][1] = fmaf(w[y], v4[y].y, acc[k][1]);
                acc[k][2] = fmaf(w[y], v4[y].z, acc[k][2]);
                acc[k][3] = fmaf(w[y], v4[y].w, acc[k][3]);
              }
            }
          }
        };
        if (t_ways == 1) add(0, kGenTile);
        else add(my_part * (kGenTile / t_ways), (my_part + 1) * (kGenTile / t_ways));
      }
      __syncthreads();
      if (stages == 1 && x + 1 < s.ntiles) load_tile(s.tile0 + x + 1, 0);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int c = warp + kGenThreads / 32 * k;
      if (c >= s.cols) break;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) l[k] += __shfl_xor_sync(0xFFFFFFFFu, l[k], o);
      if (lane == 0) {
        sh_l[c] = l[k];
        sh_m[c] = m[k];
      }
    }
    if (t_ways > 1) {  // the tokens' parts of the output, through the tiles' place
      float4* sums_at = reinterpret_cast<float4*>(smem);
      if (pv_active && my_part > 0) {
#pragma unroll
        for (int k = 0; k < C; ++k)
          sums_at[((my_part - 1) * groups * C + my_c + k) * dv + my_d / 4] =
              make_float4(acc[k][0], acc[k][1], acc[k][2], acc[k][3]);
      }
      __syncthreads();
      if (my_part == 0) {
        for (int y = 0; y < t_ways - 1; ++y) {
#pragma unroll
          for (int k = 0; k < C; ++k) {
            const float4 w = sums_at[(y * groups * C + my_c + k) * dv + my_d / 4];
            acc[k][0] += w.x;
            acc[k][1] += w.y;
            acc[k][2] += w.z;
            acc[k][3] += w.w;
          }
        }
      }
    }
    __syncthreads();
    // ---- the item's result, or this part's ----
    if (my_part == 0) {
#pragma unroll
      for (int k = 0; k < C; ++k) {
        const int c = my_c + k;
        if (c >= s.cols) break;
        if (s.slot < 0) {
          const float inv = sh_l[c] == 0.0f ? 0.0f : 1.0f / sh_l[c];
          store4(static_cast<T*>(a.out) + out_index(a, s, c) * a.D + my_d,
                 make_float4(acc[k][0] * inv, acc[k][1] * inv, acc[k][2] * inv, acc[k][3] * inv));
        } else {
          *reinterpret_cast<float4*>(a.part + ((size_t)s.slot * a.ct + c) * a.D + my_d) =
              make_float4(acc[k][0], acc[k][1], acc[k][2], acc[k][3]);
        }
      }
    }
    if (tid < s.cols) {
      if (s.slot < 0) {
        if (a.lse) a.lse[out_index(a, s, tid)] = row_lse(sh_m[tid], sh_l[tid]);
      } else {
        // scores that are all NaN leave no maximum, but a sum: a part that saw something has a finite one
        a.part_stat[(size_t)s.slot * a.ct + tid] =
            make_float2(sh_l[tid] == 0.0f ? sh_m[tid] : fmaxf(sh_m[tid], kNoMax), sh_l[tid]);
      }
    }
    if (s.slot >= 0) {
      __syncthreads();
      if (tid == 0) last = arrive_part(a, s) ? 1 : 0;
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
// The general kernel's CTAs per SM (228 KB, 1 KB of it reserved per CTA and some
// for its static arrays).
static int general_ctas_per_sm(int D, int dtype) {
  return D <= 64 && general_smem(D, element_size(dtype), 2) <= 112 * 1024 ? 2 : 1;
}

struct AttendGeometry {
  size_t part_off, stat_off, bytes;
};

// Room for the parts (two per CTA) of whichever kernel serves the shape: which one
// does depends on the cache's pages and strides too.  The counters come first, as
// many for every shape: a workspace may serve several in turn.
static AttendGeometry attend_geometry(int cols, int D, int dtype) {
  size_t columns = (size_t)2 * kAttendMaxSms * general_ctas_per_sm(D, dtype) * kGenCols;
  if (attend_tc_may_serve(D, dtype)) {
    const int ct = attend_tc_columns(cols);
    columns = std::max(columns, (size_t)2 * kAttendMaxSms * attend_tc_ctas_per_sm(D, ct) * ct);
  }
  AttendGeometry g{};
  g.part_off = (2 * kAttendMaxSms * 4 + 255) / 256 * 256;
  g.stat_off = g.part_off + (columns * D * 4 + 255) / 256 * 256;
  g.bytes = g.stat_off + (columns * 8 + 255) / 256 * 256;
  return g;
}

static bool attend_shape_ok(int B, int K, int q_heads, int kv_heads, int D, int dtype) {
  return rows_shape_ok(B, K) && kv_heads >= 1 && q_heads >= kv_heads && q_heads % kv_heads == 0 &&
         q_heads / kv_heads <= SPEC_MAX_GROUP && D >= 1 && D <= SPEC_MAX_HEAD_DIM &&
         (dtype == SPEC_BF16 || dtype == SPEC_F32) && D * element_size(dtype) % 16 == 0;
}

template <typename T, int C>
static cudaError_t launch_general(const AttendLaunch& a, cudaStream_t stream) {
  const int esize = (int)sizeof(T);
  const int stages = general_smem(a.D, esize, 2) <= 220 * 1024 ? 2 : 1;  // two where they fit
  const size_t smem = general_smem(a.D, esize, stages);
  static std::atomic<size_t> raised[kMaxDevices];
  const cudaError_t err = raise_smem(attend_general_kernel<T, C>, smem, raised);
  if (err != cudaSuccess) return err;
  return launch_after_previous(attend_general_kernel<T, C>, dim3(a.ctas), dim3(kGenThreads), smem, stream, a, stages);
}

// A thread's columns: kGenThreads / (D / 4) threads share the item's.
template <typename T>
static cudaError_t launch_general(const AttendLaunch& a, cudaStream_t stream) {
  return a.D <= 64 ? launch_general<T, 2>(a, stream)
                   : a.D <= 128 ? launch_general<T, 4>(a, stream) : launch_general<T, 8>(a, stream);
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
  a.g_inverse = (uint32_t)(((1ull << 32) + a.G - 1) / a.G);
  a.D = cache->head_dim;
  a.table = page_table;
  a.rows = RowLayout{row_offsets, depth, pos_base, B, K};
  a.c2 = (float)(1.4426950408889634 * (double)scale);
  // a window longer than the table hides nothing, and sinks end with the table
  const int table_end = max_pages * cache->page_size;
  a.window = window > table_end ? 0 : window;
  a.sinks = std::min(sinks, table_end);
  a.out = out;
  a.lse = lse_out;
  a.status = status;
  char* base = static_cast<char*>(ws);
  a.arrived = reinterpret_cast<uint32_t*>(base);
  a.part = reinterpret_cast<float*>(base + g.part_off);
  a.part_stat = reinterpret_cast<float2*>(base + g.stat_off);
  const int sms = std::min(device_sms(), kAttendMaxSms);
  const bool tc = attend_tc_serves(a.D, cache->dtype, a.page_size, a.head_b, a.token_b, a.page_b);
  a.ct = tc ? attend_tc_columns((K + 1) * a.G) : kGenCols;
  a.ctas = sms * (tc ? attend_tc_ctas_per_sm(a.D, a.ct) : general_ctas_per_sm(a.D, cache->dtype));
  a.grain = tc ? attend_tc_grain(a.page_size) : 1;
  // a list per head, if that leaves no more than one CTA in sixteen idle: 64
  // requests of 64 heads over 8, D = 128, 4,096 positions, lists / one list, us: a
  // token 166 / 171, 8 rows 181 / 191, 17 rows 250 / 295, 32 rows 335 / 385
  a.lists = 1;
  if (a.ctas % a.Hkv <= a.ctas / 16) {
    a.lists = a.Hkv;
    a.ctas -= a.ctas % a.Hkv;
  }
  // What dividing the items costs, in tiles of the kernel (a tile takes 1 to 2 us): a
  // part's writing and its share of the join grow with the columns.  Measured with
  // these rules / without them, us: a token of 8 heads over 1, 16,384 positions, D =
  // 128: 22 / 37; 17 rows of it, 8,192: 45 / 111; 32 rows, 16,384: 60 / 265; 8
  // requests of 17 rows, 64 heads over 8, 1,024: 31 / 47; 4 of 256 rows, 32 over 8,
  // 4,096: 94 / 100; in fp32, 4 of 8 rows, 8 over 2, D = 64, 3,000: 31 / 35.
  a.part_cost = tc ? 4 : 2;
  a.item_cost = tc ? 4 : 1;
  a.part_tiles = (tc ? 200.0f : 400.0f) / (float)(tc ? a.ct : std::min(a.ct, (K + 1) * a.G));
  const cudaError_t err = tc                              ? launch_attend_tc(a, stream)
                          : cache->dtype == SPEC_F32      ? launch_general<float>(a, stream)
                                                          : launch_general<__nv_bfloat16>(a, stream);
  return err == cudaSuccess && cudaGetLastError() == cudaSuccess ? SPEC_OK : SPEC_ERR_CUDA;
}
