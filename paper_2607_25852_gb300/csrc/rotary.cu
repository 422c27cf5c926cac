// rotary.cu -- rotary positions: the rows' queries and keys turned by the angles
// of their positions, the keys and the values straight into their pages.
//
// Element pair d of a head, (a, b), at position P becomes
//   amplitude (a cos t - b sin t, b cos t + a sin t),  t = P f_d.
// The angle is needed modulo a turn only, so f_d / 2 pi is rounded once to a
// multiple of 2^-64 turns and multiplied by P in 64-bit integers: what overflows
// is whole turns, and the product is exact (a position of 2^20 in fp32 loses the
// angle's last 17 bits, and fp64 arithmetic is slow here).  cos and sin are then
// CUDA's sincospif of the angle in half turns.
//
// A CTA takes up to 8 rows: a thread each finds their places, all compute their
// angles, and then a thread has the same elements of every few heads, row after
// row, with their angles in registers.  (A row per CTA spent 700 instructions per
// warp on three vectors: 16 chunks of 256 rows, 100 MB, 43 us; now 25.8, 3.9 TB/s.)
// Bound by the issue of loads and stores and the HBM for many rows, by three round
// trips (position, page, data) and the launch for few: one row 3.8 us, 1,088 rows of
// 32 + 8 heads of 128 8.9.
#include <algorithm>
#include <cmath>

#include "paged.cuh"
#include "tensor_core.cuh"

namespace spec {

namespace {

constexpr int kRotaryThreads = 256;
constexpr int kRotaryRows = 8;  // of a CTA, at most

struct RotaryLaunch {
  const char *x, *k_new, *v_new;  // k_new, v_new null without a cache
  char *out, *k, *v;              // k and v of the layer
  int64_t x_row, out_row, k_row, v_row;  // bytes between rows
  int64_t page_b, token_b, head_b;
  int heads, kv_heads, D;
  int pairs;                      // rotary_dim / 2
  int batch;                      // rows of a CTA
  int pages, page_size, max_pages;
  bool in_place;                  // out is x: what is not turned stays
  float amplitude;
  const double* frequencies;
  const int32_t* table;
  RowLayout rows;
  int32_t* status;
};

// W elements as one load or store.
template <typename T, int W>
struct alignas(sizeof(T) * W) Pack {
  T e[W];
};
template <typename T, int W>
__device__ __forceinline__ Pack<T, W> load_pack(const char* p) {
  return *reinterpret_cast<const Pack<T, W>*>(p);
}
template <typename T, int W>
__device__ __forceinline__ void store_pack(char* p, const Pack<T, W>& v) {
  *reinterpret_cast<Pack<T, W>*>(p) = v;
}
__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void from_float(float x, float* to) { *to = x; }
__device__ __forceinline__ void from_float(float x, __nv_bfloat16* to) { *to = __float2bfloat16_rn(x); }

// Cosine and sine, times the amplitude, of position P's turn of a pair.
__device__ __forceinline__ float2 turn(double frequency, int64_t P, float amplitude, int32_t* status) {
  double turns = frequency * 0.15915494309189533577;  // 1 / (2 pi)
  turns -= rint(turns);
  if (!(fabs(turns) <= 0.5)) {  // not finite
    report(status, SPEC_ERR_BAD_INPUT);
    turns = 0.0;
  }
  const int64_t step = __double2ll_rn(turns * 18446744073709551616.0);  // half a turn saturates, 2^-64 off
  const int64_t phase = (int64_t)((uint64_t)P * (uint64_t)step);
  float s, c;
  sincospif((float)phase * 1.0842021724855044e-19f, &s, &c);  // 2^-63: in half turns
  return make_float2(amplitude * c, amplitude * s);
}

struct RowPlace {
  int64_t row, pos;  // row -1: skipped
  int64_t at;        // the key's and value's bytes into the layer; -1: nowhere
};

__device__ __forceinline__ RowPlace row_place(const RotaryLaunch& p, unsigned r) {
  const unsigned K1 = (unsigned)p.rows.K + 1;
  RowPlace t{-1, 0, -1};
  if (r >= (unsigned)p.rows.B * K1) return t;
  const int i = (int)(r / K1), j = (int)(r - (unsigned)i * K1);
  const RequestRows q = request_rows(p.rows, i);
  if (!q.ok) {
    if (j == 0) report(p.status, SPEC_ERR_BAD_INPUT);
    return t;
  }
  t.pos = q.p + j;
  if (j >= q.count || t.pos < 0) return t;
  if (t.pos >> 32) {
    report(p.status, SPEC_ERR_BAD_INPUT);
    return t;
  }
  t.row = q.row0 + j;
  if (!p.k_new) return t;
  int page = -1, slot = 0;
  if (t.pos < (int64_t)p.max_pages * p.page_size) {
    slot = (int)t.pos / p.page_size;
    page = __ldg(p.table + (size_t)i * p.max_pages + slot);
  }
  if (page >= 0 && page < p.pages)
    t.at = (int64_t)page * p.page_b + (int64_t)((int)t.pos - slot * p.page_size) * p.token_b;
  else
    report(p.status, SPEC_ERR_BAD_INPUT);
  return t;
}

// kInter: neighbouring elements are a pair, and a unit is one pack of W
// elements.  Otherwise elements d and d + pairs are, and a unit is two packs of W
// elements, one of each half (W divides the half), or one of those that stay.
template <typename T, int W, bool kInter>
__global__ void __launch_bounds__(kRotaryThreads, 4) rotary_kernel(const RotaryLaunch p) {
  constexpr int E = (int)sizeof(T), kU = kInter ? 3 : W * (int)sizeof(T) == 16 ? 1 : 2;  // heads in flight
  constexpr int kPairs = kInter ? (W + 1) / 2 : W;
  __shared__ alignas(16) float cs[kRotaryRows][SPEC_MAX_HEAD_DIM / 2], sn[kRotaryRows][SPEC_MAX_HEAD_DIM / 2];
  __shared__ RowPlace places[kRotaryRows];
  const int tid = threadIdx.x;
  pdl_wait_prerequisites();
  pdl_launch_dependents();
  if (tid < p.batch) places[tid] = row_place(p, blockIdx.x * (unsigned)p.batch + tid);
  // ---- a thread has unit u of every hstep-th head ----
  const int turned = kInter ? (2 * p.pairs + W - 1) / W : p.pairs / W;  // a head's units with turned elements
  const int units = kInter ? p.D / W : turned + (p.D - 2 * p.pairs) / W;
  const int hstep = kRotaryThreads / units, h0 = tid / units, u = tid - h0 * units;
  const int heads = h0 < hstep ? p.heads + (p.k_new ? p.kv_heads : 0) : 0;
  const bool turns = u < turned;
  const int at0 = (kInter || turns ? u * W : 2 * p.pairs + (u - turned) * W) * E;  // within a head
  const int at1 = (p.pairs + u * W) * E, head = p.D * E;
  const int vecs = head / 16, vstep = kRotaryThreads / vecs, v0 = tid / vecs, vu = (tid - v0 * vecs) * 16;
  const int values = p.k_new && v0 < vstep ? p.kv_heads : 0;
  __syncthreads();
  for (int x = tid; x < p.batch * p.pairs; x += kRotaryThreads) {
    const int y = x / p.pairs, d = x - y * p.pairs;
    if (places[y].row < 0) continue;
    const float2 t = turn(__ldg(p.frequencies + d), places[y].pos, p.amplitude, p.status);
    cs[y][d] = t.x;
    sn[y][d] = t.y;
  }
  __syncthreads();
#pragma unroll 1
  for (int y = 0; y < p.batch; ++y) {
    const int64_t row = places[y].row, at = places[y].at;
    if (row < 0) continue;
    const char *x = p.x + row * p.x_row, *k_from = p.k_new + row * p.k_row, *v_from = p.v_new + row * p.v_row;
    char *out = p.out + row * p.out_row, *k_to = p.k + at, *v_to = p.v + at;
    Pack<T, W> a[kU], b[kU];
    auto load = [&](int h, Pack<T, W>& a, Pack<T, W>& b) {
      const char* from = h < p.heads ? x + h * head : k_from + (h - p.heads) * head;
      a = load_pack<T, W>(from + at0);
      if (!kInter && turns) b = load_pack<T, W>(from + at1);
    };
#pragma unroll
    for (int z = 0; z < kU; ++z)
      if (h0 + z * hstep < heads) load(h0 + z * hstep, a[z], b[z]);
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    if (v0 < values) v = ldg_stream(v_from + v0 * head + vu);
    float c[kPairs], s[kPairs];
#pragma unroll
    for (int e = 0; e < kPairs; ++e) c[e] = cs[y][(u * kPairs + e) & (SPEC_MAX_HEAD_DIM / 2 - 1)], s[e] = sn[y][(u * kPairs + e) & (SPEC_MAX_HEAD_DIM / 2 - 1)];
#pragma unroll 1
    for (int h = h0; h < heads; h += kU * hstep) {
#pragma unroll
      for (int z = 0; z < kU; ++z) {
        const int w = h + z * hstep;
        if (w >= heads) break;
        if (w >= p.heads && at < 0) break;
        char* to = w < p.heads ? out + w * head : k_to + (w - p.heads) * p.head_b;
        if (!turns) {
          if (!(p.in_place && w < p.heads)) store_pack<T, W>(to + at0, a[z]);
        } else {
#pragma unroll
          for (int e = 0; e < kPairs; ++e) {
            if (kInter && u * kPairs + e >= p.pairs) break;  // the rest of this pack stays
            T *f = &a[z].e[kInter ? 2 * e % W : e], *g = kInter ? &a[z].e[(2 * e + 1) % W] : &b[z].e[e];
            const float f0 = to_float(*f), g0 = to_float(*g);
            from_float(fmaf(f0, c[e], -g0 * s[e]), f);
            from_float(fmaf(g0, c[e], f0 * s[e]), g);
          }
          store_pack<T, W>(to + at0, a[z]);
          if (!kInter) store_pack<T, W>(to + at1, b[z]);
        }
        if (w + kU * hstep < heads) load(w + kU * hstep, a[z], b[z]);
      }
    }
    if (at < 0) continue;
    for (int h = v0; h < values; h += vstep) {
      if (h > v0) v = ldg_stream(v_from + h * head + vu);
      *reinterpret_cast<uint4*>(v_to + h * p.head_b + vu) = v;
    }
  }
}

template <typename T>
cudaError_t launch_rotary(const RotaryLaunch& p, bool interleaved, cudaStream_t stream) {
  const long long rows = (long long)p.rows.B * (p.rows.K + 1);
  const dim3 grid((unsigned)((rows + p.batch - 1) / p.batch)), block(kRotaryThreads);
  constexpr int W = 16 / (int)sizeof(T);
  if (interleaved) return launch_after_previous(rotary_kernel<T, W, true>, grid, block, 0, stream, p);
  // The widest packs that divide the half that is turned, as its two halves lie that far apart; 4,096 rows of 12 + 12
  // heads of 96 in fp32, all turned, take 26 us with four elements a pack.
  if (p.pairs % W == 0) return launch_after_previous(rotary_kernel<T, W, false>, grid, block, 0, stream, p);
  if (p.pairs % (W / 2) == 0) return launch_after_previous(rotary_kernel<T, W / 2, false>, grid, block, 0, stream, p);
  if (p.pairs % 2 == 0) return launch_after_previous(rotary_kernel<T, 2, false>, grid, block, 0, stream, p);
  return launch_after_previous(rotary_kernel<T, 1, false>, grid, block, 0, stream, p);
}

bool rows_ok(const void* p, int64_t stride, int heads, int head_dim, int64_t e) {
  return p && (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && stride * e % 16 == 0 &&
         stride >= (int64_t)heads * head_dim && stride <= (INT64_MAX >> 32);
}

bool rotation_ok(const double* frequencies, int rotary_dim, int head_dim, float amplitude) {
  return frequencies && rotary_dim >= 2 && rotary_dim % 2 == 0 && rotary_dim <= head_dim && std::isfinite(amplitude);
}

int run_rotary(RotaryLaunch& p, int dtype, int interleaved, cudaStream_t stream) {
  // A row per CTA up to 12 rows per SM, eight from 48 per SM on: the tables of a CTA are worth their time where the rows
  // are many.  Rows of 32 + 8 heads of 128, one per CTA / this / eight: 512 5.2 / 5.1 / 12.8 us, 2,048 14.9 / 12.4 /
  // 15.7, 4,096 28.2 / 23.5 / 26.4, 16,384 113 / 98 / 98.
  p.batch = (int)std::min<long long>(kRotaryRows, std::max<long long>(1, (long long)p.rows.B * (p.rows.K + 1) / (6 * device_sms())));
  const cudaError_t err = dtype == SPEC_F32 ? launch_rotary<float>(p, interleaved != 0, stream)
                                            : launch_rotary<__nv_bfloat16>(p, interleaved != 0, stream);
  return err == cudaSuccess && cudaGetLastError() == cudaSuccess ? SPEC_OK : SPEC_ERR_CUDA;
}

}  // namespace

}  // namespace spec

extern "C" int spec_rotary_frequencies(int rotary_dim, double base, int scaling, double factor,
                                       int64_t original_positions, double low, double high, double* out) {
  using std::isfinite;
  if (rotary_dim < 2 || rotary_dim % 2 != 0 || rotary_dim > SPEC_MAX_HEAD_DIM || !(base > 1.0) || !isfinite(base) || !out)
    return SPEC_ERR_INVALID_ARG;
  if (scaling < SPEC_ROTARY_PLAIN || scaling > SPEC_ROTARY_RAMP) return SPEC_ERR_INVALID_ARG;
  if (scaling != SPEC_ROTARY_PLAIN && (!(factor >= 1.0) || !isfinite(factor))) return SPEC_ERR_INVALID_ARG;
  if (scaling == SPEC_ROTARY_BASE && rotary_dim < 4) return SPEC_ERR_INVALID_ARG;
  if (scaling == SPEC_ROTARY_RAMP && (original_positions < 1 || !(low > 0.0) || !(high > low) || !isfinite(high)))
    return SPEC_ERR_INVALID_ARG;
  if (scaling == SPEC_ROTARY_BASE) base *= std::pow(factor, (double)rotary_dim / (rotary_dim - 2));
  for (int d = 0; d < rotary_dim / 2; ++d) {
    double f = std::pow(base, -2.0 * d / rotary_dim);
    if (scaling == SPEC_ROTARY_LINEAR) f /= factor;
    if (scaling == SPEC_ROTARY_RAMP) {
      const double turns = (double)original_positions * f / 6.283185307179586477;
      const double keep = std::fmin(1.0, std::fmax(0.0, (turns - low) / (high - low)));
      f = f * keep + f / factor * (1.0 - keep);
    }
    out[d] = f;
  }
  return SPEC_OK;
}

extern "C" int spec_rotary(const void* x, int64_t x_row_stride, int heads, int head_dim, int dtype,
                           const double* frequencies, int rotary_dim, int interleaved, float amplitude,
                           const int32_t* row_offsets, const int32_t* depth, const int64_t* pos_base, int B, int K,
                           void* out, int64_t out_row_stride, int32_t* status, cudaStream_t stream) {
  spec::NvtxRange range("spec_rotary");
  using namespace spec;
  if (!rows_shape_ok(B, K) || (dtype != SPEC_BF16 && dtype != SPEC_F32) || heads < 1 || heads > (1 << 16) ||
      head_dim < 1 || head_dim > SPEC_MAX_HEAD_DIM || head_dim * element_size(dtype) % 16 != 0)
    return SPEC_ERR_INVALID_ARG;
  const int64_t e = element_size(dtype);
  if (!rotation_ok(frequencies, rotary_dim, head_dim, amplitude) || !pos_base ||
      !rows_ok(x, x_row_stride, heads, head_dim, e) || !rows_ok(out, out_row_stride, heads, head_dim, e))
    return SPEC_ERR_INVALID_ARG;
  if (out == x && out_row_stride != x_row_stride) return SPEC_ERR_INVALID_ARG;
  RotaryLaunch p{};
  p.x = static_cast<const char*>(x);
  p.out = static_cast<char*>(out);
  p.x_row = x_row_stride * e;
  p.out_row = out_row_stride * e;
  p.heads = heads;
  p.D = head_dim;
  p.pairs = rotary_dim / 2;
  p.in_place = out == x;
  p.amplitude = amplitude;
  p.frequencies = frequencies;
  p.rows = RowLayout{row_offsets, depth, pos_base, B, K};
  p.status = status;
  return run_rotary(p, dtype, interleaved, stream);
}

extern "C" int spec_rotary_append(const spec_cache* cache, int layer, const void* q, int64_t q_row_stride, int q_heads,
                                  const void* k_new, int64_t k_row_stride, const void* v_new, int64_t v_row_stride,
                                  const double* frequencies, int rotary_dim, int interleaved, float amplitude,
                                  const int32_t* row_offsets, const int32_t* depth, const int64_t* pos_base,
                                  const int32_t* page_table, int max_pages, int B, int K, void* q_out,
                                  int64_t q_out_row_stride, int32_t* status, cudaStream_t stream) {
  spec::NvtxRange range("spec_rotary_append");
  using namespace spec;
  if (!cache_ok(cache) || layer < 0 || layer >= cache->layers || !rows_shape_ok(B, K) ||
      !table_shape_ok(B, max_pages, cache->pages, cache->page_size) || cache->kv_heads > (1 << 16))
    return SPEC_ERR_INVALID_ARG;
  const int64_t e = element_size(cache->dtype);
  const int D = cache->head_dim;
  if (!rotation_ok(frequencies, rotary_dim, D, amplitude) || !pos_base || !page_table ||
      !rows_ok(k_new, k_row_stride, cache->kv_heads, D, e) || !rows_ok(v_new, v_row_stride, cache->kv_heads, D, e))
    return SPEC_ERR_INVALID_ARG;
  if (q_heads < 0 || q_heads > (1 << 16) || (q_heads == 0) != (q == nullptr) || (q_heads == 0) != (q_out == nullptr))
    return SPEC_ERR_INVALID_ARG;
  if (q_heads && (!rows_ok(q, q_row_stride, q_heads, D, e) || !rows_ok(q_out, q_out_row_stride, q_heads, D, e) ||
                  (q == q_out && q_row_stride != q_out_row_stride)))
    return SPEC_ERR_INVALID_ARG;
  RotaryLaunch p{};
  p.x = static_cast<const char*>(q);
  p.out = static_cast<char*>(q_out);
  p.x_row = q_row_stride * e;
  p.out_row = q_out_row_stride * e;
  p.k_new = static_cast<const char*>(k_new);
  p.v_new = static_cast<const char*>(v_new);
  p.k_row = k_row_stride * e;
  p.v_row = v_row_stride * e;
  p.k = static_cast<char*>(cache->k) + layer * cache->layer_stride * e;
  p.v = static_cast<char*>(cache->v) + layer * cache->layer_stride * e;
  p.page_b = cache->page_stride * e;
  p.token_b = cache->token_stride * e;
  p.head_b = cache->head_stride * e;
  p.heads = q_heads;
  p.kv_heads = cache->kv_heads;
  p.D = D;
  p.pairs = rotary_dim / 2;
  p.pages = cache->pages;
  p.page_size = cache->page_size;
  p.max_pages = max_pages;
  p.in_place = q == q_out;
  p.amplitude = amplitude;
  p.frequencies = frequencies;
  p.table = page_table;
  p.rows = RowLayout{row_offsets, depth, pos_base, B, K};
  p.status = status;
  return run_rotary(p, cache->dtype, interleaved, stream);
}
