// What spec_attend's CTAs share out, without the attention: each block finds its
// share, lists its segments and arrives for its parts, those from `stop` on by
// arrive_for_rest, as a CTA does whose wait gave up.  For test_gpu_attend_shares.py.
#include "attend.cuh"

namespace {

struct Listed {
  int32_t request, head, col0, cols, tile0, ntiles, count, slot, first_cta, step, parts, cta;
};

template <int TT>
__global__ void shares_kernel(const spec::AttendLaunch a, const int32_t* stop, Listed* out, int most, int32_t* total) {
  using namespace spec;
  __shared__ Share share;
  __shared__ ShareSums sums;
  find_share<TT>(a, &share, &sums);
  if (threadIdx.x != 0) return;
  const int done = stop[blockIdx.x];
  Walk<TT> walk(a, share);
  Segment s;
  for (int n = 0; walk.next(&s); ++n) {
    const int at = atomicAdd(total, 1);
    if (at < most)
      out[at] = Listed{s.request, s.head, s.col0, s.cols, s.tile0, s.ntiles, s.tiles.count, s.slot, s.first_cta, s.step,
                       s.parts, (int)blockIdx.x};
    if (n < done && s.slot >= 0) arrive_part(a, s);
    walk.advance();
  }
  arrive_for_rest<TT>(a, share, done);
}

}  // namespace

extern "C" int attend_shares(int tile, int threads, int G, int Hkv, int page_size, int max_pages, int B, int K, int window,
                             int sinks, int grain, int ct, int ctas, int lists, int part_cost, int item_cost,
                             float part_tiles, const int32_t* row_offsets, const int32_t* depth, const int64_t* pos,
                             uint32_t* arrived, const int32_t* stop, void* out, int most, int32_t* total,
                             int32_t* status) {
  using namespace spec;
  AttendLaunch a{};
  a.page_size = page_size;
  a.max_pages = max_pages;
  a.Hq = Hkv * G;
  a.Hkv = Hkv;
  a.G = G;
  a.g_inverse = (uint32_t)(((1ull << 32) + G - 1) / G);
  a.rows = RowLayout{row_offsets, depth, pos, B, K};
  a.window = window;
  a.sinks = sinks;
  a.grain = grain;
  a.status = status;
  a.ct = ct;
  a.arrived = arrived;
  a.ctas = ctas;
  a.lists = lists;
  a.part_cost = part_cost;
  a.item_cost = item_cost;
  a.part_tiles = part_tiles;
  if (tile == 64) shares_kernel<64><<<ctas, threads>>>(a, stop, static_cast<Listed*>(out), most, total);
  else shares_kernel<128><<<ctas, threads>>>(a, stop, static_cast<Listed*>(out), most, total);
  return (int)cudaGetLastError();
}
