// Attention over paged 4-bit rows under masks: a new row sees all rows ahead of its request's new ones, and those of the new ones that its
// mask names (a tree of drafted tokens).  The kernels of pages_attn_tile.h.
#include "pages_attn_tile.h"

namespace lococo {
namespace {

using namespace pages_detail;

template <typename T>
__global__ __launch_bounds__(kRowsThreads) void pages_tree_rows_k(PagesAttnArgs a, TreeMasks tm) {
  attn_rows<T, true>(a, tm);
}
template <typename T, int D, int QB>
__global__ __launch_bounds__(64 * kTileWaves, 2) void pages_tree_tile_k(TileArgs g, TreeMasks tm) {
  attn_tile<T, D, QB, true>(g, tm);
}
template <typename T, int D, int TR, int WAVES>
__global__ __launch_bounds__(256) void pages_tree_join_k(TileArgs g, int32_t rows) {
  attn_join<T, D, TR, WAVES, true>(g, rows);
}

template <typename T, int D, int TR>
hipError_t launch_tile(const TileArgs& g, const TreeMasks& tm, const TilePlan& p, hipStream_t s) {
  const unsigned join = (unsigned)join_groups(p, g.a.pg.Hkv);
  pages_tree_tile_k<T, D, TR / 16><<<(unsigned)tile_groups(p, g.a.pg.Hkv), kTileThreads, 0, s>>>(g, tm);
  if (join) {
    if (p.splits > 16) pages_tree_join_k<T, D, TR, 4><<<join, kJoinThreads, 0, s>>>(g, p.rows);
    else pages_tree_join_k<T, D, TR, 1><<<join, kJoinThreads, 0, s>>>(g, p.rows);
  }
  return hipGetLastError();
}
template <typename T, int D>
hipError_t launch_tiles(const TileArgs& g, const TreeMasks& tm, const TilePlan& p, hipStream_t s) {
  if constexpr (!std::is_same<T, float>::value) {
    if (p.tr == 32) return launch_tile<T, D, 32>(g, tm, p, s);
  }
  return launch_tile<T, D, 16>(g, tm, p, s);
}

}  // namespace

hipError_t launch_pages_attn_tree(int dtype, const PagesAttnArgs& a, const uint32_t* masks, int32_t words, void* workspace, hipStream_t s) {
  const TreeMasks tm{masks, words};
  if (tile_fits(a.pg.d)) {
    const TilePlan p = tile_plan(dtype, a);
    TileArgs g{a, p.splits, p.chunk, (int32_t)p.slots, p.by_request, (float*)workspace, (float*)workspace + p.rows_all * a.pg.d};
    if (dtype == LOCOCO_F32) return a.pg.d == 64 ? launch_tiles<float, 64>(g, tm, p, s) : launch_tiles<float, 128>(g, tm, p, s);
    return a.pg.d == 64 ? launch_tiles<__bf16, 64>(g, tm, p, s) : launch_tiles<__bf16, 128>(g, tm, p, s);
  }
  const dim3 grid((unsigned)rows_groups(a.tokens), (unsigned)a.pg.Hq);
  if (dtype == LOCOCO_F32) pages_tree_rows_k<float><<<grid, kRowsThreads, 0, s>>>(a, tm);
  else pages_tree_rows_k<__bf16><<<grid, kRowsThreads, 0, s>>>(a, tm);
  return hipGetLastError();
}

}  // namespace lococo
