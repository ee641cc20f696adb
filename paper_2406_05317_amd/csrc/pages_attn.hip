// Attention over paged 4-bit rows, every new row seeing the rows up to and at its own position: the kernels of pages_attn_tile.h.
#include "pages_attn_tile.h"

namespace lococo {
namespace {

using namespace pages_detail;

template <typename T>
__global__ __launch_bounds__(kRowsThreads) void pages_attn_rows_k(PagesAttnArgs a) {
  attn_rows<T, false>(a, TreeMasks{});
}
template <typename T, int D, int QB>
__global__ __launch_bounds__(64 * kTileWaves, 2) void pages_attn_tile_k(TileArgs g) {
  attn_tile<T, D, QB, false>(g, TreeMasks{});
}
template <typename T, int D, int TR, int WAVES>
__global__ __launch_bounds__(256) void pages_attn_join_k(TileArgs g, int32_t rows) {
  attn_join<T, D, TR, WAVES, false>(g, rows);
}

template <typename T, int D, int TR>
hipError_t launch_tile(const TileArgs& g, const TilePlan& p, hipStream_t s) {
  const unsigned join = (unsigned)join_groups(p, g.a.pg.Hkv);
  pages_attn_tile_k<T, D, TR / 16><<<(unsigned)tile_groups(p, g.a.pg.Hkv), kTileThreads, 0, s>>>(g);
  if (join) {
    if (p.splits > 16) pages_attn_join_k<T, D, TR, 4><<<join, kJoinThreads, 0, s>>>(g, p.rows);
    else pages_attn_join_k<T, D, TR, 1><<<join, kJoinThreads, 0, s>>>(g, p.rows);
  }
  return hipGetLastError();
}
template <typename T, int D>
hipError_t launch_tiles(const TileArgs& g, const TilePlan& p, hipStream_t s) {
  if constexpr (!std::is_same<T, float>::value) {
    if (p.tr == 32) return launch_tile<T, D, 32>(g, p, s);
  }
  return launch_tile<T, D, 16>(g, p, s);
}

}  // namespace

bool pages_attn_fits(int dtype, const PagesAttnArgs& a) {
  if ((int64_t)a.tokens * a.pg.group > 0x7fffffff) return false;             // rows of a kv head are counted in 32 bits
  if (!tile_fits(a.pg.d)) return rows_groups(a.tokens) * kRowsThreads <= kLaunchThreads;
  const TilePlan p = tile_plan(dtype, a);
  return tile_groups(p, a.pg.Hkv) * kTileThreads <= kLaunchThreads && join_groups(p, a.pg.Hkv) * kJoinThreads <= kLaunchThreads;
}

size_t pages_attn_workspace_bytes(int dtype, const PagesAttnArgs& a) {
  if (!tile_fits(a.pg.d)) return 0;
  const TilePlan p = tile_plan(dtype, a);
  return p.splits > 1 ? p.rows_all * (a.pg.d + 2) * sizeof(float) : 0;
}

hipError_t launch_pages_attn(int dtype, const PagesAttnArgs& a, void* workspace, hipStream_t s) {
  if (tile_fits(a.pg.d)) {
    const TilePlan p = tile_plan(dtype, a);
    TileArgs g{a, p.splits, p.chunk, (int32_t)p.slots, p.by_request, (float*)workspace, (float*)workspace + p.rows_all * a.pg.d};
    if (dtype == LOCOCO_F32) return a.pg.d == 64 ? launch_tiles<float, 64>(g, p, s) : launch_tiles<float, 128>(g, p, s);
    return a.pg.d == 64 ? launch_tiles<__bf16, 64>(g, p, s) : launch_tiles<__bf16, 128>(g, p, s);
  }
  const dim3 grid((unsigned)rows_groups(a.tokens), (unsigned)a.pg.Hq);
  if (dtype == LOCOCO_F32) pages_attn_rows_k<float><<<grid, kRowsThreads, 0, s>>>(a);
  else pages_attn_rows_k<__bf16><<<grid, kRowsThreads, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace lococo
