// Attention over paged 4-bit rows under masks: a new row sees all rows ahead of its request's new ones, and those of the new ones that its
// mask names (a tree of drafted tokens).  The kernels' tiles are those of pages_attn_tile.h.
#include "pages_attn_tile.h"

namespace lococo {
namespace {

using namespace pages_detail;

template <typename T>
__global__ __launch_bounds__(kRowsThreads) void pages_tree_rows_k(PagesAttnArgs a, TreeMasks tm) {
  attn_rows<T, true>(a, tm);
}
// little work: a workgroup to a tile and a part of the keys, dealt out as in lococo_pages_attn
template <typename T, int D, int QB>
__global__ __launch_bounds__(64 * kTileWaves, 2) void pages_tree_tile_k(TileArgs g, TreeMasks tm) {
  attn_tile<T, D, QB, true>(g, tm);
}
template <typename T, int D, int TR, int WAVES>
__global__ __launch_bounds__(256) void pages_tree_join_k(TileArgs g, int32_t rows) {
  attn_join<T, D, TR, WAVES, true>(g, rows);
}

// ---------------------------------------------------------------------------------------------------------------------------------
// Much work: a launch ahead reads what the requests hold and deals it out, to workgroups of four waves,
//   of a request of up to kAlone steps of 64 keys, one to four of its row tiles: a wave works through a tile by itself and writes it;
//   of a longer one, one to a tile and a part of its keys, of about `per` steps a wave: the waves take steps in turn and meet at the end.
// `per` is such that the parts of all long requests are about kParts: a request that is far longer than the others is cut into as many more.
// Long ones go first, so that short ones fill up the end.  A tile in p parts has more than (p - 1) of their length: over all tiles in several
// parts these are 2 kParts at most, and the tiles kParts at most.
// 32 requests of 128 .. 8192 rows, trees of 8 .. 64, 8 kv heads of 4: 84 us a call against 94 dealt out as in lococo_pages_attn; 64 requests of 200
// .. 8000 with 8 new rows 76 against 91; one request of 131072 rows beside 31 of 500: 145 against 1033.  Nearly even lengths, which the host cannot
// tell, lose by it: 16 requests of up to 4000, 32 heads, 61 against 53; 8 of 8000 with 64 new rows 122 against 116.  The launch ahead takes
// 7 - 8 us, the tiles (79 us of the 84) what their vector instructions do: some 500 for 64 keys of 32 rows, beside 104 matrix products (some 1.2 us a
// step of a wave, two of them on a SIMD); shorter parts add their starts, longer ones wait at the end (kAlone 16, kParts 1024: 84 us for 79).
constexpr int kAlone = 8, kParts = 512, kLeastSteps = 2, kDealThreads = 1024;
constexpr int32_t kNoParts = kPagesCap / kTileKeys + 1;                      // steps of any request

struct Item {                                  // of a workgroup
  int32_t req, first, fresh, held, kvh, tile, key_lo, key_hi;
  int32_t part;                                // where it keeps its part of the tile; -1: it has all of it; -2: four tiles, a wave each
  int32_t spare[3];
};
struct Join { int32_t first, fresh, kvh, tile, part, parts, spare[2]; };
struct Dealt {                                 // ahead of the parts in the workspace
  int32_t items, joins, spare[62];
  Join join[kParts];
  Item item[1];                                // as many as the launch has workgroups
};

struct DealtArgs {
  TileArgs t;                                  // part_o, part_ml: [part][row]
  TreeMasks tm;
  Dealt* dealt;
  int32_t groups;
};

// running sums over the workgroup, a thread's own left out, cut off at kPagesCap
__device__ __forceinline__ int32_t scan(int32_t x, int32_t* all, int32_t* part) {
  const int l = threadIdx.x & 63, w = threadIdx.x >> 6;
  int32_t s = x;
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) {
    const int32_t y = __shfl_up(s, k);
    if (l >= k) s = add_cap(s, y);
  }
  int32_t e = __shfl_up(s, 1);
  if (l == 0) e = 0;
  __syncthreads();                               // the last sum's parts have been read
  if (l == 63) part[w] = s;
  __syncthreads();
  int32_t before = 0, sum = 0;
#pragma unroll
  for (int k = 0; k < kDealThreads / 64; ++k) {
    if (k == w) before = sum;
    sum = add_cap(sum, part[k]);
  }
  *all = sum;
  return add_cap(before, e);
}

template <int TR>
__global__ __launch_bounds__(kDealThreads) void pages_tree_deal_k(DealtArgs g) {
  __shared__ int32_t part[kDealThreads / 64], lists[3][kPagesMaxRequests];
  const PagesAttnArgs& a = g.t.a;
  const int tid = threadIdx.x, l = tid & 63, w = tid >> 6;
  const int per_thread = (a.n + kDealThreads - 1) / kDealThreads, i0 = min(tid * per_thread, a.n), i1 = min(i0 + per_thread, a.n);
  struct Request { int32_t first, fresh, held, tiles, steps; };
  auto request = [&](int32_t i) {
    Request r;
    r.first = min(max(a.starts[i], 0), a.tokens);
    r.fresh = min(max(a.starts[i + 1], r.first), a.tokens) - r.first;
    r.held = min(max(a.held[i], 0), a.table_pages << a.pg.page_shift);
    r.tiles = (int32_t)(((int64_t)r.fresh * a.pg.group + TR - 1) / TR);
    r.steps = (r.held + kTileKeys - 1) / kTileKeys;
    return r;
  };
  auto cap = [](int64_t x) { return (int32_t)min(x, (int64_t)kPagesCap); };
  int32_t work = 0, all_work;
  for (int i = i0; i < i1; ++i) {
    const Request r = request(i);
    if (r.steps > kAlone) work = add_cap(work, cap((int64_t)r.tiles * r.steps));
  }
  scan(work, &all_work, part);
  const int64_t even = ((int64_t)all_work * a.pg.Hkv + kParts * kTileWaves - 1) / (kParts * kTileWaves);
  // steps of a part
  const int32_t per = kTileWaves * (all_work < kPagesCap ? (int32_t)min(max(even, (int64_t)kLeastSteps), (int64_t)kNoParts) : kNoParts);
  auto parts_of = [&](const Request& r) { return (r.steps + per - 1) / per; };
  int32_t n_long = 0, n_alone = 0, n_kept = 0, n_joins = 0, all_long, all_alone, all_kept, all_joins;
  for (int i = i0; i < i1; ++i) {
    const Request r = request(i);
    if (r.steps <= kAlone) {
      n_alone = add_cap(n_alone, (r.tiles + kTileWaves - 1) / kTileWaves);
      continue;
    }
    const int32_t parts = parts_of(r), x = cap((int64_t)r.tiles * parts);
    n_long = add_cap(n_long, x);
    if (parts > 1) {
      n_kept = add_cap(n_kept, x);
      n_joins = add_cap(n_joins, r.tiles);
    }
  }
  n_long = scan(n_long, &all_long, part);
  n_alone = scan(n_alone, &all_alone, part);
  n_kept = scan(n_kept, &all_kept, part);
  n_joins = scan(n_joins, &all_joins, part);
  // starts that do not ascend may ask for more than there is room for: no work, then
  const int64_t items = ((int64_t)all_long + all_alone) * a.pg.Hkv;
  const bool fits = items <= g.groups && (int64_t)all_kept * a.pg.Hkv <= 2 * kParts && (int64_t)all_joins * a.pg.Hkv <= kParts;
  if (tid == 0 && blockIdx.x == 0) {
    g.dealt->items = fits ? (int32_t)items : 0;
    g.dealt->joins = fits ? all_joins * a.pg.Hkv : 0;
  }
  if (!fits) return;
  for (int i = i0; i < i1; ++i) {
    const Request r = request(i);
    const int32_t parts = parts_of(r);
    lists[0][i] = r.steps <= kAlone ? n_alone : n_long;
    lists[1][i] = n_kept;
    lists[2][i] = n_joins;
    if (r.steps <= kAlone) {
      n_alone += (r.tiles + kTileWaves - 1) / kTileWaves;
    } else {
      n_long += r.tiles * parts;
      if (parts > 1) {
        n_kept += r.tiles * parts;
        n_joins += r.tiles;
      }
    }
  }
  __syncthreads();
  // every workgroup has counted all of it; the items are written by all, a wave to a request
  for (int i = blockIdx.x * (kDealThreads / 64) + w; i < a.n; i += gridDim.x * (kDealThreads / 64)) {
    const Request r = request(i);
    const bool alone = r.steps <= kAlone;
    const int32_t parts = alone ? 1 : parts_of(r), share = (r.steps + parts - 1) / max(parts, 1) * kTileKeys;
    const int32_t mine = alone ? (r.tiles + kTileWaves - 1) / kTileWaves : r.tiles * parts;
    // a request's items: kv heads, then parts, then tiles, so that neighbours read the same keys
    const int32_t at = alone ? all_long * a.pg.Hkv + lists[0][i] * a.pg.Hkv : lists[0][i] * a.pg.Hkv;
    for (int32_t x = l; x < mine * a.pg.Hkv; x += 64) {
      const int32_t kvh = x / mine, y = x - kvh * mine, p = alone ? 0 : y / r.tiles, tile = alone ? y * kTileWaves : y - p * r.tiles;
      const int32_t kept = lists[1][i] * a.pg.Hkv + (kvh * r.tiles + tile) * parts;
      g.dealt->item[at + x] = Item{i, r.first, r.fresh, r.held, kvh, tile, min(p * share, r.held), min((p + 1) * share, r.held),
                                   alone ? -2 : parts == 1 ? -1 : kept + p, {0, 0, 0}};
      if (parts > 1 && p == 0) g.dealt->join[(lists[2][i] * a.pg.Hkv) + kvh * r.tiles + tile] = Join{r.first, r.fresh, kvh, tile, kept, parts, {0, 0}};
    }
  }
}

template <typename T, int D, int QB>
__global__ __launch_bounds__(64 * kTileWaves, 2) void pages_tree_item_k(DealtArgs g) {
  constexpr int TR = 16 * QB;
  const PagesAttnArgs& a = g.t.a;
  // workgroups are dealt round-robin to the eight XCDs: eight neighbours of 64 to each
  const int32_t b = blockIdx.x, number = (b & ~63) + (b & 7) * 8 + (b >> 3 & 7);
  if (number >= g.dealt->items) return;
  const Item& it = g.dealt->item[number];
  const int32_t part = it.part;
  TileJob job;
  job.req = it.req;
  job.first = it.first;
  job.fresh = it.fresh;
  job.held = job.keys = it.held;
  job.row0 = it.tile * TR;
  if (part == -2) {
    job.row0 += TR * (int32_t)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    job.rows = (int32_t)min((int64_t)job.fresh * a.pg.group - job.row0, (int64_t)TR);
    if (job.rows > 0) attn_piece<T, D, QB, true, 1>(g.t, g.tm, job, it.kvh, 0, job.keys, true, 0, threadIdx.x);
    return;
  }
  job.rows = (int32_t)min((int64_t)job.fresh * a.pg.group - job.row0, (int64_t)TR);
  attn_piece<T, D, QB, true, kTileWaves>(g.t, g.tm, job, it.kvh, it.key_lo, it.key_hi, part < 0, (int64_t)max(part, 0) * TR, threadIdx.x);
}

// The parts of a tile to one, in their order: a workgroup to 16 rows of a tile, 16 lanes to a row.
template <typename T, int D, int TR>
__global__ __launch_bounds__(256) void pages_tree_items_join_k(DealtArgs g) {
  constexpr int PER = D / 16, AHEAD = 4;
  const PagesAttnArgs& a = g.t.a;
  const int32_t number = blockIdx.x / (TR / 16);
  if (number >= g.dealt->joins) return;
  const Join& it = g.dealt->join[number];
  const int32_t r = blockIdx.x % (TR / 16) * 16 + threadIdx.x / 16, col = threadIdx.x % 16 * PER, parts = it.parts;
  const int32_t row = it.tile * TR + r;
  if (row >= (int64_t)it.fresh * a.pg.group) return;
  const int64_t row0 = (int64_t)it.part * TR + r;
  float best = kNoRef, total = 0.f, y[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) y[i] = 0.f;
  for (int32_t k0 = 0; k0 < parts; k0 += AHEAD) {
    f32x2 st[AHEAD];
    f4 v[AHEAD][PER / 4];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      const int64_t pr = row0 + (int64_t)min(k0 + j, parts - 1) * TR;
      st[j] = *(const f32x2*)(g.t.part_ml + 2 * pr);
#pragma unroll
      for (int i = 0; i < PER / 4; ++i) v[j][i] = *(const f4*)(g.t.part_o + pr * D + col + 4 * i);
    }
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      if (k0 + j >= parts) break;
      const float next = fmaxf(best, st[j][0]), keep = __builtin_amdgcn_exp2f(best - next), f = __builtin_amdgcn_exp2f(st[j][0] - next);
      best = next;
      total = total * keep + st[j][1] * f;
#pragma unroll
      for (int i = 0; i < PER; ++i) y[i] = y[i] * keep + v[j][i / 4][i % 4] * f;
    }
  }
  const int32_t x = row / a.pg.group, token = it.first + x, ob = token < a.o.t ? 0 : token / a.o.t, ot = token - ob * a.o.t;
  T* out = (T*)a.o.p + ob * a.o.sb + (it.kvh * a.pg.group + row - x * a.pg.group) * a.o.sh + ot * a.o.st + col;
  const float inv = total == 0.f ? 0.f : 1.f / total;
#pragma unroll
  for (int i = 0; i < PER; ++i) out[i] = (T)(y[i] * inv);
}

struct TreePlan { bool dealt; TilePlan tiles; int64_t groups; size_t dealt_bytes; };
TreePlan tree_plan(int dtype, const PagesAttnArgs& a) {
  TreePlan p{};
  p.tiles = tile_plan(dtype, a);
  const int64_t tiles = (int64_t)a.tokens * a.pg.group / p.tiles.tr + std::min(a.n, a.tokens);
  p.groups = (tiles * a.pg.Hkv + kParts + 63) / 64 * 64;
  // what the requests would cost if all were as long as the longest: steps of the waves that are resident
  const int64_t steps = tiles * a.pg.Hkv * (((int64_t)a.max_held + kTileKeys - 1) / kTileKeys) / (2 * kTileWaves * (int64_t)cu_count());
  p.dealt = a.max_held > kAlone * kTileKeys && steps >= 16 && p.groups * kTileThreads <= kLaunchThreads;
  p.dealt_bytes = (sizeof(Dealt) + (size_t)p.groups * sizeof(Item) + 255) / 256 * 256;
  return p;
}

template <typename T, int D, int TR>
hipError_t launch_tile(const PagesAttnArgs& a, const TreeMasks& tm, const TreePlan& p, void* workspace, hipStream_t s) {
  if (!p.dealt) {
    const TilePlan& t = p.tiles;
    const TileArgs g{a, t.splits, t.chunk, (int32_t)t.slots, t.by_request, (float*)workspace, (float*)workspace + t.rows_all * D};
    const unsigned join = (unsigned)join_groups(t, a.pg.Hkv);
    pages_tree_tile_k<T, D, TR / 16><<<(unsigned)tile_groups(t, a.pg.Hkv), kTileThreads, 0, s>>>(g, tm);
    if (join) {
      if (t.splits > 16) pages_tree_join_k<T, D, TR, 4><<<join, kJoinThreads, 0, s>>>(g, t.rows);
      else pages_tree_join_k<T, D, TR, 1><<<join, kJoinThreads, 0, s>>>(g, t.rows);
    }
    return hipGetLastError();
  }
  float* parts = (float*)((char*)workspace + p.dealt_bytes);
  const DealtArgs g{TileArgs{a, 0, 0, 0, 0, parts, parts + 2 * (size_t)kParts * TR * D}, tm, (Dealt*)workspace, (int32_t)p.groups};
  pages_tree_deal_k<TR><<<(unsigned)std::min((a.n + 15) / 16, 16), kDealThreads, 0, s>>>(g);
  pages_tree_item_k<T, D, TR / 16><<<(unsigned)p.groups, kTileThreads, 0, s>>>(g);
  pages_tree_items_join_k<T, D, TR><<<kParts * (TR / 16), kJoinThreads, 0, s>>>(g);
  return hipGetLastError();
}
template <typename T, int D>
hipError_t launch_tiles(const PagesAttnArgs& a, const TreeMasks& tm, const TreePlan& p, void* workspace, hipStream_t s) {
  if constexpr (!std::is_same<T, float>::value) {
    if (p.tiles.tr == 32) return launch_tile<T, D, 32>(a, tm, p, workspace, s);
  }
  return launch_tile<T, D, 16>(a, tm, p, workspace, s);
}

}  // namespace

size_t pages_attn_tree_workspace_bytes(int dtype, const PagesAttnArgs& a) {
  if (!tile_fits(a.pg.d)) return 0;
  const TreePlan p = tree_plan(dtype, a);
  // what does for a larger max_held does for a smaller one
  const size_t plain = pages_attn_workspace_bytes(dtype, a);
  return p.dealt ? std::max(plain, p.dealt_bytes + 2 * (size_t)kParts * p.tiles.tr * (a.pg.d + 2) * sizeof(float)) : plain;
}

hipError_t launch_pages_attn_tree(int dtype, const PagesAttnArgs& a, const uint32_t* masks, int32_t words, void* workspace, hipStream_t s) {
  const TreeMasks tm{masks, words};
  if (tile_fits(a.pg.d)) {
    const TreePlan p = tree_plan(dtype, a);
    if (dtype == LOCOCO_F32) return a.pg.d == 64 ? launch_tiles<float, 64>(a, tm, p, workspace, s) : launch_tiles<float, 128>(a, tm, p, workspace, s);
    return a.pg.d == 64 ? launch_tiles<__bf16, 64>(a, tm, p, workspace, s) : launch_tiles<__bf16, 128>(a, tm, p, workspace, s);
  }
  const dim3 grid((unsigned)rows_groups(a.tokens), (unsigned)a.pg.Hq);
  if (dtype == LOCOCO_F32) pages_tree_rows_k<float><<<grid, kRowsThreads, 0, s>>>(a, tm);
  else pages_tree_rows_k<__bf16><<<grid, kRowsThreads, 0, s>>>(a, tm);
  return hipGetLastError();
}

}  // namespace lococo
