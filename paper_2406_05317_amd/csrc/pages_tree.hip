// The numbers of a turn in which requests bring trees of drafted tokens: positions and masks of a tree's rows, and what becomes of the pages
// once some of the rows are kept.
#include "pages.h"

#include <algorithm>

namespace lococo {
namespace {

constexpr int kWords = kPagesMaxTree / 32;

__device__ __forceinline__ void rows_of(const int32_t* starts, int32_t tokens, int32_t i, int32_t* first, int32_t* fresh) {
  *first = min(max(starts[i], 0), tokens);
  *fresh = min(max(starts[i + 1], *first), tokens) - *first;
}

// ---------------------------------------------------------------------------------------------------------------------------------
// Positions and masks.  A workgroup to a request, a lane to a row: it holds the row's mask, its depth and the row it has got up to, and takes
// over what that one holds, so that it gets twice as far up each time: as many rounds as the depth has binary digits.  The workgroups behind
// the last request's see to the rows of nobody.  Bound by the launch: 3 us for 32 trees of 8 rows,
// 5.5 for 512 of up to 64.
template <int W>
__global__ void pages_tree_k(PagesTreeArgs a) {
  __shared__ uint32_t bits[32 * W][W];
  __shared__ int32_t depth[32 * W], up[32 * W];
  const int32_t x = threadIdx.x;
  if ((int32_t)blockIdx.x >= a.n) {
    const int32_t lo = min(max(a.starts[0], 0), a.tokens), hi = min(max(a.starts[a.n], lo), a.tokens);
    const int64_t step = (int64_t)(gridDim.x - a.n) * blockDim.x;
    for (int64_t i = (int64_t)(blockIdx.x - a.n) * blockDim.x + x; i < a.tokens; i += step) {
      if (i >= lo && i < hi) continue;
      a.positions[i] = -1;
      for (int k = 0; k < a.words; ++k) a.masks[i * a.words + k] = 0;
    }
    return;
  }
  int32_t first, fresh;
  rows_of(a.starts, a.tokens, blockIdx.x, &first, &fresh);
  const int32_t rows = min(fresh, 32 * a.words), base = a.bases ? a.bases[blockIdx.x] : max(a.held[blockIdx.x], 0) - fresh;
  // a parent is a row ahead of its child
  int32_t to = -1, deep = 0;
  uint32_t mine[W];
  if (x < rows) {
    const int32_t p = a.parents[first + x];
    to = p >= 0 && p < x ? p : -1;
    deep = to >= 0;
#pragma unroll
    for (int k = 0; k < W; ++k) bits[x][k] = mine[k] = k == x >> 5 ? 1u << (x & 31) : 0u;
    depth[x] = deep;
    up[x] = to;
  }
  while (__syncthreads_or(to >= 0)) {
    int32_t next = -1;
    if (to >= 0) {
#pragma unroll
      for (int k = 0; k < W; ++k) mine[k] |= bits[to][k];
      deep += depth[to];
      next = up[to];
    }
    __syncthreads();
    if (to >= 0) {
#pragma unroll
      for (int k = 0; k < W; ++k) bits[x][k] = mine[k];
      depth[x] = deep;
      up[x] = to = next;
    }
  }
  for (int32_t i = x; i < fresh; i += blockDim.x) {                          // rows behind what a mask can name: nobody's
    const bool real = i < rows;                                               // (the lane's own row: i is x)
    a.positions[first + i] = real && base >= 0 ? base + deep : -1;
#pragma unroll
    for (int k = 0; k < W; ++k)
      if (k < a.words) a.masks[(int64_t)(first + i) * a.words + k] = real ? mine[k] : 0u;
  }
}

// ---------------------------------------------------------------------------------------------------------------------------------
// Keeping.  A wave to a request: the kept rows close up, in their order, on the places its new rows have had.
// Bound by the launches: rows 2.7 us, ring 4 us for 32 requests, 10.5 for 256 and 63 for 4096 (one workgroup, whose waves take the requests in turn),
// moving 3.3 us.
constexpr int kKeepWaves = 4;

__global__ __launch_bounds__(64 * kKeepWaves) void pages_keep_rows_k(PagesKeepArgs a) {
  const int32_t i = blockIdx.x * kKeepWaves + (threadIdx.x >> 6), l = threadIdx.x & 63;
  if (i >= a.n) {
    // rows of nobody
    const int32_t lo = min(max(a.starts[0], 0), a.tokens), hi = min(max(a.starts[a.n], lo), a.tokens);
    const int64_t waves = (int64_t)gridDim.x * kKeepWaves - a.n;
    for (int64_t x = (int64_t)(i - a.n) * 64 + l; x < a.tokens; x += waves * 64) {
      if (x >= lo && x < hi) continue;
      a.sources[x] = a.targets[x] = -1;
    }
    return;
  }
  int32_t first, fresh;
  rows_of(a.starts, a.tokens, i, &first, &fresh);
  const int32_t most = a.table_pages << a.page_shift, held = min(max(a.held[i], 0), most);
  // a request that the plan refused has no places for its rows
  const bool served = fresh > 0 && fresh <= held && a.slots[first] >= 0;
  int32_t kept = 0;
  for (int32_t x0 = 0; x0 < fresh; x0 += 64) {
    const int32_t x = x0 + l;
    const bool keep = served && x < fresh && a.kept[first + x] != 0;
    const uint64_t all = __ballot(keep);
    const int32_t rank = kept + __popcll(all & ((1ull << l) - 1));
    int32_t from = -1, to = -1;
    if (keep && rank != x) {
      from = a.slots[first + x];
      to = a.slots[first + rank];
    }
    if (x < fresh) {
      a.sources[first + x] = from;
      a.targets[first + x] = to;
    }
    kept += __popcll(all);
  }
  if (l == 0) a.held_after[i] = served ? held - fresh + kept : held;
}

// Pages behind a request's last row go back behind the ring's last free one, request by request: one workgroup, a running sum over the
// requests (saturating, as in the plan), a wave to a request that gives some.
constexpr int kRingThreads = 1024;

__global__ __launch_bounds__(kRingThreads) void pages_keep_ring_k(PagesKeepArgs a) {
  __shared__ int32_t off[kPagesMaxRequests], part[kRingThreads / 64], kept;
  const int tid = threadIdx.x, l = tid & 63, w = tid >> 6;
  const int32_t R = a.page_rows, sh = a.page_shift, most = a.table_pages << sh;
  const int per = (a.n + kRingThreads - 1) / kRingThreads, i0 = min(tid * per, a.n), i1 = min(i0 + per, a.n);
  if (tid == 0) kept = 0;
  __syncthreads();
  auto give = [&](int32_t i) {
    const int32_t held = min(max(a.held[i], 0), most);
    return ((held + R - 1) >> sh) - ((a.held_after[i] + R - 1) >> sh);
  };
  int32_t mine = 0, rows = 0;
  for (int i = i0; i < i1; ++i) {
    int32_t first, fresh;
    rows_of(a.starts, a.tokens, i, &first, &fresh);
    const int32_t held = min(max(a.held[i], 0), most);
    if (fresh > 0 && fresh <= held && a.slots[first] >= 0) rows += a.held_after[i] - (held - fresh);
    mine = add_cap(mine, give(i));
  }
  if (rows) atomicAdd(&kept, rows);            // whole numbers: any order gives the same
  int32_t sum = mine;
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) {
    const int32_t y = __shfl_up(sum, k);
    if (l >= k) sum = add_cap(sum, y);
  }
  int32_t at = __shfl_up(sum, 1);
  if (l == 0) at = 0;
  if (l == 63) part[w] = sum;
  __syncthreads();
  int32_t all = 0;
  for (int k = 0; k < kRingThreads / 64; ++k) {
    if (k == w) at = add_cap(all, at);
    all = add_cap(all, part[k]);
  }
  for (int i = i0; i < i1; ++i) {
    off[i] = at;
    at = add_cap(at, give(i));
  }
  __syncthreads();
  const int64_t head = a.ends[0], tail = a.ends[1];
  const int32_t P = a.n_pages, tail_at = (int32_t)(((tail % P) + P) % P);
  if (tid == 0) {
    a.ends_after[0] = head;
    a.ends_after[1] = tail + all;
    a.totals[0] = kept;
    a.totals[1] = all;
  }
  for (int i = w; i < a.n; i += kRingThreads / 64) {
    const int32_t n = give(i), page0 = (a.held_after[i] + R - 1) >> sh;
    for (int32_t j = l; j < n; j += 64) a.ring[((int64_t)tail_at + off[i] + j) % P] = a.tables[(int64_t)i * a.table_pages + page0 + j];
  }
}

// ---------------------------------------------------------------------------------------------------------------------------------
// Rows from slot to slot, as they lie.  A wave to a request and a kv head, d / 32 lanes to a row: 16 bytes of codes and a scale byte of K and
// of V each.  Rows move in their order, as many at a time as a wave has lanes for: a row goes to the place of one that is ahead of it, so
// what a later batch reads no earlier one has written.
constexpr int kMoveWaves = 4;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

__global__ __launch_bounds__(64 * kMoveWaves) void pages_move_k(PagesMoveArgs a) {
  __shared__ int32_t lists[kMoveWaves][64][2];
  const PagesView& pg = a.pg;
  const int l = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int32_t heads = (pg.Hkv + kMoveWaves - 1) / kMoveWaves, i = blockIdx.x / heads, h = (blockIdx.x - i * heads) * kMoveWaves + w;
  if (h >= pg.Hkv) return;                       // nothing below meets the other waves
  int32_t first, fresh;
  rows_of(a.starts, a.tokens, i, &first, &fresh);
  const int32_t lanes = pg.d / 32, batch = 64 / lanes, k = l / lanes, c = l - k * lanes, slots = pg.n_pages << pg.page_shift;
  for (int32_t x0 = 0; x0 < fresh; x0 += 64) {
    const int32_t x = x0 + l;
    const int32_t from = x < fresh ? a.sources[first + x] : -1, to = x < fresh ? a.targets[first + x] : -1;
    const bool moves = from >= 0 && from < slots && to >= 0 && to < slots && from != to;
    const uint64_t all = __ballot(moves);
    const int32_t n = __popcll(all);
    if (n == 0) continue;
    __builtin_amdgcn_wave_barrier();
    if (moves) {
      const int32_t r = __popcll(all & ((1ull << l) - 1));
      lists[w][r][0] = from;
      lists[w][r][1] = to;
    }
    __builtin_amdgcn_wave_barrier();
    for (int32_t r0 = 0; r0 < n; r0 += batch) {
      const bool real = k < batch && r0 + k < n;
      const int32_t src = real ? lists[w][r0 + k][0] : 0, dst = real ? lists[w][r0 + k][1] : 0;
      const int64_t sp = ((int64_t)(src >> pg.page_shift) * pg.Hkv + h) * pg.page_rows, dp = ((int64_t)(dst >> pg.page_shift) * pg.Hkv + h) * pg.page_rows;
      const int32_t sr = src & (pg.page_rows - 1), dr = dst & (pg.page_rows - 1);
      const int64_t sc = (sp + sr) * (pg.d / 2) + 16 * c, dc = (dp + dr) * (pg.d / 2) + 16 * c;
      const int64_t ss = sp * lanes + (int64_t)c * pg.page_rows + sr, ds = dp * lanes + (int64_t)c * pg.page_rows + dr;
      u32x4 kc, vc;
      uint8_t ks, vs;
      if (real) {
        kc = *(const u32x4*)(pg.k_codes + sc);
        vc = *(const u32x4*)(pg.v_codes + sc);
        ks = pg.k_scales[ss];
        vs = pg.v_scales[ss];
      }
      __builtin_amdgcn_wave_barrier();           // all of a batch is read ahead of what it writes
      if (real) {
        *(u32x4*)(pg.k_codes + dc) = kc;
        *(u32x4*)(pg.v_codes + dc) = vc;
        pg.k_scales[ds] = ks;
        pg.v_scales[ds] = vs;
      }
    }
  }
}

int64_t move_groups(const PagesView& pg, int32_t n) { return (int64_t)n * ((pg.Hkv + kMoveWaves - 1) / kMoveWaves); }

}  // namespace

hipError_t launch_pages_tree(const PagesTreeArgs& a, hipStream_t s) {
  const unsigned spare = (unsigned)std::min<int64_t>(std::max<int64_t>(a.tokens / 4096, 1), 64), grid = (unsigned)a.n + spare;
  switch (a.words) {
    case 1: pages_tree_k<1><<<grid, 64, 0, s>>>(a); break;
    case 2: pages_tree_k<2><<<grid, 64, 0, s>>>(a); break;
    case 3:
    case 4: pages_tree_k<4><<<grid, 128, 0, s>>>(a); break;
    default: pages_tree_k<kWords><<<grid, 32 * kWords, 0, s>>>(a); break;
  }
  return hipGetLastError();
}

hipError_t launch_pages_keep(const PagesKeepArgs& a, hipStream_t s) {
  const unsigned spare = (unsigned)std::min<int64_t>(std::max<int64_t>(a.tokens / 4096, 1), 64);
  pages_keep_rows_k<<<((unsigned)a.n + spare + kKeepWaves - 1) / kKeepWaves, 64 * kKeepWaves, 0, s>>>(a);
  pages_keep_ring_k<<<1, kRingThreads, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_pages_move(const PagesMoveArgs& a, hipStream_t s) {
  pages_move_k<<<(unsigned)move_groups(a.pg, a.n), 64 * kMoveWaves, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace lococo
