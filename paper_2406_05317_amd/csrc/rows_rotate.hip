// Norm and position rotation of query and key rows, and the way back.
#include "rotate.h"

#include <algorithm>

namespace lococo {
namespace {

using namespace rotate_detail;

// cosines and sines of the workgroup's positions, to LDS
__device__ __forceinline__ void fill_table(float2* table, const RotateView& rv, const int32_t* positions, int32_t tokens, int32_t t,
                                           int32_t token0, int32_t lt) {
  const int32_t half = rv.r / 2;
  for (int32_t i = threadIdx.x; i < half << lt; i += kRotateThreads) {
    const int32_t x = i / half, token = min(token0 + x, tokens - 1);
    const int32_t pos = positions ? positions[token] : token % t;
    float s, c;
    cos_sin(pos, rv.freqs[i - x * half], &c, &s);
    table[i] = make_float2(c, s);
  }
}
// a lane's four of them
template <int KIND>
__device__ __forceinline__ void read_table(const float2* table, const Pairs<KIND>& pr, int32_t sub, float (&c)[4], float (&s)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    c[i] = 1.f;
    s[i] = 0.f;
    if (pr.turned(i)) {
      const float2 v = table[sub * pr.half + pr.q0 + i];
      c[i] = v.x;
      s[i] = v.y;
    }
  }
}

// A workgroup takes 2^lt positions and a block of q's or k's heads, (256 / P) >> lt of them side by side, a lane's rows two at a time.
// Bound by memory: 16384 positions of 40 heads, 336 MB in 67 us (5.0 TB/s; a large copy 5.1; 97 us where a lane loaded its eight channels'
// partners beside them and multiplied by the weights); 32 positions 4 us.

template <typename T, int KIND>
__global__ __launch_bounds__(kRotateThreads) void rows_rotate_k(RotateArgs a) {
  __shared__ float2 table[kRotateTable];
  const RotateView& rv = a.rv;
  const int32_t all = a.blocks[0] + a.blocks[1], tile = blockIdx.x / all, blk = blockIdx.x - tile * all;
  const int part = blk >= a.blocks[0];
  const int32_t h0 = (blk - (part ? a.blocks[0] : 0)) * a.sh.hb, h1 = min(h0 + a.sh.hb, rv.heads[part]);
  const int32_t lp = a.sh.lp, lt = a.sh.lt, grp = threadIdx.x >> lp, lane = threadIdx.x & ((1 << lp) - 1);
  const int32_t token0 = tile << lt, sub = grp & ((1 << lt) - 1), token = token0 + sub, step = (kRotateThreads >> lp) >> lt;
  fill_table(table, rv, a.positions, a.tokens, a.t, token0, lt);
  __syncthreads();
  const Pairs<KIND> pr{4 * lane, rv.r / 2, rv.r, rv.d};
  const bool active = pr.in() && token < a.tokens && (!a.positions || a.positions[min(token, a.tokens - 1)] >= 0);
  float c[4], s[4];
  read_table(table, pr, sub, c, s);
  // times the weights: with xhat = one x, which is not large, y_a = xhat_a ca - xhat_b sb, y_b = xhat_b cb + xhat_a sa
  const T* weights = (const T*)rv.w[part];
  const bool banks = weights && rv.ws[part];
  float ca[4], cb[4], sa[4], sb[4];
  auto weigh = [&](int32_t h) {
    float wa[4] = {1.f, 1.f, 1.f, 1.f}, wb[4] = {1.f, 1.f, 1.f, 1.f};
    if (weights && pr.in()) pr.load(weights + h * rv.ws[part], wa, wb);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      ca[i] = c[i] * wa[i];
      sa[i] = s[i] * wa[i];
      cb[i] = c[i] * wb[i];
      sb[i] = s[i] * wb[i];
    }
  };
  if (!banks) weigh(0);
  const T* in = row_at<T>(a.in[part], active ? token : 0, 0);
  T* out = const_cast<T*>(row_at<T>(a.out[part], active ? token : 0, 0));
  for (int32_t h = h0 + (grp >> lt); h < h1; h += kAhead * step) {
    float xa[kAhead][4], xb[kAhead][4];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
#pragma unroll
      for (int i = 0; i < 4; ++i) xa[k][i] = xb[k][i] = 0.f;
      if (active && h + k * step < h1) pr.load(in + (h + k * step) * a.in[part].sh, xa[k], xb[k]);
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (h + k * step >= h1) break;
      if (banks) weigh(h + k * step);
      const float one = rv.norm ? one_over_root(xa[k], xb[k], lp, rv) : 1.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float na = one * xa[k][i], nb = one * xb[k][i];
        xa[k][i] = fmaf(na, ca[i], -nb * sb[i]);
        xb[k][i] = fmaf(nb, cb[i], na * sa[i]);
      }
      if (active) pr.store(out + (h + k * step) * a.out[part].sh, xa[k], xb[k]);
    }
  }
}

// The way back: g_n = the upstream gradient turned the other way; with xhat = x * one, one = 1 / sqrt(mean(x^2) + eps),
//   d_w += g_n xhat (over all rows),  d_x = one * (w g_n - xhat mean(w g_n xhat)).
// Both means are sums over the row taken side by side.  A workgroup adds up its rows' part of d_w, once over its rows in LDS at the end, and
// leaves it for rows_rotate_weights_k: no atomics, the same bits every time.  d_w is a sum over all rows of all heads: in fp32 over the eight
// or fewer that a lane has of one tile (of eight tiles, where it has one of each), beyond them in 64 bits, a workgroup's part rounded to fp32.
// In fp32 throughout it was twice as far from the exact sum.  Bound by memory: 16384 positions of 40 heads, 839 MB in 168 us (5.0 TB/s), the
// weights' parts 9 more; with half as many workgroups 171, with a quarter 188.
constexpr int kBackRows = 8;                   // rows whose part of d_w a lane adds up in fp32

template <typename T, int KIND>
__global__ __launch_bounds__(kRotateThreads, 4) void rows_rotate_back_k(RotateBackArgs a) {
  __shared__ float2 table[kRotateTable];
  __shared__ double gws[kRotateThreads * 8];
  const RotateView& rv = a.rv;
  const int32_t blk = blockIdx.x / a.chunks, chunk = blockIdx.x - blk * a.chunks;
  const int part = blk >= a.blocks[0];
  const int32_t h0 = (blk - (part ? a.blocks[0] : 0)) * a.sh.hb, h1 = min(h0 + a.sh.hb, rv.heads[part]);
  const int32_t lp = a.sh.lp, lt = a.sh.lt, grp = threadIdx.x >> lp, lane = threadIdx.x & ((1 << lp) - 1);
  const int32_t sub = grp & ((1 << lt) - 1), step = (kRotateThreads >> lp) >> lt;
  const Pairs<KIND> pr{4 * lane, rv.r / 2, rv.r, rv.d};
  const bool in = pr.in(), banks = rv.ws[part] != 0;
  const T* weights = (const T*)rv.w[part];
  float wa[4] = {1.f, 1.f, 1.f, 1.f}, wb[4] = {1.f, 1.f, 1.f, 1.f};
  if (weights && !banks && in) pr.load(weights, wa, wb);
  // a lane's sums in 64 bits lie in LDS: in registers they would cost a fourth of the waves
  double* mine = gws + threadIdx.x;
#pragma unroll
  for (int i = 0; i < 8; ++i) mine[i * kRotateThreads] = 0.0;
  float gwa[4] = {0.f, 0.f, 0.f, 0.f}, gwb[4] = {0.f, 0.f, 0.f, 0.f};
  auto add = [&] {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      mine[i * kRotateThreads] += gwa[i];
      mine[(4 + i) * kRotateThreads] += gwb[i];
      gwa[i] = gwb[i] = 0.f;
    }
  };
  for (int32_t k = 0; k < a.tiles; ++k) {
    if (k && k % a.stretch == 0) add();
    const int64_t first = ((int64_t)chunk * a.tiles + k) << lt;
    if (first >= a.tokens) break;              // the same for all lanes
    const int32_t token0 = (int32_t)first, token = token0 + sub;
    __syncthreads();                           // the last tile's table has been read
    fill_table(table, rv, a.positions, a.tokens, a.t, token0, lt);
    __syncthreads();
    const bool real = in && token < a.tokens, active = real && (!a.positions || a.positions[token] >= 0);
    float c[4], s[4];
    read_table(table, pr, sub, c, s);
    const int32_t b = real ? token / a.t : 0, t = real ? token - b * a.t : 0;
    const int64_t at = ((int64_t)b * rv.heads[part] * a.t + t) * rv.d, head = (int64_t)a.t * rv.d;
    const T* rows = row_at<T>(a.in[part], active ? token : 0, 0);
    for (int32_t h = h0 + (grp >> lt); h < h1; h += kAhead * step) {
      float ga[kAhead][4], gb[kAhead][4], xa[kAhead][4], xb[kAhead][4];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
#pragma unroll
        for (int i = 0; i < 4; ++i) ga[j][i] = gb[j][i] = xa[j][i] = xb[j][i] = 0.f;
        const int32_t hj = h + j * step;
        if (active && hj < h1) {
          pr.load(a.gy[part] + at + hj * head, ga[j], gb[j]);
          if (rv.norm) pr.load(rows + hj * a.in[part].sh, xa[j], xb[j]);
        }
      }
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const int32_t hj = h + j * step;
        if (hj >= h1) break;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float ya = ga[j][i], yb = gb[j][i];
          ga[j][i] = fmaf(ya, c[i], yb * s[i]);
          gb[j][i] = fmaf(yb, c[i], -ya * s[i]);
        }
        if (rv.norm) {
          if (banks && in) pr.load(weights + hj * rv.ws[part], wa, wb);
          float sq = 0.f, dot = 0.f;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            sq = fmaf(xa[j][i], xa[j][i], fmaf(xb[j][i], xb[j][i], sq));
            dot = fmaf(wa[i] * ga[j][i], xa[j][i], fmaf(wb[i] * gb[j][i], xb[j][i], dot));
          }
          sq = row_sum(sq, lp);
          dot = row_sum(dot, lp);
          float one = rsqrtf(sq * (1.f / (float)rv.d) + rv.eps), mean = one * dot * (1.f / (float)rv.d);
          if (!(sq < INFINITY && fabsf(dot) < INFINITY)) {
            one = one_of_large(xa[j], xb[j], lp, rv);
            dot = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) dot = fmaf(wa[i] * ga[j][i], xa[j][i] * one, fmaf(wb[i] * gb[j][i], xb[j][i] * one, dot));
            mean = row_sum(dot, lp) * (1.f / (float)rv.d);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float ha = xa[j][i] * one, hb = xb[j][i] * one;
            gwa[i] = fmaf(ga[j][i], ha, gwa[i]);
            gwb[i] = fmaf(gb[j][i], hb, gwb[i]);
            ga[j][i] = one * fmaf(wa[i], ga[j][i], -ha * mean);
            gb[j][i] = one * fmaf(wb[i], gb[j][i], -hb * mean);
          }
        }
        if (real) pr.store(a.gx[part] + at + hj * head, ga[j], gb[j]);        // a row of nobody: zeros
      }
    }
  }
  if (!a.gw[part]) return;
  add();
  double dw[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) dw[i] = mine[i * kRotateThreads];
  __syncthreads();
  if (in)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      gws[grp * rv.d + pr.first(i)] = dw[i];
      gws[grp * rv.d + pr.second(i)] = dw[4 + i];
    }
  __syncthreads();
  for (int32_t c = threadIdx.x; c < rv.d; c += kRotateThreads) {
    double sum = 0.0;
    for (int32_t k = 0; k < kRotateThreads >> lp; ++k) sum += gws[k * rv.d + c];
    a.parts[((int64_t)blk * a.chunks + chunk) * rv.d + c] = (float)sum;
  }
}

// The parts of a weight's gradient to one, in 64 bits and a fixed order, and onto what is there: a workgroup to 16 columns of a bank of
// weights, lanes of four columns, eight rows on their way at once.
constexpr int kWeightThreads = 1024, kWeightCols = 16, kWeightRows = 8;

__global__ __launch_bounds__(kWeightThreads) void rows_rotate_weights_k(RotateBackArgs a) {
  constexpr int LANES = kWeightCols / 4, SIDE = kWeightThreads / LANES;
  __shared__ double sums[SIDE][kWeightCols];
  const RotateView& rv = a.rv;
  // banks: q's (one, or one a head), then k's
  const int32_t cols = (rv.d + kWeightCols - 1) / kWeightCols, bank = blockIdx.x / cols, c0 = (blockIdx.x - bank * cols) * kWeightCols;
  const int32_t banks = rv.ws[0] ? rv.heads[0] : 1;
  const int part = bank >= banks;
  const int32_t head = bank - (part ? banks : 0);
  if (!a.gw[part]) return;
  const int32_t first = (part ? a.blocks[0] : 0) + (rv.ws[part] ? head : 0), rows = (rv.ws[part] ? 1 : a.blocks[part]) * a.chunks;
  const int32_t k = threadIdx.x / LANES, c = 4 * (threadIdx.x % LANES);
  const float* at = a.parts + (int64_t)first * a.chunks * rv.d + c0 + c;
  double sum[4] = {0.0, 0.0, 0.0, 0.0};
  if (c0 + c < rv.d)
    for (int32_t i = k; i < rows; i += kWeightRows * SIDE) {
      float x[kWeightRows][4];
#pragma unroll
      for (int j = 0; j < kWeightRows; ++j) read4(at + (int64_t)min(i + j * SIDE, rows - 1) * rv.d, x[j]);
#pragma unroll
      for (int j = 0; j < kWeightRows; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] += i + j * SIDE < rows ? x[j][e] : 0.f;
    }
#pragma unroll
  for (int e = 0; e < 4; ++e) sums[k][c + e] = sum[e];
  for (int32_t n = SIDE / 2; n >= 1; n /= 2) {
    __syncthreads();
    if (k < n)
#pragma unroll
      for (int e = 0; e < 4; ++e) sums[k][c + e] = sum[e] += sums[k + n][c + e];
  }
  if (k == 0 && c0 + c < rv.d)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float* gw = a.gw[part] + head * rv.ws[part] + c0 + c + e;
      *gw = (float)(*gw + sum[e]);
    }
}

struct BackPlan { RotateShape sh; int32_t blocks[2], chunks, tiles; };
BackPlan back_plan(const RotateView& rv, int32_t tokens) {
  BackPlan p{};
  p.sh.lp = lanes_log(rv.d);
  p.sh.lt = 8 - p.sh.lp;                       // positions alone: a workgroup's rows of a head lie side by side
  const bool banks = rv.ws[0] || rv.ws[1];
  p.sh.hb = banks ? 1 : kBackRows;
  int64_t blocks = 0;
  for (int i = 0; i < 2; ++i) blocks += p.blocks[i] = (rv.heads[i] + p.sh.hb - 1) / p.sh.hb;
  const int64_t tiles = std::max<int64_t>(((int64_t)tokens + (1 << p.sh.lt) - 1) >> p.sh.lt, 1);
  const int64_t most = std::max<int64_t>(16 * (int64_t)cu_count() / blocks, 1), chunks = std::min(tiles, most);
  p.tiles = (int32_t)((tiles + chunks - 1) / chunks);
  p.chunks = (int32_t)((tiles + p.tiles - 1) / p.tiles);
  return p;
}

template <int KIND>
void rotate(int dtype, const RotateArgs& a, unsigned grid, hipStream_t s) {
  if (dtype == LOCOCO_F32) rows_rotate_k<float, KIND><<<grid, kRotateThreads, 0, s>>>(a);
  else rows_rotate_k<__bf16, KIND><<<grid, kRotateThreads, 0, s>>>(a);
}
template <int KIND>
void rotate_back(int dtype, const RotateBackArgs& a, unsigned grid, hipStream_t s) {
  if (dtype == LOCOCO_F32) rows_rotate_back_k<float, KIND><<<grid, kRotateThreads, 0, s>>>(a);
  else rows_rotate_back_k<__bf16, KIND><<<grid, kRotateThreads, 0, s>>>(a);
}

// How the forward pass is laid out: all 256 / P rows of a workgroup at positions of their own and 16 heads in turn, where that fills the
// device; else a row each, one position and heads side by side.
struct RotatePlan { RotateShape sh; int32_t blocks[2]; int64_t groups; };
RotatePlan rotate_plan(const RotateView& rv, int32_t tokens) {
  RotatePlan p{};
  p.sh.lp = lanes_log(rv.d);
  const int32_t rows = kRotateThreads >> p.sh.lp;
  auto lay = [&](int32_t lt, int32_t hb) {
    p.sh.lt = lt;
    p.sh.hb = hb;
    for (int i = 0; i < 2; ++i) p.blocks[i] = (rv.heads[i] + hb - 1) / hb;
    p.groups = (((int64_t)tokens + (1 << lt) - 1) >> lt) * (p.blocks[0] + p.blocks[1]);
  };
  lay(8 - p.sh.lp, 16);
  if (p.groups < 2 * (int64_t)cu_count()) lay(0, rows);
  return p;
}

}  // namespace

bool rows_rotate_fits(const RotateView& rv, int32_t tokens) { return rotate_plan(rv, tokens).groups * kRotateThreads <= 0xffffffffll; }

hipError_t launch_rows_rotate(int dtype, RotateArgs a, hipStream_t s) {
  const RotatePlan p = rotate_plan(a.rv, a.tokens);
  a.sh = p.sh;
  a.blocks[0] = p.blocks[0];
  a.blocks[1] = p.blocks[1];
  const unsigned grid = (unsigned)p.groups;
  switch (pair_kind(a.rv.r, a.rv.adjacent)) {
    case kHalves4: rotate<kHalves4>(dtype, a, grid, s); break;
    case kHalves: rotate<kHalves>(dtype, a, grid, s); break;
    case kAdjacent: rotate<kAdjacent>(dtype, a, grid, s); break;
  }
  return hipGetLastError();
}

size_t rows_rotate_workspace_bytes(const RotateView& rv, int32_t tokens) {
  size_t most = 0;                               // of a call for both, and for either alone
  for (int only = 0; only < 3; ++only) {
    RotateView one = rv;
    if (only < 2) one.heads[only] = 0;
    if (one.heads[0] + one.heads[1] == 0) continue;
    const BackPlan p = back_plan(one, tokens);
    most = std::max(most, (size_t)(p.blocks[0] + p.blocks[1]) * p.chunks * rv.d * sizeof(float));
  }
  return most;
}

hipError_t launch_rows_rotate_backward(int dtype, RotateBackArgs a, void* workspace, hipStream_t s) {
  const BackPlan p = back_plan(a.rv, a.tokens);
  a.sh = p.sh;
  a.blocks[0] = p.blocks[0];
  a.blocks[1] = p.blocks[1];
  a.chunks = p.chunks;
  a.tiles = p.tiles;
  a.stretch = kBackRows / p.sh.hb;
  a.parts = (float*)workspace;
  const unsigned grid = (unsigned)((p.blocks[0] + p.blocks[1]) * p.chunks);
  switch (pair_kind(a.rv.r, a.rv.adjacent)) {
    case kHalves4: rotate_back<kHalves4>(dtype, a, grid, s); break;
    case kHalves: rotate_back<kHalves>(dtype, a, grid, s); break;
    case kAdjacent: rotate_back<kAdjacent>(dtype, a, grid, s); break;
  }
  if (a.gw[0] || a.gw[1]) {
    const unsigned banks = (unsigned)((a.rv.ws[0] ? a.rv.heads[0] : 1) + (a.rv.ws[1] ? a.rv.heads[1] : 1));
    rows_rotate_weights_k<<<banks * (unsigned)((a.rv.d + kWeightCols - 1) / kWeightCols), kWeightThreads, 0, s>>>(a);
  }
  return hipGetLastError();
}

}  // namespace lococo
