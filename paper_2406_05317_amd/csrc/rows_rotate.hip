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
    sincospif(half_turns(pos, rv.freqs[i - x * half]), &s, &c);
    table[i] = make_float2(c, s);
  }
}

// one over the root of a row's mean square where the squares leave fp32
__device__ __forceinline__ float one_of_large(const float (&x)[8], int32_t lp, const RotateView& rv) {
  double sum = 0.0;
#pragma unroll
  for (int i = 0; i < 8; ++i) sum = fma((double)x[i], (double)x[i], sum);
  return (float)(1.0 / sqrt(row_sum(sum, lp) / rv.d + rv.eps));
}

// A workgroup takes 2^lt positions and a block of q's or k's heads, (256 / P) >> lt of them at a time.  Bound by memory.
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
  const bool in = 8 * lane < rv.d, there = token < a.tokens && (!a.positions || a.positions[min(token, a.tokens - 1)] >= 0);
  const Partners<KIND> pr{8 * lane, rv.r / 2, rv.r};
  float c[8], s[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    c[i] = 1.f;
    s[i] = 0.f;
    if (in && pr.turned(i)) {
      const float2 v = table[sub * (rv.r / 2) + pr.pair(i)];
      c[i] = v.x;
      s[i] = pr.second(i) ? v.y : -v.y;
    }
  }
  const T* weights = (const T*)rv.w[part];
  const bool active = in && there;
  for (int32_t h = h0 + (grp >> lt); h < h1; h += step) {
    float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, p[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    const T* row = row_at<T>(a.in[part], active ? token : 0, h);
    if (active) {
      read8(row + 8 * lane, x);
      pr.load(row, x, p);
    }
    if (rv.norm) {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) sum = fmaf(x[i], x[i], sum);
      sum = row_sum(sum, lp);
      float one = 1.f / sqrtf(sum / (float)rv.d + rv.eps);
      if (sum == INFINITY) one = one_of_large(x, lp, rv);
      if (weights && in) {
        const T* w = weights + h * rv.ws[part];
        float own[8], other[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        read8(w + 8 * lane, own);
        pr.load(w, own, other);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          x[i] *= one;
          x[i] *= own[i];
          p[i] *= one;
          p[i] *= other[i];
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          x[i] *= one;
          p[i] *= one;
        }
      }
    }
    if (active) {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = pr.turned(i) ? fmaf(x[i], c[i], p[i] * s[i]) : x[i];
      write8(const_cast<T*>(row_at<T>(a.out[part], token, h)) + 8 * lane, x);
    }
  }
}

// The way back: g_n = the upstream gradient turned the other way; with xhat = x * one, one = 1 / sqrt(mean(x^2) + eps),
//   d_w += g_n xhat (over all rows),  d_x = one * (w g_n - xhat mean(w g_n xhat)).
// Both means are sums over the row taken side by side.  A workgroup adds up its rows' part of d_w in registers, once over its rows in LDS at
// the end, and leaves it for rows_rotate_weights_k: no atomics, the same bits every time.  Bound by memory.
template <typename T, int KIND>
__global__ __launch_bounds__(kRotateThreads) void rows_rotate_back_k(RotateBackArgs a) {
  __shared__ float2 table[kRotateTable];
  __shared__ float gws[kRotateThreads * 8];
  const RotateView& rv = a.rv;
  const int32_t blk = blockIdx.x / a.chunks, chunk = blockIdx.x - blk * a.chunks;
  const int part = blk >= a.blocks[0];
  const int32_t h0 = (blk - (part ? a.blocks[0] : 0)) * a.sh.hb, h1 = min(h0 + a.sh.hb, rv.heads[part]);
  const int32_t lp = a.sh.lp, lt = a.sh.lt, grp = threadIdx.x >> lp, lane = threadIdx.x & ((1 << lp) - 1);
  const int32_t sub = grp & ((1 << lt) - 1), step = (kRotateThreads >> lp) >> lt;
  const bool in = 8 * lane < rv.d;
  const Partners<KIND> pr{8 * lane, rv.r / 2, rv.r};
  const T* weights = (const T*)rv.w[part];
  float gw[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  for (int32_t k = 0; k < a.tiles; ++k) {
    const int64_t first = ((int64_t)chunk * a.tiles + k) << lt;
    if (first >= a.tokens) break;              // the same for all lanes
    const int32_t token0 = (int32_t)first, token = token0 + sub;
    __syncthreads();                           // the last tile's table has been read
    fill_table(table, rv, a.positions, a.tokens, a.t, token0, lt);
    __syncthreads();
    const bool real = token < a.tokens, there = real && (!a.positions || a.positions[token] >= 0);
    float c[8], s[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      c[i] = 1.f;
      s[i] = 0.f;
      if (in && pr.turned(i)) {
        const float2 v = table[sub * (rv.r / 2) + pr.pair(i)];
        c[i] = v.x;
        s[i] = pr.second(i) ? -v.y : v.y;
      }
    }
    const int32_t b = real ? token / a.t : 0, t = real ? token - b * a.t : 0;
    for (int32_t h = h0 + (grp >> lt); h < h1; h += step) {
      const int64_t at = (((int64_t)b * rv.heads[part] + h) * a.t + t) * rv.d;
      float g[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, p[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      const bool active = in && there;
      if (active) {
        const float* gy = a.gy[part] + at;
        read8(gy + 8 * lane, g);
        pr.load(gy, g, p);
#pragma unroll
        for (int i = 0; i < 8; ++i) g[i] = pr.turned(i) ? fmaf(g[i], c[i], p[i] * s[i]) : g[i];
      }
      if (rv.norm) {
        float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, w[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
        if (active) read8(row_at<T>(a.in[part], token, h) + 8 * lane, x);
        if (weights && in) read8(weights + h * rv.ws[part] + 8 * lane, w);
        float sq = 0.f, dot = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          sq = fmaf(x[i], x[i], sq);
          dot = fmaf(w[i] * g[i], x[i], dot);
        }
        sq = row_sum(sq, lp);
        dot = row_sum(dot, lp);
        float one = 1.f / sqrtf(sq / (float)rv.d + rv.eps);
        if (sq == INFINITY) one = one_of_large(x, lp, rv);
        float mean = one * dot / (float)rv.d;
        if (sq == INFINITY) {                  // so may the other sum have been
          dot = 0.f;
#pragma unroll
          for (int i = 0; i < 8; ++i) dot = fmaf(w[i] * g[i], x[i] * one, dot);
          mean = row_sum(dot, lp) / (float)rv.d;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float hat = x[i] * one;
          gw[i] = fmaf(g[i], hat, gw[i]);
          g[i] = one * fmaf(w[i], g[i], -hat * mean);
        }
      }
      if (in && real) write8(a.gx[part] + at + 8 * lane, g);                  // a row of nobody: zeros
    }
  }
  if (!a.gw[part]) return;
  float* mine = gws + (grp * rv.d + 8 * lane);
  if (in)
#pragma unroll
    for (int i = 0; i < 8; ++i) mine[i] = gw[i];
  __syncthreads();
  for (int32_t c = threadIdx.x; c < rv.d; c += kRotateThreads) {
    float sum = 0.f;
    for (int32_t k = 0; k < kRotateThreads >> lp; ++k) sum += gws[k * rv.d + c];
    a.parts[((int64_t)blk * a.chunks + chunk) * rv.d + c] = sum;
  }
}

// The parts of a weight's gradient to one, in a fixed order, and onto what is there: a workgroup to a bank of weights.
__global__ __launch_bounds__(1024) void rows_rotate_weights_k(RotateBackArgs a) {
  __shared__ float sums[1024];
  const RotateView& rv = a.rv;
  // banks: q's (one, or one a head), then k's
  const int32_t banks = rv.ws[0] ? rv.heads[0] : 1;
  const int part = (int32_t)blockIdx.x >= banks;
  const int32_t head = blockIdx.x - (part ? banks : 0);
  if (!a.gw[part]) return;
  const int32_t first = (part ? a.blocks[0] : 0) + (rv.ws[part] ? head : 0), rows = (rv.ws[part] ? 1 : a.blocks[part]) * a.chunks;
  const float* at = a.parts + (int64_t)first * a.chunks * rv.d;
  const int32_t side = 1024 / rv.d, k = threadIdx.x / rv.d, c = threadIdx.x - k * rv.d;
  float sum = 0.f;
  if (k < side)
    for (int32_t i = k; i < rows; i += side) sum += at[(int64_t)i * rv.d + c];
  sums[threadIdx.x] = sum;
  __syncthreads();
  if (threadIdx.x >= rv.d) return;
  sum = 0.f;
  for (int32_t i = 0; i < side; ++i) sum += sums[i * rv.d + threadIdx.x];
  a.gw[part][head * rv.ws[part] + threadIdx.x] += sum;
}

int32_t lanes_log(int32_t d) {
  int32_t lp = 0;
  while (8 << lp < d) ++lp;
  return lp;
}

struct BackPlan { RotateShape sh; int32_t blocks[2], chunks, tiles; };
BackPlan back_plan(const RotateView& rv, int32_t tokens) {
  BackPlan p{};
  p.sh.lp = lanes_log(rv.d);
  p.sh.lt = 8 - p.sh.lp;                       // positions alone: a workgroup's rows of a head lie side by side
  const bool banks = rv.ws[0] || rv.ws[1];
  p.sh.hb = banks ? 1 : 8;
  int64_t blocks = 0;
  for (int i = 0; i < 2; ++i) blocks += p.blocks[i] = (rv.heads[i] + p.sh.hb - 1) / p.sh.hb;
  const int64_t tiles = std::max<int64_t>(((int64_t)tokens + (1 << p.sh.lt) - 1) >> p.sh.lt, 1);
  const int64_t most = std::max<int64_t>(8 * (int64_t)cu_count() / blocks, 1), chunks = std::min(tiles, most);
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
// workgroups of the forward pass: blocks of eight heads
int64_t rotate_groups(const RotateView& rv, int32_t tokens) {
  const int64_t tile = 1 << (8 - lanes_log(rv.d));
  return (tokens + tile - 1) / tile * ((rv.heads[0] + 7) / 8 + (rv.heads[1] + 7) / 8);
}

}  // namespace

bool rows_rotate_fits(const RotateView& rv, int32_t tokens) { return rotate_groups(rv, tokens) * kRotateThreads <= 0xffffffffll; }

hipError_t launch_rows_rotate(int dtype, RotateArgs a, hipStream_t s) {
  a.sh.lp = lanes_log(a.rv.d);
  a.sh.lt = 8 - a.sh.lp;
  a.sh.hb = 8;
  for (int i = 0; i < 2; ++i) a.blocks[i] = (a.rv.heads[i] + a.sh.hb - 1) / a.sh.hb;
  const unsigned grid = (unsigned)rotate_groups(a.rv, a.tokens);
  switch (pair_kind(a.rv.r, a.rv.adjacent)) {
    case kHalves8: rotate<kHalves8>(dtype, a, grid, s); break;
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
  a.parts = (float*)workspace;
  const unsigned grid = (unsigned)((p.blocks[0] + p.blocks[1]) * p.chunks);
  switch (pair_kind(a.rv.r, a.rv.adjacent)) {
    case kHalves8: rotate_back<kHalves8>(dtype, a, grid, s); break;
    case kHalves: rotate_back<kHalves>(dtype, a, grid, s); break;
    case kAdjacent: rotate_back<kAdjacent>(dtype, a, grid, s); break;
  }
  if (a.gw[0] || a.gw[1]) {
    const unsigned banks = (unsigned)((a.rv.ws[0] ? a.rv.heads[0] : 1) + (a.rv.ws[1] ? a.rv.heads[1] : 1));
    rows_rotate_weights_k<<<banks, 1024, 0, s>>>(a);
  }
  return hipGetLastError();
}

}  // namespace lococo
