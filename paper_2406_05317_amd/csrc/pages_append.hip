// New rows into the pages: q rows normed and turned, k rows normed, turned and to 4 bits, v rows to 4 bits, in one pass.
#include "pages_codes.h"
#include "rotate.h"

#include <algorithm>

namespace lococo {
namespace {

using namespace rotate_detail;

struct AppendArgs {
  PagesView pg;
  RotateView rv;
  RotateShape sh;
  RowsView q, k, v, qo;
  int32_t tokens, blocks_q, blocks_kv;         // blocks of heads: q's, k's, v's
  const int32_t* slots;
  const int32_t* positions;
};

// an fp32 number whose rounding to fewer bits is x's: x rounded, its last bit set where that is not x (the neighbour on x's side, then)
__device__ __forceinline__ float to_odd(double x) {
  const float y = (float)x;
  const double e = x - (double)y;
  uint32_t bits = __float_as_uint(y);
  if ((e > 0.0 || e < 0.0) && !(bits & 1u)) bits += (e > 0.0) == (x > 0.0) ? 1u : 0xffffffffu;
  return __uint_as_float(bits);
}

// Keys go to 4 bits by the codes nearest to their exact values.  A value as fp32 arithmetic has it, off by some 2^-23, would now and then lie
// on the other side of a border between two codes: norm and rotation of keys are in 64 bits, and so are their cosines and sines (computed once
// for all heads of a position; vector instructions of 64 bits go as fast as those of 32).  A key's pairs lie half a row apart, its blocks of 32 do
// not: it goes through LDS on the way.  A workgroup takes 2^lt positions and a block of q's, k's or v's heads.
template <typename T, int KIND>
__global__ __launch_bounds__(kRotateThreads) void pages_append_k(AppendArgs a) {
  __shared__ double2 table[kRotateTable];
  __shared__ __align__(16) float turned[kRotateThreads * 8];
  const RotateView& rv = a.rv;
  const PagesView& pg = a.pg;
  const int32_t all = a.blocks_q + 2 * a.blocks_kv, tile = blockIdx.x / all, blk = blockIdx.x - tile * all;
  const int part = blk < a.blocks_q ? 0 : blk < a.blocks_q + a.blocks_kv ? 1 : 2;
  const int32_t h0 = (part == 0 ? blk : part == 1 ? blk - a.blocks_q : blk - a.blocks_q - a.blocks_kv) * a.sh.hb;
  const int32_t h1 = min(h0 + a.sh.hb, part ? pg.Hkv : pg.Hq);
  const int32_t lp = a.sh.lp, lt = a.sh.lt, grp = threadIdx.x >> lp, lane = threadIdx.x & ((1 << lp) - 1);
  const int32_t token0 = tile << lt, sub = grp & ((1 << lt) - 1), step = (kRotateThreads >> lp) >> lt, half = rv.r / 2;
  const int32_t token = min(token0 + sub, a.tokens - 1), slot = a.slots[token], pos = a.positions[token];
  const bool real = 8 * lane < rv.d && token0 + sub < a.tokens;
  const int32_t page = slot >> pg.page_shift, prow = slot & (pg.page_rows - 1);
  const bool active = part ? real && slot >= 0 && page < pg.n_pages : real && pos >= 0;
  auto write = [&](const float (&x)[8], int32_t h, uint8_t* codes, uint8_t* scales) {
    uint32_t byte;
    const uint32_t code = four_bits(x, &byte);
    if (!active) return;
    const int64_t at = (int64_t)page * pg.Hkv + h;
    *(uint32_t*)(codes + (at * pg.page_rows + prow) * (pg.d / 2) + 4 * lane) = code;
    if ((lane & 3) == 0) scales[(at * (pg.d / 32) + lane / 4) * pg.page_rows + prow] = (uint8_t)byte;
  };
  if (part == 2) {
    const T* row = row_at<T>(a.v, active ? token : 0, 0) + 8 * lane;
    for (int32_t h = h0 + (grp >> lt); h < h1; h += kAhead * step) {
      float x[kAhead][8];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[j][i] = 0.f;
        if (active && h + j * step < h1) read8(row + (h + j * step) * a.v.sh, x[j]);
      }
#pragma unroll
      for (int j = 0; j < kAhead; ++j)
        if (h + j * step < h1) write(x[j], h + j * step, pg.v_codes, pg.v_scales);
    }
    return;
  }
  const Pairs<KIND> pr{4 * lane, half, rv.r, rv.d};
  auto load = [&](const T* row, int64_t sh, int32_t h, float (&xa)[kAhead][4], float (&xb)[kAhead][4]) {
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
#pragma unroll
      for (int i = 0; i < 4; ++i) xa[j][i] = xb[j][i] = 0.f;
      if (active && h + j * step < h1) pr.load(row + (h + j * step) * sh, xa[j], xb[j]);
    }
  };
  const T* weights = (const T*)rv.w[part];
  const int64_t ws = rv.ws[part];
  float wa[4] = {1.f, 1.f, 1.f, 1.f}, wb[4] = {1.f, 1.f, 1.f, 1.f};
  if (weights && !ws && pr.in()) pr.load(weights, wa, wb);
  for (int32_t i = threadIdx.x; i < half << lt; i += kRotateThreads) {
    const int32_t x = i / half, p = a.positions[min(token0 + x, a.tokens - 1)];
    const float f = rv.freqs[i - x * half];
    if (part) {
      double s, c;
      sincos((double)p * (double)f, &s, &c);
      table[i] = make_double2(c, s);
    } else {
      float s, c;
      sincospif(half_turns(p, f), &s, &c);
      ((float2*)table)[i] = make_float2(c, s);
    }
  }
  __syncthreads();
  if (part == 0) {
    float c[4], s[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 v = pr.turned(i) ? ((const float2*)table)[sub * half + pr.q0 + i] : make_float2(1.f, 0.f);
      c[i] = v.x;
      s[i] = v.y;
    }
    const T* row = row_at<T>(a.q, active ? token : 0, 0);
    T* out = const_cast<T*>(row_at<T>(a.qo, active ? token : 0, 0));
    for (int32_t h = h0 + (grp >> lt); h < h1; h += kAhead * step) {
      float xa[kAhead][4], xb[kAhead][4];
      load(row, a.q.sh, h, xa, xb);
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const int32_t hj = h + j * step;
        if (hj >= h1) break;
        if (ws && pr.in()) pr.load(weights + hj * ws, wa, wb);
        const float one = rv.norm ? one_over_root(xa[j], xb[j], lp, rv) : 1.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float na = xa[j][i] * one * wa[i], nb = xb[j][i] * one * wb[i];
          xa[j][i] = fmaf(na, c[i], -nb * s[i]);
          xb[j][i] = fmaf(nb, c[i], na * s[i]);
        }
        if (active) pr.store(out + hj * a.qo.sh, xa[j], xb[j]);
      }
    }
    return;
  }
  double c[4], s[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const double2 v = pr.turned(i) ? table[sub * half + pr.q0 + i] : make_double2(1.0, 0.0);
    c[i] = v.x;
    s[i] = v.y;
  }
  const T* row = row_at<T>(a.k, active ? token : 0, 0);
  float* mine = turned + grp * rv.d;
  for (int32_t h = h0 + (grp >> lt); h < h1; h += kAhead * step) {
    float xa[kAhead][4], xb[kAhead][4];
    load(row, a.k.sh, h, xa, xb);
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int32_t hj = h + j * step;
      if (hj >= h1) break;
      if (ws && pr.in()) pr.load(weights + hj * ws, wa, wb);
      double one = 1.0;
      if (rv.norm) {
        double sum = 0.0;
#pragma unroll
        for (int i = 0; i < 4; ++i) sum = fma((double)xa[j][i], (double)xa[j][i], fma((double)xb[j][i], (double)xb[j][i], sum));
        one = 1.0 / sqrt(row_sum(sum, lp) / rv.d + (double)rv.eps);
      }
      if (pr.in())
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const double na = (double)xa[j][i] * (double)wa[i], nb = (double)xb[j][i] * (double)wb[i];
          mine[pr.first(i)] = to_odd(one * fma(na, c[i], -nb * s[i]));
          mine[pr.second(i)] = to_odd(one * fma(nb, c[i], na * s[i]));
        }
      __builtin_amdgcn_wave_barrier();           // a row's lanes share a wave
      float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      if (pr.in()) read8(mine + 8 * lane, x);
      __builtin_amdgcn_wave_barrier();
      write(x, hj, pg.k_codes, pg.k_scales);
    }
  }
}

template <int KIND>
void append(int dtype, const AppendArgs& a, unsigned grid, hipStream_t s) {
  if (dtype == LOCOCO_F32) pages_append_k<float, KIND><<<grid, kRotateThreads, 0, s>>>(a);
  else pages_append_k<__bf16, KIND><<<grid, kRotateThreads, 0, s>>>(a);
}

// As the forward pass of lococo_rows_rotate: positions side by side and heads in turn where that fills the device, else a row each.
struct AppendPlan { RotateShape sh; int32_t blocks_q, blocks_kv; int64_t groups; };
AppendPlan append_plan(const PagesView& pg, int32_t tokens) {
  AppendPlan p{};
  p.sh.lp = lanes_log(pg.d);
  auto lay = [&](int32_t lt, int32_t hb) {
    p.sh.lt = lt;
    p.sh.hb = hb;
    p.blocks_q = (pg.Hq + hb - 1) / hb;
    p.blocks_kv = (pg.Hkv + hb - 1) / hb;
    p.groups = (((int64_t)tokens + (1 << lt) - 1) >> lt) * (p.blocks_q + 2 * p.blocks_kv);
  };
  lay(8 - p.sh.lp, 16);
  if (p.groups < 2 * (int64_t)cu_count()) lay(0, kRotateThreads >> p.sh.lp);
  return p;
}

}  // namespace

bool pages_append_fits(const PagesView& pg, int32_t tokens) { return append_plan(pg, tokens).groups * kRotateThreads <= 0xffffffffll; }

hipError_t launch_pages_append(int dtype, const PagesView& pg, const RotateView& rv, const RowsView& q, const RowsView& k, const RowsView& v,
                               const RowsView& qo, int32_t tokens, const int32_t* slots, const int32_t* positions, hipStream_t s) {
  const AppendPlan p = append_plan(pg, tokens);
  AppendArgs a{pg, rv, p.sh, q, k, v, qo, tokens, p.blocks_q, p.blocks_kv, slots, positions};
  const unsigned grid = (unsigned)p.groups;
  switch (pair_kind(rv.r, rv.adjacent)) {
    case kHalves4: append<kHalves4>(dtype, a, grid, s); break;
    case kHalves: append<kHalves>(dtype, a, grid, s); break;
    case kAdjacent: append<kAdjacent>(dtype, a, grid, s); break;
  }
  return hipGetLastError();
}

}  // namespace lococo
