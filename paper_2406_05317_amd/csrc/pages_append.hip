// New rows into the pages: q rows normed and turned, k rows normed, turned and to 4 bits, v rows to 4 bits, in one pass.
#include "pages_codes.h"
#include "rotate.h"

#include <algorithm>

namespace lococo {
namespace {

using namespace rotate_detail;

typedef __attribute__((ext_vector_type(4))) float f4;

struct AppendArgs {
  PagesView pg;
  RotateView rv;
  RotateShape sh;
  RowsView q, k, v, qo;
  int32_t tokens, tiles, blocks_q, blocks_kv;  // tiles of positions; blocks of q's heads, of k's and v's
  const int32_t* slots;
  const int32_t* positions;
};

// Borders between codes, and between scales, have three bits behind the first: an fp32 number with others decides as the value it was rounded
// from.  One without takes the neighbour on that value's side, unless it is that value.
__device__ __forceinline__ bool may_be_border(float y) { return (__float_as_uint(y) << 12) == 0 && y != 0.f; }
__device__ __forceinline__ float off_border(float y, double x) {
  const double e = x - (double)y;
  const uint32_t bits = __float_as_uint(y);
  return may_be_border(y) && (e > 0.0 || e < 0.0) ? __uint_as_float(bits + ((e > 0.0) == (x > 0.0) ? 1u : 0xffffffffu)) : y;
}

// Keys go to 4 bits by the codes nearest to their exact values.  A value as fp32 arithmetic has it, off by some 2^-23, would now and then lie
// on the other side of a border between two codes: norm and rotation of keys are in 64 bits, and so are their cosines and sines (computed once
// for all heads of a position; vector instructions of 64 bits go as fast as those of 32).  A key's pairs lie half a row apart, its blocks of 32 do
// not: it goes through LDS on the way.  A workgroup takes 2^lt positions and a block of q's, k's or v's heads, a lane's rows two at a time,
// the next two on their way.  8186 prompt rows of 32 heads, bf16: 304 MB in 83 us (3.7 TB/s; a large copy 5.1), of it q alone 37, v 20, k 47: keys
// wait for their chain of 64-bit arithmetic, LDS and conversion, with four waves to a SIMD by their registers (five spill: 181 us).  Keys' workgroups,
// the longest, go first (92 us mixed with the others).  With norm and weights 97 us; fp32 rows, 571 MB, 138 us and 144.  32 tokens: 5 us, three
// trips to memory and the functions of 64 bits.
template <typename T, int KIND>
__global__ __launch_bounds__(kRotateThreads, KIND == kHalves ? 3 : 4) void pages_append_k(AppendArgs a) {
  __shared__ double2 table[kRotateTable];
  __shared__ __align__(16) float turned[kRotateThreads * 8];
  const RotateView& rv = a.rv;
  const PagesView& pg = a.pg;
  // keys, which take longest, ahead of the others
  const int32_t blk = blockIdx.x / a.tiles, tile = blockIdx.x - blk * a.tiles;
  const int part = blk < a.blocks_kv ? 1 : blk < a.blocks_kv + a.blocks_q ? 0 : 2;
  const int32_t h0 = (part == 1 ? blk : part == 0 ? blk - a.blocks_kv : blk - a.blocks_q - a.blocks_kv) * a.sh.hb;
  const int32_t h1 = min(h0 + a.sh.hb, part ? pg.Hkv : pg.Hq);
  const int32_t lp = a.sh.lp, lt = a.sh.lt, grp = threadIdx.x >> lp, lane = threadIdx.x & ((1 << lp) - 1);
  const int32_t token0 = tile << lt, sub = grp & ((1 << lt) - 1), step = (kRotateThreads >> lp) >> lt, half = rv.r / 2;
  const int32_t token = min(token0 + sub, a.tokens - 1), slot = a.slots[token], pos = a.positions[token];
  const bool real = 8 * lane < rv.d && token0 + sub < a.tokens;
  const int32_t page = slot >> pg.page_shift, prow = slot & (pg.page_rows - 1);
  const bool active = part ? real && slot >= 0 && page < pg.n_pages : real && pos >= 0;
  // where a lane's codes go, head h0's, and its block's scale; from there by heads
  const int64_t at = ((int64_t)(active ? page : 0) * pg.Hkv + h0 + (grp >> lt)) * pg.page_rows;
  uint8_t* codes = (part == 2 ? pg.v_codes : pg.k_codes) + (at + prow) * (pg.d / 2) + 4 * lane;
  uint8_t* scales = (part == 2 ? pg.v_scales : pg.k_scales) + at * (pg.d / 32) + lane / 4 * pg.page_rows + prow;
  const int32_t codes_on = step * pg.page_rows * (pg.d / 2), scales_on = step * pg.page_rows * (pg.d / 32);
  auto write = [&](const float (&x)[8]) {      // the next head's
    uint32_t byte;
    const uint32_t code = four_bits(x, &byte);
    if (active) {
      *(uint32_t*)codes = code;
      if ((lane & 3) == 0) *scales = (uint8_t)byte;
    }
    codes += codes_on;
    scales += scales_on;
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
        if (h + j * step < h1) write(x[j]);
    }
    return;
  }
  const Pairs<KIND> pr{4 * lane, half, rv.r, rv.d};
  RawPairs<T, KIND> raw[kAhead] = {};          // rows that are left out stay zeros
  auto load = [&](const T* row, int64_t sh, int32_t h) {
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
      if (active && h + j * step < h1) pr.load(row + (h + j * step) * sh, raw[j]);
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
      sincospi(half_turns(p, f), &s, &c);
      table[i] = make_double2(c, s);
    } else {
      float s, c;
      cos_sin(p, f, &c, &s);
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
    load(row, a.q.sh, h0 + (grp >> lt));
    for (int32_t h = h0 + (grp >> lt); h < h1; h += kAhead * step) {
      float xa[kAhead][4], xb[kAhead][4];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) pr.unpack(raw[j], xa[j], xb[j]);
      load(row, a.q.sh, h + kAhead * step);     // the next ones, while these are at work
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
  const T* row = row_at<T>(a.k, active ? token : 0, 0);
  float* mine = turned + grp * rv.d;
  load(row, a.k.sh, h0 + (grp >> lt));
  for (int32_t h = h0 + (grp >> lt); h < h1; h += kAhead * step) {
    RawPairs<T, KIND> now[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) now[j] = raw[j];
    load(row, a.k.sh, h + kAhead * step);
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int32_t hj = h + j * step;
      if (hj >= h1) break;
      float xa[4], xb[4];
      pr.unpack(now[j], xa, xb);
      if (ws && pr.in()) pr.load(weights + hj * ws, wa, wb);
      double one = 1.0;
      if (rv.norm) {
        double sum = 0.0;
#pragma unroll
        for (int i = 0; i < 4; ++i) sum = fma((double)xa[i], (double)xa[i], fma((double)xb[i], (double)xb[i], sum));
        one = 1.0 / sqrt(row_sum(sum, lp) / rv.d + (double)rv.eps);
      }
      double na[4], nb[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        na[i] = xa[i];
        nb[i] = xb[i];
      }
      if (weights)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          na[i] *= (double)wa[i];
          nb[i] *= (double)wb[i];
        }
      bool border = false;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const double2 v = pr.turned(i) ? table[sub * half + pr.q0 + i] : make_double2(1.0, 0.0);
        const double ya = fma(na[i], v.x, -nb[i] * v.y), yb = fma(nb[i], v.x, na[i] * v.y);
        na[i] = rv.norm ? one * ya : ya;
        nb[i] = rv.norm ? one * yb : yb;
        xa[i] = (float)na[i];
        xb[i] = (float)nb[i];
        border |= may_be_border(xa[i]) || may_be_border(xb[i]);
      }
      if (border)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          xa[i] = off_border(xa[i], na[i]);
          xb[i] = off_border(xb[i], nb[i]);
        }
      if (pr.in())
#pragma unroll
        for (int i = 0; i < (KIND == kHalves4 ? 1 : 4); ++i) {
          if constexpr (KIND == kHalves4) {
            *(f4*)(mine + pr.first(0)) = f4{xa[0], xa[1], xa[2], xa[3]};
            *(f4*)(mine + pr.second(0)) = f4{xb[0], xb[1], xb[2], xb[3]};
          } else {
            mine[pr.first(i)] = xa[i];
            mine[pr.second(i)] = xb[i];
          }
        }
      __builtin_amdgcn_wave_barrier();           // a row's lanes share a wave
      float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      if (pr.in()) {
        const f4 lo = *(const f4*)(mine + 8 * lane), hi = *(const f4*)(mine + 8 * lane + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[i] = lo[i];
          x[4 + i] = hi[i];
        }
      }
      __builtin_amdgcn_wave_barrier();
      write(x);
    }
  }
}

template <int KIND>
void append(int dtype, const AppendArgs& a, unsigned grid, hipStream_t s) {
  if (dtype == LOCOCO_F32) pages_append_k<float, KIND><<<grid, kRotateThreads, 0, s>>>(a);
  else pages_append_k<__bf16, KIND><<<grid, kRotateThreads, 0, s>>>(a);
}

// As the forward pass of lococo_rows_rotate: positions side by side and heads in turn where that fills the device, else a row each.
struct AppendPlan { RotateShape sh; int32_t tiles, blocks_q, blocks_kv; int64_t groups; };
AppendPlan append_plan(const PagesView& pg, int32_t tokens) {
  AppendPlan p{};
  p.sh.lp = lanes_log(pg.d);
  auto lay = [&](int32_t lt, int32_t hb) {
    p.sh.lt = lt;
    p.sh.hb = hb;
    p.blocks_q = (pg.Hq + hb - 1) / hb;
    p.blocks_kv = (pg.Hkv + hb - 1) / hb;
    p.tiles = (int32_t)(((int64_t)tokens + (1 << lt) - 1) >> lt);
    p.groups = (int64_t)p.tiles * (p.blocks_q + 2 * p.blocks_kv);
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
  AppendArgs a{pg, rv, p.sh, q, k, v, qo, tokens, p.tiles, p.blocks_q, p.blocks_kv, slots, positions};
  const unsigned grid = (unsigned)p.groups;
  switch (pair_kind(rv.r, rv.adjacent)) {
    case kHalves4: append<kHalves4>(dtype, a, grid, s); break;
    case kHalves: append<kHalves>(dtype, a, grid, s); break;
    case kAdjacent: append<kAdjacent>(dtype, a, grid, s); break;
  }
  return hipGetLastError();
}

}  // namespace lococo
