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
  int32_t tokens, blocks;                      // blocks of heads: q's, k's and v's, one after the other
  const int32_t* slots;
  const int32_t* positions;
};

// the fp32 number nearest to x towards zero, its last bit set where that is not x: rounding it to fewer bits is rounding x to them
__device__ __forceinline__ float to_odd(double x) {
  const float y = __double2float_rz(x);
  return (double)y == x || y != y ? y : __uint_as_float(__float_as_uint(y) | 1u);
}

// Keys go to 4 bits by the codes nearest to their exact values.  A value as fp32 arithmetic has it, off by some 2^-23, would now and then lie
// on the other side of a border between two codes: norm and rotation of keys are in 64 bits, and so are the cosines and sines (computed once
// for all heads of a position).  A workgroup takes 2^lt positions and a block of heads.  Bound by memory.
template <typename T, int KIND>
__global__ __launch_bounds__(kRotateThreads) void pages_append_k(AppendArgs a) {
  __shared__ double2 table[kRotateTable];
  const RotateView& rv = a.rv;
  const PagesView& pg = a.pg;
  const int32_t tile = blockIdx.x / a.blocks, blk = blockIdx.x - tile * a.blocks, all = pg.Hq + 2 * pg.Hkv;
  const int32_t h0 = blk * a.sh.hb, h1 = min(h0 + a.sh.hb, all);
  const int32_t lp = a.sh.lp, lt = a.sh.lt, grp = threadIdx.x >> lp, lane = threadIdx.x & ((1 << lp) - 1);
  const int32_t token0 = tile << lt, sub = grp & ((1 << lt) - 1), step = (kRotateThreads >> lp) >> lt, half = rv.r / 2;
  if (h0 < pg.Hq + pg.Hkv)                     // values are not turned
    for (int32_t i = threadIdx.x; i < half << lt; i += kRotateThreads) {
      const int32_t x = i / half, token = min(token0 + x, a.tokens - 1);
      double s, c;
      sincos((double)a.positions[token] * (double)rv.freqs[i - x * half], &s, &c);
      table[i] = make_double2(c, s);
    }
  __syncthreads();
  const int32_t token = min(token0 + sub, a.tokens - 1), slot = a.slots[token], pos = a.positions[token];
  const bool in = 8 * lane < rv.d, real = in && token0 + sub < a.tokens;
  const int32_t page = slot >> pg.page_shift, prow = slot & (pg.page_rows - 1);
  const bool placed = real && slot >= 0 && page < pg.n_pages;
  const Partners<KIND> pr{8 * lane, half, rv.r};
  for (int32_t hh = h0 + (grp >> lt); hh < h1; hh += step) {
    const int part = hh < pg.Hq ? 0 : hh < pg.Hq + pg.Hkv ? 1 : 2;
    const int32_t h = hh - (part == 0 ? 0 : part == 1 ? pg.Hq : pg.Hq + pg.Hkv);
    const bool active = part ? placed : real && pos >= 0;
    float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, p[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    const T* row = row_at<T>(part == 0 ? a.q : part == 1 ? a.k : a.v, active ? token : 0, h);
    if (active) read8(row + 8 * lane, x);
    if (part < 2) {
      if (active) pr.load(row, x, p);
      double y[8];
      double one = 1.0;
      if (rv.norm) {
        double sum = 0.0;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum = fma((double)x[i], (double)x[i], sum);
        one = 1.0 / sqrt(row_sum(sum, lp) / rv.d + (double)rv.eps);
      }
      float own[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f}, other[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
      const T* weights = (const T*)rv.w[part];
      if (weights && in) {
        const T* w = weights + h * rv.ws[part];
        read8(w + 8 * lane, own);
        pr.load(w, own, other);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        y[i] = (double)x[i] * (double)own[i] * one;
        if (pr.turned(i) && in) {
          const double2 v = table[sub * half + pr.pair(i)];
          const double z = (double)p[i] * (double)other[i] * one;
          y[i] = fma(y[i], v.x, pr.second(i) ? z * v.y : -z * v.y);
        }
      }
      if (part == 0) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = (float)y[i];
        if (active) write8(const_cast<T*>(row_at<T>(a.qo, token, h)) + 8 * lane, x);
        continue;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = to_odd(y[i]);
    }
    uint32_t byte;
    const uint32_t code = four_bits(x, &byte);
    if (!placed) continue;
    const int64_t at = (int64_t)page * pg.Hkv + h;
    *(uint32_t*)((part == 2 ? pg.v_codes : pg.k_codes) + (at * pg.page_rows + prow) * (pg.d / 2) + 4 * lane) = code;
    if ((lane & 3) == 0) (part == 2 ? pg.v_scales : pg.k_scales)[(at * (pg.d / 32) + lane / 4) * pg.page_rows + prow] = (uint8_t)byte;
  }
}

template <int KIND>
void append(int dtype, const AppendArgs& a, unsigned grid, hipStream_t s) {
  if (dtype == LOCOCO_F32) pages_append_k<float, KIND><<<grid, kRotateThreads, 0, s>>>(a);
  else pages_append_k<__bf16, KIND><<<grid, kRotateThreads, 0, s>>>(a);
}

RotateShape append_shape(const PagesView& pg) {
  RotateShape sh{};
  while (8 << sh.lp < pg.d) ++sh.lp;
  sh.lt = 0;
  sh.hb = 1 << (8 - sh.lp);
  return sh;
}
int64_t append_groups(const PagesView& pg, int32_t tokens) {
  const RotateShape sh = append_shape(pg);
  return (((int64_t)tokens + (1 << sh.lt) - 1) >> sh.lt) * ((pg.Hq + 2 * pg.Hkv + sh.hb - 1) / sh.hb);
}

}  // namespace

bool pages_append_fits(const PagesView& pg, int32_t tokens) { return append_groups(pg, tokens) * kRotateThreads <= 0xffffffffll; }

hipError_t launch_pages_append(int dtype, const PagesView& pg, const RotateView& rv, const RowsView& q, const RowsView& k, const RowsView& v,
                               const RowsView& qo, int32_t tokens, const int32_t* slots, const int32_t* positions, hipStream_t s) {
  AppendArgs a{pg, rv, append_shape(pg), q, k, v, qo, tokens, 0, slots, positions};
  a.blocks = (pg.Hq + 2 * pg.Hkv + a.sh.hb - 1) / a.sh.hb;
  const unsigned grid = (unsigned)append_groups(pg, tokens);
  switch (pair_kind(rv.r, rv.adjacent)) {
    case kHalves8: append<kHalves8>(dtype, a, grid, s); break;
    case kHalves: append<kHalves>(dtype, a, grid, s); break;
    case kAdjacent: append<kAdjacent>(dtype, a, grid, s); break;
  }
  return hipGetLastError();
}

}  // namespace lococo
