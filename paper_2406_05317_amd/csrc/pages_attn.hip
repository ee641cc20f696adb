// Attention over paged 4-bit rows: o = softmax(scale q K^T) V for the new rows of a batch of requests of different lengths.
#include "pages.h"

#include <type_traits>

namespace lococo {
namespace {

typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

constexpr float kLog2e = 1.4426950408889634f;

// the request a token of the call belongs to: the last one that begins at or before it
__device__ __forceinline__ int request_of(const int32_t* starts, int n, int32_t x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (starts[mid] <= x) lo = mid; else hi = mid;
  }
  return lo;
}

// ---------------------------------------------------------------------------------------------------------------------------------
// Any head_dim that is a multiple of 32: a wave to a query row, a lane to a key, vector arithmetic in fp32.
constexpr int kRowsWaves = 4;

template <typename T>
__global__ __launch_bounds__(64 * kRowsWaves) void pages_attn_rows_k(PagesAttnArgs a) {
  __shared__ float qs[kRowsWaves][kPagesMaxHeadDim], ps[kRowsWaves][64];
  __shared__ int64_t at[kRowsWaves][64];
  const int l = threadIdx.x & 63, w = threadIdx.x >> 6;
  const PagesView& pg = a.pg;
  const int32_t token = blockIdx.x * kRowsWaves + w, h = blockIdx.y, kvh = h / pg.group;
  if (token >= a.tokens) return;                 // nothing below meets the other waves
  const int req = request_of(a.starts, a.n, token);
  const int32_t stop = a.starts[req + 1];
  if (token >= stop) return;                     // behind the last request
  const int32_t held = min(max(a.held[req], 0), a.table_pages << pg.page_shift);
  const int32_t seen = max(held - (stop - token) + 1, 0);                   // rows the query sees
  const int32_t b = token / a.q.t, t = token - b * a.q.t;
  const T* q = (const T*)a.q.p + b * a.q.sb + h * a.q.sh + t * a.q.st;
  for (int i = l; i < pg.d; i += 64) qs[w][i] = (float)q[i] * (pg.scale * kLog2e);
  float m = -INFINITY, sum = 0.f;
  f32x2 acc[2] = {{0.f, 0.f}, {0.f, 0.f}};       // columns 2 (l + 64 i), + 1
  const int32_t* table = a.tables + (int64_t)req * a.table_pages;
  for (int32_t j0 = 0; j0 < seen; j0 += 64) {
    const int32_t j = j0 + l;
    const int32_t page = j < seen ? table[j >> pg.page_shift] : -1;
    const bool there = (uint32_t)page < (uint32_t)pg.n_pages;
    const int32_t row = j & (pg.page_rows - 1);
    const int64_t pr = ((int64_t)page * pg.Hkv + kvh) * pg.page_rows + row;
    float s = -INFINITY;
    if (there) {
      const u32x4* codes = (const u32x4*)(pg.k_codes + pr * (pg.d / 2));
      const uint8_t* scales = pg.k_scales + (pr - row) * (pg.d / 32) + row;
      s = 0.f;
      for (int c = 0; c < pg.d / 32; ++c) {
        const u32x4 x = codes[c];
        const float sc = __uint_as_float((uint32_t)scales[c * pg.page_rows] << 23);
        const float* y = qs[w] + 32 * c;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const f32x2 z[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(x[i], sc, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(x[i], sc, 1),
                              __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(x[i], sc, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(x[i], sc, 3)};
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            s = fmaf(z[k][0], y[8 * i + 2 * k], s);
            s = fmaf(z[k][1], y[8 * i + 2 * k + 1], s);
          }
        }
      }
    }
    float top = s;
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) top = fmaxf(top, __shfl_xor(top, k));
    const float ref = fmaxf(m, top), use = ref == -INFINITY ? 0.f : ref;    // nothing seen yet: 0 - (-inf) stays out of it
    const float keep = __builtin_amdgcn_exp2f(m - use), p = there ? __builtin_amdgcn_exp2f(s - use) : 0.f;
    m = ref;
    sum = sum * keep + p;
#pragma unroll
    for (int i = 0; i < 2; ++i) acc[i] = {acc[i][0] * keep, acc[i][1] * keep};
    ps[w][l] = p;
    at[w][l] = there ? pr : -1;
    __builtin_amdgcn_wave_barrier();
    const int32_t rows = min(seen - j0, 64);
    for (int r = 0; r < rows; ++r) {
      const int64_t vr = at[w][r];
      if (vr < 0) continue;
      const int32_t vrow = (j0 + r) & (pg.page_rows - 1);
      const float pr1 = ps[w][r];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int c = l + 64 * i;
        if (c < pg.d / 2) {
          const uint32_t x = pg.v_codes[vr * (pg.d / 2) + c];
          const float sc = __uint_as_float((uint32_t)pg.v_scales[(vr - vrow) * (pg.d / 32) + (c / 16) * pg.page_rows + vrow] << 23);
          const f32x2 z = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(x, sc, 0);
          acc[i] = {fmaf(pr1, z[0], acc[i][0]), fmaf(pr1, z[1], acc[i][1])};
        }
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) sum += __shfl_xor(sum, k);
  const int32_t ob = token / a.o.t, ot = token - ob * a.o.t;
  T* o = (T*)a.o.p + ob * a.o.sb + h * a.o.sh + ot * a.o.st;
  const float inv = sum == 0.f ? 0.f : 1.f / sum;                           // a row that sees nothing: zeros
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int c = l + 64 * i;
    if (c < pg.d / 2) {
      o[2 * c] = (T)(acc[i][0] * inv);
      o[2 * c + 1] = (T)(acc[i][1] * inv);
    }
  }
}

}  // namespace

size_t pages_attn_workspace_bytes(int dtype, const PagesAttnArgs& a) { return 0; }

hipError_t launch_pages_attn(int dtype, const PagesAttnArgs& a, void* workspace, hipStream_t s) {
  const dim3 grid((unsigned)((a.tokens + kRowsWaves - 1) / kRowsWaves), (unsigned)a.pg.Hq);
  if (dtype == LOCOCO_F32) pages_attn_rows_k<float><<<grid, 64 * kRowsWaves, 0, s>>>(a);
  else pages_attn_rows_k<__bf16><<<grid, 64 * kRowsWaves, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace lococo
