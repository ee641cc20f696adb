// The plan of a turn over paged requests, and rows to 4 bits and back.
#include "pages.h"

#include <type_traits>

namespace lococo {
namespace {

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(4), aligned(4))) float f32x4_any;      // fp32 rows begin at any float

// ---------------------------------------------------------------------------------------------------------------------------------
// Plan.  Three running sums over the requests give every row's place: of the new rows (where a request's rows begin in the call), of
// the pages needed (which of the free ones are whose) and of the pages given back.  Every workgroup computes them all, n numbers from
// the L2, and places a share of the rows, one a lane where the device holds that many: no workgroup waits for another, and one launch
// does.  What this call writes no part of it reads: a request's new table entries lie behind the ones it reads, what is given back goes
// to the ring behind its free part.
// Sums saturate at kPagesCap (addition cut off at a bound is associative for numbers >= 0): lengths that make no sense stay sums that
// refuse.  Bound by the launch and some three round trips to memory: 5.3 us for 32 requests with a row each, 7.8 us for 512 with 52 K rows.
constexpr int kPlanThreads = 256;

__device__ __forceinline__ int32_t add_cap(int32_t a, int32_t b) { return min(a + b, kPagesCap); }

// exclusive running sums of two numbers a thread over the workgroup; the totals in *t0, *t1
__device__ __forceinline__ void scan_two(int32_t& x0, int32_t& x1, int32_t* t0, int32_t* t1, int32_t (*part)[2]) {
  const int tid = threadIdx.x, l = tid & 63, w = tid >> 6;
  int32_t s0 = x0, s1 = x1;
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) {
    const int32_t y0 = __shfl_up(s0, k), y1 = __shfl_up(s1, k);
    if (l >= k) {
      s0 = add_cap(s0, y0);
      s1 = add_cap(s1, y1);
    }
  }
  int32_t e0 = __shfl_up(s0, 1), e1 = __shfl_up(s1, 1);
  if (l == 0) e0 = e1 = 0;
  __syncthreads();                               // the last sum's parts have been read
  if (l == 63) {
    part[w][0] = s0;
    part[w][1] = s1;
  }
  __syncthreads();
  int32_t b0 = 0, b1 = 0, a0 = 0, a1 = 0;
#pragma unroll
  for (int k = 0; k < kPlanThreads / 64; ++k) {
    if (k == w) { b0 = a0; b1 = a1; }
    a0 = add_cap(a0, part[k][0]);
    a1 = add_cap(a1, part[k][1]);
  }
  x0 = add_cap(b0, e0);
  x1 = add_cap(b1, e1);
  *t0 = a0;
  *t1 = a1;
}

__global__ __launch_bounds__(kPlanThreads) void pages_plan_k(PagesPlanArgs a) {
  extern __shared__ int32_t lists[];
  __shared__ int32_t part[kPlanThreads / 64][2], sums[3];
  int32_t* start = lists;                        // first row of a request in the call
  int32_t* held = lists + a.n;                   // rows it holds; -1 - rows where it ends
  int32_t* off = lists + 2 * a.n;                // its first page among those taken (-1: refused), or given back
  const int tid = threadIdx.x, n = a.n, R = a.page_rows, sh = a.page_shift;
  const int per = (n + kPlanThreads - 1) / kPlanThreads, i0 = min(tid * per, n), i1 = min(i0 + per, n);
  const int32_t most = a.table_pages << sh;      // rows a table has room for
  if (tid < 3) sums[tid] = 0;

  int32_t mine = 0, none = 0, rows, unused;
  for (int i = i0; i < i1; ++i) {
    const int32_t w = a.new_rows[i], h = min(max(a.held[i], 0), most);
    held[i] = w < 0 ? -1 - h : h;
    start[i] = min(max(w, 0), kPagesCap);        // the number of rows, for now
    mine = add_cap(mine, start[i]);
  }
  scan_two(mine, none, &rows, &unused, part);
  int32_t want = 0, give = 0;
  for (int i = i0, at = mine; i < i1; ++i) {
    const int32_t cnt = start[i], h = held[i];
    start[i] = at;
    at = add_cap(at, cnt);
    if (h < 0) {
      give = add_cap(give, (-1 - h + R - 1) >> sh);
    } else {
      const int32_t after = (h + cnt + R - 1) >> sh;
      if (at <= a.tokens && after <= a.table_pages) want = add_cap(want, after - ((h + R - 1) >> sh));
    }
  }
  int32_t all_want, all_give;
  scan_two(want, give, &all_want, &all_give, part);
  const int64_t head = a.ends[0], tail = a.ends[1];
  const int32_t avail = (int32_t)min(max(tail - head, (int64_t)0), (int64_t)a.n_pages);
  int32_t taken = 0, refused = 0, laid = 0;
  for (int i = i0; i < i1; ++i) {
    const int32_t h = held[i];
    if (h < 0) {
      off[i] = give;
      give = add_cap(give, (-1 - h + R - 1) >> sh);
      continue;
    }
    const int32_t cnt = (i + 1 < n ? start[i + 1] : rows) - start[i];       // written ahead of the second sum's barriers
    const int32_t after = (h + cnt + R - 1) >> sh;
    const bool fits = add_cap(start[i], cnt) <= a.tokens && after <= a.table_pages;
    const int32_t need = fits ? after - ((h + R - 1) >> sh) : 0;
    const bool ok = fits && (need == 0 || add_cap(want, need) <= avail);
    off[i] = ok ? want : -1;
    want = add_cap(want, need);
    if (blockIdx.x == 0) {
      taken += ok ? need : 0;
      laid += ok ? cnt : 0;
      refused += !ok;
      a.held_after[i] = ok ? h + cnt : h;
    }
  }
  if (blockIdx.x == 0) {
    for (int i = i0; i < i1; ++i) {
      a.starts[i] = min(start[i], a.tokens);
      if (held[i] < 0) a.held_after[i] = 0;
    }
    if (taken) atomicAdd(&sums[0], taken);       // whole numbers: any order gives the same
    if (laid) atomicAdd(&sums[1], laid);
    if (refused) atomicAdd(&sums[2], refused);
  }
  __syncthreads();
  if (blockIdx.x == 0 && tid == 0) {
    a.starts[n] = min(rows, a.tokens);
    a.ends_after[0] = head + sums[0];
    a.ends_after[1] = tail + all_give;
    a.totals[0] = sums[1];
    a.totals[1] = sums[0];
    a.totals[2] = all_give;
    a.totals[3] = sums[2];
  }
  const int32_t P = a.n_pages, head_at = (int32_t)(((head % P) + P) % P), tail_at = (int32_t)(((tail % P) + P) % P);
  for (int64_t x = blockIdx.x * kPlanThreads + tid; x < a.tokens; x += gridDim.x * kPlanThreads) {
    int32_t slot = -1, pos = -1;
    if (x < rows) {
      int lo = 0, hi = n;                        // the last request that begins at or before row x: requests without rows begin with
      while (hi - lo > 1) {                      // the one behind them
        const int mid = (lo + hi) >> 1;
        if (start[mid] <= x) lo = mid; else hi = mid;
      }
      const int32_t h = held[lo], o = off[lo];
      if (h >= 0 && o >= 0) {
        pos = h + (int32_t)x - start[lo];
        const int32_t j = pos >> sh, had = (h + R - 1) >> sh;
        int32_t page;
        if (j < had) {
          page = a.tables[(int64_t)lo * a.table_pages + j];
        } else {
          const int64_t r = (int64_t)head_at + o + (j - had);
          page = a.ring[r >= P ? r - P : r];
          if ((pos & (R - 1)) == 0) a.tables[(int64_t)lo * a.table_pages + j] = page;   // the row that opens it enters it
        }
        if ((uint32_t)page < (uint32_t)P) slot = (page << sh) + (pos & (R - 1));
      }
    }
    a.slots[x] = slot;
    a.positions[x] = pos;
  }
  // pages given back: a wave to a request
  const int waves = gridDim.x * (kPlanThreads / 64);
  for (int i = blockIdx.x * (kPlanThreads / 64) + (tid >> 6); i < n; i += waves) {
    if (held[i] >= 0) continue;
    const int32_t pages = (-1 - held[i] + R - 1) >> sh;
    for (int32_t j = tid & 63; j < pages; j += 64)
      a.ring[((int64_t)tail_at + off[i] + j) % P] = a.tables[(int64_t)i * a.table_pages + j];
  }
}

// ---------------------------------------------------------------------------------------------------------------------------------
// Rows to 4 bits.  A block of 32 values has the scale 2^E, E = floor(log2 of the largest magnitude) - 2, one more where that magnitude
// exceeds 1.75 times its power of two: then no value is more than 7 steps of the scale, and the largest code, 6, is off by no more than
// half a step of its own binade.  x 2^-E is exact and the conversion rounds to the nearest code, ties to even, so the codes follow from
// the values alone.  Four lanes share a block, eight values each: every access is contiguous over a row; a lane takes a row's K and V, two
// requests on their way instead of one (2048 rows of 32 heads there and back 22.4 us with a lane to either, 20.1 so).  Bound by memory: 42 MB
// in 10.5 us stored, 9.4 us loaded (4.0 and 4.5 TB/s; a large copy 5.1).
constexpr int kRowThreads = 256;
constexpr int32_t kMinExp = -100, kMaxExp = 125;     // of a scale: blocks of nothing but smaller values are zeros; 6 times it is finite

template <typename T>
__device__ __forceinline__ void read8(const T* p, float (&x)[8]) {
  if constexpr (std::is_same<T, float>::value) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const f32x4_any v = *(const f32x4_any*)(p + 4 * i);
#pragma unroll
      for (int k = 0; k < 4; ++k) x[4 * i + k] = v[k];
    }
  } else {
    const u32x4 v = *(const u32x4*)p;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(v[i] << 16);
      x[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
    }
  }
}

template <typename T>
__device__ __forceinline__ const T* row_of(const RowsView& r, int32_t token, int32_t head) {
  const int32_t b = token < r.t ? 0 : token / r.t, t = token - b * r.t;
  return (const T*)r.p + b * r.sb + head * r.sh + t * r.st;
}

template <typename T>
__global__ __launch_bounds__(kRowThreads) void pages_store_k(PagesView pg, RowsView k, RowsView v, int32_t tokens, const int32_t* slots) {
  const int32_t token = blockIdx.x * blockDim.y + threadIdx.y, c = threadIdx.x, head = blockIdx.y;
  if (token >= tokens) return;                   // the four lanes of a block leave together
  const int32_t slot = slots[token];
  const int32_t page = slot >> pg.page_shift, row = slot & (pg.page_rows - 1);
  if (slot < 0 || page >= pg.n_pages) return;
  float x[2][8];
  read8(row_of<T>(k, token, head) + 8 * c, x[0]);
  read8(row_of<T>(v, token, head) + 8 * c, x[1]);
  const int64_t at = (int64_t)page * pg.Hkv + head;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    uint32_t top = 0;                            // magnitudes as whole numbers: their order, with infinities and NaN on top
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[j][i]) & 0x7fffffffu);
    top = max(top, (uint32_t)__shfl_xor((int)top, 1));
    top = max(top, (uint32_t)__shfl_xor((int)top, 2));
    const int32_t e = (int32_t)(top >> 23) - 127 - 2 + ((top & 0x7fffffu) > 0x600000u);
    const uint32_t byte = top >= 0x7f800000u ? 255u : (uint32_t)(min(max(e, kMinExp), kMaxExp) + 127);
    uint32_t code = 0;
    if (byte != 255u) {
      const float s = __uint_as_float(byte << 23);
      code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[j][0], x[j][1], s, 0);
      code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[j][2], x[j][3], s, 1);
      code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[j][4], x[j][5], s, 2);
      code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[j][6], x[j][7], s, 3);
    }
    *(uint32_t*)((j ? pg.v_codes : pg.k_codes) + (at * pg.page_rows + row) * (pg.d / 2) + 4 * c) = code;
    if ((c & 3) == 0) (j ? pg.v_scales : pg.k_scales)[(at * (pg.d / 32) + c / 4) * pg.page_rows + row] = (uint8_t)byte;
  }
}

template <typename T>
__global__ __launch_bounds__(kRowThreads) void pages_load_k(PagesView pg, RowsView k, RowsView v, int32_t tokens, const int32_t* slots) {
  const int32_t token = blockIdx.x * blockDim.y + threadIdx.y, c = threadIdx.x, head = blockIdx.y;
  if (token >= tokens) return;
  const int32_t slot = slots[token];
  const int32_t page = slot >> pg.page_shift, row = slot & (pg.page_rows - 1);
  uint32_t code[2] = {0, 0}, byte[2] = {127, 127};
  if (slot >= 0 && page < pg.n_pages) {
    const int64_t at = (int64_t)page * pg.Hkv + head, codes = (at * pg.page_rows + row) * (pg.d / 2) + 4 * c,
                  scale = (at * (pg.d / 32) + c / 4) * pg.page_rows + row;
    code[0] = *(const uint32_t*)(pg.k_codes + codes);
    code[1] = *(const uint32_t*)(pg.v_codes + codes);
    byte[0] = pg.k_scales[scale];
    byte[1] = pg.v_scales[scale];
  }
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const float s = __uint_as_float(byte[j] << 23);
    T* out = const_cast<T*>(row_of<T>(j ? v : k, token, head)) + 8 * c;
    if constexpr (std::is_same<T, float>::value) {
      const f32x2 y[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[j], s, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[j], s, 1),
                          __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[j], s, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[j], s, 3)};
#pragma unroll
      for (int i = 0; i < 2; ++i) *(f32x4_any*)(out + 4 * i) = f32x4_any{y[2 * i][0], y[2 * i][1], y[2 * i + 1][0], y[2 * i + 1][1]};
    } else {
      u32x4 y;
      y[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code[j], s, 0));
      y[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code[j], s, 1));
      y[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code[j], s, 2));
      y[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code[j], s, 3));
      *(u32x4*)out = y;
    }
  }
}

// lanes of a row along x, rows along y (a workgroup is a whole number of waves where head_dim is a power of two)
dim3 row_block(const PagesView& pg) { return dim3((unsigned)(pg.d / 8), (unsigned)(kRowThreads / (pg.d / 8))); }
dim3 row_grid(const PagesView& pg, int32_t tokens) {
  const int rows = kRowThreads / (pg.d / 8);
  return dim3((unsigned)((tokens + rows - 1) / rows), (unsigned)pg.Hkv);
}

}  // namespace

hipError_t launch_pages_plan(const PagesPlanArgs& a, hipStream_t s) {
  const unsigned want = (unsigned)((a.tokens + kPlanThreads - 1) / kPlanThreads), most = 2u * (unsigned)cu_count();
  const unsigned grid = want < 1 ? 1u : want < most ? want : most;
  pages_plan_k<<<grid, kPlanThreads, 3 * sizeof(int32_t) * (size_t)a.n, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_pages_store(int dtype, const PagesView& pg, const RowsView& k, const RowsView& v, int32_t tokens,
                              const int32_t* slots, hipStream_t s) {
  if (dtype == LOCOCO_F32) pages_store_k<float><<<row_grid(pg, tokens), row_block(pg), 0, s>>>(pg, k, v, tokens, slots);
  else pages_store_k<__bf16><<<row_grid(pg, tokens), row_block(pg), 0, s>>>(pg, k, v, tokens, slots);
  return hipGetLastError();
}

hipError_t launch_pages_load(int dtype, const PagesView& pg, const RowsView& k, const RowsView& v, int32_t tokens,
                             const int32_t* slots, hipStream_t s) {
  if (dtype == LOCOCO_F32) pages_load_k<float><<<row_grid(pg, tokens), row_block(pg), 0, s>>>(pg, k, v, tokens, slots);
  else pages_load_k<__bf16><<<row_grid(pg, tokens), row_block(pg), 0, s>>>(pg, k, v, tokens, slots);
  return hipGetLastError();
}

}  // namespace lococo
