// Paged 4-bit rows: what the kernels of pages.hip and pages_attn.hip and the host side share.  Nothing here is public.
//
// A page holds page_rows rows of every kv head, K and V apart.  Codes [page][kv head][row][d / 2], value 2 i of a row in the low four
// bits of byte i; scale bytes [page][kv head][d / 32][row]: a row's 32-value blocks lie page_rows bytes apart, so that the eight or
// sixteen rows a lane takes as one operand have their scales side by side.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "lococo_internal.h"

namespace lococo {

struct PagesView {
  uint8_t* k_codes;
  uint8_t* k_scales;
  uint8_t* v_codes;
  uint8_t* v_scales;
  int32_t n_pages, page_rows, page_shift;   // page_rows = 1 << page_shift
  int32_t Hq, Hkv, group, d;
  float scale;                              // of the attention's scores
};

// rows of a [b, heads, t, d] tensor counted b * t + t'
struct RowsView {
  void* p;
  int64_t sb, sh, st;
  int32_t t;
};

struct PagesPlanArgs {
  int32_t n, tokens, table_pages, page_rows, page_shift, n_pages;
  const int32_t* new_rows;
  const int32_t* held;
  int32_t* tables;
  int32_t* ring;
  const int64_t* ends;
  int32_t* held_after;
  int64_t* ends_after;
  int32_t* starts;
  int32_t* slots;
  int32_t* positions;
  int32_t* totals;
};

struct PagesAttnArgs {
  PagesView pg;
  RowsView q, o;
  int32_t n, tokens, table_pages, max_new, max_held;
  const int32_t* tables;
  const int32_t* starts;
  const int32_t* held;
};

// positions and masks of a turn's trees
struct PagesTreeArgs {
  int32_t n, tokens, words;
  const int32_t* starts;
  const int32_t* held;
  const int32_t* bases;                        // null: held less the new rows
  const int32_t* parents;
  uint32_t* masks;
  int32_t* positions;
};

// what becomes of a turn's rows and pages once some of the rows are kept
struct PagesKeepArgs {
  int32_t n, tokens, table_pages, page_rows, page_shift, n_pages;
  const int32_t* starts;
  const int32_t* held;
  const int32_t* slots;
  const int32_t* kept;
  const int32_t* tables;
  int32_t* ring;
  const int64_t* ends;
  int32_t* held_after;
  int64_t* ends_after;
  int32_t* sources;
  int32_t* targets;
  int32_t* totals;
};

struct PagesMoveArgs {
  PagesView pg;
  int32_t n, tokens;
  const int32_t* starts;
  const int32_t* sources;
  const int32_t* targets;
};

constexpr int kPagesMaxRequests = 4096;       // the plan's lists lie in LDS
constexpr int kPagesMaxHeadDim = 256;
constexpr int kPagesMinRows = 16, kPagesMaxRows = 1024;
constexpr int32_t kPagesCap = 0x3fffffff;     // rows of a call, slots, rows of a request: below
constexpr int kPagesMaxTree = 256;            // new rows of a request that masks can name, a multiple of 32

// ---- what their kernels share
typedef __attribute__((ext_vector_type(4))) uint32_t w4;
typedef __attribute__((ext_vector_type(4), aligned(4))) float f4_any;          // fp32 rows begin at any float

// sums of numbers >= 0 cut off at kPagesCap
__device__ __forceinline__ int32_t add_cap(int32_t x, int32_t y) { return min(x + y, kPagesCap); }

// a head's row of a call's token
template <typename T>
__device__ __forceinline__ const T* row_at(const RowsView& r, int32_t token, int32_t head) {
  const int32_t b = token < r.t ? 0 : token / r.t, t = token - b * r.t;
  return (const T*)r.p + b * r.sb + head * r.sh + t * r.st;
}

// eight values of a row: bf16 rows begin at multiples of 16 bytes
template <typename T>
__device__ __forceinline__ void read8(const T* p, float (&x)[8]) {
  if constexpr (std::is_same<T, float>::value) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const f4_any v = *(const f4_any*)(p + 4 * i);
#pragma unroll
      for (int k = 0; k < 4; ++k) x[4 * i + k] = v[k];
    }
  } else {
    const w4 v = *(const w4*)p;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(v[i] << 16);
      x[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
    }
  }
}

// ---- pages.hip
hipError_t launch_pages_plan(const PagesPlanArgs& a, hipStream_t s);
// k and v rows to their slots (store) or from them (load); a slot outside the pages is skipped, or read as zeros
hipError_t launch_pages_store(int dtype, const PagesView& pg, const RowsView& k, const RowsView& v, int32_t tokens,
                              const int32_t* slots, hipStream_t s);
hipError_t launch_pages_load(int dtype, const PagesView& pg, const RowsView& k, const RowsView& v, int32_t tokens,
                             const int32_t* slots, hipStream_t s);
// ---- pages_tree.hip
hipError_t launch_pages_tree(const PagesTreeArgs& a, hipStream_t s);
hipError_t launch_pages_keep(const PagesKeepArgs& a, hipStream_t s);
hipError_t launch_pages_move(const PagesMoveArgs& a, hipStream_t s);
// ---- pages_attn.hip
bool pages_attn_fits(int dtype, const PagesAttnArgs& a);     // a launch takes the work
size_t pages_attn_workspace_bytes(int dtype, const PagesAttnArgs& a);
hipError_t launch_pages_attn(int dtype, const PagesAttnArgs& a, void* workspace, hipStream_t s);
// ---- pages_attn_tree.hip: the same sizes (those that pages_attn_fits), a mask of `words` words for each of the call's rows
size_t pages_attn_tree_workspace_bytes(int dtype, const PagesAttnArgs& a);
hipError_t launch_pages_attn_tree(int dtype, const PagesAttnArgs& a, const uint32_t* masks, int32_t words, void* workspace, hipStream_t s);

}  // namespace lococo
