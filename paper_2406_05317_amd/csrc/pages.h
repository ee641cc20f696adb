// Paged 4-bit rows: what the kernels of pages.hip and pages_attn.hip and the host side share.  Nothing here is public.
//
// A page holds page_rows rows of every kv head, K and V apart.  Codes [page][kv head][row][d / 2], value 2 i of a row in the low four
// bits of byte i; scale bytes [page][kv head][d / 32][row]: a row's 32-value blocks lie page_rows bytes apart, so that the eight or
// sixteen rows a lane takes as one operand have their scales side by side.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

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

constexpr int kPagesMaxRequests = 4096;       // the plan's lists lie in LDS
constexpr int kPagesMaxHeadDim = 256;
constexpr int kPagesMinRows = 16, kPagesMaxRows = 1024;
constexpr int32_t kPagesCap = 0x3fffffff;     // rows of a call, slots, rows of a request: below

// ---- pages.hip
hipError_t launch_pages_plan(const PagesPlanArgs& a, hipStream_t s);
// k and v rows to their slots (store) or from them (load); a slot outside the pages is skipped, or read as zeros
hipError_t launch_pages_store(int dtype, const PagesView& pg, const RowsView& k, const RowsView& v, int32_t tokens,
                              const int32_t* slots, hipStream_t s);
hipError_t launch_pages_load(int dtype, const PagesView& pg, const RowsView& k, const RowsView& v, int32_t tokens,
                             const int32_t* slots, hipStream_t s);
// ---- pages_attn.hip
bool pages_attn_fits(int dtype, const PagesAttnArgs& a);     // a launch takes the work
size_t pages_attn_workspace_bytes(int dtype, const PagesAttnArgs& a);
hipError_t launch_pages_attn(int dtype, const PagesAttnArgs& a, void* workspace, hipStream_t s);

}  // namespace lococo
