// Attention over paged 4-bit rows: o = softmax(scale q K^T) V for the new rows of a batch of requests of different lengths.  What a new
// row sees of its request: the rows up to and at its own position (pages_attn.hip), or all rows ahead of the new ones and those of the new
// ones that its mask names (TREE: pages_attn_tree.hip).
#pragma once

#include "mfma_util.h"
#include "pages.h"

#include <algorithm>
#include <type_traits>

namespace lococo {
namespace pages_detail {

// the masks of a call's new rows: bit j of the `words` words of a row is its request's new row j
struct TreeMasks {
  const uint32_t* masks;
  int32_t words;
};
// A row's mask as a tile has it in LDS: a word ahead of it for the rows that all see, zeros behind it.  16 consecutive bits from new row
// j0 on (below 0: rows ahead of the new ones).
constexpr int kMaskWords = kPagesMaxTree / 32;
struct TileMask { uint32_t w[kMaskWords + 2]; };
__device__ __forceinline__ uint32_t mask_bits(const TileMask& row, int32_t j0) {
  const int32_t w = j0 >> 5;
  const uint32_t lo = row.w[min(max(w + 1, 0), kMaskWords + 1)], hi = row.w[min(max(w + 2, 0), kMaskWords + 1)];
  return (uint32_t)((((uint64_t)hi << 32) | lo) >> (j0 & 31)) & 0xffffu;
}

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
constexpr int kRowsWaves = 4, kRowsThreads = 64 * kRowsWaves;

template <typename T, bool TREE>
__device__ __forceinline__ void attn_rows(const PagesAttnArgs& a, const TreeMasks& tm) {
  __shared__ float qs[kRowsWaves][kPagesMaxHeadDim], ps[kRowsWaves][64];
  __shared__ int64_t at[kRowsWaves][64];
  const int l = threadIdx.x & 63, w = threadIdx.x >> 6;
  const PagesView& pg = a.pg;
  const int32_t token = blockIdx.x * kRowsWaves + w, h = blockIdx.y, kvh = h / pg.group;
  if (token >= a.tokens) return;                 // nothing below meets the other waves
  const int req = request_of(a.starts, a.n, token);
  const int32_t stop = min(a.starts[req + 1], a.tokens);
  if (token < a.starts[req] || token >= stop) return;                       // nobody's: ahead of the first request, behind the last
  const int32_t held = min(max(a.held[req], 0), a.table_pages << pg.page_shift);
  const int32_t ahead = held - (stop - a.starts[req]);                      // TREE: rows ahead of the new ones
  const int32_t seen = TREE ? held : max(held - (stop - token) + 1, 0);     // rows the query sees, or may
  const uint32_t* mask = TREE ? tm.masks + (int64_t)token * tm.words : nullptr;
  const int32_t b = token / a.q.t, t = token - b * a.q.t;
  const T* q = (const T*)a.q.p + b * a.q.sb + h * a.q.sh + t * a.q.st;
  for (int i = l; i < pg.d; i += 64) qs[w][i] = (float)q[i] * (pg.scale * kLog2e);
  float m = -INFINITY, sum = 0.f;
  f32x2 acc[2] = {{0.f, 0.f}, {0.f, 0.f}};       // columns 2 (l + 64 i), + 1
  const int32_t* table = a.tables + (int64_t)req * a.table_pages;
  for (int32_t j0 = 0; j0 < seen; j0 += 64) {
    const int32_t j = j0 + l;
    const int32_t page = j < seen ? table[j >> pg.page_shift] : -1;
    bool there = (uint32_t)page < (uint32_t)pg.n_pages;
    if (TREE && j >= ahead) {
      const int32_t x = j - ahead;
      there = there && x < 32 * tm.words && (mask[x >> 5] >> (x & 31) & 1u);
    }
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

// ---------------------------------------------------------------------------------------------------------------------------------
// head_dim 64 and 128: matrix instructions.  A workgroup takes TR = 16 QB query rows that share a kv head (the new rows of a request
// times the heads of the group) and a part of the keys; its four waves take the 64-key tiles of that part in turn, each for all the
// query rows with a running softmax of its own, and meet once, at the end.  No wave waits for another before that, nothing passes
// through LDS on the way: codes go from memory to operand registers.
//
//   scores, transposed: S^T [64 keys x 16 queries] = K Q^T.  Lane (m = l % 16, g = l / 16) loads the codes of keys 4 m + t, t = 0 .. 3,
//     columns g D/4 .. + D/4 - 1, which as bf16 (the conversion applies the scale; scale times code is exact in bf16) are the operand of
//     key 4 m + t in MFMA t; the query operands take the columns in the same order.  The result has in lane (query l % 16, g) the keys
//     16 g + 4 i + t: 16 consecutive ones.
//   so the probabilities are where the second product, O^T = V^T P^T, wants them: lane (query, g) holds keys 16 g + 8 c + 0 .. 7 of
//     step c.  Its other operand, V^T, wants in lane (column, g) those keys' values of one column: lane (m, g) loads, for its 16 keys,
//     the D/32 bytes of columns D/16 m .. + D/16 - 1 and pairs two keys' values of a column after the conversion.
//
// Running softmax: the reference a row's exponentials are taken against is set 8 (in powers of two) above a tile's largest score and moves
// only when a later one passes it, exact after the final division: no exponential exceeds 1, and what they weigh, up to 6 * 2^125, does
// not leave fp32 by them.  Probabilities enter their product as the sum of two bf16 numbers (16 bits), for fp32
// rows of three (all 24 bits), as their queries do.  One alone would save a third of the MFMAs (prompts of 2000 tokens 0.81 ms for 0.99 then),
// but is off by as much as the rounding of a bf16 result wherever one key carries a column, be it by its probability or, as where new
// rows stand beside the averages of a compressed memory, by the size of its value.  Two are off by 2^-16 of the sum of |p v|: below a bf16
// result's own rounding unless the values cancel to less than 2^-8 of that sum.  The row's sum is taken of the same numbers, by a product
// with ones: no vector instruction adds.
//
// Bound, single tokens: by memory and by the start and end of a workgroup, some 7 us: 131072 keys of 8 heads, 143 MB, 27.6 us
// (5.1 TB/s), and 4 for the join.  Many rows: by the instructions around 104 MFMAs a tile of 64 keys x 32 rows (vector port 68 % busy,
// matrix pipe 44 %): 3349 tokens on up to 14 K keys of 32 heads 0.97 - 1.01 ms, 670 - 700 TFLOP/s (4 d flops a pair).  Each wave asks
// for the codes of V a whole tile ahead; those of K for the next tile go into the registers the scores have just been taken from.
constexpr int kTileWaves = 4, kTileKeys = 64;
constexpr float kNoRef = -3.0e38f;             // below any score
constexpr float kRefAhead = 8.f;               // of a row's reference over the scores it was taken from

typedef __attribute__((ext_vector_type(4))) float f4;

struct TileArgs {
  PagesAttnArgs a;
  int32_t splits, chunk;                       // parts of the keys at most, keys of a part at least
  int32_t slots;                               // row tiles at most
  int32_t by_request;                          // 1: a tile to a request
  float* part_o;                               // [slot][kv head][part][row][D]
  float* part_ml;                              // the same rows: reference, sum
};

// What a workgroup works on.  Row r of a request is query head r % group of its new row r / group.
struct TileJob {
  int32_t req, row0, rows, first, fresh, held; // rows of the tile; the request's first row of the call, its new rows, rows held
  int32_t keys;                                // keys its last row sees; TREE: any row may
};

// The slot request i's tiles begin at.  A request with rows opens one tile more than its whole ones at most, and moves min(i, starts) on by
// one at least: its tiles never reach into the next one's.  Requests without rows, of which there may be thousands, take no slot.
template <int TR>
__device__ __forceinline__ int32_t first_slot(const PagesAttnArgs& a, int32_t i) {
  const int32_t at = a.starts[i];
  return (int32_t)((int64_t)at * a.pg.group / TR) + min(i, at);
}

template <int TR, bool TREE>
__device__ __forceinline__ bool tile_job(const TileArgs& g, int32_t slot, TileJob* j) {
  const PagesAttnArgs& a = g.a;
  int32_t req = slot, tile = 0;
  if (!g.by_request) {
    // the last request that begins at or before the slot, 64 candidates at a look (one trip to memory, two with more than 64 requests)
    const int l = threadIdx.x & 63;
    req = 0;
#pragma unroll
    for (int step = 64; step; step = step == 64 ? 1 : 0) {
      if (step == 64 && a.n <= 64) continue;
      const int32_t at = first_slot<TR>(a, min(req + l * step, a.n - 1));
      req += max(__popcll(__ballot(req + l * step < a.n && at <= slot)) - 1, 0) * step;
    }
    req = __builtin_amdgcn_readfirstlane(req);
    tile = slot - first_slot<TR>(a, req);
    if (tile < 0) return false;
  }
  j->req = req;
  j->first = min(max(a.starts[req], 0), a.tokens);
  j->fresh = min(max(a.starts[req + 1], j->first), a.tokens) - j->first;
  j->row0 = tile * TR;
  const int64_t left = (int64_t)j->fresh * a.pg.group - (int64_t)tile * TR;
  if (left <= 0) return false;
  j->rows = (int32_t)min(left, (int64_t)TR);
  j->held = min(max(a.held[req], 0), a.table_pages << a.pg.page_shift);
  j->keys = TREE ? j->held : max(j->held - j->fresh + (j->row0 + j->rows - 1) / a.pg.group + 1, 0);
  return true;
}
// keys of a part, and how many parts there are (one at least): all from what the join knows as well
__device__ __forceinline__ int32_t part_keys(const TileArgs& g, int32_t keys) {
  const int32_t even = ((keys + g.splits - 1) / g.splits + kTileKeys - 1) / kTileKeys * kTileKeys;
  return max(even, g.chunk);
}
__device__ __forceinline__ int32_t parts_of(const TileArgs& g, int32_t keys) {
  return max((keys + part_keys(g, keys) - 1) / part_keys(g, keys), 1);
}

template <int BYTES>
struct Bytes;
template <>
struct Bytes<16> { typedef u32x4 type; };
template <>
struct Bytes<8> { typedef u32x2 type; };
template <>
struct Bytes<4> { typedef uint32_t type; };
template <>
struct Bytes<2> { typedef uint16_t type; };

// the codes and scales of a tile, as a lane holds them
template <int D>
struct KeyCodes {
  typename Bytes<D / 8>::type c[4];            // keys 4 m + t
  uint32_t scales;                             // a byte each
};
template <int D>
struct ValueCodes {
  typename Bytes<D / 32>::type c[16];          // keys 16 g + x
  u32x4 scales;
};

// key t's bf16 operand of a step: 8 values
template <int D>
__device__ __forceinline__ bf16x8 k_operand(const KeyCodes<D>& k, int t, int step, float scale) {
  const uint32_t w = k.c[t][step];
  u32x4 r;
  r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0));
  r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1));
  r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2));
  r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3));
  return __builtin_bit_cast(bf16x8, r);
}
template <int B>
__device__ __forceinline__ uint32_t v_pair(uint32_t code, float scale) {      // columns 2 B, 2 B + 1 of a key
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, B));
}
__device__ __forceinline__ float scale_byte(uint32_t w, int i) { return __uint_as_float((i < 3 ? w << (23 - 8 * i) : w >> 1) & 0x7f800000u); }

__device__ __forceinline__ f4 mfma16(bf16x8 a, bf16x8 b, f4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// the largest over the four lanes that hold a query's keys
__device__ __forceinline__ float max_groups(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return max_halves(x);
}

// the page of a key: -1 where there is none, and behind the keys at hand (without a branch: an entry is read in any case)
__device__ __forceinline__ int32_t page_of(const PagesAttnArgs& a, const int32_t* table, int32_t key, int32_t keys) {
  const int32_t page = table[max(min(key, keys - 1), 0) >> a.pg.page_shift];
  const bool in = (key < keys) & ((uint32_t)page < (uint32_t)a.pg.n_pages);
  return in ? page : -1;
}

// (rows of a page are always there; a lane without a page reads page 0 and has its keys masked)
template <int D>
__device__ __forceinline__ void load_k(KeyCodes<D>& k, const PagesView& pg, int32_t kvh, int32_t key0, int32_t page, int m, int g) {
  const int32_t row = (key0 + 4 * m) & (pg.page_rows - 1);
  const int64_t at = ((int64_t)max(page, 0) * pg.Hkv + kvh) * pg.page_rows;
  const uint8_t* codes = pg.k_codes + (at + row) * (D / 2) + g * (D / 8);
#pragma unroll
  for (int t = 0; t < 4; ++t) k.c[t] = *(const typename Bytes<D / 8>::type*)(codes + t * (D / 2));
  k.scales = *(const uint32_t*)(pg.k_scales + at * (D / 32) + (g * (D / 4) / 32) * pg.page_rows + row);
}
template <int D>
__device__ __forceinline__ void load_v(ValueCodes<D>& v, const PagesView& pg, int32_t kvh, int32_t key0, int32_t page, int m, int g) {
  const int32_t row = (key0 + 16 * g) & (pg.page_rows - 1);
  const int64_t at = ((int64_t)max(page, 0) * pg.Hkv + kvh) * pg.page_rows;
  const uint8_t* codes = pg.v_codes + (at + row) * (D / 2) + m * (D / 32);
#pragma unroll
  for (int x = 0; x < 16; ++x) v.c[x] = *(const typename Bytes<D / 32>::type*)(codes + x * (D / 2));
  v.scales = *(const u32x4*)(pg.v_scales + at * (D / 32) + (m * (D / 16) / 32) * pg.page_rows + row);
}

// A tile's work on the keys key_lo .. key_hi - 1: to o where that is all it sees, else as a part, rows from part_row on.  WAVES waves take 64
// keys in turn and meet at the end; one alone, for which it is all, writes from where the products left its results.  tid: threadIdx.x.
template <typename T, int D, int QB, bool TREE, int WAVES>
__device__ __forceinline__ void attn_piece(const TileArgs& g, const TreeMasks& tm, const TileJob& job, int32_t kvh, int32_t key_lo, int32_t key_hi,
                                           bool whole_job, int64_t part_row, int tid) {
  constexpr int PARTS = std::is_same<T, float>::value ? 3 : 1, PROBS = PARTS == 3 ? 3 : 2, TR = 16 * QB, STEPS = D / 32, COLS = D / 16, LD = D + 4;
  __shared__ __align__(16) float joined[WAVES > 1 ? WAVES : 1][WAVES > 1 ? TR : 1][LD];
  __shared__ float ml[WAVES > 1 ? WAVES : 1][WAVES > 1 ? TR : 1][2];
  constexpr int OWN = WAVES == 1 ? kTileWaves : 1;                            // waves that work alone have arrays of their own
  __shared__ int32_t nan_keys[OWN][D / 32];          // first visible key whose 32 values of V stand for NaN, among the tiles that mask;
  __shared__ uint32_t nan_news[OWN][TREE ? D / 32 : 1][kMaskWords];                 // TREE: among those ahead of the new ones.  And new ones
  __shared__ TileMask mask_rows[OWN][TREE ? TR : 1];
  const PagesAttnArgs& a = g.a;
  const PagesView& pg = a.pg;
  const int l = tid & 63, own = WAVES == 1 ? __builtin_amdgcn_readfirstlane(tid >> 6) : 0, w = WAVES == 1 ? 0 : __builtin_amdgcn_readfirstlane(tid >> 6),
            m = l & 15, grp = l >> 4;
  auto& nan_key = nan_keys[own];
  auto& nan_new = nan_news[own];
  auto& masks = mask_rows[own];
  if constexpr (WAVES == 1) tid = l;
  auto meet = [] {                               // LDS as it is written so far
    if constexpr (WAVES == 1) {
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    } else {
      __syncthreads();
    }
  };
  if (tid < D / 32) nan_key[tid] = 0x7fffffff;
  if constexpr (TREE) {
    if (tid < D / 32 * kMaskWords) (&nan_new[0][0])[tid] = 0;
    if (key_hi > job.held - job.fresh)
      for (int i = tid; i < TR * (kMaskWords + 2); i += 64 * WAVES) {
        const int r = i / (kMaskWords + 2), k = i % (kMaskWords + 2) - 1;
        const int64_t token = job.first + (job.row0 + r) / pg.group;
        masks[r].w[k + 1] = r >= job.rows || k >= tm.words ? 0u : k < 0 ? 0xffffffffu : tm.masks[token * tm.words + k];
      }
  }
  meet();

  // queries: row 16 qb + m, columns grp D/4 + 8 step ..
  bf16x8 q[QB][PARTS][STEPS];
  int32_t last[QB];                            // the key a row's query stands at
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    const int32_t r = 16 * qb + m, row = job.row0 + r;
    const bool real = r < job.rows;
    const int32_t x = row / pg.group, token = job.first + x, b = token < a.q.t ? 0 : token / a.q.t, t = token - b * a.q.t;
    last[qb] = real ? job.held - job.fresh + x : -1;
    const T* qr = (const T*)a.q.p + (real ? b * a.q.sb + (kvh * pg.group + row - x * pg.group) * a.q.sh + t * a.q.st : 0) + grp * (D / 4);
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      if constexpr (PARTS == 1) {
        u32x4 v = {0, 0, 0, 0};
        if (real) v = *(const u32x4*)(qr + 8 * s);
        q[qb][0][s] = __builtin_bit_cast(bf16x8, v);
      } else {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = real ? (float)qr[8 * s + i] : 0.f;
        bf16x8 part[PARTS];
        split_parts<PARTS>(v, part);
#pragma unroll
        for (int p = 0; p < PARTS; ++p) q[qb][p][s] = part[p];
      }
    }
  }
  const float c = pg.scale * kLog2e;
  const int32_t ahead = job.held - job.fresh;                                 // TREE: rows ahead of the new ones
  const int32_t whole = TREE ? ahead : job.held - job.fresh + job.row0 / pg.group + 1;     // keys every row of the tile sees
  const int32_t* table = a.tables + (int64_t)job.req * a.table_pages;
  float ref[QB];
  f4 o[QB][COLS], sum[QB];                     // sum: the same number in all four places of a lane
  constexpr int kStride = WAVES * kTileKeys;
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    ref[qb] = kNoRef;
    sum[qb] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < COLS; ++j) o[qb][j] = f4{0.f, 0.f, 0.f, 0.f};
  }
  int32_t key0 = key_lo + w * kTileKeys;
  int32_t kp = page_of(a, table, key0 + 4 * m, key_hi);
  KeyCodes<D> kc;
  if (key0 < key_hi) load_k<D>(kc, pg, kvh, key0, kp, m, grp);
  kp = page_of(a, table, key0 + kStride + 4 * m, key_hi);
  // one tile: vp is the page of a lane's keys
  auto tile = [&](const ValueCodes<D>& vc, int32_t vp) {
    // a wave in either product goes ahead of one in its softmax: the matrix pipe is given work while vector instructions wait (prompts
    // 1 to 2 % shorter, 77 tokens on 3 K keys 4 to 6 %)
    __builtin_amdgcn_s_setprio(1);
    f4 s[QB][4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const float sc = scale_byte(kc.scales, t);
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) s[qb][t] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int st = 0; st < STEPS; ++st) {
        const bf16x8 k = k_operand<D>(kc, t, st, sc);
#pragma unroll
        for (int qb = 0; qb < QB; ++qb)
#pragma unroll
          for (int p = PARTS - 1; p >= 0; --p) s[qb][t] = mfma16(k, q[qb][p][st], s[qb][t]);
      }
    }
    if (key0 + kStride < key_hi) load_k<D>(kc, pg, kvh, key0 + kStride, kp, m, grp);     // the next tile's, into the same registers
    kp = page_of(a, table, key0 + 2 * kStride + 4 * m, key_hi);
    u32x4 vs = vc.scales;
    if (key0 + kTileKeys > min(whole, key_hi) || __any(vp < 0)) {
      // keys behind a row's own, behind the part, or without a page: no score, and a V that is zero times something finite.  A key that
      // only some rows see may stand for NaN: taken out of the product here and put into those rows at the end.
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) {
        const int32_t lim = vp < 0 ? -1 : TREE ? key_hi - 1 : min(last[qb], key_hi - 1);
        const uint32_t bits = TREE && key_hi > ahead ? mask_bits(masks[TREE ? 16 * qb + m : 0], key0 + 16 * grp - ahead) : 0xffffu;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const bool in = key0 + 16 * grp + 4 * i + t <= lim && (!TREE || (bits >> (4 * i + t) & 1u));
            s[qb][t][i] = in ? s[qb][t][i] : -INFINITY;
          }
      }
#pragma unroll
      for (int x = 0; x < 16; ++x) {
        const int32_t key = key0 + 16 * grp + x;
        const bool in = vp >= 0 && key < key_hi, odd = (vs[x / 4] >> (8 * (x % 4)) & 255u) == 255u;
        if (!TREE || key < ahead) {
          if (in && odd) atomicMin(&nan_key[m * (D / 16) / 32], key);
        } else if (in && odd && key - ahead < 32 * tm.words) {
          atomicOr(&nan_new[m * (D / 16) / 32][(key - ahead) >> 5], 1u << ((key - ahead) & 31));
        }
        if (!in || odd) vs[x / 4] &= ~(255u << (8 * (x % 4)));
      }
    }
    __builtin_amdgcn_s_setprio(0);
    float top[QB];
    bool grown = false;
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      top[qb] = s[qb][0][0];
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) top[qb] = fmaxf(top[qb], s[qb][t][i]);
      top[qb] *= c;
      grown |= top[qb] > ref[qb];
    }
    if (__any(grown)) {
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) {
        const float next = fmaxf(ref[qb], max_groups(top[qb]) + kRefAhead), keep = __builtin_amdgcn_exp2f(ref[qb] - next);
        ref[qb] = next;
        sum[qb] = f4{sum[qb][0] * keep, sum[qb][1] * keep, sum[qb][2] * keep, sum[qb][3] * keep};
#pragma unroll
        for (int j = 0; j < COLS; ++j) o[qb][j] = f4{o[qb][j][0] * keep, o[qb][j][1] * keep, o[qb][j][2] * keep, o[qb][j][3] * keep};
      }
    }
    bf16x8 p[QB][PROBS][2], one;
#pragma unroll
    for (int i = 0; i < 8; ++i) one[i] = (__bf16)1.f;
#pragma unroll
    for (int qb = 0; qb < QB; ++qb)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float e[8];                             // keys 16 grp + 8 h + 4 i + t
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int t = 0; t < 4; ++t) e[4 * i + t] = __builtin_amdgcn_exp2f(fmaf(s[qb][t][2 * h + i], c, -ref[qb]));
        bf16x8 part[PROBS];
        split_parts<PROBS>(e, part);
#pragma unroll
        for (int k = 0; k < PROBS; ++k) p[qb][k][h] = part[k];
#pragma unroll
        for (int k = PROBS - 1; k >= 0; --k) sum[qb] = mfma16(one, p[qb][k][h], sum[qb]);
      }

    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float sc[8];
#pragma unroll
      for (int x = 0; x < 8; ++x) sc[x] = scale_byte(vs[2 * h + x / 4], x % 4);
      auto columns = [&](auto byte) {
        constexpr int B = decltype(byte)::value;
        uint32_t y[8];
#pragma unroll
        for (int x = 0; x < 8; ++x) y[x] = v_pair<B>(vc.c[8 * h + x], sc[x]);
        u32x4 op[2];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          op[0][x] = __builtin_amdgcn_perm(y[2 * x + 1], y[2 * x], 0x05040100u);
          op[1][x] = __builtin_amdgcn_perm(y[2 * x + 1], y[2 * x], 0x07060302u);
        }
#pragma unroll
        for (int k = PROBS - 1; k >= 0; --k)
#pragma unroll
          for (int qb = 0; qb < QB; ++qb)
#pragma unroll
            for (int j = 0; j < 2; ++j) o[qb][2 * B + j] = mfma16(__builtin_bit_cast(bf16x8, op[j]), p[qb][k][h], o[qb][2 * B + j]);
      };
      columns(std::integral_constant<int, 0>());
      columns(std::integral_constant<int, 1>());
      if constexpr (D == 128) {
        columns(std::integral_constant<int, 2>());
        columns(std::integral_constant<int, 3>());
      }
    }
    __builtin_amdgcn_s_setprio(0);
    key0 += kStride;
  };
  if (key0 < key_hi) {
    // the codes of V are on their way a whole tile ahead
    int32_t vp = page_of(a, table, key0 + 16 * grp, key_hi), vp1 = page_of(a, table, key0 + kStride + 16 * grp, key_hi);
    ValueCodes<D> even, odd;
    load_v<D>(even, pg, kvh, key0, vp, m, grp);
    while (true) {
      int32_t vp2 = page_of(a, table, key0 + 2 * kStride + 16 * grp, key_hi);
      if (key0 + kStride < key_hi) load_v<D>(odd, pg, kvh, key0 + kStride, vp1, m, grp);
      tile(even, vp);
      if (key0 >= key_hi) break;
      if constexpr (QB == 2) {                 // two tiles a turn would not fit the registers
        even = odd;
        vp = vp1;
        vp1 = vp2;
      } else {
        vp = vp2;
        vp2 = page_of(a, table, key0 + 2 * kStride + 16 * grp, key_hi);
        if (key0 + kStride < key_hi) load_v<D>(even, pg, kvh, key0 + kStride, vp, m, grp);
        tile(odd, vp1);
        if (key0 >= key_hi) break;
        vp1 = vp2;
      }
    }
  }

  // o[qb][j][i] is column COLS (4 grp + i) + j of row 16 qb + m
  if constexpr (WAVES == 1) {
    meet();
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      const int32_t r = 16 * qb + m, row = job.row0 + r, x = row / pg.group, at = TREE ? 0x7ffffffe : job.held - job.fresh + x;
      if (r >= job.rows) continue;
      const float inv = sum[qb][0] == 0.f ? 0.f : 1.f / sum[qb][0];           // a row that sees nothing: zeros
      const int32_t token = job.first + x, ob = token < a.o.t ? 0 : token / a.o.t, ot = token - ob * a.o.t;
      T* out = (T*)a.o.p + ob * a.o.sb + (kvh * pg.group + row - x * pg.group) * a.o.sh + ot * a.o.st;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int col = COLS * (4 * grp + i), block = col / 32;
        bool odd = at >= nan_key[block];
        if (TREE && key_hi > ahead)
          for (int32_t k = 0; k < kMaskWords; ++k) odd |= (nan_new[TREE ? block : 0][k] & masks[TREE ? r : 0].w[k + 1]) != 0;
        __align__(16) T z[COLS];
#pragma unroll
        for (int j = 0; j < COLS; ++j) {
          if (odd) o[qb][j][i] = NAN;
          z[j] = (T)(o[qb][j][i] * inv);
        }
        if constexpr (PARTS == 1) {
          *(typename Bytes<COLS * 2>::type*)(out + col) = *(typename Bytes<COLS * 2>::type*)z;
        } else {
#pragma unroll
          for (int j = 0; j < COLS; ++j) out[col + j] = z[j];
        }
      }
    }
    return;
  }
  // the waves' results to one
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    if (grp == 0) {
      ml[w][16 * qb + m][0] = ref[qb];
      ml[w][16 * qb + m][1] = sum[qb][0];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < COLS; j += 4)
        *(f4*)&joined[w][16 * qb + m][COLS * (4 * grp + i) + j] = f4{o[qb][j][i], o[qb][j + 1][i], o[qb][j + 2][i], o[qb][j + 3][i]};
  }
  __syncthreads();
  constexpr int PER = TR * D / (64 * WAVES);                             // columns of a thread
  const int r = tid / (D / PER), col = tid % (D / PER) * PER;
  if (r >= job.rows) return;
  float best = ml[0][r][0];
#pragma unroll
  for (int k = 1; k < WAVES; ++k) best = fmaxf(best, ml[k][r][0]);
  float y[PER], total = 0.f;
#pragma unroll
  for (int i = 0; i < PER; ++i) y[i] = 0.f;
#pragma unroll
  for (int k = 0; k < WAVES; ++k) {
    const float keep = __builtin_amdgcn_exp2f(ml[k][r][0] - best);
    total += ml[k][r][1] * keep;
#pragma unroll
    for (int i = 0; i < PER; ++i) y[i] += joined[k][r][col + i] * keep;
  }
  const int32_t row = job.row0 + r, x = row / pg.group, at = TREE ? 0x7ffffffe : job.held - job.fresh + x;
#pragma unroll
  for (int i = 0; i < PER; ++i)
    if (at >= nan_key[(col + i) / 32]) y[i] = NAN;
  if (TREE && key_hi > ahead) {
    for (int32_t k = 0; k < kMaskWords; ++k)
#pragma unroll
      for (int i = 0; i < PER; ++i)
        if (nan_new[TREE ? (col + i) / 32 : 0][k] & masks[TREE ? r : 0].w[k + 1]) y[i] = NAN;
  }
  if (!whole_job) {
    const int64_t pr = part_row + r;
#pragma unroll
    for (int i = 0; i < PER; i += 4) *(f4*)(g.part_o + pr * D + col + i) = f4{y[i], y[i + 1], y[i + 2], y[i + 3]};
    if (col == 0) {
      g.part_ml[2 * pr] = best;
      g.part_ml[2 * pr + 1] = total;
    }
    return;
  }
  const float inv = total == 0.f ? 0.f : 1.f / total;                         // a row that sees nothing: zeros
  const int32_t token = job.first + x, ob = token < a.o.t ? 0 : token / a.o.t, ot = token - ob * a.o.t;
  T* out = (T*)a.o.p + ob * a.o.sb + (kvh * pg.group + row - x * pg.group) * a.o.sh + ot * a.o.st + col;
  __align__(16) T z[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) z[i] = (T)(y[i] * inv);
  if constexpr (PARTS == 1) {
    constexpr int V = PER * 2 < 16 ? PER * 2 : 16;
#pragma unroll
    for (int i = 0; i < PER * 2 / V; ++i) ((typename Bytes<V>::type*)out)[i] = ((typename Bytes<V>::type*)z)[i];
  } else {
#pragma unroll
    for (int i = 0; i < PER; ++i) out[i] = z[i];
  }
}

// A workgroup's tile and part of the keys, by its number.
template <typename T, int D, int QB, bool TREE>
__device__ __forceinline__ void attn_tile(const TileArgs& g, const TreeMasks& tm) {
  constexpr int TR = 16 * QB;
  const PagesView& pg = g.a.pg;
  const int item = xcd_item(blockIdx.x, gridDim.x);
  // neighbours, on one XCD: the kv heads of a part where a request is one tile (their scales share cache lines), else the tiles that
  // read the same keys
  const int32_t kvh = g.by_request ? item % pg.Hkv : item / g.slots / g.splits;
  const int32_t rest = g.by_request ? item / pg.Hkv : item % (g.slots * g.splits);
  const int32_t slot = g.by_request ? rest / g.splits : rest % g.slots, split = g.by_request ? rest % g.splits : rest / g.slots;
  TileJob job;
  if (!tile_job<TR, TREE>(g, slot, &job)) return;
  const int32_t per = part_keys(g, job.keys), parts = parts_of(g, job.keys);
  if (split >= parts) return;
  const int32_t key_lo = split * per, key_hi = min(key_lo + per, job.keys);
  attn_piece<T, D, QB, TREE, kTileWaves>(g, tm, job, kvh, key_lo, key_hi, parts == 1, (((int64_t)slot * pg.Hkv + kvh) * g.splits + split) * TR,
                             threadIdx.x);
}

// The parts of a row to one, in their order.  WAVES waves to a row, which take its parts in turn: one where there are few, so that four
// rows share a workgroup.  A lane holds the reference and the sum of one part, all lanes the columns of every part.
template <typename T, int D, int TR, int WAVES, bool TREE>
__device__ __forceinline__ void attn_join(const TileArgs& g, int32_t rows) {
  typedef __attribute__((ext_vector_type(D / 64))) float cols;
  __shared__ float sums[4][D], stat[4][2];
  const PagesAttnArgs& a = g.a;
  const PagesView& pg = a.pg;
  const int l = threadIdx.x & 63, w = threadIdx.x >> 6, first = WAVES == 4 ? w : 0;
  const int32_t per = (rows + 4 / WAVES - 1) / (4 / WAVES);                   // workgroups to a tile of a kv head
  const int32_t kvh = blockIdx.x % pg.Hkv, slot = blockIdx.x / pg.Hkv / per, r = blockIdx.x / pg.Hkv % per * (4 / WAVES) + (WAVES == 4 ? 0 : w);
  TileJob job;
  if (!tile_job<TR, TREE>(g, slot, &job) || r >= job.rows) return;
  const int32_t parts = parts_of(g, job.keys);
  if (parts == 1) return;
  const int64_t pr = ((int64_t)slot * pg.Hkv + kvh) * g.splits * TR + r;
  float best = kNoRef, total = 0.f;
  cols y;
#pragma unroll
  for (int i = 0; i < D / 64; ++i) y[i] = 0.f;
  for (int32_t k0 = first; k0 < parts; k0 += 64 * WAVES) {
    const int32_t mine = k0 + l * WAVES, n = min((parts - k0 + WAVES - 1) / WAVES, 64);
    const bool real = mine < parts;
    const f32x2 st = real ? *(const f32x2*)(g.part_ml + 2 * (pr + (int64_t)mine * TR)) : f32x2{kNoRef, 0.f};
    // eight parts' columns on their way at once, the first ones beside the references; what is over is the last part times a lane's 0
    const float* at = g.part_o + (pr + (int64_t)k0 * TR) * D + l * (D / 64);
    auto load = [&](int32_t k, cols (&v)[8]) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = *(const cols*)(at + (int64_t)min(k + j, n - 1) * WAVES * TR * D);
    };
    cols v[8];
    load(0, v);
    float top = st[0];
#pragma unroll
    for (int i = 1; i < 64; i <<= 1) top = fmaxf(top, __shfl_xor(top, i));
    const float next = fmaxf(best, top), keep = __builtin_amdgcn_exp2f(best - next), f = real ? __builtin_amdgcn_exp2f(st[0] - next) : 0.f;
    best = next;
    float sum = st[1] * f;
#pragma unroll
    for (int i = 1; i < 64; i <<= 1) sum += __shfl_xor(sum, i);
    total = total * keep + sum;
#pragma unroll
    for (int i = 0; i < D / 64; ++i) y[i] *= keep;
    for (int32_t k = 0; k < n; k += 8) {
      if (k) load(k, v);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float fk = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f), k + j));
#pragma unroll
        for (int i = 0; i < D / 64; ++i) y[i] += v[j][i] * fk;
      }
    }
  }
  if constexpr (WAVES == 4) {
#pragma unroll
    for (int i = 0; i < D / 64; ++i) sums[w][l * (D / 64) + i] = y[i];
    if (l == 0) {
      stat[w][0] = best;
      stat[w][1] = total;
    }
    __syncthreads();
    if (w) return;
    best = fmaxf(fmaxf(stat[0][0], stat[1][0]), fmaxf(stat[2][0], stat[3][0]));
    total = 0.f;
#pragma unroll
    for (int i = 0; i < D / 64; ++i) y[i] = 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float f = __builtin_amdgcn_exp2f(stat[k][0] - best);
      total += stat[k][1] * f;
#pragma unroll
      for (int i = 0; i < D / 64; ++i) y[i] += sums[k][l * (D / 64) + i] * f;
    }
  }
  const int32_t row = job.row0 + r, x = row / pg.group, token = job.first + x, ob = token < a.o.t ? 0 : token / a.o.t, ot = token - ob * a.o.t;
  T* out = (T*)a.o.p + ob * a.o.sb + (kvh * pg.group + row - x * pg.group) * a.o.sh + ot * a.o.st + l * (D / 64);
  const float inv = total == 0.f ? 0.f : 1.f / total;
#pragma unroll
  for (int i = 0; i < D / 64; ++i) out[i] = (T)(y[i] * inv);
}

constexpr int64_t kLaunchThreads = 0xffffffffll;                            // of a launch's dimension at most
inline int64_t rows_groups(int32_t tokens) { return ((int64_t)tokens + kRowsWaves - 1) / kRowsWaves; }

inline bool tile_fits(int d) { return d == 64 || d == 128; }

// How the work is dealt out.  Row tiles of 32 where a request has more than 16 rows (new rows times the group) and rows are bf16.
// Parts of the keys, of 256 at least (one tile a wave):
//  - none where the longest request is short.  One part takes about 5 us and 1.15 us for 256 keys more, 1.7 where all compute units are
//    busy; joining parts takes 4.  One request, 8 kv heads: 512 keys 7.6 us whole and 9.2 in parts, 1024 keys 10.2 and 9.3; 32 requests:
//    1024 keys 13 and 18 us, 2048 keys 18 and 25.
//  - else as many as bring the launch to the workgroups that are resident at once, two a compute unit: more of them only add their
//    starts and ends (a request of 131072 keys, 8 heads of 4: 37 us, with twice as many 42), unless requests differ in length: those of a
//    batch of single tokens are cut half as long, so that short ones make room (32 requests of 128 .. 8192 keys: 27 us, without 36).
// One number of parts holds for all requests, from the longest and from how many tiles there are.  So one that is far longer than the others
// is cut into too few: 131072 keys, 8 kv heads of 4, take 33 us alone, 262 beside 31 single tokens on up to 8192 and 778 beside 63.
constexpr int kPartTiles = 8;                  // a workspace holds parts of so many times the tiles that are resident: 68 MB at d = 128
struct TilePlan { int tr, rows, splits, chunk, by_request; int64_t slots; size_t rows_all; };
inline TilePlan tile_plan(int dtype, const PagesAttnArgs& a) {
  TilePlan p{};
  const int64_t most = (int64_t)a.max_new * a.pg.group;
  p.tr = dtype != LOCOCO_BF16 || most <= 16 ? 16 : 32;
  const int tr = p.tr;
  p.by_request = most <= tr;
  p.rows = (int)(most < tr ? most : tr);
  p.slots = p.by_request ? a.n : (int64_t)a.tokens * a.pg.group / tr + std::min(a.n, a.tokens);     // (first_slot)
  // tiles that have rows, about (one at least: a call without rows asks for its workspace as well)
  const int64_t units = (p.by_request ? a.n : std::max<int64_t>(((int64_t)a.tokens * a.pg.group + tr - 1) / tr, 1)) * a.pg.Hkv;
  const int64_t keys = a.max_held > 0 ? a.max_held : 1;
  constexpr int64_t kLeast = kTileWaves * kTileKeys;
  // not fewer parts for more keys: a workspace for many takes fewer
  const int64_t resident = 2 * (int64_t)cu_count(), target = p.by_request && a.n > 1 && units < resident ? 2 * resident : resident;
  const int64_t whole = 2 * units >= resident ? 2048 : 768;
  // slots may be more than tiles: parts lie in the workspace by slot, and what they take there is bounded (two requests of 33 and 7 rows
  // on 131072 keys among 510 without rows, 8 kv heads: 66 MB and 263 us; bounded at a quarter of that, 705 us)
  const int64_t room = kPartTiles * resident / std::max<int64_t>(p.slots * a.pg.Hkv, 1);
  const int64_t want = keys <= whole ? 1 : std::max<int64_t>(std::min(target / units, room), 1);
  const int64_t splits = std::min(want, (keys + kLeast - 1) / kLeast);
  p.splits = (int)splits;
  p.chunk = (int)std::max<int64_t>(kLeast, ((keys + splits - 1) / splits + kTileKeys - 1) / kTileKeys * kTileKeys);
  p.rows_all = (size_t)p.slots * a.pg.Hkv * p.splits * tr;
  return p;
}

constexpr int kTileThreads = 64 * kTileWaves, kJoinThreads = 256;
// workgroups of the two launches; the join takes a row with a wave, or with four where there are many parts
inline int64_t tile_groups(const TilePlan& p, int Hkv) { return p.slots * Hkv * p.splits; }
inline int64_t join_groups(const TilePlan& p, int Hkv) {
  return p.splits == 1 ? 0 : p.slots * Hkv * (p.splits > 16 ? p.rows : (p.rows + 3) / 4);
}

}  // namespace pages_detail
}  // namespace lococo
