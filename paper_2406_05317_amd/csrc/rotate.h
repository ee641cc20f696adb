// Norm and position rotation of query and key rows: what the kernels of rows_rotate.hip and pages_append.hip share.  Nothing here is public.
//
//   n = x / sqrt(mean(x^2) + eps) * w        (or n = x)
//   y_a = n_a cos - n_b sin, y_b = n_b cos + n_a sin        (a, b) the two channels of pair i, the angle position * freqs[i]
//
// A row is P lanes of eight consecutive channels (P a power of two, lanes behind the row idle), so that a mean is a few exchanges inside a
// wave and every access is 16 bytes or more.  What a lane's channels are turned against it loads once more, from where the lane beside it
// has just had it fetched.  A workgroup's rows stand at few positions: their cosines and sines are computed once, to LDS, for all heads.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "pages.h"

namespace lococo {

struct RotateView {
  const float* freqs;                          // radians a position, r / 2 of them
  const void* w[2];                            // norm weights of q, k (or null): head h's at h * ws
  int64_t ws[2];
  int32_t heads[2];
  int32_t d, r, adjacent, norm;
  float eps;
};

constexpr int kRotateThreads = 256, kRotateMaxDim = 256;
constexpr int kRotateTable = 1024;             // pairs of a workgroup's positions: 256 / P of them, 4 P pairs each at most

// how a workgroup of 256 / P rows at a time is laid out: 2^lt positions, the rest heads side by side
struct RotateShape {
  int32_t lp, lt;                              // P = 2^lp lanes to a row
  int32_t hb;                                  // heads of a workgroup
};

namespace rotate_detail {

typedef __attribute__((ext_vector_type(4))) uint32_t w4;
typedef __attribute__((ext_vector_type(4), aligned(4))) float f4_any;          // fp32 rows begin at any float

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
template <typename T>
__device__ __forceinline__ void write8(T* p, const float (&x)[8]) {
  if constexpr (std::is_same<T, float>::value) {
#pragma unroll
    for (int i = 0; i < 2; ++i) *(f4_any*)(p + 4 * i) = f4_any{x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]};
  } else {
    __align__(16) __bf16 y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = (__bf16)x[i];
    *(w4*)p = *(const w4*)y;
  }
}

template <typename T>
__device__ __forceinline__ const T* row_at(const RowsView& r, int32_t token, int32_t head) {
  const int32_t b = token < r.t ? 0 : token / r.t, t = token - b * r.t;
  return (const T*)r.p + b * r.sb + head * r.sh + t * r.st;
}

// Which channels a lane's, c0 .. c0 + 7, are turned against.
enum PairKind {
  kHalves8,                                    // channels j and j + r / 2, r / 2 a multiple of 8: a lane's are all first ones, all second ones
  kHalves,                                     // or not turned at all; any other r
  kAdjacent                                    // channels 2 j and 2 j + 1: pairs do not leave a lane
};
template <int KIND>
struct Partners {
  int32_t c0, half, r;
  __device__ __forceinline__ int32_t pair(int i) const {
    const int32_t c = c0 + i;
    return KIND == kAdjacent ? c >> 1 : c < half ? c : c - half;
  }
  __device__ __forceinline__ bool turned(int i) const { return c0 + (KIND == kHalves8 ? 0 : i) < r; }
  __device__ __forceinline__ bool second(int i) const { return KIND == kAdjacent ? i & 1 : c0 + (KIND == kHalves8 ? 0 : i) >= half; }
  // the partners of the lane's channels in a row of a type, `own` those channels
  template <typename T>
  __device__ __forceinline__ void load(const T* row, const float (&own)[8], float (&x)[8]) const {
    if constexpr (KIND == kAdjacent) {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = own[i ^ 1];
    } else if constexpr (KIND == kHalves8) {
      if (c0 < r) read8(row + (c0 < half ? c0 + half : c0 - half), x);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (c0 + i < r) x[i] = (float)row[c0 + i < half ? c0 + i + half : c0 + i - half];
    }
  }
};
inline PairKind pair_kind(int32_t r, int32_t adjacent) { return adjacent ? kAdjacent : r % 16 ? kHalves : kHalves8; }

// whole turns left out of the angle in 64 bits (position * frequency is exact there): half turns in [-1, 1]
__device__ __forceinline__ float half_turns(int32_t position, float freq) {
  const double h = (double)position * (double)freq * 0.31830988618379067154;
  return (float)(h - 2.0 * rint(h * 0.5));
}

// sums over the P lanes of a row
template <typename R>
__device__ __forceinline__ R row_sum(R x, int32_t lp) {
  for (int k = 1; k < 1 << lp; k <<= 1) x += __shfl_xor(x, k);
  return x;
}

}  // namespace rotate_detail

struct RotateArgs {
  RotateView rv;
  RotateShape sh;
  RowsView in[2], out[2];                      // q, k
  const int32_t* positions;                    // null: a row's number in its batch entry
  int32_t tokens, t;
  int32_t blocks[2];                           // workgroups to a tile of positions for q's heads, for k's
};

struct RotateBackArgs {
  RotateView rv;
  RotateShape sh;
  RowsView in[2];
  const float* gy[2];                          // [b, heads, t, d]
  float* gx[2];
  float* gw[2];                                // null: not wanted
  const int32_t* positions;
  int32_t tokens, t;
  int32_t blocks[2];
  int32_t chunks, tiles;                       // workgroups to a block of heads, tiles of positions to a workgroup
  float* parts;                                // [block][chunk][d]
};

// ---- rows_rotate.hip
bool rows_rotate_fits(const RotateView& rv, int32_t tokens);   // a launch takes the rows
hipError_t launch_rows_rotate(int dtype, RotateArgs a, hipStream_t s);
size_t rows_rotate_workspace_bytes(const RotateView& rv, int32_t tokens);
hipError_t launch_rows_rotate_backward(int dtype, RotateBackArgs a, void* workspace, hipStream_t s);

// ---- pages_append.hip
bool pages_append_fits(const PagesView& pg, int32_t tokens);
// q rows to out, k and v rows (turned, as they are) to their slots
hipError_t launch_pages_append(int dtype, const PagesView& pg, const RotateView& rv, const RowsView& q, const RowsView& k, const RowsView& v,
                               const RowsView& qo, int32_t tokens, const int32_t* slots, const int32_t* positions, hipStream_t s);

}  // namespace lococo
