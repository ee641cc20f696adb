// Norm and position rotation of query and key rows: what the kernels of rows_rotate.hip and pages_append.hip share.  Nothing here is public.
//
//   n = x / sqrt(mean(x^2) + eps) * w        (or n = x)
//   y_a = n_a cos - n_b sin, y_b = n_b cos + n_a sin        (a, b) the two channels of pair i, the angle position * freqs[i]
//
// A row is P lanes of four pairs (P a power of two, lanes behind the row idle): both channels of a pair are a lane's own, a mean is a few
// exchanges inside a wave.  A workgroup's rows stand at few positions: their cosines and sines are computed once, to LDS, for all heads, and a
// lane keeps its four pairs' in registers from head to head, times the weights where all heads share them.
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
inline int32_t lanes_log(int32_t d) {
  int32_t lp = 0;
  while (8 << lp < d) ++lp;
  return lp;
}

namespace rotate_detail {

typedef __attribute__((ext_vector_type(2))) uint32_t w2;

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
__device__ __forceinline__ void read4(const T* p, float (&x)[4]) {
  if constexpr (std::is_same<T, float>::value) {
    const f4_any v = *(const f4_any*)p;
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = v[k];
  } else {
    const w2 v = *(const w2*)p;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      x[2 * k] = __uint_as_float(v[k] << 16);
      x[2 * k + 1] = __uint_as_float(v[k] & 0xffff0000u);
    }
  }
}
template <typename T>
__device__ __forceinline__ void write4(T* p, const float (&x)[4]) {
  if constexpr (std::is_same<T, float>::value) {
    *(f4_any*)p = f4_any{x[0], x[1], x[2], x[3]};
  } else {
    __align__(8) __bf16 y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = (__bf16)x[i];
    *(w2*)p = *(const w2*)y;
  }
}

// The four pairs of a lane, q0 .. q0 + 3 of the row's d / 2; those from r / 2 on are not turned.
enum PairKind {
  kHalves4,                                    // channels q and q + r / 2, r a multiple of 8; not turned: halves of the rest, likewise
  kHalves,                                     // any other r; the rest two by two
  kAdjacent                                    // channels 2 q and 2 q + 1
};
// a lane's eight channels as they were loaded: what waits for its turn takes no more registers than it has bytes
template <typename T, int KIND>
struct RawPairs {
  typename std::conditional<std::is_same<T, float>::value, f4_any, w2>::type a, b;
};
template <typename T>
struct RawPairs<T, kHalves> {
  T a[4], b[4];
};

template <int KIND>
struct Pairs {
  int32_t q0, half, r, d;
  __device__ __forceinline__ bool in() const { return 2 * q0 < d; }
  __device__ __forceinline__ bool turned(int i) const { return q0 + (KIND == kHalves4 ? 0 : i) < half; }
  __device__ __forceinline__ int32_t first(int i) const {
    const int32_t q = q0 + i;
    return KIND == kAdjacent ? 2 * q : q < half ? q : KIND == kHalves4 ? half + q : 2 * q;
  }
  __device__ __forceinline__ int32_t second(int i) const {
    const int32_t q = q0 + i;
    return KIND == kAdjacent ? 2 * q + 1 : q < half ? q + half : KIND == kHalves4 ? q + d / 2 : 2 * q + 1;
  }
  template <typename T>
  __device__ __forceinline__ void load(const T* row, float (&a)[4], float (&b)[4]) const {
    if constexpr (KIND == kHalves4) {
      read4(row + first(0), a);
      read4(row + second(0), b);
    } else if constexpr (KIND == kAdjacent) {
      float x[8];
      read8(row + 2 * q0, x);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        a[i] = x[2 * i];
        b[i] = x[2 * i + 1];
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        a[i] = (float)row[first(i)];
        b[i] = (float)row[second(i)];
      }
    }
  }
  template <typename T>
  __device__ __forceinline__ void load(const T* row, RawPairs<T, KIND>& x) const {
    if constexpr (KIND == kHalves) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x.a[i] = row[first(i)];
        x.b[i] = row[second(i)];
      }
    } else if constexpr (KIND == kHalves4) {
      x.a = *(const decltype(x.a)*)(row + first(0));
      x.b = *(const decltype(x.b)*)(row + second(0));
    } else if constexpr (std::is_same<T, float>::value) {
      x.a = *(const f4_any*)(row + 2 * q0);
      x.b = *(const f4_any*)(row + 2 * q0 + 4);
    } else {
      const w4 v = *(const w4*)(row + 2 * q0);
      x.a = w2{v[0], v[1]};
      x.b = w2{v[2], v[3]};
    }
  }
  template <typename T>
  __device__ __forceinline__ void unpack(const RawPairs<T, KIND>& x, float (&a)[4], float (&b)[4]) const {
    float y[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (KIND == kHalves) {
        y[i] = (float)x.a[i];
        y[4 + i] = (float)x.b[i];
      } else if constexpr (std::is_same<T, float>::value) {
        y[i] = x.a[i];
        y[4 + i] = x.b[i];
      } else {
        y[i] = __uint_as_float(i & 1 ? x.a[i / 2] & 0xffff0000u : x.a[i / 2] << 16);
        y[4 + i] = __uint_as_float(i & 1 ? x.b[i / 2] & 0xffff0000u : x.b[i / 2] << 16);
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      a[i] = KIND == kAdjacent ? y[2 * i] : y[i];
      b[i] = KIND == kAdjacent ? y[2 * i + 1] : y[4 + i];
    }
  }
  template <typename T>
  __device__ __forceinline__ void store(T* row, const float (&a)[4], const float (&b)[4]) const {
    if constexpr (KIND == kHalves4) {
      write4(row + first(0), a);
      write4(row + second(0), b);
    } else if constexpr (KIND == kAdjacent) {
      float x[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[2 * i] = a[i];
        x[2 * i + 1] = b[i];
      }
      write8(row + 2 * q0, x);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        row[first(i)] = (T)a[i];
        row[second(i)] = (T)b[i];
      }
    }
  }
};
inline PairKind pair_kind(int32_t r, int32_t adjacent) { return adjacent ? kAdjacent : r % 8 ? kHalves : kHalves4; }

// The angle position * freq in half turns, whole turns left out: in [-1, 1] or little beyond, off by some 2^-53 at any position and at
// frequencies up to 2^24.  The product has up to 55 bits and 1 / pi has no end, so both are sums of two numbers: what a product leaves over is
// an fma.
__device__ __forceinline__ double half_turns(int32_t position, float freq) {
  constexpr double kHi = 0.3183098861837907, kLo = -1.9678676675182486e-17;    // of 1 / pi
  const double p = position, f = freq, a = p * f, h = a * kHi;
  return h - 2.0 * rint(h * 0.5) + (fma(a, kHi, -h) + fma(a, kLo, fma(p, f, -a) * kHi));
}

// Its cosine and sine in fp32, right to two steps of their own size.  They are taken of what it is from the nearest quarter turn, y in
// [-pi / 4, pi / 4], which rounds to fp32 by 2^-25 or less and near a zero of either by less (rounded in half turns up to 1, by 2^-25 of them, results
// were twice as far from exact ones).  sin y = y + y^3 P(y^2), cos y = 1 - y^2 / 2 + y^4 Q(y^2): P and Q of degree two by least maximum error, 0.06 u
// and 0.002 u of the results.
__device__ __forceinline__ void cos_sin(int32_t position, float freq, float* c, float* s) {
  const double h = half_turns(position, freq), quarters = rint(2.0 * h);
  const int32_t k = (int32_t)quarters;
  const float y = (float)((h - 0.5 * quarters) * 3.141592653589793), z = y * y;
  const float si = fmaf(y * z, fmaf(z, fmaf(z, -0.00019517137843649834f, 0.008332177065312862f), -0.16666655242443085f), y);
  const float co = fmaf(z, fmaf(z, fmaf(z, fmaf(z, 2.4438271793769673e-05f, -0.0013887366512790322f), 0.04166664555668831f), -0.5f), 1.f);
  const float a = k & 1 ? -si : co, b = k & 1 ? co : si;
  *c = k & 2 ? -a : a;
  *s = k & 2 ? -b : b;
}

// sums over the P lanes of a row; in fp32 up to 16 lanes without a trip through the LDS crossbar
template <int CTRL>
__device__ __forceinline__ float beside(float x) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float row_sum(float x, int32_t lp) {
  if (lp > 0) x += beside<0xb1>(x);            // lanes 1, 0, 3, 2 of four
  if (lp > 1) x += beside<0x4e>(x);            // lanes 2, 3, 0, 1
  if (lp > 2) x += beside<0x141>(x);           // eight, the other way round: the other four's sum
  if (lp > 3) x += beside<0x140>(x);           // sixteen
  if (lp > 4) x += __shfl_xor(x, 16);
  return x;
}
__device__ __forceinline__ double row_sum(double x, int32_t lp) {
  for (int k = 1; k < 1 << lp; k <<= 1) x += __shfl_xor(x, k);
  return x;
}

// one over the root of a row's mean square; again in 64 bits where the squares leave 32
__device__ __forceinline__ float one_of_large(const float (&a)[4], const float (&b)[4], int32_t lp, const RotateView& rv) {
  double sum = 0.0;
#pragma unroll
  for (int i = 0; i < 4; ++i) sum = fma((double)a[i], (double)a[i], fma((double)b[i], (double)b[i], sum));
  return (float)(1.0 / sqrt(row_sum(sum, lp) / rv.d + rv.eps));
}
__device__ __forceinline__ float one_over_root(const float (&a)[4], const float (&b)[4], int32_t lp, const RotateView& rv) {
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) sum = fmaf(a[i], a[i], fmaf(b[i], b[i], sum));
  sum = row_sum(sum, lp);
  return sum == INFINITY ? one_of_large(a, b, lp, rv) : rsqrtf(sum * (1.f / (float)rv.d) + rv.eps);
}

constexpr int kAhead = 2;                      // rows of a lane on their way at once

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
  int32_t stretch;                             // tiles whose part of d_w a lane adds up in fp32
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
