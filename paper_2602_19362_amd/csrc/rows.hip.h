// Rows of channels ([row][channel], any distance between rows, from any element on), which the embedding and the residual stream's
// kernels share.
#pragma once

#include "heads.hip.h"

namespace oapl {

// One [rows][d] operand; the stride in bytes.
struct Rows {
  char* p;
  int64_t stride;
  template <class T>
  __device__ __forceinline__ T* row(int64_t i) const { return (T*)(p + i * stride); }
};

// W neighbouring channels, as they are stored and in 32 bits: eight where everything is bf16, four where something is fp32, so that a
// wavefront's access of 16 bytes a lane covers whole lines.  Rows may start at any element: memory takes accesses of 8 and 16 bytes at any
// address, aligned ones at full rate.
template <class T, int W>
struct RawOf {
  typedef T type __attribute__((ext_vector_type(W)));
  typedef uint32_t words __attribute__((ext_vector_type(W * sizeof(T) / 4), aligned(sizeof(T))));      // anywhere in memory
};
template <class T, int W>
using Raw = typename RawOf<T, W>::type;

template <int W>
struct Piece {
  float v[W];
};

template <class R>
__device__ __forceinline__ auto widened(const R& raw) {
  constexpr int W = sizeof(R) / sizeof(raw[0]);
  Piece<W> x;
#pragma unroll
  for (int i = 0; i < W; ++i) x.v[i] = (float)raw[i];
  return x;
}

// Channels c .. c + W - 1 of a row of d.  WHOLE: d is a multiple of W, and lanes behind the row's end repeat its last piece: their loads need no
// branch, which would keep those after it waiting (16411 rows of 768 bf16 channels in 128 lanes backwards 76 us with branches, 44 without).
// Otherwise there are zeros behind the end.  ONCE: an access that leaves nothing in the caches.
template <int W, bool WHOLE, bool ONCE = false, class T>
__device__ __forceinline__ Raw<T, W> load_raw(const T* row, int c, int d) {
  typedef typename RawOf<T, W>::words words;
  if (WHOLE || c + W <= d) {
    const words* at = (const words*)(row + (WHOLE ? min(c, d - W) : c));
    if constexpr (ONCE) return __builtin_bit_cast(Raw<T, W>, __builtin_nontemporal_load(at));
    else return __builtin_bit_cast(Raw<T, W>, *at);
  }
  Raw<T, W> x = {};
#pragma unroll
  for (int i = 0; i < W; ++i)
    if (c + i < d) x[i] = row[c + i];
  return x;
}
template <int W, bool WHOLE, bool ONCE = false, class T>
__device__ __forceinline__ Piece<W> load_piece(const T* row, int c, int d) {
  return widened(load_raw<W, WHOLE, ONCE>(row, c, d));
}

// Rounding to bf16 is to nearest even, once, of values held in 32 bits until then.
template <int W, bool ONCE = false, class T>
__device__ __forceinline__ void store_whole(T* p, const Piece<W>& x) {
  typedef typename RawOf<T, W>::words words;
  Raw<T, W> b;
#pragma unroll
  for (int i = 0; i < W; ++i) b[i] = (T)x.v[i];
  if constexpr (ONCE) __builtin_nontemporal_store(__builtin_bit_cast(words, b), (words*)p);
  else *(words*)p = __builtin_bit_cast(words, b);
}
template <int W, bool WHOLE, bool ONCE = false, class T>
__device__ __forceinline__ void store_piece(T* row, int c, int d, const Piece<W>& x) {
  if (c + W <= d) {
    store_whole<W, ONCE>(row + c, x);
  } else if constexpr (!WHOLE) {
#pragma unroll
    for (int i = 0; i < W; ++i)
      if (c + i < d) row[c + i] = (T)x.v[i];
  }
}

// Sum over a group of 16 lanes, or over a wavefront, in every lane and in a fixed order: rows of 16 lanes by rotations, then pairs of rows
// and of halves trade places.
template <int LANES>
__device__ __forceinline__ float lanes_total(float v) {
  static_assert(LANES == 16 || LANES == 64, "a row of lanes, or a wavefront");
  v = group_sum(v);
  if constexpr (LANES == 64) {
    v += __shfl_xor(v, 16, 64);
    v += __shfl_xor(v, 32, 64);
  }
  return v;
}

}  // namespace oapl
