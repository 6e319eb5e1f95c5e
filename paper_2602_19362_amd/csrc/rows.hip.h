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

// Rows of d channels in pieces of W: d is a multiple of W, has a part of a piece more, or may be anything, fewer than W too.
enum Form { kWhole, kRagged, kAny };

// Channels c .. c + W - 1 of a row of d.  Loads of whole and ragged rows need no branch, which would keep those after it waiting (16411 rows of
// 768 bf16 channels in 128 lanes backwards 76 us with branches, 44 without; 16000 of 333 52 and 24): lanes behind the row's last W channels load
// those.  In ragged rows `own` drops what the lane before holds of them; lanes behind a whole row's end repeat its last piece.  Of rows of any
// width, the part behind the end is zero.  ONCE: an access that leaves nothing in the caches.
template <int W, Form FORM, bool ONCE = false, class T>
__device__ __forceinline__ Raw<T, W> load_raw(const T* row, int c, int d) {
  typedef typename RawOf<T, W>::words words;
  if (FORM != kAny || c + W <= d) {
    const words* at = (const words*)(row + (FORM != kAny ? min(c, d - W) : c));
    if constexpr (ONCE) return __builtin_bit_cast(Raw<T, W>, __builtin_nontemporal_load(at));
    else return __builtin_bit_cast(Raw<T, W>, *at);
  }
  Raw<T, W> x = {};
#pragma unroll
  for (int i = 0; i < W; ++i)
    if (c + i < d) x[i] = row[c + i];
  return x;
}
// What was loaded, once it is there: a ragged row's last piece begins at c, with zeros behind the row's end.
template <Form FORM, class R>
__device__ __forceinline__ R own(const R& raw, int c, int d) {
  if constexpr (FORM != kRagged) return raw;
  constexpr int W = sizeof(R) / sizeof(raw[0]), N = sizeof(R) / 4, PER = W / N;
  typedef uint32_t words __attribute__((ext_vector_type(N)));
  words x = __builtin_bit_cast(words, raw);
  const int before = min(max(c + W - d, 0), W), whole = before / PER;          // channels to drop, and words of them
#pragma unroll
  for (int step = 4; step >= 1; step /= 2)
    if (step <= N)
#pragma unroll
      for (int k = 0; k < N; ++k) x[k] = whole & step ? (k + step < N ? x[k + step] : 0u) : x[k];
  if constexpr (PER == 2)
#pragma unroll
    for (int k = 0; k < N; ++k) x[k] = before & 1 ? (k + 1 < N ? x[k + 1] << 16 | x[k] >> 16 : x[k] >> 16) : x[k];
  return __builtin_bit_cast(R, x);
}
template <int W, Form FORM, bool ONCE = false, class T>
__device__ __forceinline__ Piece<W> load_piece(const T* row, int c, int d) {
  return widened(own<FORM>(load_raw<W, FORM, ONCE>(row, c, d), c, d));
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
template <int W, Form FORM, bool ONCE = false, class T>
__device__ __forceinline__ void store_piece(T* row, int c, int d, const Piece<W>& x) {
  if (c + W <= d) {
    store_whole<W, ONCE>(row + c, x);
  } else if constexpr (FORM != kWhole) {
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
