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

// Eight channels in 32 bits.  Rows may start at any element: memory takes 16-byte accesses at any address, aligned ones at full rate.
struct Eight {
  float v[8];
};

__device__ __forceinline__ void load8(Eight& x, const float* p) {
  __builtin_memcpy(x.v, p, 32);
}
__device__ __forceinline__ void load8(Eight& x, const bf16_t* p) {
  bf16x8 b;
  __builtin_memcpy(&b, p, 16);
#pragma unroll
  for (int i = 0; i < 8; ++i) x.v[i] = (float)b[i];
}
// Rounding to bf16 is to nearest even, once, of values held in 32 bits until then.
__device__ __forceinline__ void store8(float* p, const Eight& x) {
  __builtin_memcpy(p, x.v, 32);
}
__device__ __forceinline__ void store8(bf16_t* p, const Eight& x) {
  bf16x8 b;
#pragma unroll
  for (int i = 0; i < 8; ++i) b[i] = (bf16_t)x.v[i];
  __builtin_memcpy(p, &b, 16);
}

// Channels c .. c + 7 of a row of d, zeros behind its end.
template <class T>
__device__ __forceinline__ Eight load_piece(const T* row, int c, int d) {
  Eight x = {};
  if (c + 8 <= d) {
    load8(x, row + c);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < d) x.v[i] = (float)row[c + i];
  }
  return x;
}
template <class T>
__device__ __forceinline__ void store_piece(T* row, int c, int d, const Eight& x) {
  if (c + 8 <= d) {
    store8(row + c, x);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < d) row[c + i] = (T)x.v[i];
  }
}

// Sum over a wavefront, in every lane, in a fixed order: rows of 16 lanes by rotations, then pairs of rows and of halves trade places.
__device__ __forceinline__ float wave_total(float v) {
  v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x128, 0xf, 0xf, false));
  v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x124, 0xf, 0xf, false));
  v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x122, 0xf, 0xf, false));
  v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x121, 0xf, 0xf, false));
  v += __shfl_xor(v, 16, 64);
  return v + __shfl_xor(v, 32, 64);
}

}  // namespace oapl
