// Tensors of heads ([token][head][channel], any token and head stride) and the packed sequences they hold: what the
// norm-and-rotation kernels and the attention kernels share.
#pragma once

#include "common.hip.h"

namespace oapl {

constexpr int kMaxHeadDim = 128;

// One [tokens][heads][D] operand; strides in bytes.
struct Heads {
  char* p;
  int64_t token, head;
  __device__ __forceinline__ char* row(int64_t t, int h) const { return p + t * token + h * head; }
};

__device__ __forceinline__ f32x4 load4(const float* p) { return *(const f32x4*)p; }
__device__ __forceinline__ f32x4 load4(const bf16_t* p) {
  const bf16x4 v = *(const bf16x4*)p;
  return f32x4{(float)v[0], (float)v[1], (float)v[2], (float)v[3]};
}
// Rounding to bf16 is to nearest even, once, of a value held in 32 bits until then.
__device__ __forceinline__ void store4(float* p, f32x4 v) { *(f32x4*)p = v; }
__device__ __forceinline__ void store4(bf16_t* p, f32x4 v) {
  *(bf16x4*)p = bf16x4{(bf16_t)v[0], (bf16_t)v[1], (bf16_t)v[2], (bf16_t)v[3]};
}

// Sum over the 16 lanes of a group, in every lane: rotations by 8, 4, 2 and 1 of a row of lanes.
__device__ __forceinline__ float group_sum(float v) {
  v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x128, 0xf, 0xf, false));
  v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x124, 0xf, 0xf, false));
  v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x122, 0xf, 0xf, false));
  v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x121, 0xf, 0xf, false));
  return v;
}

__device__ __forceinline__ float quiet_nan() { return __builtin_nanf(""); }

}  // namespace oapl
