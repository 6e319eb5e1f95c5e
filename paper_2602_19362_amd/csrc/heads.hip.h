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

__device__ __forceinline__ float quiet_nan() { return __builtin_nanf(""); }

}  // namespace oapl
