// The norm of many tensors together, and the tensors scaled to a length.
//
//   N = sqrt(sum over tensors of sum_i g_i^2),      g <- g max_norm / N  where N is finite and larger than max_norm
//
// Bound by memory: the gradients are read once for the norm and once for the scaling, and written once.  Squares are taken and added up in
// 64 bits, so that no gradient's square is too large or too small for its sum; every workgroup has a fixed share of the tensors, and the
// shares are added in a fixed order.
#pragma once

#include "rows.hip.h"

namespace oapl {

constexpr int kClipTensors = 96;        // of one launch: their list is an argument
constexpr int kClipChunk = 16384;       // elements that a workgroup takes at a time
constexpr int kClipGrid = 2048;         // workgroups of a launch, at most

struct ClipTensor {
  const void* data;
  void* out;
  int64_t n;
  uint32_t first;                       // chunks of the tensors before it
  int32_t dtype;
};
struct ClipArgs {
  ClipTensor t[kClipTensors];
  int32_t count, sums;                  // tensors; sums in all
  uint32_t chunks;
  double* sum;                          // of every workgroup of every launch; this launch's begin at `mine`
  int32_t mine;
  float max_norm;
  const float* norm;                    // given, or nullptr: from the sums
  float* norm_out;
};

template <class F>
__device__ __forceinline__ void clip_chunks(const ClipArgs& p, F f) {
  for (uint32_t chunk = blockIdx.x; chunk < p.chunks; chunk += gridDim.x) {
    int lo = 0, hi = p.count - 1;                   // the last tensor that begins at or before the chunk
    while (lo < hi) {
      const int mid = (lo + hi + 1) / 2;
      if (p.t[mid].first <= chunk) lo = mid;
      else hi = mid - 1;
    }
    const ClipTensor& t = p.t[lo];
    const int64_t from = (int64_t)(chunk - t.first) * kClipChunk;
    const int n = (int)(t.n - from < kClipChunk ? t.n - from : kClipChunk);
    if (t.dtype == 1) f((const bf16_t*)t.data + from, (bf16_t*)t.out + from, n);
    else f((const float*)t.data + from, (float*)t.out + from, n);
  }
}

__device__ __forceinline__ double clip_block_sum(double v) {
  __shared__ double all[4];
  v = wave_sum(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) all[threadIdx.x >> 6] = v;
  __syncthreads();
  return ((all[0] + all[1]) + all[2]) + all[3];
}

__global__ __launch_bounds__(256) void k_grad_squares(const ClipArgs p) {
  double sum = 0.0;
  clip_chunks(p, [&](const auto* x, auto*, int n) {
    for (int i = threadIdx.x * 8; i < n; i += 256 * 8) {
      const Eight v = load_piece(x, i, n);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum += (double)v.v[e] * (double)v.v[e];
    }
  });
  sum = clip_block_sum(sum);
  if (threadIdx.x == 0) p.sum[p.mine + blockIdx.x] = sum;
}

// The norm, the same in every thread of every workgroup: all of the sums in one order.
__device__ __forceinline__ float clip_norm(const ClipArgs& p) {
  if (p.norm) return *p.norm;
  double v = 0.0;
  for (int i = threadIdx.x; i < p.sums; i += 256) v += p.sum[i];
  return (float)sqrt(clip_block_sum(v));
}

__global__ __launch_bounds__(256) void k_grad_norm(const ClipArgs p) {
  const float norm = clip_norm(p);
  if (threadIdx.x == 0) *p.norm_out = norm;
}

// The factor is a number of 64 bits, and so is its product with a gradient until that is rounded: 32 bits would hold a factor below 2^-126 in
// fewer bits.
__global__ __launch_bounds__(256) void k_grad_scale(const ClipArgs p) {
  const float norm = clip_norm(p);
  if (p.norm_out && blockIdx.x == 0 && threadIdx.x == 0) *p.norm_out = norm;
  const bool clips = norm > p.max_norm && norm <= 3.4028235e38f;
  const double factor = clips ? (double)p.max_norm / (double)norm : 1.0;
  clip_chunks(p, [&](const auto* x, auto* y, int n) {
    if (!clips && (const void*)x == (const void*)y) return;
    for (int i = threadIdx.x * 8; i < n; i += 256 * 8) {
      Eight v = load_piece(x, i, n);
      if (clips) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v.v[e] = (float)((double)v.v[e] * factor);
      }
      store_piece(y, i, n, v);
    }
  });
}

}  // namespace oapl
