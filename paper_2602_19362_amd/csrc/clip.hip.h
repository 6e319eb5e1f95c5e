// The norm of many tensors together, and the tensors scaled to a length.
//
//   N = sqrt(sum over tensors of sum_i g_i^2),      g <- g max_norm / N  where N is finite and larger than max_norm
//
// Bound by memory: the gradients are read once for the norm and once for the scaling, and written once (98 tensors of 6.3 GB, into others: 19
// GB in 3.1 ms, 6.1 TB/s).  Squares are taken and added up in 64 bits, so that no gradient's square is too large or too small for its sum;
// every workgroup has a fixed share of the tensors, and the shares are added in a fixed order.
#pragma once

#include "rows.hip.h"

namespace oapl {

constexpr int kClipTensors = 112;       // of one launch: their list is an argument, of less than 4 KB
constexpr int kClipGrid = 2048;         // workgroups that have sums, at most

struct ClipTensor {
  const void* data;
  void* out;
  int64_t n;
  uint32_t first;                       // chunks of the tensors before it
  int32_t bf16;
};
struct ClipArgs {
  ClipTensor t[kClipTensors];
  int32_t count, chunk;                 // tensors; elements that a workgroup takes at a time, a multiple of 2048
  uint32_t chunks;
  int32_t mine, sums;                   // where this launch's sums begin, and how many there are in all
  double* sum;                          // of every workgroup of every launch
  float max_norm;
  const float* norm;                    // given, or nullptr: from the sums
  float* norm_out;
};
static_assert(sizeof(ClipArgs) <= 4096 - 256, "launch arguments");

// f(data, out, elements) of a chunk.
template <class F>
__device__ __forceinline__ void clip_chunk(const ClipArgs& p, uint32_t chunk, F f) {
  int lo = 0, hi = p.count - 1;                   // the last tensor that begins at or before the chunk: an empty one has none
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (p.t[mid].first <= chunk) lo = mid;
    else hi = mid - 1;
  }
  const ClipTensor& t = p.t[lo];
  const int64_t from = (int64_t)(chunk - t.first) * p.chunk;
  const int n = (int)(t.n - from < p.chunk ? t.n - from : p.chunk);
  if (t.bf16) f((const bf16_t*)t.data + from, (bf16_t*)t.out + from, n);
  else f((const float*)t.data + from, (float*)t.out + from, n);
}

__device__ __forceinline__ double clip_block_sum(double v) {
  __shared__ double all[4];
  v = wave_sum(v);
  if ((threadIdx.x & 63) == 0) all[threadIdx.x >> 6] = v;
  __syncthreads();
  return ((all[0] + all[1]) + all[2]) + all[3];
}

// A workgroup's sum over every gridDim.x-th chunk.  98 tensors of 6.3 GB: 6.6 TB/s.  ONCE: past the caches.
template <bool ONCE>
__global__ __launch_bounds__(256) void k_grad_squares(const ClipArgs p) {
  double sum = 0.0;
  for (uint32_t chunk = blockIdx.x; chunk < p.chunks; chunk += gridDim.x)
    clip_chunk(p, chunk, [&](const auto* x, auto*, int n) {
      constexpr int W = 16 / sizeof(*x);
#pragma unroll 4
      for (int i = threadIdx.x * W; i < n; i += 256 * W) {
        const Piece<W> v = load_piece<W, kAny, ONCE>(x, i, n);
#pragma unroll
        for (int e = 0; e < W; ++e) sum += (double)v.v[e] * (double)v.v[e];
      }
    });
  sum = clip_block_sum(sum);
  if (threadIdx.x == 0) p.sum[p.mine + blockIdx.x] = sum;
}

// The norm, the same in every thread of every workgroup: all of the sums in one order.
__device__ __forceinline__ float clip_norm(const ClipArgs& p) {
  if (p.norm) return *p.norm;
  double v = 0.0;
#pragma unroll 8
  for (int i = threadIdx.x; i < p.sums; i += 256) v += p.sum[i];
  return (float)sqrt(clip_block_sum(v));
}

__global__ __launch_bounds__(256) void k_grad_norm(const ClipArgs p) {
  const float norm = clip_norm(p);
  if (threadIdx.x == 0) *p.norm_out = norm;
}

// The last chunks first: of what was read for the norm, those are still in the memory-side cache.  The same 98 tensors: 5.9 TB/s (5.7 with one
// piece at a time).  The factor is a number of 64 bits, and so is its product with a gradient until that is rounded (for bf16 to 32 bits first,
// which moves the last rounding by 2^-24): 32 bits would hold a factor below 2^-126 in fewer bits.
template <bool LOAD_ONCE, bool STORE_ONCE>
__global__ __launch_bounds__(256) void k_grad_scale(const ClipArgs p) {
  const float norm = clip_norm(p);
  if (p.norm_out && blockIdx.x == 0 && threadIdx.x == 0) *p.norm_out = norm;
  const bool clips = norm > p.max_norm && norm <= 3.4028235e38f;
  const double factor = clips ? (double)p.max_norm / (double)norm : 1.0;
  const uint32_t chunk = blockIdx.y * gridDim.x + blockIdx.x;
  if (chunk < p.chunks)
    clip_chunk(p, p.chunks - 1 - chunk, [&](const auto* x, auto* y, int n) {
      if (!clips && (const void*)x == (const void*)y) return;
      constexpr int W = 16 / sizeof(*x);
      // two pieces a lane, loaded before one is stored, which might be what the other is loaded from for all the compiler knows
      const auto scale = [&](auto form, auto pieces, int at) {
        constexpr Form FORM = form;
        constexpr int PIECES = pieces;
        Piece<W> v[PIECES];
#pragma unroll
        for (int i = 0; i < PIECES; ++i) v[i] = load_piece<W, FORM, LOAD_ONCE>(x, at + i * 256 * W, n);
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
          if (clips) {
#pragma unroll
            for (int e = 0; e < W; ++e) v[i].v[e] = (float)((double)v[i].v[e] * factor);
          }
          store_piece<W, FORM, STORE_ONCE>(y, at + i * 256 * W, n, v[i]);
        }
      };
      int at = threadIdx.x * W;
      for (; at + 256 * W + W <= n; at += 2 * 256 * W) scale(std::integral_constant<Form, kWhole>{}, std::integral_constant<int, 2>{}, at);
      for (; at < n; at += 256 * W) scale(std::integral_constant<Form, kAny>{}, std::integral_constant<int, 1>{}, at);
    });
}

}  // namespace oapl
