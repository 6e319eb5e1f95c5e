// A block's output added to the residual stream, and the root-mean-square norms before and behind the block, in one pass over the rows.
//
//   z = y r(y) o y_gain  (or y),   x' = x + scale gate o z,   n = gain o x' r(x'),   r(a) = (mean_c a_c^2 + eps)^(-1/2)
//
// Backwards, with v = x' r(x'), u = gain o dn, w = y r(y), t = y_gain o dz:
//
//   dX = dx' + r (u - v mean_c(u o v)),   dz = scale gate o dX,   dy = r(y) (t - w mean_c(t o w))  (or dz)
//   dgain = sum dn o v,   dy_gain = sum dz o w,   dgate = scale z o dX (summed over tokens where they share the gate)
//
// Bound by memory: every row is read once and written once, and stays in registers in between, in 32 bits; a row's sums are the only
// thing that its lanes exchange.
#pragma once

#include "rows.hip.h"

namespace oapl {

struct ResidualNormArgs {
  Rows x, y, gate;            // x: of the gradient, the stream behind the block; y.p, gate.p == nullptr: no block, no gate
  Rows x_out, out;            // forward: results; backwards: gradients of them (nullptr: none)
  Rows dx, dy, dgate;         // backwards: results
  const void *gain, *y_gain;  // nullptr: no norm
  float* partials;            // backwards: [workgroups][2][d], of dgain and of sum dX o w (times a token's gate)
  int64_t T;
  int d;
  float scale, eps;
};

// Sum over the THREADS lanes of a row, in all of them.  `turn`, kept by the caller, alternates between two places: a wavefront that is
// ahead writes to the other one, and cannot be two sums ahead of a barrier, so that one barrier a sum is enough.
template <int THREADS>
__device__ __forceinline__ float row_total(float v, int& turn) {
  v = wave_total(v);
  if constexpr (THREADS > 64) {
    __shared__ float all[2][THREADS / 64];
    turn ^= 1;
    if ((threadIdx.x & 63) == 0) all[turn][threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int i = 0; i < THREADS / 64; ++i) v += all[turn][i];
  }
  return v;
}

__device__ __forceinline__ float square_sum(const Eight& x) {
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) s += x.v[i] * x.v[i];
  return s;
}

// TX: the residual stream's type, T: the block's and the norms'.  THREADS lanes hold a row, eight channels in each of PIECES pieces.
template <class TX, class T, int THREADS, int PIECES>
__global__ __launch_bounds__(THREADS < 256 ? 256 : THREADS) void k_residual_norm_fwd(const ResidualNormArgs p) {
  constexpr int ROWS = THREADS < 256 ? 256 / THREADS : 1;
  const int lane = threadIdx.x % THREADS, d = p.d;
  int turn = 0;
  for (int64_t t = (int64_t)blockIdx.x * ROWS + threadIdx.x / THREADS; t < p.T; t += (int64_t)gridDim.x * ROWS) {
    Eight x[PIECES], y[PIECES];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int c = (i * THREADS + lane) * 8;
      x[i] = load_piece(p.x.row<TX>(t), c, d);
      if (p.y.p) y[i] = load_piece(p.y.row<T>(t), c, d);
    }
    if (p.y.p) {
      float r = p.scale;
      if (p.y_gain) {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < PIECES; ++i) sum += square_sum(y[i]);
        r *= rsqrtf(row_total<THREADS>(sum, turn) / (float)d + p.eps);
      }
#pragma unroll
      for (int i = 0; i < PIECES; ++i) {
        const int c = (i * THREADS + lane) * 8;
        if (p.y_gain) {
          const Eight g = load_piece((const T*)p.y_gain, c, d);
#pragma unroll
          for (int e = 0; e < 8; ++e) y[i].v[e] *= g.v[e];
        }
        if (p.gate.p) {
          const Eight g = load_piece(p.gate.row<T>(t), c, d);
#pragma unroll
          for (int e = 0; e < 8; ++e) y[i].v[e] *= g.v[e];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) x[i].v[e] += r * y[i].v[e];
        store_piece(p.x_out.row<TX>(t), c, d, x[i]);
      }
    }
    if (p.gain) {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < PIECES; ++i) sum += square_sum(x[i]);
      const float r = rsqrtf(row_total<THREADS>(sum, turn) / (float)d + p.eps);
#pragma unroll
      for (int i = 0; i < PIECES; ++i) {
        const int c = (i * THREADS + lane) * 8;
        const Eight g = load_piece((const T*)p.gain, c, d);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[i].v[e] *= r * g.v[e];
        store_piece(p.out.row<T>(t), c, d, x[i]);
      }
    }
  }
}

template <class TX, class T, int THREADS, int PIECES>
__global__ __launch_bounds__(THREADS < 256 ? 256 : THREADS) void k_residual_norm_bwd(const ResidualNormArgs p) {
  constexpr int ROWS = THREADS < 256 ? 256 / THREADS : 1;
  const int lane = threadIdx.x % THREADS, d = p.d;
  int turn = 0;
  Eight sum_gain[PIECES] = {}, sum_block[PIECES] = {};
  for (int64_t t = (int64_t)blockIdx.x * ROWS + threadIdx.x / THREADS; t < p.T; t += (int64_t)gridDim.x * ROWS) {
    Eight dx[PIECES], v[PIECES], u[PIECES];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int c = (i * THREADS + lane) * 8;
      dx[i] = p.x_out.p ? load_piece(p.x_out.row<TX>(t), c, d) : Eight{};
      if (p.gain) v[i] = load_piece(p.x.row<TX>(t), c, d), u[i] = load_piece(p.out.row<T>(t), c, d);
    }
    if (p.gain) {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < PIECES; ++i) sum += square_sum(v[i]);
      const float r = rsqrtf(row_total<THREADS>(sum, turn) / (float)d + p.eps);
      float m = 0.f;
#pragma unroll
      for (int i = 0; i < PIECES; ++i) {
        const Eight g = load_piece((const T*)p.gain, (i * THREADS + lane) * 8, d);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          v[i].v[e] *= r;
          sum_gain[i].v[e] += u[i].v[e] * v[i].v[e];
          u[i].v[e] *= g.v[e];
          m += u[i].v[e] * v[i].v[e];
        }
      }
      m = row_total<THREADS>(m, turn) / (float)d;
#pragma unroll
      for (int i = 0; i < PIECES; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) dx[i].v[e] += r * (u[i].v[e] - v[i].v[e] * m);
    }
#pragma unroll
    for (int i = 0; i < PIECES; ++i) store_piece(p.dx.row<TX>(t), (i * THREADS + lane) * 8, d, dx[i]);
    if (!p.y.p) continue;
    // from here on dx is dz, v is w (or y)
    float r = 1.f;
#pragma unroll
    for (int i = 0; i < PIECES; ++i)
      if (p.y_gain || p.gate.p) v[i] = load_piece(p.y.row<T>(t), (i * THREADS + lane) * 8, d);
    if (p.y_gain) {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < PIECES; ++i) sum += square_sum(v[i]);
      r = rsqrtf(row_total<THREADS>(sum, turn) / (float)d + p.eps);
    }
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int c = (i * THREADS + lane) * 8;
      Eight g;
#pragma unroll
      for (int e = 0; e < 8; ++e) dx[i].v[e] *= p.scale, g.v[e] = 1.f;
      if (p.y_gain) g = load_piece((const T*)p.y_gain, c, d);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i].v[e] *= r;
      if (p.gate.p) {
        const Eight gate = load_piece(p.gate.row<T>(t), c, d);
        if (p.dgate.p) {
          Eight dg;
#pragma unroll
          for (int e = 0; e < 8; ++e) dg.v[e] = dx[i].v[e] * v[i].v[e] * g.v[e];
          store_piece(p.dgate.row<T>(t), c, d, dg);
        } else {
          // the sum for a gate that all tokens share; both it and the gain's gradient come out of it
#pragma unroll
          for (int e = 0; e < 8; ++e) sum_block[i].v[e] += dx[i].v[e] * v[i].v[e];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) dx[i].v[e] *= gate.v[e];
      }
      if (p.y_gain) {
        if (!p.gate.p || p.dgate.p) {
#pragma unroll
          for (int e = 0; e < 8; ++e) sum_block[i].v[e] += dx[i].v[e] * v[i].v[e];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          dx[i].v[e] *= g.v[e];
          m += dx[i].v[e] * v[i].v[e];
        }
      }
    }
    if (p.y_gain) {
      m = row_total<THREADS>(m, turn) / (float)d;
#pragma unroll
      for (int i = 0; i < PIECES; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) dx[i].v[e] = r * (dx[i].v[e] - v[i].v[e] * m);
    }
#pragma unroll
    for (int i = 0; i < PIECES; ++i) store_piece(p.dy.row<T>(t), (i * THREADS + lane) * 8, d, dx[i]);
  }
  if (!p.partials) return;
#pragma unroll
  for (int i = 0; i < PIECES; ++i) {
    const int c = (i * THREADS + lane) * 8;
    float* to = p.partials + ((int64_t)blockIdx.x * ROWS + threadIdx.x / THREADS) * 2 * d;
    store_piece(to, c, d, sum_gain[i]);
    store_piece(to + d, c, d, sum_block[i]);
  }
}

// The gains' and a shared gate's gradients from the workgroups' sums, in a fixed order and in 64 bits: a workgroup for 16 channels, 64
// slices of the sums.  With a shared gate the second sum S = sum scale dX o w: dy_gain = gate o S, dgate = y_gain o S.
template <class T>
__global__ __launch_bounds__(1024) void k_norm_gain_grads(const float* __restrict__ partials, int n, int d, const T* gate, const T* y_gain,
                                                          float* dgain, float* dy_gain, float* dgate) {
  __shared__ double all[64][17];
  const int at = blockIdx.x * 16 + (threadIdx.x & 15), slice = threadIdx.x >> 4;
  double v = 0.0;
  if (at < 2 * d)
#pragma unroll 8
    for (int i = slice; i < n; i += 64) v += partials[(int64_t)i * 2 * d + at];
  all[slice][threadIdx.x & 15] = v;
  __syncthreads();
  if (slice > 0 || at >= 2 * d) return;
  v = 0.0;
#pragma unroll 8
  for (int i = 0; i < 64; ++i) v += all[i][threadIdx.x & 15];
  if (at < d) {
    if (dgain) dgain[at] = (float)v;
    return;
  }
  const int c = at - d;
  if (dy_gain) dy_gain[c] = (float)(dgate ? v * (double)(float)gate[c] : v);
  if (dgate) dgate[c] = (float)(y_gain ? v * (double)(float)y_gain[c] : v);
}

}  // namespace oapl
