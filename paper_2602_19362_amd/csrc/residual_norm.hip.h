// A block's output added to the residual stream, and the root-mean-square norms before and behind the block, in one pass over the rows.
//
//   z = y r(y) o y_gain  (or y),   x' = x + scale gate o z,   n = gain o x' r(x'),   r(a) = (mean_c a_c^2 + eps)^(-1/2)
//
// Backwards, with v = x' r(x'), u = gain o dn, w = y r(y), t = y_gain o dz:
//
//   dX = dx' + r (u - v mean_c(u o v)),   dz = scale gate o dX,   dy = r(y) (t - w mean_c(t o w))  (or dz)
//   dgain = sum dn o v,   dy_gain = sum dz o w,   dgate = scale z o dX (summed over tokens where they share the gate)
//
// Bound by memory: every row is read once and written once, and stays in registers in between; a row's sums are the only thing that its
// lanes exchange.  16411 tokens, d = 4096 in bf16: forward 538 MB in 93 us (5.8 TB/s; a large copy reaches 4.9), backward 807 MB in 153 us with
// the sums over tokens, which take 5 of them.
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

// Sum over the lanes of a row, in all of them: LANES, or the workgroup's (0).  `turn`, kept by the caller, alternates between two places: a
// wavefront that is ahead writes to the other one, and cannot be two sums ahead of a barrier, so that one barrier a sum is enough.
template <int LANES>
__device__ __forceinline__ float row_total(float v, int& turn) {
  v = lanes_total<LANES ? LANES : 64>(v);
  if constexpr (LANES == 0) {
    __shared__ float all[2][16];
    turn ^= 1;
    if ((threadIdx.x & 63) == 0) all[turn][threadIdx.x >> 6] = v;
    __syncthreads();
    const int wave = threadIdx.x & 15;
    v = lanes_total<16>(wave < (int)blockDim.x / 64 ? all[turn][wave] : 0.f);
  }
  return v;
}

template <int W>
__device__ __forceinline__ float dot(const Piece<W>& a, const Piece<W>& b) {
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < W; ++i) s += a.v[i] * b.v[i];
  return s;
}

// A row's lanes and where they are: 16 of them, a wavefront, or (LANES == 0) a workgroup, as many as the row has pieces for.
template <int LANES>
struct RowLanes {
  static constexpr int kRows = LANES ? 256 / LANES : 1;      // of a workgroup
  int lane, lanes, row;
  __device__ __forceinline__ RowLanes()
      : lane(LANES ? threadIdx.x % LANES : threadIdx.x), lanes(LANES ? LANES : blockDim.x), row(LANES ? threadIdx.x / LANES : 0) {}
};

// TX: the residual stream's type, T: the block's and the norms'.  A lane holds W channels in each of PIECES pieces of a row; MOST lanes a workgroup.
template <class TX, class T, int W, int LANES, int MOST, int PIECES, Form FORM>
__global__ __launch_bounds__(MOST) void k_residual_norm_fwd(const ResidualNormArgs p) {
  const RowLanes<LANES> at;
  constexpr int ROWS = at.kRows;
  const int lane = at.lane, lanes = at.lanes, d = p.d;
  int turn = 0;
  if (const int64_t t = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * ROWS + at.row; t < p.T) {
    Raw<TX, W> rx[PIECES];
    Raw<T, W> ry[PIECES] = {}, rg[PIECES] = {};
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int c = (i * lanes + lane) * W;
      rx[i] = load_raw<W, FORM>(p.x.row<TX>(t), c, d);
      if (p.y.p) ry[i] = load_raw<W, FORM>(p.y.row<T>(t), c, d);
      if (p.gate.p) rg[i] = load_raw<W, FORM>(p.gate.row<T>(t), c, d);
    }
    Piece<W> x[PIECES];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int c = (i * lanes + lane) * W;
      ry[i] = own<FORM>(ry[i], c, d), rg[i] = own<FORM>(rg[i], c, d);
      x[i] = widened(own<FORM>(rx[i], c, d));
    }
    if (p.y.p) {
      float r = p.scale;
      if (p.y_gain) {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < PIECES; ++i) sum += (i * lanes + lane) * W < d ? dot(widened(ry[i]), widened(ry[i])) : 0.f;
        r *= rsqrtf(row_total<LANES>(sum, turn) / (float)d + p.eps);
      }
#pragma unroll
      for (int i = 0; i < PIECES; ++i) {
        const int c = (i * lanes + lane) * W;
        Piece<W> y = widened(ry[i]);
        if (p.y_gain) {
          const Piece<W> g = load_piece<W, FORM>((const T*)p.y_gain, c, d);
#pragma unroll
          for (int e = 0; e < W; ++e) y.v[e] *= g.v[e];
        }
        if (p.gate.p) {
#pragma unroll
          for (int e = 0; e < W; ++e) y.v[e] *= (float)rg[i][e];
        }
#pragma unroll
        for (int e = 0; e < W; ++e) x[i].v[e] += r * y.v[e];
        store_piece<W, FORM>(p.x_out.row<TX>(t), c, d, x[i]);
      }
    }
    if (p.gain) {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < PIECES; ++i) sum += (i * lanes + lane) * W < d ? dot(x[i], x[i]) : 0.f;
      const float r = rsqrtf(row_total<LANES>(sum, turn) / (float)d + p.eps);
#pragma unroll
      for (int i = 0; i < PIECES; ++i) {
        const int c = (i * lanes + lane) * W;
        const Piece<W> g = load_piece<W, FORM>((const T*)p.gain, c, d);
#pragma unroll
        for (int e = 0; e < W; ++e) x[i].v[e] *= r * g.v[e];
        store_piece<W, FORM>(p.out.row<T>(t), c, d, x[i]);
      }
    }
  }
}

// What a row's gradient is made of, as it is stored.
template <class TX, class T, int W, int PIECES>
struct NormRow {
  Raw<TX, W> dx[PIECES], x[PIECES];
  Raw<T, W> dn[PIECES], y[PIECES], gate[PIECES];
};

template <class TX, class T, int W, int LANES, int MOST, int PIECES, Form FORM>
__global__ __launch_bounds__(MOST) void k_residual_norm_bwd(const ResidualNormArgs p) {
  const RowLanes<LANES> at;
  constexpr int ROWS = at.kRows;
  const int lane = at.lane, lanes = at.lanes, d = p.d;
  int turn = 0;
  Piece<W> sum_gain[PIECES] = {}, sum_block[PIECES] = {};
  Raw<T, W> gain[PIECES] = {}, y_gain[PIECES] = {};
#pragma unroll
  for (int i = 0; i < PIECES; ++i) {
    const int c = (i * lanes + lane) * W;
    if (p.gain) gain[i] = own<FORM>(load_raw<W, FORM>((const T*)p.gain, c, d), c, d);
    if (p.y_gain) y_gain[i] = own<FORM>(load_raw<W, FORM>((const T*)p.y_gain, c, d), c, d);
  }
  typedef NormRow<TX, T, W, PIECES> Row;
  const auto load = [&](Row& row, int64_t t) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int c = (i * lanes + lane) * W;
      row.dx[i] = Raw<TX, W>{};
      if (p.gain) row.x[i] = load_raw<W, FORM>(p.x.row<TX>(t), c, d), row.dn[i] = load_raw<W, FORM>(p.out.row<T>(t), c, d);
      if (p.x_out.p) row.dx[i] = load_raw<W, FORM>(p.x_out.row<TX>(t), c, d);
      if (p.y.p) row.y[i] = load_raw<W, FORM>(p.y.row<T>(t), c, d);
      if (p.gate.p) row.gate[i] = load_raw<W, FORM>(p.gate.row<T>(t), c, d);
    }
  };
  const int64_t first = (int64_t)blockIdx.x * ROWS + at.row, step = (int64_t)gridDim.x * ROWS;
  // the next row is under way while one is worked on, as far as there are registers for it
  constexpr bool AHEAD = MOST < 1024 || (W == 8 && PIECES == 1);
  Row row, next;
  if (AHEAD && first < p.T) load(next, first);
  for (int64_t t = first; t < p.T; t += step) {
    if (AHEAD) row = next;
    else load(row, t);
    if (AHEAD && t + step < p.T) load(next, t + step);
    Piece<W> dx[PIECES];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int c = (i * lanes + lane) * W;
      row.x[i] = own<FORM>(row.x[i], c, d), row.dn[i] = own<FORM>(row.dn[i], c, d);
      row.y[i] = own<FORM>(row.y[i], c, d), row.gate[i] = own<FORM>(row.gate[i], c, d);
      dx[i] = widened(own<FORM>(row.dx[i], c, d));
    }
    if (p.gain) {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < PIECES; ++i) sum += (i * lanes + lane) * W < d ? dot(widened(row.x[i]), widened(row.x[i])) : 0.f;
      const float r = rsqrtf(row_total<LANES>(sum, turn) / (float)d + p.eps);
      Piece<W> v[PIECES], u[PIECES];
      float m = 0.f;
#pragma unroll
      for (int i = 0; i < PIECES; ++i) {
        v[i] = widened(row.x[i]), u[i] = widened(row.dn[i]);
#pragma unroll
        for (int e = 0; e < W; ++e) {
          v[i].v[e] *= r;
          sum_gain[i].v[e] += u[i].v[e] * v[i].v[e];
          u[i].v[e] *= (float)gain[i][e];
        }
        m += (i * lanes + lane) * W < d ? dot(u[i], v[i]) : 0.f;
      }
      m = row_total<LANES>(m, turn) / (float)d;
#pragma unroll
      for (int i = 0; i < PIECES; ++i)
#pragma unroll
        for (int e = 0; e < W; ++e) dx[i].v[e] += r * (u[i].v[e] - v[i].v[e] * m);
    }
#pragma unroll
    for (int i = 0; i < PIECES; ++i) store_piece<W, FORM>(p.dx.row<TX>(t), (i * lanes + lane) * W, d, dx[i]);
    if (p.y.p) {
      // from here on dx is dz
      float r = 1.f;
      if (p.y_gain) {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < PIECES; ++i) sum += (i * lanes + lane) * W < d ? dot(widened(row.y[i]), widened(row.y[i])) : 0.f;
        r = rsqrtf(row_total<LANES>(sum, turn) / (float)d + p.eps);
      }
      float m = 0.f;
      Piece<W> w[PIECES];
#pragma unroll
      for (int i = 0; i < PIECES; ++i) {
        const int c = (i * lanes + lane) * W;
        w[i] = widened(row.y[i]);
#pragma unroll
        for (int e = 0; e < W; ++e) dx[i].v[e] *= p.scale, w[i].v[e] *= r;
        // the second sum: of a gate that all tokens share, from which both its gradient and the gain's come, or the gain's
        if (p.gate.p && p.dgate.p) {
          Piece<W> dg;
#pragma unroll
          for (int e = 0; e < W; ++e) {
            dg.v[e] = dx[i].v[e] * w[i].v[e] * (p.y_gain ? (float)y_gain[i][e] : 1.f);
            dx[i].v[e] *= (float)row.gate[i][e];
          }
          store_piece<W, FORM>(p.dgate.row<T>(t), c, d, dg);
        }
#pragma unroll
        for (int e = 0; e < W; ++e) sum_block[i].v[e] += dx[i].v[e] * w[i].v[e];
        if (p.gate.p && !p.dgate.p) {
#pragma unroll
          for (int e = 0; e < W; ++e) dx[i].v[e] *= (float)row.gate[i][e];
        }
        if (p.y_gain) {
#pragma unroll
          for (int e = 0; e < W; ++e) dx[i].v[e] *= (float)y_gain[i][e];
          m += c < d ? dot(dx[i], w[i]) : 0.f;
        }
      }
      if (p.y_gain) {
        m = row_total<LANES>(m, turn) / (float)d;
#pragma unroll
        for (int i = 0; i < PIECES; ++i)
#pragma unroll
          for (int e = 0; e < W; ++e) dx[i].v[e] = r * (dx[i].v[e] - w[i].v[e] * m);
      }
#pragma unroll
      for (int i = 0; i < PIECES; ++i) store_piece<W, FORM>(p.dy.row<T>(t), (i * lanes + lane) * W, d, dx[i]);
    }
  }
  if (!p.partials) return;
  float* to = p.partials + (int64_t)blockIdx.x * 2 * d;
  if constexpr (ROWS == 1) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      store_piece<W, FORM>(to, (i * lanes + lane) * W, d, sum_gain[i]);
      store_piece<W, FORM>(to + d, (i * lanes + lane) * W, d, sum_block[i]);
    }
  } else {
    // the workgroup's rows, added in their order
    __shared__ float all[ROWS][2][LANES * PIECES * W];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      store_whole<W>(&all[at.row][0][(i * lanes + lane) * W], sum_gain[i]);
      store_whole<W>(&all[at.row][1][(i * lanes + lane) * W], sum_block[i]);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * d; i += 256) {
      float v = 0.f;
#pragma unroll
      for (int r = 0; r < ROWS; ++r) v += all[r][i >= d][i >= d ? i - d : i];
      to[i] = v;
    }
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
