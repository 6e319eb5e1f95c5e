// Root-mean-square norm of every query and key head, and the position rotation, in one pass over the projection's rows.
//
//   y = R(pos) (g o x r),   r = (mean_c x_c^2 + eps)^(-1/2)
//
// R turns channel pairs (i, i + rot / 2), i < rot / 2, by the token's angles; channels from rot on stay.  Backwards, with
// u = R^T dy and t = g o u:
//
//   dx = r (t - x r^2 mean_c(t_c x_c)),   dg = sum over tokens and heads of u o x r
//
// Bound by memory: a row is read once and written once (backwards two are read), all arithmetic is in 32 bits on registers.
// A head's D channels are D / 8 lanes of a group of 16; a lane holds four channels and the four that they are turned with, so the
// rotation needs no other lane, and a mean is four exchanges.  A wavefront is on one token at a time (its angles are loaded
// once) and its four groups take the token's heads in turn.
#pragma once

#include "heads.hip.h"

namespace oapl {

struct NormRopeArgs {
  Heads q, k, v;               // the projection's rows; v.p == nullptr: no values to copy
  Heads q_out, k_out, v_out;   // backwards: dy of q and k (v_out unused)
  Heads dq, dk;                // backwards: results
  const int32_t* positions;
  const float* cos_sin;        // [n_pos][rot]: cosines, then sines
  const void *q_gain, *k_gain; // nullptr: no norm
  const int64_t* rows;         // rows of k_out and v_out that tokens go to; nullptr: their own
  int64_t n_rows;              // ... of how many
  float* partials;             // backwards: [workgroups][2][D]
  int64_t T, n_pos;
  int hq, hk, D, rot;
  int parts;                   // wavefronts that share a token's heads
  float eps;
};

// Sum over the 16 lanes of a group, in every lane.
__device__ __forceinline__ float group_sum(float v) {
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) v += __shfl_xor(v, o, 16);
  return v;
}
__device__ __forceinline__ float dot4(f32x4 a, f32x4 b) { return a[0] * b[0] + a[1] * b[1] + a[2] * b[2] + a[3] * b[3]; }

// Where a lane's two pieces of four channels lie, and whether it has any: lanes below rot / 8 hold pairs that are turned
// together, the others eight channels in a row.
struct Pieces {
  int a, b;
  bool any, turned;
  __device__ __forceinline__ Pieces(int lane16, int D, int rot) {
    const int pairs = rot >> 3;
    turned = lane16 < pairs;
    any = lane16 * 8 < D;
    a = turned ? lane16 * 4 : rot + (lane16 - pairs) * 8;
    b = turned ? (rot >> 1) + lane16 * 4 : a + 4;
  }
};

// A token's cosines and sines for a lane's pairs; false (and NaN) where its position has none.
__device__ __forceinline__ void token_angles(const NormRopeArgs& p, const Pieces& at, int64_t t, f32x4& c, f32x4& s) {
  const int32_t pos = p.positions[t];
  const float bad = pos >= 0 && pos < p.n_pos ? 0.f : quiet_nan();
  c = f32x4{1.f, 1.f, 1.f, 1.f} + bad;
  s = f32x4{0.f, 0.f, 0.f, 0.f};
  if (at.turned && bad == 0.f) {
    const float* row = p.cos_sin + (int64_t)pos * p.rot + at.a;
    c = load4(row);
    s = load4(row + (p.rot >> 1));
  }
}

template <class T>
__global__ __launch_bounds__(256) void k_qk_norm_rope_fwd(const NormRopeArgs p) {
  const int lane = threadIdx.x & 63, group = lane >> 4;
  const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int64_t t = unit / p.parts;
  if (t >= p.T) return;
  const Pieces at(lane & 15, p.D, p.rot);
  f32x4 cos, sin;
  token_angles(p, at, t, cos, sin);
  const int64_t to = p.rows ? p.rows[t] : t;
  const bool kept = !p.rows || (to >= 0 && to < p.n_rows);
  const int heads = p.hq + p.hk + (p.v.p ? p.hk : 0);
  f32x4 gq[2] = {}, gk[2] = {};
  if (p.q_gain && at.any) {
    gq[0] = load4((const T*)p.q_gain + at.a), gq[1] = load4((const T*)p.q_gain + at.b);
    gk[0] = load4((const T*)p.k_gain + at.a), gk[1] = load4((const T*)p.k_gain + at.b);
  }
  for (int h = (int)(unit % p.parts) * 4 + group; h < heads; h += p.parts * 4) {
    const bool query = h < p.hq, value = h >= p.hq + p.hk;
    const T* x = (const T*)(query ? p.q.row(t, h) : value ? p.v.row(t, h - p.hq - p.hk) : p.k.row(t, h - p.hq));
    T* y = (T*)(query ? p.q_out.row(t, h) : value ? p.v_out.row(to, h - p.hq - p.hk) : p.k_out.row(to, h - p.hq));
    f32x4 a = {}, b = {};
    if (at.any) a = load4(x + at.a), b = load4(x + at.b);
    if (!value) {
      if (p.q_gain) {
        const float r = rsqrtf(group_sum(dot4(a, a) + dot4(b, b)) / (float)p.D + p.eps);
        a = a * r * (query ? gq[0] : gk[0]);
        b = b * r * (query ? gq[1] : gk[1]);
      }
      const f32x4 turned = a * cos - b * sin;
      b = b * cos + a * sin;
      a = turned;
    }
    if (at.any && (query || kept)) store4(y + at.a, a), store4(y + at.b, b);
  }
}

template <class T>
__global__ __launch_bounds__(256) void k_qk_norm_rope_bwd(const NormRopeArgs p) {
  const int lane = threadIdx.x & 63, group = lane >> 4;
  const Pieces at(lane & 15, p.D, p.rot);
  f32x4 gq[2] = {}, gk[2] = {}, sum_q[2] = {}, sum_k[2] = {};
  if (p.q_gain && at.any) {
    gq[0] = load4((const T*)p.q_gain + at.a), gq[1] = load4((const T*)p.q_gain + at.b);
    gk[0] = load4((const T*)p.k_gain + at.a), gk[1] = load4((const T*)p.k_gain + at.b);
  }
  const int heads = p.hq + p.hk;
  for (int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); unit < p.T * p.parts; unit += (int64_t)gridDim.x * 4) {
    const int64_t t = unit / p.parts;
    f32x4 cos, sin;
    token_angles(p, at, t, cos, sin);
    for (int h = (int)(unit % p.parts) * 4 + group; h < heads; h += p.parts * 4) {
      const bool query = h < p.hq;
      const T* x = (const T*)(query ? p.q.row(t, h) : p.k.row(t, h - p.hq));
      const T* dy = (const T*)(query ? p.q_out.row(t, h) : p.k_out.row(t, h - p.hq));
      T* dx = (T*)(query ? p.dq.row(t, h) : p.dk.row(t, h - p.hq));
      f32x4 a = {}, b = {}, da = {}, db = {};
      if (at.any) a = load4(x + at.a), b = load4(x + at.b), da = load4(dy + at.a), db = load4(dy + at.b);
      f32x4 ua = da * cos + db * sin, ub = db * cos - da * sin;
      if (p.q_gain) {
        const float r = rsqrtf(group_sum(dot4(a, a) + dot4(b, b)) / (float)p.D + p.eps);
        const f32x4 xa = a * r, xb = b * r;
        if (query) sum_q[0] += ua * xa, sum_q[1] += ub * xb;
        else sum_k[0] += ua * xa, sum_k[1] += ub * xb;
        ua = ua * (query ? gq[0] : gk[0]);
        ub = ub * (query ? gq[1] : gk[1]);
        const float m = group_sum(dot4(ua, xa) + dot4(ub, xb)) / (float)p.D;
        ua = (ua - xa * m) * r;
        ub = (ub - xb * m) * r;
      }
      if (at.any) store4(dx + at.a, ua), store4(dx + at.b, ub);
    }
  }
  if (!p.partials) return;
  // the workgroup's 16 groups, added in their order
  __shared__ float all[16][2][kMaxHeadDim];
  const int g = threadIdx.x >> 4;
  if (at.any) {
    store4(&all[g][0][at.a], sum_q[0]), store4(&all[g][0][at.b], sum_q[1]);
    store4(&all[g][1][at.a], sum_k[0]), store4(&all[g][1][at.b], sum_k[1]);
  }
  __syncthreads();
  const int which = threadIdx.x >> 7, c = threadIdx.x & 127;
  if (c < p.D) {
    float v = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) v += all[i][which][c];
    p.partials[((int64_t)blockIdx.x * 2 + which) * p.D + c] = v;
  }
}

// The gains' gradients from the workgroups' sums, in a fixed order, in 64 bits: one workgroup for each channel of each gain.
__global__ __launch_bounds__(64) void k_gain_grads(const float* __restrict__ partials, int n, int D, float* __restrict__ dq_gain,
                                                   float* __restrict__ dk_gain) {
  const int which = blockIdx.x / D, c = blockIdx.x % D;
  double v = 0.0;
  for (int i = threadIdx.x; i < n; i += 64) v += partials[((int64_t)i * 2 + which) * D + c];
  v = wave_sum(v);
  if (threadIdx.x == 0) (which ? dk_gain : dq_gain)[c] = (float)v;
}

}  // namespace oapl
