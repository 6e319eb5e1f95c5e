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
  // What the sine of a rotation multiplies: channels that are not rotated have no partner, and what is not finite in one is not the other's.
  __device__ __forceinline__ f32x4 partner(f32x4 x) const { return turned ? x : f32x4{}; }
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

// Heads that a group of lanes has under way together: more bytes in flight.  16411 tokens of 32 + 8 heads of 128 in bf16, 1 / 2 / 3:
// backwards 113 / 108 / 139 us, forward 71 / 73 / 72.
constexpr int kRopeHeads = 2;

// 16411 tokens of 32 + 8 heads of 128 in bf16: 336 MB in 73 us, 4.6 TB/s (in fp32 671 MB in 134, 5.0); a large copy reaches 5.07.  8 tokens 3.7 us, the
// launch.
template <class T>
__global__ __launch_bounds__(256) void k_qk_norm_rope_fwd(const NormRopeArgs p) {
  const int lane = threadIdx.x & 63, group = lane >> 4;
  const int64_t unit = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 4 + (threadIdx.x >> 6);
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
  const int step = p.parts * 4;
  for (int h0 = (int)(unit % p.parts) * 4 + group; h0 < heads; h0 += step * kRopeHeads) {
    f32x4 a[kRopeHeads], b[kRopeHeads];
#pragma unroll
    for (int i = 0; i < kRopeHeads; ++i) {
      const int h = h0 + i * step;
      a[i] = b[i] = f32x4{};
      if (h >= heads || !at.any) continue;
      const T* x = (const T*)(h < p.hq ? p.q.row(t, h) : h < p.hq + p.hk ? p.k.row(t, h - p.hq) : p.v.row(t, h - p.hq - p.hk));
      a[i] = load4(x + at.a), b[i] = load4(x + at.b);
    }
#pragma unroll
    for (int i = 0; i < kRopeHeads; ++i) {
      const int h = h0 + i * step;
      const bool query = h < p.hq, value = h >= p.hq + p.hk;
      if (p.q_gain && !value) {
        const float r = rsqrtf(group_sum(dot4(a[i], a[i]) + dot4(b[i], b[i])) / (float)p.D + p.eps);
        a[i] = a[i] * r * (query ? gq[0] : gk[0]);
        b[i] = b[i] * r * (query ? gq[1] : gk[1]);
      }
      const f32x4 ta = at.partner(a[i]), tb = at.partner(b[i]);
      const f32x4 x = value ? a[i] : a[i] * cos - tb * sin, y = value ? b[i] : b[i] * cos + ta * sin;
      if (h >= heads || !at.any || !(query || kept)) continue;
      T* z = (T*)(query ? p.q_out.row(t, h) : value ? p.v_out.row(to, h - p.hq - p.hk) : p.k_out.row(to, h - p.hq));
      store4(z + at.a, x), store4(z + at.b, y);
    }
  }
}

// The same tokens: 504 MB in 102 us, 4.9 TB/s, with the workgroups' sums for the gains.
template <class T>
__global__ __launch_bounds__(256) void k_qk_norm_rope_bwd(const NormRopeArgs p) {
  const int lane = threadIdx.x & 63, group = lane >> 4;
  const Pieces at(lane & 15, p.D, p.rot);
  f32x4 gq[2] = {}, gk[2] = {}, sum_q[2] = {}, sum_k[2] = {};
  if (p.q_gain && at.any) {
    gq[0] = load4((const T*)p.q_gain + at.a), gq[1] = load4((const T*)p.q_gain + at.b);
    gk[0] = load4((const T*)p.k_gain + at.a), gk[1] = load4((const T*)p.k_gain + at.b);
  }
  const int heads = p.hq + p.hk, step = p.parts * 4;
  for (int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); unit < p.T * p.parts; unit += (int64_t)gridDim.x * 4) {
    const int64_t t = unit / p.parts;
    f32x4 cos, sin;
    token_angles(p, at, t, cos, sin);
    for (int h0 = (int)(unit % p.parts) * 4 + group; h0 < heads; h0 += step * kRopeHeads) {
      f32x4 a[kRopeHeads], b[kRopeHeads], da[kRopeHeads], db[kRopeHeads];
#pragma unroll
      for (int i = 0; i < kRopeHeads; ++i) {
        const int h = h0 + i * step;
        a[i] = b[i] = da[i] = db[i] = f32x4{};
        if (h >= heads || !at.any) continue;
        const T* x = (const T*)(h < p.hq ? p.q.row(t, h) : p.k.row(t, h - p.hq));
        const T* dy = (const T*)(h < p.hq ? p.q_out.row(t, h) : p.k_out.row(t, h - p.hq));
        a[i] = load4(x + at.a), b[i] = load4(x + at.b), da[i] = load4(dy + at.a), db[i] = load4(dy + at.b);
      }
#pragma unroll
      for (int i = 0; i < kRopeHeads; ++i) {
        const int h = h0 + i * step;
        const bool query = h < p.hq;
        f32x4 ua = da[i] * cos + at.partner(db[i]) * sin, ub = db[i] * cos - at.partner(da[i]) * sin;
        if (p.q_gain) {
          // (a head behind the last holds zeros, which without eps have no norm)
          const float norm = rsqrtf(group_sum(dot4(a[i], a[i]) + dot4(b[i], b[i])) / (float)p.D + p.eps), r = h < heads ? norm : 0.f;
          const f32x4 xa = a[i] * r, xb = b[i] * r;
          if (query) sum_q[0] += ua * xa, sum_q[1] += ub * xb;
          else sum_k[0] += ua * xa, sum_k[1] += ub * xb;      // of a head behind the last: zeros
          ua = ua * (query ? gq[0] : gk[0]);
          ub = ub * (query ? gq[1] : gk[1]);
          const float m = group_sum(dot4(ua, xa) + dot4(ub, xb)) / (float)p.D;
          ua = (ua - xa * m) * r;
          ub = (ub - xb * m) * r;
        }
        if (h >= heads || !at.any) continue;
        T* dx = (T*)(query ? p.dq.row(t, h) : p.dk.row(t, h - p.hq));
        store4(dx + at.a, ua), store4(dx + at.b, ub);
      }
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

// The gains' gradients from the workgroups' sums, in a fixed order: a workgroup for 16 channels, 64 slices of the workgroups, whose
// sums are added in 64 bits.  Bound by its launch and a chain of loads: 4 us behind the call above.
__global__ __launch_bounds__(1024) void k_gain_grads(const float* __restrict__ partials, int n, int D, float* __restrict__ dq_gain,
                                                     float* __restrict__ dk_gain) {
  __shared__ double all[64][17];
  const int at = blockIdx.x * 16 + (threadIdx.x & 15), slice = threadIdx.x >> 4;
  double v = 0.0;
  if (at < 2 * D)
#pragma unroll 8
    for (int i = slice; i < n; i += 64) v += partials[(int64_t)i * 2 * D + at];
  all[slice][threadIdx.x & 15] = v;
  __syncthreads();
  if (slice > 0 || at >= 2 * D) return;
  v = 0.0;
#pragma unroll 8
  for (int i = 0; i < 64; ++i) v += all[i][threadIdx.x & 15];
  (at < D ? dq_gain : dk_gain)[at < D ? at : at - D] = (float)v;
}

}  // namespace oapl
