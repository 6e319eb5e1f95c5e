// Soft-max attention over packed sequences, forward and backward, for bf16 and fp32 (32 x 32 matrix instructions of either).
//
// With z_ij = scale q_i . k_j over the keys j that query i sees (all of its sequence's, or, causal, j <= i + n_k - n_q):
//
//   lse_i = ln sum_j e^z_ij,   P_ij = e^(z_ij - lse_i),   o_i = sum_j P_ij v_j
//   D_i = do_i . o_i,   dS_ij = P_ij (do_i . v_j - D_i)
//   dv_j = sum_i P_ij do_i,   dq_i = scale sum_j dS_ij k_j,   dk_j = scale sum_i dS_ij q_i
//
// A row that sees no key has o = 0, lse = -infinity and no part in any gradient.
//
// A "row" is a (query token, head) pair of one key head: the heads that share a key head are rows of the same tile, next to
// each other, so its keys and values are staged once for all of them, and the sums over shared heads in dk and dv are sums
// over rows.  Products are taken so that a lane of the result owns one row (forward, dq) or one key (dk, dv): what a lane
// holds of z is then already an operand of the next product, whose contraction runs over the keys (rows) in the order in which
// the lane holds them, and the soft-max needs one exchange between the two halves of a wavefront.
#pragma once

#include "heads.hip.h"

namespace oapl {

constexpr float kLn2f = 0.69314718055994531f;

struct AttnArgs {
  Heads q, k, v, o, dout, dq, dk, dv;   // o: written forward, read backward
  float* lse;                           // [Tq][hq]; read backward; nullptr: not wanted (forward)
  float* delta;                         // [Tq][hq] D_i, between the two backward kernels
  const int64_t *q_offsets, *k_offsets, *k_used;
  int* status;
  int64_t Tq, Tk;
  int n_seq, hq, hk, g, D, causal;
  float scale;
};

// ---------------------------------------------------------------------------------------------------------------- sequences
// Tiles of B rows over the packed sequences: sequence i has ids floor(first row / B) + i and up, one more than its rows can
// need, so ids are found from the offsets alone (no list of tiles is made) and some have no rows.
template <int B>
__host__ __device__ __forceinline__ int64_t tile_ids(int64_t rows, int n_seq) { return rows / B + n_seq; }

struct SeqTile {
  int64_t q0, k0;   // first token of the sequence's queries and keys
  int nq, nk;       // its lengths
  int first;        // the tile's first row (key), counted in the sequence
};

// Offsets start at 0, do not fall, and end at the number of tokens; cached lengths lie within their sequences' room.  Every
// wavefront looks for itself, so nothing has to be launched before the kernel that computes.
__device__ __forceinline__ bool sequences_ok(const AttnArgs& p) {
  bool bad = false;
  for (int i = threadIdx.x & 63; i < p.n_seq; i += 64) {
    const int64_t a = p.q_offsets[i], b = p.q_offsets[i + 1], c = p.k_offsets[i], d = p.k_offsets[i + 1];
    bad |= (i == 0 && (a != 0 || c != 0)) || b < a || d < c || (i == p.n_seq - 1 && (b != p.Tq || d != p.Tk));
    if (p.k_used) bad |= p.k_used[i] < 0 || p.k_used[i] > d - c;
  }
  return __ballot(bad) == 0;
}

// Whose tile `id` is, by a search over the first ids of the sequences, 64 at a time; `off` and `per` say what tiles are cut from
// (rows: query offsets times heads in a group; keys: key offsets).  Only after sequences_ok.
template <int B>
__device__ __forceinline__ SeqTile find_tile(const AttnArgs& p, const int64_t* __restrict__ off, int per, int64_t id) {
  int lo = 0, n = p.n_seq;                       // the last sequence in [lo, lo + n) whose first id is not above `id`
  const int lane = threadIdx.x & 63;
  while (n > 1) {
    const int step = (n + 63) >> 6, i = lane * step;
    const bool not_above = i < n && off[lo + i] * per / B + (lo + i) <= id;
    const int k = __popcll(__ballot(not_above)) - 1;   // first ids rise with the sequence: a prefix of the lanes
    lo += k * step;
    n = n - k * step < step ? n - k * step : step;
  }
  SeqTile t;
  t.q0 = p.q_offsets[lo];
  t.k0 = p.k_offsets[lo];
  t.nq = (int)(p.q_offsets[lo + 1] - t.q0);
  t.nk = (int)(p.k_used ? p.k_used[lo] : p.k_offsets[lo + 1] - t.k0);
  const int64_t first = (id - (off[lo] * per / B + lo)) * B, rows = (off[lo + 1] - off[lo]) * per;
  t.first = (int)(first < rows ? first : rows);
  return t;
}

// Malformed sequences: the outputs are NaN.  Workgroups share the tokens.
template <class T>
__device__ __forceinline__ void poison(const Heads& x, int64_t tokens, int heads, int D) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < tokens * heads * (D / 4); i += (int64_t)gridDim.x * 256) {
    const int64_t th = i / (D / 4);
    store4((T*)x.row(th / heads, (int)(th % heads)) + i % (D / 4) * 4, f32x4{} + quiet_nan());
  }
}
__device__ __forceinline__ void poison(float* x, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) x[i] = quiet_nan();
}

// ---------------------------------------------------------------------------------------------------------------- fragments
// Eight contracted elements of one row (A) or column (B) of a 32 x 32 x 16 product; element j of lane l meets element j of the
// other operand's lanes in the same half of the wavefront, so any order of the contraction serves that is the same in both.
struct FragF32 { f32x4 x[2]; };
template <class T> struct FragOf;
template <> struct FragOf<bf16_t> { typedef bf16x8 type; };
template <> struct FragOf<float> { typedef FragF32 type; };

__device__ __forceinline__ f32x16 mma(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 mma(const FragF32& a, const FragF32& b, f32x16 c) {
#pragma unroll
  for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.x[j >> 2][j & 3], b.x[j >> 2][j & 3], c, 0, 0, 0);
  return c;
}

// Rows (keys) 8 (i / 4) + 4 half + i % 4 of a 32 x 32 result are in accumulator i; eight of them in a row, as an operand.
__device__ __forceinline__ void pack(const f32x16& c, int chunk, bf16x8& f) {
#pragma unroll
  for (int j = 0; j < 8; ++j) f[j] = (bf16_t)c[chunk * 8 + j];
}
__device__ __forceinline__ void pack(const f32x16& c, int chunk, FragF32& f) {
#pragma unroll
  for (int j = 0; j < 8; ++j) f.x[j >> 2][j & 3] = c[chunk * 8 + j];
}

// A row's channels of one k-step from memory (nullptr: zeros).
__device__ __forceinline__ void load_frag(const char* row, int c, int D, bf16x8& f) {
  f = bf16x8{};
  if (row && c < D) f = *(const bf16x8*)(row + c * 2);
}
__device__ __forceinline__ void load_frag(const char* row, int c, int D, FragF32& f) {
  f = FragF32{};
  if (row && c < D) f.x[0] = *(const f32x4*)(row + c * 4), f.x[1] = *(const f32x4*)(row + c * 4 + 16);
}
__device__ __forceinline__ float dot(const bf16x8& a, const bf16x8& b) {
  float s = 0.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) s = fmaf((float)a[j], (float)b[j], s);
  return s;
}
__device__ __forceinline__ float dot(const FragF32& a, const FragF32& b) {
  float s = 0.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) s = fmaf(a.x[j >> 2][j & 3], b.x[j >> 2][j & 3], s);
  return s;
}

// A tile of R rows of DP channels in LDS.  16-byte chunk c of row r lies at chunk c ^ swizzle(r): fetches of one chunk of many
// rows, and transposing fetches of four rows of one column range, both touch every bank once.
template <class T, int DP>
struct Tile {
  static constexpr int kPitch = DP * (int)sizeof(T), kChunks = kPitch / 16;
  __device__ static __forceinline__ int swizzle(int r) {
    return kChunks >= 16 ? (r & 3) << 2 | (r >> 2 & 3) : (r >> 1 & 1) << 2 | (r >> 2 & 3);
  }
  __device__ static __forceinline__ int at(int r, int c) { return r * kPitch + ((c ^ swizzle(r)) << 4); }

  // Rows [0, rows) of heads' rows at `p`, `stride` bytes apart, zeros behind them and behind channel D.
  template <int R>
  __device__ static __forceinline__ void fill(lds_char_ptr lds, const char* p, int64_t stride, int rows, int D) {
#pragma unroll 4
    for (int i = threadIdx.x; i < R * kChunks; i += 256) {
      const int r = i / kChunks, c = i % kChunks;
      u32x4 v = {};
      if (r < rows && c * 16 < D * (int)sizeof(T)) v = *(const u32x4*)(p + r * stride + c * 16);
      *(__attribute__((address_space(3))) u32x4*)(lds + at(r, c)) = v;
    }
  }

  // Operand of rows r0 + lane % 32, contracted over the 16 channels of step kk.
  __device__ static __forceinline__ void rows(lds_char_ptr lds, int r0, int kk, bf16x8& f) {
    const int lane = threadIdx.x & 63;
    f = *(__attribute__((address_space(3))) bf16x8*)(lds + at(r0 + (lane & 31), kk * 2 + (lane >> 5)));
  }
  __device__ static __forceinline__ void rows(lds_char_ptr lds, int r0, int kk, FragF32& f) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int x = 0; x < 2; ++x)
      f.x[x] = *(__attribute__((address_space(3))) f32x4*)(lds + at(r0 + (lane & 31), kk * 4 + (lane >> 5) * 2 + x));
  }

  // Operand of channels c0 + lane % 32, contracted over rows r0 .. r0 + 15 in the order of a result's accumulators.
  // bf16: of the 16 lanes of a group, lane 4e + a points at four channels of row e, and lane i receives channel i of four rows.
  __device__ static __forceinline__ void columns(lds_char_ptr lds, int r0, int c0, bf16x8& f) {
    typedef __attribute__((address_space(3))) bf16x4* ptr;
    const int lane = threadIdx.x & 63;
    const int r = r0 + (lane >> 5) * 4 + (lane >> 2 & 3), c = c0 + (lane >> 4 & 1) * 16 + (lane & 3) * 4;
    const bf16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((ptr)(lds + at(r, c >> 3) + (c & 4) * 2));
    const bf16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((ptr)(lds + at(r + 8, c >> 3) + (c & 4) * 2));
    f = __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
  }
  __device__ static __forceinline__ void columns(lds_char_ptr lds, int r0, int c0, FragF32& f) {
    const int lane = threadIdx.x & 63, c = c0 + (lane & 31);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int r = r0 + (lane >> 5) * 4 + (j & 3) + (j >> 2) * 8;
      f.x[j >> 2][j & 3] = *(__attribute__((address_space(3))) float*)(lds + at(r, c >> 2) + (c & 3) * 4);
    }
  }
};

__device__ __forceinline__ float other_half(float v) { return __shfl_xor(v, 32, 64); }

// Four consecutive channels a lane: a result whose columns are rows (keys) of `row`.
template <class T, int DB>
__device__ __forceinline__ void store_columns(char* row, const f32x16 (&acc)[DB], float factor, int D) {
  if (!row) return;
  const int half = threadIdx.x >> 5 & 1;
#pragma unroll
  for (int b = 0; b < DB; ++b)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = b * 32 + i * 8 + half * 4;
      if (c < D) store4((T*)row + c, f32x4{acc[b][i * 4], acc[b][i * 4 + 1], acc[b][i * 4 + 2], acc[b][i * 4 + 3]} * factor);
    }
}

// What a lane of the forward and dq kernels knows of its row.
struct Row {
  int token, head;   // head in the group
  int sees;          // keys that it sees; 0 behind the sequence's end
  __device__ __forceinline__ Row(const AttnArgs& p, const SeqTile& t, int row) {
    const bool any = row < t.nq * p.g;
    token = any ? row / p.g : 0;
    head = any ? row % p.g : 0;
    const int n = p.causal ? token + 1 + t.nk - t.nq : t.nk;
    sees = !any ? 0 : n < 0 ? 0 : n < t.nk ? n : t.nk;
    exists = any;
  }
  bool exists;
};

// Keys that the last row of a tile of B rows sees: no row sees more.
template <int B>
__device__ __forceinline__ int tile_sees(const AttnArgs& p, const SeqTile& t) {
  if (!p.causal) return t.nk;
  const int rows = t.nq * p.g, last = (t.first + B < rows ? t.first + B : rows) - 1;
  const int n = last / p.g + 1 + t.nk - t.nq;
  return n < 0 ? 0 : n < t.nk ? n : t.nk;
}

constexpr int kKeys = 64;   // keys staged at a time

// ---------------------------------------------------------------------------------------------------------------- forward
// A workgroup: 128 rows, 32 a wavefront, over all keys that they see.
template <class T, int DP>
__global__ __launch_bounds__(256) void k_attn_fwd(const AttnArgs p) {
  typedef typename FragOf<T>::type Frag;
  typedef Tile<T, DP> Lds;
  constexpr int B = 128, KS = DP / 16, DB = DP / 32;
  extern __shared__ char smem[];
  const lds_char_ptr ks = (lds_char_ptr)smem, vs = ks + kKeys * Lds::kPitch;
  const bool ok = sequences_ok(p);
  if (blockIdx.x == 0 && threadIdx.x == 0) *p.status = ok ? 0 : kErrOffsets;
  if (!ok) {
    poison<T>(p.o, p.Tq, p.hq, p.D);
    if (p.lse) poison(p.lse, p.Tq * p.hq);
    return;
  }
  const int kh = blockIdx.x % p.hk;
  const SeqTile t = find_tile<B>(p, p.q_offsets, p.g, tile_ids<B>(p.Tq * p.g, p.n_seq) - 1 - blockIdx.x / p.hk);
  if (t.first >= t.nq * p.g) return;
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const Row row(p, t, t.first + (threadIdx.x >> 6) * 32 + (lane & 31));
  const int head = kh * p.g + row.head;
  Frag q[KS];
#pragma unroll
  for (int kk = 0; kk < KS; ++kk) load_frag(row.exists ? p.q.row(t.q0 + row.token, head) : nullptr, kk * 16 + half * 8, p.D, q[kk]);
  f32x16 o[DB] = {};
  float m = kNegHuge, l = 0.f;     // l: this half's keys
  const float scale2 = p.scale * kLog2e;
  const int sees = tile_sees<B>(p, t);
  for (int j0 = 0; j0 < sees; j0 += kKeys) {
    __syncthreads();
    Lds::template fill<kKeys>(ks, p.k.row(t.k0 + j0, kh), p.k.token, t.nk - j0, p.D);
    Lds::template fill<kKeys>(vs, p.v.row(t.k0 + j0, kh), p.v.token, t.nk - j0, p.D);
    __syncthreads();
    f32x16 s[2] = {};
#pragma unroll
    for (int kk = 0; kk < KS; ++kk)
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        Frag f;
        Lds::rows(ks, b * 32, kk, f);
        s[b] = mma(f, q[kk], s[b]);
      }
    float top = kNegHuge;
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int key = j0 + b * 32 + (i >> 2) * 8 + half * 4 + (i & 3);
        s[b][i] = key < row.sees ? s[b][i] * scale2 : -__builtin_inff();
        top = fmaxf(top, s[b][i]);
      }
    top = fmaxf(m, fmaxf(top, other_half(top)));
    const float old = __builtin_amdgcn_exp2f(m - top);
    m = top;
    l *= old;
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[b][i] = __builtin_amdgcn_exp2f(s[b][i] - m);
        l += s[b][i];
      }
#pragma unroll
    for (int d = 0; d < DB; ++d) o[d] *= old;
#pragma unroll
    for (int c = 0; c < kKeys / 16; ++c) {
      Frag f, w;
      pack(s[c >> 1], c & 1, w);
#pragma unroll
      for (int d = 0; d < DB; ++d) {
        Lds::columns(vs, c * 16, d * 32, f);
        o[d] = mma(f, w, o[d]);
      }
    }
  }
  l += other_half(l);
  if (!row.exists) return;
  store_columns<T>(p.o.row(t.q0 + row.token, head), o, l > 0.f ? 1.f / l : l == 0.f ? 0.f : l, p.D);
  if (p.lse && half == 0)
    p.lse[(t.q0 + row.token) * p.hq + head] = l == 0.f ? -__builtin_inff() : (m + __builtin_amdgcn_logf(l)) * kLn2f;
}

// ---------------------------------------------------------------------------------------------------------------- backward
// D_i and dq: a workgroup has 128 rows, as forward.
template <class T, int DP>
__global__ __launch_bounds__(256) void k_attn_dq(const AttnArgs p) {
  typedef typename FragOf<T>::type Frag;
  typedef Tile<T, DP> Lds;
  constexpr int B = 128, KS = DP / 16, DB = DP / 32;
  extern __shared__ char smem[];
  const lds_char_ptr ks = (lds_char_ptr)smem, vs = ks + kKeys * Lds::kPitch;
  const bool ok = sequences_ok(p);
  if (blockIdx.x == 0 && threadIdx.x == 0) *p.status = ok ? 0 : kErrOffsets;
  if (!ok) return poison<T>(p.dq, p.Tq, p.hq, p.D);
  const int kh = blockIdx.x % p.hk;
  const SeqTile t = find_tile<B>(p, p.q_offsets, p.g, tile_ids<B>(p.Tq * p.g, p.n_seq) - 1 - blockIdx.x / p.hk);
  if (t.first >= t.nq * p.g) return;
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const Row row(p, t, t.first + (threadIdx.x >> 6) * 32 + (lane & 31));
  const int head = kh * p.g + row.head;
  const int64_t token = t.q0 + row.token;
  Frag q[KS], dout[KS];
  float delta = 0.f;
#pragma unroll
  for (int kk = 0; kk < KS; ++kk) {
    Frag o;
    load_frag(row.exists ? p.q.row(token, head) : nullptr, kk * 16 + half * 8, p.D, q[kk]);
    load_frag(row.exists ? p.dout.row(token, head) : nullptr, kk * 16 + half * 8, p.D, dout[kk]);
    load_frag(row.exists ? p.o.row(token, head) : nullptr, kk * 16 + half * 8, p.D, o);
    delta += dot(o, dout[kk]);
  }
  delta += other_half(delta);
  if (row.exists && half == 0) p.delta[token * p.hq + head] = delta;
  const float scale2 = p.scale * kLog2e, lse2 = row.exists ? p.lse[token * p.hq + head] * kLog2e : 0.f;
  f32x16 dq[DB] = {};
  const int sees = tile_sees<B>(p, t);
  for (int j0 = 0; j0 < sees; j0 += kKeys) {
    __syncthreads();
    Lds::template fill<kKeys>(ks, p.k.row(t.k0 + j0, kh), p.k.token, t.nk - j0, p.D);
    Lds::template fill<kKeys>(vs, p.v.row(t.k0 + j0, kh), p.v.token, t.nk - j0, p.D);
    __syncthreads();
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      f32x16 s = {}, dp = {};
#pragma unroll
      for (int kk = 0; kk < KS; ++kk) {
        Frag f;
        Lds::rows(ks, b * 32, kk, f);
        s = mma(f, q[kk], s);
        Lds::rows(vs, b * 32, kk, f);
        dp = mma(f, dout[kk], dp);
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int key = j0 + b * 32 + (i >> 2) * 8 + half * 4 + (i & 3);
        s[i] = key < row.sees ? __builtin_amdgcn_exp2f(s[i] * scale2 - lse2) * (dp[i] - delta) : 0.f;
      }
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        Frag f, w;
        pack(s, c, w);
#pragma unroll
        for (int d = 0; d < DB; ++d) {
          Lds::columns(ks, b * 32 + c * 16, d * 32, f);
          dq[d] = mma(f, w, dq[d]);
        }
      }
    }
  }
  if (row.exists) store_columns<T>(p.dq.row(token, head), dq, p.scale, p.D);
}

// dk and dv: a workgroup has 128 keys, 32 a wavefront, over all rows that see any of them.
template <class T, int DP>
__global__ __launch_bounds__(256) void k_attn_dkdv(const AttnArgs p) {
  typedef typename FragOf<T>::type Frag;
  typedef Tile<T, DP> Lds;
  constexpr int B = 128, KS = DP / 16, DB = DP / 32, R = 32;
  extern __shared__ char smem[];
  const lds_char_ptr qs = (lds_char_ptr)smem, ds = qs + R * Lds::kPitch;
  typedef __attribute__((address_space(3))) float* lds_f32;
  typedef __attribute__((address_space(3))) int* lds_i32;
  const lds_f32 lse2s = (lds_f32)(ds + R * Lds::kPitch), deltas = lse2s + R;
  const lds_i32 seess = (lds_i32)(deltas + R);
  if (!sequences_ok(p)) {
    poison<T>(p.dk, p.Tk, p.hk, p.D);
    return poison<T>(p.dv, p.Tk, p.hk, p.D);
  }
  const int kh = blockIdx.x % p.hk;
  const SeqTile t = find_tile<B>(p, p.k_offsets, 1, blockIdx.x / p.hk);
  if (t.first >= t.nk) return;
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const int key = t.first + (threadIdx.x >> 6) * 32 + (lane & 31);
  const bool exists = key < t.nk;
  Frag k[KS], v[KS];
#pragma unroll
  for (int kk = 0; kk < KS; ++kk) {
    load_frag(exists ? p.k.row(t.k0 + key, kh) : nullptr, kk * 16 + half * 8, p.D, k[kk]);
    load_frag(exists ? p.v.row(t.k0 + key, kh) : nullptr, kk * 16 + half * 8, p.D, v[kk]);
  }
  f32x16 dk[DB] = {}, dv[DB] = {};
  const float scale2 = p.scale * kLog2e;
  const int rows = t.nq * p.g;
  // the first token that sees the tile's first key
  const int from = p.causal && t.first > t.nk - t.nq ? t.first - (t.nk - t.nq) : 0;
  for (int r0 = from * p.g / R * R; r0 < rows; r0 += R) {
    __syncthreads();
#pragma unroll 4
    for (int i = threadIdx.x; i < R * Lds::kChunks; i += 256) {
      const int r = i / Lds::kChunks, c = i % Lds::kChunks, x = r0 + r;
      u32x4 a = {}, b = {};
      if (x < rows && c * 16 < p.D * (int)sizeof(T)) {
        a = *(const u32x4*)(p.q.row(t.q0 + x / p.g, kh * p.g + x % p.g) + c * 16);
        b = *(const u32x4*)(p.dout.row(t.q0 + x / p.g, kh * p.g + x % p.g) + c * 16);
      }
      *(__attribute__((address_space(3))) u32x4*)(qs + Lds::at(r, c)) = a;
      *(__attribute__((address_space(3))) u32x4*)(ds + Lds::at(r, c)) = b;
    }
    if (threadIdx.x < R) {
      const Row row(p, t, r0 + threadIdx.x);
      const int64_t i = (t.q0 + row.token) * p.hq + kh * p.g + row.head;
      lse2s[threadIdx.x] = row.exists ? p.lse[i] * kLog2e : 0.f;
      deltas[threadIdx.x] = row.exists ? p.delta[i] : 0.f;
      seess[threadIdx.x] = row.sees;
    }
    __syncthreads();
    f32x16 s = {}, dp = {};
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) {
      Frag f;
      Lds::rows(qs, 0, kk, f);
      s = mma(f, k[kk], s);
      Lds::rows(ds, 0, kk, f);
      dp = mma(f, v[kk], dp);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int r = (i >> 2) * 8 + half * 4 + (i & 3);
      s[i] = key < seess[r] ? __builtin_amdgcn_exp2f(s[i] * scale2 - lse2s[r]) : 0.f;
      dp[i] = key < seess[r] ? s[i] * (dp[i] - deltas[r]) : 0.f;
    }
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      Frag f, w;
      pack(s, c, w);
#pragma unroll
      for (int d = 0; d < DB; ++d) {
        Lds::columns(ds, c * 16, d * 32, f);
        dv[d] = mma(f, w, dv[d]);
      }
      pack(dp, c, w);
#pragma unroll
      for (int d = 0; d < DB; ++d) {
        Lds::columns(qs, c * 16, d * 32, f);
        dk[d] = mma(f, w, dk[d]);
      }
    }
  }
  if (!exists) return;
  store_columns<T>(p.dk.row(t.k0 + key, kh), dk, p.scale, p.D);
  store_columns<T>(p.dv.row(t.k0 + key, kh), dv, 1.f, p.D);
}

}  // namespace oapl
