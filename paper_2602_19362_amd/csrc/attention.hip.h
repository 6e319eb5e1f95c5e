// Soft-max attention over packed sequences, forward and backward, for bf16 and fp32 (matrix instructions of 16 x 16 results).
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
// the lane holds them, and the soft-max needs one exchange between the quarters of a wavefront.
//
// Scores, maxima, sums, accumulators, log-sum-exp and D_i are 32 bits wide.  In bf16, P (before it is divided by its sum) and dS are rounded
// once, because they are operands of the next product and the matrix cores take both in one type: an error of 2^-8 of each term at most,
// where q, k, v and the results carry as much, and 32-bit products would take nine times as long.  Outputs are rounded once, at the end; partial
// results of splits are kept in 32 bits.
#pragma once

#include "gemm_bf16.hip.h"   // vmcnt_imm, lds_read_transposed
#include "heads.hip.h"

namespace oapl {

constexpr float kLn2f = 0.69314718055994531f;

struct AttnArgs {
  Heads q, k, v, o, dout, dq, dk, dv;   // o: written forward, read backward
  float* lse;                           // [Tq][hq]; read backward; nullptr: not wanted (forward)
  float *lse2, *delta;                  // [hk][Tq][g] log-sum-exp in base 2 and D_i, between the two backward kernels
  const int64_t *q_offsets, *k_offsets, *k_used;
  int* status;
  int64_t Tq, Tk;
  float *partials, *part_sums;          // of splits
  int n_seq, hq, hk, g, D, causal;
  int splits;                           // of the keys of a tile of rows (forward, dq), or of the rows of a tile of keys
  uint32_t g_mul;                       // quotients by g, see by_group
  int g_shift;
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

// A number that all lanes hold alike, for the scalar unit.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int64_t uniform(int64_t x) {
  return (int64_t)((uint64_t)(uint32_t)uniform((int)(x >> 32)) << 32 | (uint32_t)uniform((int)x));
}

// Tiles of rows, or of keys.
enum TileOf { kOfRows, kOfKeys };

__device__ __forceinline__ SeqTile tile_of(const AttnArgs& p, int seq, TileOf what, int64_t first) {
  SeqTile t;
  t.q0 = uniform(p.q_offsets[seq]);
  t.k0 = uniform(p.k_offsets[seq]);
  t.nq = uniform((int)(p.q_offsets[seq + 1] - t.q0));
  t.nk = uniform((int)(p.k_used ? p.k_used[seq] : p.k_offsets[seq + 1] - t.k0));
  const int64_t end = what == kOfRows ? (int64_t)t.nq * p.g : t.nk;
  t.first = uniform((int)(first < end ? first : end));
  return t;
}

// Offsets start at 0, do not fall, and end at the number of tokens; cached lengths lie within their sequences' room.  Of up to kLookedAt
// sequences every wavefront looks for itself, so nothing has to be launched before the kernel that computes.
struct SeqEnds {
  int64_t q0, q1, k0, k1, used;      // of one sequence; zeros behind the last
  __device__ __forceinline__ SeqEnds(const AttnArgs& p, int i) {
    q0 = q1 = k0 = k1 = used = 0;
    if (i >= p.n_seq) return;
    q0 = p.q_offsets[i], q1 = p.q_offsets[i + 1], k0 = p.k_offsets[i], k1 = p.k_offsets[i + 1];
    used = p.k_used ? p.k_used[i] : k1 - k0;
  }
  __device__ __forceinline__ bool bad(const AttnArgs& p, int i) const {
    return (i == 0 && (q0 != 0 || k0 != 0)) || q1 < q0 || k1 < k0 || (i == p.n_seq - 1 && (q1 != p.Tq || k1 != p.Tk)) || used < 0 ||
           used > k1 - k0;
  }
};

// Of more, that would be work by the square of their number (all offsets for every sequence's tiles): one workgroup looks first, and
// the others find in the status word what it saw.  16384 tokens, 8 heads of 64 channels, forward / backward, every wavefront / one workgroup:
// 128 sequences 32 / 85 and 34 / 82 us; 256, 31 / 83 and 29 / 72; 1024, 181 / 300 and 90 / 177; 4096, 1450 / 2410 and 290 / 600.
constexpr int kLookedAt = 128;
__global__ __launch_bounds__(1024) void k_attn_check(const AttnArgs p) {
  bool bad = false;
#pragma unroll 4
  for (int i = threadIdx.x; i < p.n_seq; i += 1024) bad |= SeqEnds(p, i).bad(p, i);
  const int any = __syncthreads_or(bad);
  if (threadIdx.x == 0) *p.status = any ? kErrOffsets : 0;
}

// The tile with this id, by a search over the first ids of (well-formed) sequences, 64 at a time.
template <int B>
__device__ __forceinline__ SeqTile find_tile(const AttnArgs& p, TileOf what, int64_t id) {
  const int64_t* __restrict__ off = what == kOfRows ? p.q_offsets : p.k_offsets;
  const int per = what == kOfRows ? p.g : 1;
  int lo = 0, n = p.n_seq;                       // the last sequence in [lo, lo + n) whose first id is not above `id`
  const int lane = threadIdx.x & 63;
  while (n > 1) {
    const int step = (n + 63) >> 6, i = lane * step;
    const bool not_above = i < n && off[lo + i] * per / B + (lo + i) <= id;
    const int k = __popcll(__ballot(not_above)) - 1;   // first ids rise with the sequence: a prefix of the lanes
    lo += k * step;
    n = n - k * step < step ? n - k * step : step;
  }
  lo = uniform(lo);
  return tile_of(p, lo, what, (id - (uniform(off[lo]) * per / B + lo)) * B);
}

// Sums over the lanes up to each one, and the largest of all.
__device__ __forceinline__ int prefix_sum(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);   // from one, two, four, eight lanes below, in rows of 16
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);   // from the row before, from the half before
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);
  return v;
}
__device__ __forceinline__ int last_lane(int v) { return __builtin_amdgcn_readlane(v, 63); }

// The tile that stands `rank`-th when all are ordered by how far they reach, longest first (in 256 levels): what a tile of rows costs is
// the keys that its last row sees, a tile of keys the queries that see its first key, and either is a closed form of the tile's
// number, so that every workgroup finds its own by a search over levels.  Long tiles that start last are what the chip
// waits for in the end.  More than 64 sequences go in the order of their ids.
enum Found { kMalformed, kNoTile, kTile };

template <int B>
__device__ __forceinline__ Found pick_tile(const AttnArgs& p, TileOf what, int rank, SeqTile& t) {
  const int lane = threadIdx.x & 63;
  const SeqEnds ends(p, lane);
  if (p.n_seq > kLookedAt) {
    if (uniform(*p.status) != 0) return kMalformed;
  } else {
    bool bad = lane < p.n_seq && ends.bad(p, lane);
    for (int i = lane + 64; i < p.n_seq; i += 64) bad |= SeqEnds(p, i).bad(p, i);
    if (__ballot(bad) != 0) return kMalformed;
  }
  if (p.n_seq > 64) {
    const int64_t last = what == kOfRows ? tile_ids<B>(p.Tq * p.g, p.n_seq) - 1 : 0;
    t = find_tile<B>(p, what, what == kOfRows ? last - rank : rank);
    return t.first < (what == kOfRows ? t.nq * p.g : t.nk) ? kTile : kNoTile;
  }
  const int nq = (int)(ends.q1 - ends.q0), nk = (int)ends.used;
  const int tiles = ((what == kOfRows ? nq * p.g : nk) + B - 1) / (unsigned)B, reach = what == kOfRows ? nk : nq;
  // the sequence's tiles that reach beyond x >= 0
  const auto beyond = [&](int x) {
    if (x >= reach) return 0;
    if (!p.causal) return tiles;
    if (what == kOfKeys) return min(tiles, (int)((max(nk - x, 0) + B - 1) / (unsigned)B));      // (more queries than keys: x may pass nk)
    const int token = x - (nk - nq);       // the first that sees more than x
    return tiles - (token > 0 ? (int)(token * p.g / (unsigned)B) : 0);
  };
  int most = reach;
#pragma unroll
  for (int x = 32; x > 0; x >>= 1) most = max(most, __shfl_xor(most, x, 64));
  const int unit = (uniform(most) + 255) / 256;
  int lo = -1, hi = 256;      // all tiles reach beyond level -1, none beyond 256; lo: more than `rank` do, hi: not
  while (hi - lo > 1) {
    const int y = (lo + hi) / 2;
    if (last_lane(prefix_sum(beyond(y * unit))) > rank) lo = y;
    else hi = y;
  }
  const int above = beyond(hi * unit), mine = (lo < 0 ? tiles : beyond(lo * unit)) - above;
  const int to = prefix_sum(mine), left = rank - last_lane(prefix_sum(above));
  if (left >= last_lane(to)) return kNoTile;
  const int seq = __ffsll((unsigned long long)__ballot(to > left)) - 1;
  const int nth = __builtin_amdgcn_readlane(above + left - (to - mine), seq);    // among the sequence's, longest first
  const auto of = [&](int64_t x) {
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), seq) << 32 |
                     (uint32_t)__builtin_amdgcn_readlane((int)x, seq));
  };
  t.q0 = of(ends.q0), t.k0 = of(ends.k0);
  t.nq = __builtin_amdgcn_readlane(nq, seq), t.nk = __builtin_amdgcn_readlane(nk, seq);
  t.first = (what == kOfRows ? __builtin_amdgcn_readlane(tiles, seq) - 1 - nth : nth) * B;
  return kTile;
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

// Inline assembly, so that an accumulator stays where it is: given the builtin the compiler moves results about in the middle of a
// sum.  What it then does not keep are the wait states around an MFMA: results are looked at behind settle(), and operands that
// vector instructions made go through ready().
__device__ __forceinline__ void mma(f32x4& c, bf16x8 a, bf16x8 b) { asm("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+v"(c) : "v"(a), "v"(b)); }
// (fp32 operands may be copied between registers just before: its wait states go with every multiplication, behind the one before.)
__device__ __forceinline__ void mma(f32x4& c, const FragF32& a, const FragF32& b) {
#pragma unroll
  for (int j = 0; j < 8; ++j) asm("s_nop 1\n\tv_mfma_f32_16x16x4_f32 %0, %1, %2, %0" : "+v"(c) : "v"(a.x[j >> 2][j & 3]), "v"(b.x[j >> 2][j & 3]));
}
// ... the first of a sum.
__device__ __forceinline__ void mma0(f32x4& c, bf16x8 a, bf16x8 b) { asm("v_mfma_f32_16x16x32_bf16 %0, %1, %2, 0" : "=&v"(c) : "v"(a), "v"(b)); }
__device__ __forceinline__ void mma0(f32x4& c, const FragF32& a, const FragF32& b) {
  asm("s_nop 1\n\tv_mfma_f32_16x16x4_f32 %0, %1, %2, 0" : "=&v"(c) : "v"(a.x[0][0]), "v"(b.x[0][0]));
#pragma unroll
  for (int j = 1; j < 8; ++j) asm("s_nop 1\n\tv_mfma_f32_16x16x4_f32 %0, %1, %2, %0" : "+v"(c) : "v"(a.x[j >> 2][j & 3]), "v"(b.x[j >> 2][j & 3]));
}
// The wait states of the slower of the two shapes: one statement that all results go into and come out of.
template <int N>
__device__ __forceinline__ void settle(f32x4 (&x)[2][N]) {
  static_assert(N == 2 || N == 4 || N == 6 || N == 8, "operands are listed");
  __builtin_amdgcn_sched_barrier(0);
  if constexpr (N == 2)
    asm volatile("s_nop 7\n\ts_nop 7" : "+v"(x[0][0]), "+v"(x[0][1]), "+v"(x[1][0]), "+v"(x[1][1]));
  else if constexpr (N == 4)
    asm volatile("s_nop 7\n\ts_nop 7" : "+v"(x[0][0]), "+v"(x[0][1]), "+v"(x[0][2]), "+v"(x[0][3]), "+v"(x[1][0]), "+v"(x[1][1]),
                 "+v"(x[1][2]), "+v"(x[1][3]));
  else if constexpr (N == 6)
    asm volatile("s_nop 7\n\ts_nop 7" : "+v"(x[0][0]), "+v"(x[0][1]), "+v"(x[0][2]), "+v"(x[0][3]), "+v"(x[0][4]), "+v"(x[0][5]),
                 "+v"(x[1][0]), "+v"(x[1][1]), "+v"(x[1][2]), "+v"(x[1][3]), "+v"(x[1][4]), "+v"(x[1][5]));
  else
    asm volatile("s_nop 7\n\ts_nop 7" : "+v"(x[0][0]), "+v"(x[0][1]), "+v"(x[0][2]), "+v"(x[0][3]), "+v"(x[0][4]), "+v"(x[0][5]),
                 "+v"(x[0][6]), "+v"(x[0][7]), "+v"(x[1][0]), "+v"(x[1][1]), "+v"(x[1][2]), "+v"(x[1][3]), "+v"(x[1][4]),
                 "+v"(x[1][5]), "+v"(x[1][6]), "+v"(x[1][7]));
}
__device__ __forceinline__ void settle(f32x4 (&x)[2], f32x4 (&y)[2]) {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_nop 7\n\ts_nop 7" : "+v"(x[0]), "+v"(x[1]), "+v"(y[0]), "+v"(y[1]));
}
__device__ __forceinline__ void ready(bf16x8 (&f)[2]) { asm volatile("s_nop 1" : "+v"(f[0]), "+v"(f[1])); }
__device__ __forceinline__ void ready(FragF32 (&f)[2]) {
  asm volatile("s_nop 1" : "+v"(f[0].x[0]), "+v"(f[0].x[1]), "+v"(f[1].x[0]), "+v"(f[1].x[1]));
}
__device__ __forceinline__ void zero(f32x4& c) {
  c = f32x4{0.f, 0.f, 0.f, 0.f};
  asm volatile("" : "+v"(c));     // here, and not in front of the multiplication that adds to it
}

__device__ __forceinline__ void pack(f32x4 a, f32x4 b, bf16x8& f) {
#pragma unroll
  for (int j = 0; j < 4; ++j) f[j] = (bf16_t)a[j], f[j + 4] = (bf16_t)b[j];
}
__device__ __forceinline__ void pack(f32x4 a, f32x4 b, FragF32& f) { f.x[0] = a, f.x[1] = b; }

// A lane's eighths of a row of D channels, in steps of 32; zeros behind channel D.
__device__ __forceinline__ void load_frag(const char* at, bf16x8& f) { f = *(const bf16x8*)at; }
__device__ __forceinline__ void load_frag(const char* at, FragF32& f) { f.x[0] = *(const f32x4*)at, f.x[1] = *(const f32x4*)(at + 16); }
template <class T, int KS, class Frag>
__device__ __forceinline__ void load_row(const char* row, int D, Frag (&f)[KS]) {
#pragma unroll
  for (int kk = 0; kk < KS; ++kk) {
    const int c = (threadIdx.x >> 4 & 3) * 8 + kk * 32;
    load_frag(row + (c < D ? c : 0) * sizeof(T), f[kk]);
    if (c >= D) f[kk] = Frag{};
  }
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

// A value that the compiler computes with where it stands, and not ahead of a loop.
__device__ __forceinline__ int fresh(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// Heads of up to DW channels (32, 64, 96, 128) lie in LDS in rows of 64 or 128.
constexpr int padded(int DW) { return DW <= 64 ? 64 : 128; }

// LDS addresses as numbers.
__device__ __forceinline__ int lds_place(lds_char_ptr p) { return (int)(uintptr_t)p; }
__device__ __forceinline__ lds_char_ptr lds_at(int place) { return (lds_char_ptr)(uintptr_t)(uint32_t)place; }

// A tile of R rows of DP channels in LDS.  16-byte chunk c of row r lies at chunk c ^ swizzle(r): fetches of one chunk of many
// rows, and transposing fetches of four rows of one column range, both touch every bank once.
template <class T, int DP>
struct Tile {
  static constexpr int kPitch = DP * (int)sizeof(T), kChunks = kPitch / 16;
  __device__ static __forceinline__ int swizzle(int r) {
    return (kChunks >= 16 ? (r & 3) << 2 : (r >> 1 & 1) << 2) | (-(r >> 2) & 3);
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

  // Operands come out of a tile (at a multiple of 256 bytes) from places that differ in a few bits of the chunk: a lane has one place
  // for each kind, and the step's bits are put in where the operand is fetched: once for all fetches of a step or, with KEEP =
  // false, each time anew, where a dozen places do not fit the registers.

  // Fetches below take a place with the step's bits in it, and what is constant of an address beside it.
  template <bool KEEP = true>
  __device__ static __forceinline__ int flip(int place, int bits) {
    if (KEEP) return place ^ bits;
    int at;
    asm volatile("v_xor_b32 %0, %1, %2" : "=v"(at) : "i"(bits), "v"(place));
    return at;
  }
  static constexpr int kRowBits = 16 * 2 * (int)sizeof(T), kColumnBits = 16 * (int)sizeof(T);   // of a step of 32 (16) channels

  // Rows lane % 16 of the 16 rows `off` bytes into the tile, contracted over 32 channels.
  __device__ static __forceinline__ int rows_place(lds_char_ptr lds, int thread) {
    const int lane = thread & 63;
    return lds_place(lds) + (lane & 15) * kPitch + (((lane >> 4) * ((int)sizeof(T) / 2) ^ swizzle(lane & 15)) << 4);
  }
  __device__ static __forceinline__ void rows(int place, int off, bf16x8& f) {
    f = *(__attribute__((address_space(3))) bf16x8*)(lds_at(place) + off);
  }
  __device__ static __forceinline__ void rows(int place, int off, FragF32& f) {
#pragma unroll
    for (int x = 0; x < 2; ++x) f.x[x] = *(__attribute__((address_space(3))) f32x4*)(lds_at(place ^ x << 4) + off);
  }

  // Channels lane % 16 of 16, contracted over 32 rows in the order in which the results of two blocks of 16 rows hold them.  bf16: of the 16 lanes of a group, lane 4e + a points at four channels of row e, and lane i receives channel i of four
  // rows.
  __device__ static __forceinline__ int columns_place(lds_char_ptr lds, int thread) {
    const int lane = thread & 63;
    if (sizeof(T) == 2) {
      const int r = (lane >> 4) * 4 + (lane >> 2 & 3);
      return lds_place(lds) + r * kPitch + (((lane >> 1 & 1) ^ swizzle(r)) << 4) + ((lane & 1) << 3);
    }
    return lds_place(lds) + (lane >> 4) * 4 * kPitch + (((lane >> 2 & 3) ^ swizzle((lane >> 4) * 4)) << 4) + ((lane & 3) << 2);
  }
  __device__ static __forceinline__ void columns(int place, int off, bf16x8& f) {
    const lds_char_ptr at = lds_at(place) + off;
    const bf16x4 x = lds_read_transposed(at), y = lds_read_transposed(at + 16 * kPitch);
    f = __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
  }
  __device__ static __forceinline__ void columns(int place, int off, FragF32& f) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      f.x[j >> 2][j & 3] = *(__attribute__((address_space(3))) float*)(lds_at(place ^ (j & 3) << 6) + off +
                                                                        ((j & 3) + (j >> 2) * 16) * kPitch);
  }
};

// Rows of one tile of R rows of DP channels on their way from memory to LDS without passing through registers: 16 bytes a lane, whole
// LDS rows a wavefront, W wavefronts together.  What lies behind the last row or channel is behind the buffer's range and reads as zeros.
template <class T, int DP, int R, int W>
struct Stager {
  typedef Tile<T, DP> Lds;
  static constexpr int kRows = 64 / Lds::kChunks;          // that a wavefront's load covers
  static constexpr int kLoads = R / (W * kRows);           // of each wavefront
  static constexpr uint32_t kOutside = 0x80000000u;        // rows of a tile span 2^30 bytes at most
  const char* base;
  int64_t stride;
  int row, wave;
  uint32_t column, columns, whole;
  __device__ __forceinline__ Stager(const char* p, int64_t token_stride, int D) : base(p), stride(token_stride) {
    const int lane = threadIdx.x & 63;
    wave = W == 1 ? 0 : uniform((int)threadIdx.x >> 6);
    row = wave * kRows + lane / Lds::kChunks;
    column = ((lane % Lds::kChunks) ^ Lds::swizzle(row)) * 16;
    columns = D * sizeof(T);
    whole = column < columns ? (uint32_t)(row * (int)stride) + column : kOutside;
  }
  // Starts the loads of rows [first, first + R), of which those from `n` on (counted from the base) do not exist.
  __device__ __forceinline__ void start(lds_char_ptr lds, int first, int n) const {
    const __amdgpu_buffer_rsrc_t r =
        __builtin_amdgcn_make_buffer_rsrc((void*)(base + first * stride), 0, kOutside, 0x00020000);
    // rows 16 apart are swizzled alike, and others by bits that do not depend on the lane
    if (W * kRows % 16 == 0 && first + R <= n) {
#pragma unroll
      for (int j = 0; j < kLoads; ++j)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void_ptr)(lds + (j * W + wave) * 1024), 16, whole, j * W * kRows * (int)stride, 0, 0);
      return;
    }
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int at = row + j * W * kRows;
      const uint32_t c = column ^ (uint32_t)Lds::swizzle(j * W * kRows) << 4;
      const uint32_t v = first + at < n && c < columns ? (uint32_t)(at * (int)stride) + c : kOutside;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void_ptr)(lds + (j * W + wave) * 1024), 16, v, 0, 0, 0);
    }
  }
};

// Everything that this wavefront started has arrived ...
__device__ __forceinline__ void staged() { __builtin_amdgcn_s_waitcnt(vmcnt_imm(0) & ~0x0F00); }      // vmcnt(0) lgkmcnt(0)
// Quotients by the group size of numbers below 2^31: (x * mul) >> shift.
__device__ __forceinline__ int by_group(const AttnArgs& p, int x) { return (int)((uint64_t)(uint32_t)x * p.g_mul >> p.g_shift); }

// What a lane of the forward and dq kernels knows of its row.
struct Row {
  int token, head;   // head in the group
  int sees;          // keys that it sees; 0 behind the sequence's end
  __device__ __forceinline__ Row(const AttnArgs& p, const SeqTile& t, int row) {
    const bool any = row < t.nq * p.g;
    token = any ? by_group(p, row) : 0;      // what reads a row that does not exist reads the sequence's first
    head = any ? row - token * p.g : 0;
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
  const int n = uniform(by_group(p, last)) + 1 + t.nk - t.nq;
  return n < 0 ? 0 : n < t.nk ? n : t.nk;
}

// Keys that every row of a tile sees.
__device__ __forceinline__ int all_rows_see(const AttnArgs& p, const SeqTile& t) {
  if (!p.causal) return t.nk;
  const int n = uniform(by_group(p, t.first)) + 1 + t.nk - t.nq;
  return n < 0 ? 0 : n < t.nk ? n : t.nk;
}

// Whether keys [from, from + KEYS) hold one that exists and that some row of the tile does not see: one that others see, or one behind the
// reach of all (which a tile of one token's heads has, too) in the step in which it ends.
template <int KEYS>
__device__ __forceinline__ bool hides(const SeqTile& t, int all_see, int from) {
  return all_see < t.nk && all_see < from + KEYS;
}

template <int WK> constexpr int fwd_keys = WK == 2 ? 64 : 32;   // keys staged at a time: forward
template <int WK> constexpr int dq_keys = WK == 4 ? 32 : 64;    // ... for dq

// ---------------------------------------------------------------------------------------------------------------- forward
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;      // fmaxf would first make quiet what may be a signalling NaN
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(d) : "v"(a), "v"(b), "v"(c));
  return d;
}

__device__ __forceinline__ void negate(bf16x8& f) {
  u32x4 x;
  __builtin_memcpy(&x, &f, 16);
  x ^= 0x80008000u;
  __builtin_memcpy(&f, &x, 16);
}
__device__ __forceinline__ void negate(FragF32& f) { f.x[0] = -f.x[0], f.x[1] = -f.x[1]; }

template <class T, int DB>
__device__ __forceinline__ void store_columns(char* row, const f32x4 (&acc)[DB], float factor, int D) {
  const int c0 = (threadIdx.x >> 4 & 3) * 4;
  if (D == DB * 16) {
#pragma unroll
    for (int b = 0; b < DB; ++b) store4((T*)row + c0 + b * 16, acc[b] * factor);
  } else {
#pragma unroll
    for (int b = 0; b < DB; ++b)
      if (c0 + b * 16 < D) store4((T*)row + c0 + b * 16, acc[b] * factor);
  }
}

// Over the four lanes that hold a row, in all of them.
template <class F>
__device__ __forceinline__ float over_row(float v, F f) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = f(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return f(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float row_max(float v) { return over_row(v, [](float a, float b) { return max3(a, a, b); }); }
__device__ __forceinline__ float row_sum(float v) { return over_row(v, [](float a, float b) { return a + b; }); }

// What is not finite in a tile's masked places.  A masked probability is 0, and 0 times a NaN or an infinity would be NaN in rows that
// do not see it.  Where a step masks anything, what is not finite becomes 0 in the tile before it is used.  Forward the
// rows that see it are remembered and their outputs made NaN in the end (a value is no part of the log-sum-exp); backwards their probabilities are
// made NaN (mark_odd).
//
// Whether this wavefront has staged any such number: its pieces of a tile (j W + wave, of 1 KiB), before the others have to be there.
template <class T, int LOADS, int W>
__device__ __forceinline__ bool staged_odd(lds_char_ptr tile) {
  typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
  const int wave = W == 1 ? 0 : uniform((int)threadIdx.x >> 6);
  uint32_t top = 0;      // the largest magnitude (of either half), as an integer
#pragma unroll
  for (int i = 0; i < LOADS; ++i) {
    const u32x4 x = *(__attribute__((address_space(3))) u32x4*)(tile + (i * W + wave) * 1024 + (threadIdx.x & 63) * 16);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (sizeof(T) == 4) top = max(top, x[j] & 0x7fffffffu);
      else top = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, top), __builtin_bit_cast(u16x2, x[j] & 0x7fff7fffu)));
    }
  }
  return __any(top >= 0x7f800000u || (sizeof(T) == 2 && (top & 0xffffu) >= 0x7f80u));
}
// ... and whether anybody of four has, in words that alternate from step to step (the slower ones may still be reading).
__device__ __forceinline__ void tell_odd(lds_char_ptr words, int parity, bool odd) {
  if ((threadIdx.x & 63) == 0) ((__attribute__((address_space(3))) uint32_t*)words)[parity * 4 + (threadIdx.x >> 6)] = odd;
}
__device__ __forceinline__ bool told_odd(lds_char_ptr words, int parity) {
  const u32x4 x = *(__attribute__((address_space(3))) u32x4*)(words + parity * 16);
  return uniform((int)(x[0] | x[1] | x[2] | x[3])) != 0;
}

// The rows of a tile of ROWS (and of the one SIZE bytes behind it, with TILES = 2) that hold any, as bits.  W wavefronts share a tile:
// all of them come here, and `words` are W words of LDS for what each has found.
template <class T, int DP, int ROWS, int W, int TILES = 1, int SIZE = 0>
__device__ __forceinline__ uint64_t clean_tile(lds_char_ptr tile, lds_char_ptr words) {
  typedef Tile<T, DP> Lds;
  typedef __attribute__((address_space(3))) u32x4* lds_u32x4;
  typedef __attribute__((address_space(3))) uint32_t* lds_u32;
  constexpr int kAtOnce = 64 / Lds::kChunks, kMine = ROWS / W;      // rows that 64 lanes cover at a time; of a wavefront
  const int wave = W == 1 ? 0 : uniform((int)threadIdx.x >> 6);
  const lds_char_ptr mine = tile + wave * kMine * Lds::kPitch + (threadIdx.x & 63) * 16;
  uint64_t odd = 0;
  const auto pieces = [&](auto&& f) {
#pragma unroll 1
    for (int i = 0; i < TILES * kMine / kAtOnce; ++i)
      f(i % (kMine / kAtOnce) * kAtOnce, (lds_u32x4)(mine + i / (kMine / kAtOnce) * SIZE + i % (kMine / kAtOnce) * 1024));
  };
  pieces([&](int row, lds_u32x4 at) {
    const u32x4 x = *at;
    bool any = false;
#pragma unroll
    for (int j = 0; j < 4; ++j) any |= (x[j] & 0x7f800000u) == 0x7f800000u || (sizeof(T) == 2 && (x[j] & 0x7f80u) == 0x7f80u);
    const uint64_t lanes = __ballot(any);
#pragma unroll
    for (int r = 0; r < kAtOnce; ++r)
      if (lanes >> (r * Lds::kChunks) & ((1ull << Lds::kChunks) - 1)) odd |= 1ull << (row + r);
  });
  if (W > 1) {
    static_assert(W == 1 || kMine <= 32, "a word holds a wavefront's rows");
    if ((threadIdx.x & 63) == 0) ((lds_u32)words)[wave] = (uint32_t)odd;
    lds_barrier();
    odd = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) odd |= (uint64_t)(uint32_t)uniform((int)((lds_u32)words)[w]) << (w * kMine);
  }
  if (odd == 0) return 0;
  pieces([&](int, lds_u32x4 at) {
    u32x4 x = *at;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (sizeof(T) == 4) {
        if ((x[j] & 0x7f800000u) == 0x7f800000u) x[j] = 0;
      } else {
        if ((x[j] & 0x7f80u) == 0x7f80u) x[j] &= 0xffff0000u;
        if ((x[j] & 0x7f800000u) == 0x7f800000u) x[j] &= 0xffffu;
      }
    }
    *at = x;
  });
  if (W > 1) lds_barrier();
  return odd;
}
__device__ __forceinline__ void mark_odd(f32x4 (&s)[2][2], uint32_t odd) {
  const int group = fresh(threadIdx.x) >> 4 & 3;
#pragma unroll
  for (int n = 0; n < 2; ++n)
#pragma unroll
    for (int x = 0; x < 8; ++x)
      if (odd >> (group * 4 + (x >> 2) * 16 + (x & 3)) & 1) s[n][x >> 2][x & 3] = quiet_nan();
}

// Scores of two blocks of 16 rows of a tile in LDS (keys, or rows) with the wavefront's 32 rows (keys): s[n][b] is the tile's block b,
// `off` bytes into it, by the wavefront's block n.  Operands are fetched three ahead of their multiplications, and after each pair of
// these comes between(i), i = 0 .. 2 KS - 1: other work for the vector unit while the matrix unit is busy.  The compiler left alone
// fetches two operands and waits for them, and puts the other work behind.
template <class Lds, int KS, class Frag, class F>
__device__ __forceinline__ void scores(f32x4 (&s)[2][2], int place, int off, const Frag (&x)[2][KS], F&& between) {
  constexpr int AHEAD = 3, N = 2 * KS;
  Frag f[N];
  const auto fetch = [&](int i) { Lds::rows(Lds::flip(place, (i >> 1) * Lds::kRowBits), off + (i & 1) * 16 * Lds::kPitch, f[i]); };
#pragma unroll
  for (int i = 0; i < (AHEAD < N ? AHEAD : N); ++i) fetch(i);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    __builtin_amdgcn_sched_barrier(0);
    if (i + AHEAD < N) fetch(i + AHEAD);
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      if (i < 2) mma0(s[n][i & 1], f[i], x[n][i >> 1]);
      else mma(s[n][i & 1], f[i], x[n][i >> 1]);
    }
    between(i);
  }
  settle(s);
}

// acc[n][d] += columns 16 d of 32 rows of a tile, contracted over those rows with w[n].
template <class Lds, int DB, class Frag, class F>
__device__ __forceinline__ void add_columns(f32x4 (&acc)[2][DB], int place, int off, const Frag (&w)[2], F&& between) {
  constexpr int AHEAD = 3, N = DB;
  Frag f[DB];
  const auto fetch = [&](int i) { Lds::columns(Lds::flip(place, i * Lds::kColumnBits), off, f[i]); };
#pragma unroll
  for (int i = 0; i < (AHEAD < N ? AHEAD : N); ++i) fetch(i);
#pragma unroll
  for (int i = 0; i < DB; ++i) {
    __builtin_amdgcn_sched_barrier(0);
    if (i + AHEAD < DB) fetch(i + AHEAD);
#pragma unroll
    for (int n = 0; n < 2; ++n) mma(acc[n][i], f[i], w[n]);
    between(i);
  }
  __builtin_amdgcn_sched_barrier(0);
}

// Both for a pair of tiles SIZE bytes apart, for where registers are short: places are made anew with every fetch, for both tiles.
template <class Lds, int KS, int SIZE, class Frag>
__device__ __forceinline__ void scores2(f32x4 (&s)[2][2], f32x4 (&t)[2][2], int place, const Frag (&x)[2][KS], const Frag (&y)[2][KS]) {
  constexpr int AHEAD = 3, N = 4 * KS;      // fetch i: channels i / 4, tile (i / 2) % 2, block i % 2
  Frag f[N];
  int at = place;
  const auto fetch = [&](int i) {
    if ((i & 3) == 0) at = Lds::template flip<false>(place, (i >> 2) * Lds::kRowBits);
    Lds::rows(at, (i >> 1 & 1) * SIZE + (i & 1) * 16 * Lds::kPitch, f[i]);
  };
#pragma unroll
  for (int i = 0; i < (AHEAD < N ? AHEAD : N); ++i) fetch(i);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    __builtin_amdgcn_sched_barrier(0);
    if (i + AHEAD < N) fetch(i + AHEAD);
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      f32x4& to = (i >> 1 & 1) ? t[n][i & 1] : s[n][i & 1];
      const Frag& by = (i >> 1 & 1) ? y[n][i >> 2] : x[n][i >> 2];
      if (i < 4) mma0(to, f[i], by);
      else mma(to, f[i], by);
    }
  }
  settle(s);
  settle(t);
}

template <class Lds, int DB, int SIZE, class Frag>
__device__ __forceinline__ void add_columns2(f32x4 (&a)[2][DB], f32x4 (&b)[2][DB], int place, const Frag (&w)[2], const Frag (&x)[2]) {
  constexpr int AHEAD = 3, N = 2 * DB;      // fetch i: channels i / 2, tile i % 2
  Frag f[N];
  int at = place;
  const auto fetch = [&](int i) {
    if ((i & 1) == 0) at = Lds::template flip<false>(place, (i >> 1) * Lds::kColumnBits);
    Lds::columns(at, (i & 1) * SIZE, f[i]);
  };
#pragma unroll
  for (int i = 0; i < (AHEAD < N ? AHEAD : N); ++i) fetch(i);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    __builtin_amdgcn_sched_barrier(0);
    if (i + AHEAD < N) fetch(i + AHEAD);
#pragma unroll
    for (int n = 0; n < 2; ++n) mma((i & 1) ? b[n][i >> 1] : a[n][i >> 1], f[i], (i & 1) ? x[n] : w[n]);
  }
  __builtin_amdgcn_sched_barrier(0);
}

// Where a row's numbers lie in workspaces: rows of a key head one after the other.
__device__ __forceinline__ int64_t packed_row(const AttnArgs& p, const SeqTile& t, int kh, int row) {
  return (kh * p.Tq + t.q0) * p.g + row;
}

// LDS of a workgroup that walks over keys: slots of a tile of keys and one of values, and (WK = 4) the same for every wavefront, later
// its results; words of tell_odd and clean_tile.
template <class T, int DP, int WK, int KEYS>
struct KeyLds {
  static constexpr int kTile = KEYS * Tile<T, DP>::kPitch, kSlots = WK == 4 && sizeof(T) == 4 ? 1 : 2;
  static constexpr int kStages = 2 * kSlots * kTile, kResults = 32 * (DP * 4 + 16);
  static constexpr int kEach = WK == 4 && kStages > kResults ? kStages : (kResults + 511) / 512 * 512;      // of a wavefront
  static constexpr int kWords = WK == 1 || (WK == 2 && kStages > 4 * kEach) ? kStages : 4 * kEach, kBytes = kWords + 48;
  static_assert(kBytes <= 160 * 1024, "LDS of one CU");
};

// Keys [begin, end) of split `split` of the n that a tile sees, in whole steps.
struct Part {
  int begin, end;
  __device__ __forceinline__ Part(int n, int splits, int split, int step) {
    const int64_t each = ((int64_t)n + (int64_t)splits * step - 1) / ((int64_t)splits * step) * step, from = split * each;
    begin = (int)(from < n ? from : n);
    end = (int)(from + each < n ? from + each : n);
  }
};

// What a workgroup does: the part of a tile's walk, the key head, the tile's rank.  Parts come first: XCDs take workgroups in turn, so one
// XCD's workgroups walk over the same part, which its L2 then holds.
struct Job {
  int part, kh, rank;
  __device__ __forceinline__ explicit Job(const AttnArgs& p) {
    const unsigned id = blockIdx.x / (unsigned)p.splits;
    part = uniform((int)(blockIdx.x - id * p.splits));
    rank = uniform((int)(id / (unsigned)p.hk));
    kh = uniform((int)id - rank * p.hk);
  }
};

// A result of one split, unnormalised: partial[split][packed row][D], and its maximum (in base 2) and sum.
__device__ __forceinline__ void store_sums(const AttnArgs& p, int part, int64_t row, float m2, float l) {
  *(float2*)(p.part_sums + (part * p.Tq * p.hq + row) * 2) = make_float2(m2, l);
}
__device__ __forceinline__ float* partial_row(const AttnArgs& p, int part, int64_t rows, int64_t row) {
  return p.partials + (part * rows + row) * p.D;
}

// WK = 1: a workgroup has 128 rows, 32 a wavefront, over all keys that they see, 32 at a time.  Three wavefronts a SIMD: one's exponentials
// run beside another's products.  Bound by the matrix cores at the clock that the power limit leaves, and by the exponentials' issue
// between them: 4 x 8192 tokens, 32 heads on 8 of 128 channels, no mask, 1081 ... 1115 TFLOP/s by box, calls in turn (a 16384^3 product of the vendor's library
// 1353), matrix cores busy 0.53 of the time at 1.7 GHz.  64 keys at a time by two wavefronts a SIMD: 5 % less.
// WK = 2, for few rounds of tiles: 64 rows, two wavefronts for either half of 64 keys; they join at the end.
// WK = 4, for few rows: the wavefronts have the same 32 rows and take the steps of 32 keys in turn, each through LDS of its own, and
// join at the end.  That is bound by reading the keys and values: 64 single tokens over up to 4096 each, 8 key heads, 599 MB in 112 us,
// 5.3 TB/s; 8 over 32768 in parts, 1.07 GB in 184 us, 5.8 TB/s (a large read reaches 5.95).  In fp32 a wavefront's LDS holds one step at a time, and
// loads wait for products: 244 us, 4.9 TB/s, and 392 us, 5.5 TB/s.
// Where tiles are few, their keys are split over workgroups whose results k_attn_join puts together.
template <class T, int DW, int WK>
__global__ __launch_bounds__(256, WK == 4 ? 1 : WK == 2 && DW > 64 ? 2 : sizeof(T) == 2 ? 3 : 2) void k_attn_fwd(const AttnArgs p) {
  constexpr bool kAlone = WK == 4;      // a wavefront stages keys for itself
  constexpr int DP = padded(DW), KEYS = fwd_keys<WK>, W = kAlone ? 1 : 4, STEP = KEYS * 4 / W;
  typedef typename FragOf<T>::type Frag;
  typedef Tile<T, DP> Lds;
  typedef Stager<T, DP, KEYS, W> Stage;
  typedef KeyLds<T, DP, WK, KEYS> Size;
  constexpr int B = 128 / WK, KS = DW / 32, DB = DW / 16, SIZE = Size::kTile;
  extern __shared__ char smem[];
  const Job job(p);
  const int kh = job.kh;
  SeqTile t;
  const Found found = pick_tile<B>(p, kOfRows, job.rank, t);
  if (blockIdx.x == 0 && threadIdx.x == 0) *p.status = found == kMalformed ? kErrOffsets : 0;
  if (found == kMalformed) {
    poison<T>(p.o, p.Tq, p.hq, p.D);
    if (p.lse) poison(p.lse, p.Tq * p.hq);
  }
  if (found != kTile) return;
  const int wave = uniform((int)threadIdx.x >> 6), half = WK == 2 ? (wave >> 1) * 32 : 0;      // of the staged keys, this wavefront's
  const lds_char_ptr lds = (lds_char_ptr)smem + (kAlone ? wave * Size::kEach : 0);     // slots of keys and values
  const Part part(tile_sees<B>(p, t), p.splits, job.part, STEP);
  const Stage ks(p.k.row(t.k0, kh), p.k.token, p.D), vs(p.v.row(t.k0, kh), p.v.token, p.D);
  int j0 = part.begin + (kAlone ? wave * KEYS : 0), slot = 0;
  const lds_char_ptr words = (lds_char_ptr)smem + Size::kWords;
  const int first_sees = all_rows_see(p, t);
  const auto masks = [&](int from) { return hides<KEYS>(t, first_sees, from); };
  const auto stage = [&](int at, int first) {
    ks.start(lds + at, first, t.nk);
    vs.start(lds + at + SIZE, first, t.nk);
  };
  if (Size::kSlots == 2 && j0 < part.end) stage(0, j0);
  const int group = threadIdx.x >> 4 & 3, row0 = t.first + wave % (4 / WK) * 32 + (threadIdx.x & 15);
  const float scale2 = p.scale == 0.f ? 1.f : fabsf(p.scale) * kLog2e;
  // Where the running maximum starts: it is scaled before a row has seen any key, and a masked score less an infinite offset would be NaN.
  const float lowest = kNegHuge / fmaxf(scale2, 1.f);
  int row_sees[2];
  Frag q[2][KS];
  f32x4 o[2][DB];
  float m[2], l[2];                                // m: the running maximum before scaling; l: this lane's keys
  int all_see = t.nk;                              // keys that every row of this wavefront sees
  int sees_odd = 0;                                // rows (bits) that see a value that is not finite
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    const Row row(p, t, row0 + n * 16);
    load_row<T>(p.q.row(t.q0 + row.token, kh * p.g + row.head), p.D, q[n]);
    if (p.scale <= 0.f) {      // products are taken with -q, or with zeros
#pragma unroll
      for (int kk = 0; kk < KS; ++kk) {
        negate(q[n][kk]);
        if (p.scale == 0.f) q[n][kk] = Frag{};
      }
    }
#pragma unroll
    for (int d = 0; d < DB; ++d) zero(o[n][d]);
    row_sees[n] = row.sees;
    if (row.exists) all_see = row.sees < all_see ? row.sees : all_see;
    m[n] = lowest;
    l[n] = 0.f;
  }
#pragma unroll
  for (int x = 8; x > 0; x >>= 1) {
    const int y = __shfl_xor(all_see, x, 64);
    all_see = y < all_see ? y : all_see;
  }
  all_see = __builtin_amdgcn_readfirstlane(all_see);
  for (; j0 < part.end; j0 += STEP, slot ^= Size::kSlots == 2 ? 2 * SIZE : 0) {
    if (Size::kSlots == 1) stage(0, j0);
    staged();
    bool odd = masks(j0) && staged_odd<T, Stage::kLoads, W>(lds + slot + SIZE);
    if (!kAlone) {
      if (masks(j0)) tell_odd(words, slot != 0, odd);
      lds_barrier();
      odd = masks(j0) && told_odd(words, slot != 0);
    }
    if (Size::kSlots == 2 && j0 + STEP < part.end) stage(slot ^ 2 * SIZE, j0 + STEP);
    const lds_char_ptr own = lds + slot + half * Lds::kPitch;
    const int k_rows = Lds::rows_place(own, threadIdx.x), v_columns = Lds::columns_place(own + SIZE, threadIdx.x);
    f32x4 s[2][2];     // [rows][keys]
    scores<Lds, KS>(s, k_rows, 0, q, [](int) {});
    if (odd) {
      const int first = __ffs((uint32_t)(clean_tile<T, DP, KEYS, W>(lds + slot + SIZE, words + 32) >> half)) - 1;
#pragma unroll
      for (int n = 0; n < 2; ++n)
        if (first >= 0 && j0 + half + first < row_sees[n]) sees_odd |= 1 << n;
    }
    if (j0 + half + 32 > all_see) {
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int x = 0; x < 8; ++x) {
          const int key = (x >> 2) * 16 + group * 4 + (x & 3);
          if (j0 + half + key >= row_sees[n]) s[n][x >> 2][x & 3] = -__builtin_inff();
        }
    }
    // The maximum that the exponentials are taken from follows only when it falls behind by 2^8: until then they stay below 2^8, and
    // what is rounded is rounded as well as below 1.
    float top[2];
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      top[n] = m[n];
#pragma unroll
      for (int x = 0; x < 8; x += 2) top[n] = max3(top[n], s[n][x >> 2][x & 3], s[n][x >> 2][(x & 3) + 1]);
      top[n] = row_max(top[n]);
    }
    if (__any(fmaxf(top[0] - m[0], top[1] - m[1]) * scale2 > 8.f)) {
      settle(o);
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const float old = __builtin_amdgcn_exp2f((m[n] - top[n]) * scale2);
        m[n] = top[n];
        l[n] *= old;
#pragma unroll
        for (int d = 0; d < DB; ++d) o[n][d] *= old;
      }
    }
    Frag w[2];
#pragma unroll
    for (int n = 0; n < 2; ++n) {
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        const float e = __builtin_amdgcn_exp2f(fmaf(s[n][x >> 2][x & 3], scale2, -m[n] * scale2));
        l[n] += e;
        s[n][x >> 2][x & 3] = e;
      }
      pack(s[n][0], s[n][1], w[n]);
    }
    ready(w);
    add_columns<Lds, DB>(o, v_columns, 0, w, [](int) {});
  }
  settle(o);
  if (__any(sees_odd)) {
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int d = 0; d < DB; ++d)
        if (sees_odd >> n & 1) o[n][d] = f32x4{} + quiet_nan();
  }
  const auto finish = [&](float m2, float l) { return l == 0.f ? -__builtin_inff() : (m2 + __builtin_amdgcn_logf(l)) * kLn2f; };
  const auto inverse = [&](float l) { return l > 0.f ? 1.f / l : l == 0.f ? 0.f : l; };
  if constexpr (WK == 1) {
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      const Row row(p, t, row0 + n * 16);
      l[n] = row_sum(l[n]);
      if (!row.exists) continue;
      const int head = kh * p.g + row.head;
      if (p.splits > 1) {
        const int64_t at = packed_row(p, t, kh, row0 + n * 16);
        store_columns<float>((char*)partial_row(p, job.part, p.Tq * p.hq, at), o[n], 1.f, p.D);
        if (group == 0) store_sums(p, job.part, at, m[n] * scale2, l[n]);
        continue;
      }
      store_columns<T>(p.o.row(t.q0 + row.token, head), o[n], inverse(l[n]), p.D);
      if (p.lse && group == 0) p.lse[(t.q0 + row.token) * p.hq + head] = finish(m[n] * scale2, l[n]);
    }
  } else {
    // The wavefronts' results in LDS, then two threads a row for each wavefront that had it.
    constexpr int PITCH = DP * 4 + 16, G = 4 / WK, C = DW / (2 * WK);
    typedef __attribute__((address_space(3))) float* lds_f32;
    typedef __attribute__((address_space(3))) f32x4* lds_f32x4;
    __syncthreads();      // everybody has read its last tile
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      l[n] = row_sum(l[n]);
      const lds_char_ptr to = (lds_char_ptr)smem + wave * Size::kEach + (n * 16 + (threadIdx.x & 15)) * PITCH;
#pragma unroll
      for (int d = 0; d < DB; ++d) *(lds_f32x4)(to + d * 64 + group * 16) = o[n][d];
      if (group == 0) {
        *(lds_f32)(to + DP * 4) = m[n] * scale2;
        *(lds_f32)(to + DP * 4 + 4) = l[n];
      }
    }
    __syncthreads();
    const int r = threadIdx.x / (2 * WK), c0 = threadIdx.x % (2 * WK) * C;
    const Row row(p, t, t.first + r);
    const lds_char_ptr from = (lds_char_ptr)smem + r / 32 * Size::kEach + r % 32 * PITCH;
    float top = kNegHuge, sum = 0.f;
#pragma unroll
    for (int w = 0; w < WK; ++w) top = fmaxf(top, *(lds_f32)(from + w * G * Size::kEach + DP * 4));
    f32x4 x[C / 4] = {};
#pragma unroll
    for (int w = 0; w < WK; ++w) {
      const float by = __builtin_amdgcn_exp2f(*(lds_f32)(from + w * G * Size::kEach + DP * 4) - top);
      sum = fmaf(*(lds_f32)(from + w * G * Size::kEach + DP * 4 + 4), by, sum);
#pragma unroll
      for (int c = 0; c < C / 4; ++c) x[c] += *(lds_f32x4)(from + w * G * Size::kEach + (c0 + c * 4) * 4) * by;
    }
    if (!row.exists) return;
    const int head = kh * p.g + row.head;
    if (p.splits > 1) {
      const int64_t at = packed_row(p, t, kh, t.first + r);
#pragma unroll
      for (int c = 0; c < C / 4; ++c)
        if (c0 + c * 4 < p.D) store4(partial_row(p, job.part, p.Tq * p.hq, at) + c0 + c * 4, x[c]);
      if (c0 == 0) store_sums(p, job.part, at, top, sum);
      return;
    }
    T* to = (T*)p.o.row(t.q0 + row.token, head);
#pragma unroll
    for (int c = 0; c < C / 4; ++c)
      if (c0 + c * 4 < p.D) store4(to + c0 + c * 4, x[c] * inverse(sum));
    if (p.lse && c0 == 0) p.lse[(t.q0 + row.token) * p.hq + head] = finish(top, sum);
  }
}

// Puts the splits of a row together: 32 lanes a row, a lane for each split's numbers (two from 33 splits on), then four channels a lane.
// Bound by its launch and two rounds of loads: 320 rows of 4 parts 4.6 us.
template <class T>
__global__ __launch_bounds__(256) void k_attn_join(const AttnArgs p) {
  if (*p.status != 0) return;      // the outputs are NaN already
  const int64_t rows = p.Tq * p.hq, row = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (row >= rows) return;
  const int lane = threadIdx.x & 31, c = lane * 4, h = (int)(row % p.g), kh = (int)(row / (p.Tq * p.g));
  const int64_t token = row / p.g - kh * p.Tq;
  float2 sums[2];
  float top = kNegHuge, sum = 0.f;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int s = lane + i * 32;
    sums[i] = s < p.splits ? *((const float2*)p.part_sums + s * rows + row) : make_float2(kNegHuge, 0.f);
    top = fmaxf(top, sums[i].x);
  }
#pragma unroll
  for (int x = 16; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor(top, x, 32));
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    sums[i].x = __builtin_amdgcn_exp2f(sums[i].x - top);
    sum = fmaf(sums[i].x, sums[i].y, sum);
  }
#pragma unroll
  for (int x = 16; x > 0; x >>= 1) sum += __shfl_xor(sum, x, 32);
  f32x4 x = {};
  const float* part = p.partials + row * p.D + (c < p.D ? c : 0);
  for (int s0 = 0; s0 < p.splits; s0 += 8) {      // eight requests at a time; behind the last split the factors are 0
    f32x4 y[8];
#pragma unroll
    for (int s = 0; s < 8; ++s) y[s] = load4(part + min(s0 + s, p.splits - 1) * rows * p.D);
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      const float by = __shfl(s0 < 32 ? sums[0].x : sums[1].x, (s0 + s) & 31, 32);
      x += y[s] * (s0 + s < p.splits ? by : 0.f);
    }
  }
  const int head = kh * p.g + h;
  if (c < p.D) store4((T*)p.o.row(token, head) + c, x * (sum > 0.f ? 1.f / sum : sum == 0.f ? 0.f : sum));
  if (p.lse && c == 0) p.lse[token * p.hq + head] = sum == 0.f ? -__builtin_inff() : (top + __builtin_amdgcn_logf(sum)) * kLn2f;
}

// A gradient that comes in parts: out[token][head] = factor * sum over splits of partial[split][key head][token][in group], in their order.
// Bound by its launch where parts are used (few rows or keys): dk and dv of 1200 keys, 2 heads, 4.4 us.
struct GradSum {
  Heads out;
  const float* partials;
  float factor;
};
template <class T>
__global__ __launch_bounds__(256) void k_attn_add(const AttnArgs p, GradSum first, GradSum second, int64_t stride, int64_t tokens, int g) {
  if (*p.status != 0) return;
  const GradSum& grad = blockIdx.y ? second : first;
  const int64_t rows = tokens * p.hk * g, row = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int c = (threadIdx.x & 31) * 4;
  if (row >= rows || c >= p.D) return;
  const int kh = (int)(row / (tokens * g));
  const int64_t token = row / g - kh * tokens;
  f32x4 x = {};
#pragma unroll 8
  for (int s = 0; s < p.splits; ++s) x += load4(grad.partials + s * stride + row * p.D + c);
  store4((T*)grad.out.row(token, kh * g + (int)(row % g)) + c, x * grad.factor);
}

// ---------------------------------------------------------------------------------------------------------------- backward
// Adds up what the N wavefronts (every 4 / N-th) have of the same 32 rows (keys), in their order, in LDS of `each` bytes a wavefront: threads
// get a share(row, first channel, sums) each.
template <int DW, int N, class F>
__device__ __forceinline__ void add_wavefronts(const f32x4 (&acc)[2][DW / 16], lds_char_ptr lds, int each, F&& share) {
  constexpr int PITCH = padded(DW) * 4 + 16, G = 4 / N, THREADS = 2 * N, C = DW / THREADS;
  typedef __attribute__((address_space(3))) f32x4* lds_f32x4;
  __syncthreads();      // everybody is done with what was there
#pragma unroll
  for (int n = 0; n < 2; ++n)
#pragma unroll
    for (int d = 0; d < DW / 16; ++d)
      *(lds_f32x4)(lds + (threadIdx.x >> 6) * each + (n * 16 + (threadIdx.x & 15)) * PITCH + d * 64 + (threadIdx.x >> 4 & 3) * 16) = acc[n][d];
  __syncthreads();
  const int r = threadIdx.x / THREADS, c0 = threadIdx.x % THREADS * C;
  f32x4 x[C / 4] = {};
#pragma unroll
  for (int w = 0; w < N; ++w)
#pragma unroll
    for (int c = 0; c < C / 4; ++c) x[c] += *(lds_f32x4)(lds + (r / 32 + w * G) * each + r % 32 * PITCH + (c0 + c * 4) * 4);
  share(r, c0, x);
}
template <class T, int N>
__device__ __forceinline__ void store_share(char* row, int c0, const f32x4 (&x)[N], float factor, int D) {
#pragma unroll
  for (int c = 0; c < N; ++c)
    if (c0 + c * 4 < D) store4((T*)row + c0 + c * 4, x[c] * factor);
}

// dq, and what the other kernel needs of a row: its log-sum-exp in base 2 and D_i.  A workgroup has 128 rows over steps of 64 keys or,
// where tiles are few, 64 rows, two wavefronts for either half of the keys (WK = 2), or 32 rows over steps of 32 keys that the wavefronts take in
// turn (WK = 4), as forward.
// dq is summed here and dk, dv in the other kernel, which computes z and dP again (seven products, not five): one kernel would add to dq in
// memory from all tiles of keys, by atomics in an order that changes, or through sums of (keys / 128) x dq's size.
// Bound by the matrix cores at the power limit: 2 x 8192 tokens, 32 heads on 8 of 128 channels, no mask, three products in 2.94 ms, 1123
// TFLOP/s, matrix cores busy 0.58 at 1.85 GHz (under the profiler; both kernels in turn without it 6.10 ... 6.40 ms, 1202 ... 1262).  fp32 operands are
// twice as wide for the same registers: at 96 channels 17 to 19 are spilled, at 128 channels 87 (WK = 4) and 165.
template <class T, int DW, int WK>
__global__ __launch_bounds__(256, 2) void k_attn_dq(const AttnArgs p) {
  constexpr bool kAlone = WK == 4;      // a wavefront stages keys for itself
  constexpr int DP = padded(DW), KEYS = dq_keys<WK>, W = kAlone ? 1 : 4, STEP = KEYS * 4 / W, PER = WK == 1 ? KEYS : 32;      // PER: a wavefront's
  typedef typename FragOf<T>::type Frag;
  typedef Tile<T, DP> Lds;
  typedef Stager<T, DP, KEYS, W> Stage;
  typedef KeyLds<T, DP, WK, KEYS> Size;
  constexpr int B = 128 / WK, KS = DW / 32, DB = DW / 16, SIZE = Size::kTile;
  extern __shared__ char smem[];
  const int wave = uniform((int)threadIdx.x >> 6), half = WK == 2 ? (wave >> 1) * 32 : 0;      // of the staged keys, this wavefront's
  const lds_char_ptr lds = (lds_char_ptr)smem + (kAlone ? wave * Size::kEach : 0), words = (lds_char_ptr)smem + Size::kWords;
  const Job job(p);
  const int kh = job.kh;
  SeqTile t;
  const Found found = pick_tile<B>(p, kOfRows, job.rank, t);
  if (blockIdx.x == 0 && threadIdx.x == 0) *p.status = found == kMalformed ? kErrOffsets : 0;
  if (found == kMalformed) poison<T>(p.dq, p.Tq, p.hq, p.D);
  if (found != kTile) return;
  const int first_sees = all_rows_see(p, t);
  const Part part(tile_sees<B>(p, t), p.splits, job.part, STEP);
  const Stage ks(p.k.row(t.k0, kh), p.k.token, p.D), vs(p.v.row(t.k0, kh), p.v.token, p.D);
  int j0 = part.begin + (kAlone ? wave * KEYS : 0), slot = 0;
  const auto stage = [&](int at, int first) {
    ks.start(lds + at, first, t.nk);
    vs.start(lds + at + SIZE, first, t.nk);
  };
  if (Size::kSlots == 2 && j0 < part.end) stage(0, j0);
  const int group = threadIdx.x >> 4 & 3, row0 = t.first + wave % (4 / WK) * 32 + (threadIdx.x & 15);
  const float scale2 = p.scale * kLog2e;
  int row_sees[2];
  Frag q[2][KS], dout[2][KS];
  float lse2[2], delta[2];
  f32x4 dq[2][DB];
  int all_see = t.nk;
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    const Row row(p, t, row0 + n * 16);
    const int64_t token = t.q0 + row.token;
    const int head = kh * p.g + row.head;
#pragma unroll
    for (int d = 0; d < DB; ++d) zero(dq[n][d]);
    delta[n] = 0.f;
    Frag o[KS];
    load_row<T>(p.q.row(token, head), p.D, q[n]);
    load_row<T>(p.dout.row(token, head), p.D, dout[n]);
    load_row<T>(p.o.row(token, head), p.D, o);
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) delta[n] += dot(o[kk], dout[n][kk]);
    delta[n] = row_sum(delta[n]);
    lse2[n] = row.exists ? p.lse[token * p.hq + head] * kLog2e : 0.f;
    if (row.exists && group == 0 && job.part == 0 && wave < 4 / WK) {
      const int64_t at = packed_row(p, t, kh, row0 + n * 16);
      p.delta[at] = delta[n];
      // of a row that sees nothing: every probability comes out as 0
      p.lse2[at] = lse2[n] == -__builtin_inff() ? __builtin_inff() : lse2[n];
    }
    row_sees[n] = row.sees;
    if (row.exists) all_see = row.sees < all_see ? row.sees : all_see;
  }
#pragma unroll
  for (int x = 8; x > 0; x >>= 1) {
    const int y = __shfl_xor(all_see, x, 64);
    all_see = y < all_see ? y : all_see;
  }
  all_see = __builtin_amdgcn_readfirstlane(all_see);
  for (; j0 < part.end; j0 += STEP, slot ^= Size::kSlots == 2 ? 2 * SIZE : 0) {
    const bool masks = hides<KEYS>(t, first_sees, j0);
    if (Size::kSlots == 1) stage(0, j0);
    staged();
    bool found_odd = masks && staged_odd<T, Stage::kLoads, W>(lds + slot);
    if (!kAlone) {
      if (masks) tell_odd(words, slot != 0, found_odd);
      lds_barrier();
      found_odd = masks && told_odd(words, slot != 0);
    }
    if (Size::kSlots == 2 && j0 + STEP < part.end) stage(slot ^ 2 * SIZE, j0 + STEP);
    const lds_char_ptr own = lds + slot + half * Lds::kPitch;
    const int k_rows = Lds::rows_place(own, threadIdx.x), k_columns = Lds::columns_place(own, threadIdx.x);
    const uint64_t odd = found_odd ? clean_tile<T, DP, KEYS, W>(lds + slot, words + 32) >> half : 0;
    f32x4 s[2][2][2], dp[2][2][2];     // [32 keys][rows][keys]
    Frag w[2][2];
    const auto finish = [&](int c, int i) {
      const int n = i >> 3, x = i & 7;
      s[c][n][x >> 2][x & 3] = __builtin_amdgcn_exp2f(fmaf(s[c][n][x >> 2][x & 3], scale2, -lse2[n])) * (dp[c][n][x >> 2][x & 3] - delta[n]);
    };
    const auto mask = [&](int c) {
      if (odd) mark_odd(s[c], (uint32_t)(odd >> (c * 32)));
      if (j0 + half + c * 32 + 32 > all_see) {
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int x = 0; x < 8; ++x) {
            const int key = (x >> 2) * 16 + group * 4 + (x & 3);
            if (j0 + half + c * 32 + key >= row_sees[n]) s[c][n][x >> 2][x & 3] = 0.f;
          }
      }
#pragma unroll
      for (int n = 0; n < 2; ++n) pack(s[c][n][0], s[c][n][1], w[c][n]);
      ready(w[c]);
    };
    // the elements [from, to) of 32 keys c that go with one of n pairs of multiplications
    const auto share = [&](int c, int from, int to, int i, int n) {
#pragma unroll
      for (int x = from + (to - from) * i / n; x < from + (to - from) * (i + 1) / n; ++x) finish(c, x);
    };
    scores<Lds, KS>(s[0], k_rows, 0, q, [](int) {});
    scores<Lds, KS>(dp[0], k_rows, SIZE, dout, [](int) {});
    if constexpr (PER == 64) {
      scores<Lds, KS>(s[1], k_rows, 32 * Lds::kPitch, q, [&](int i) { share(0, 0, 8, i, 2 * KS); });
      scores<Lds, KS>(dp[1], k_rows, SIZE + 32 * Lds::kPitch, dout, [&](int i) { share(0, 8, 16, i, 2 * KS); });
    } else {
      share(0, 0, 16, 0, 1);
    }
    mask(0);
    add_columns<Lds, DB>(dq, k_columns, 0, w[0], [&](int i) {
      if (PER == 64) share(1, 0, 16, i, DB);
    });
    if constexpr (PER == 64) {
      mask(1);
      add_columns<Lds, DB>(dq, k_columns, 32 * Lds::kPitch, w[1], [](int) {});
    }
  }
  settle(dq);
  if constexpr (WK == 1) {
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      const Row row(p, t, row0 + n * 16);
      if (!row.exists) continue;
      if (p.splits > 1) store_columns<float>((char*)partial_row(p, job.part, p.Tq * p.hq, packed_row(p, t, kh, row0 + n * 16)), dq[n], 1.f, p.D);
      else store_columns<T>(p.dq.row(t.q0 + row.token, kh * p.g + row.head), dq[n], p.scale, p.D);
    }
  } else {
    add_wavefronts<DW, WK>(dq, (lds_char_ptr)smem, Size::kEach, [&](int r, int c0, const auto& x) {
      const Row row(p, t, t.first + r);
      if (!row.exists) return;
      if (p.splits > 1) store_share<float>((char*)partial_row(p, job.part, p.Tq * p.hq, packed_row(p, t, kh, t.first + r)), c0, x, 1.f, p.D);
      else store_share<T>(p.dq.row(t.q0 + row.token, kh * p.g + row.head), c0, x, p.scale, p.D);
    });
  }
}

// Rows of two operands (queries and the output's gradient) and the rows' two numbers on their way to LDS, as Stager; what lies
// behind the sequence's last row or channel D reads as zeros.
template <class T, int DP, int R, int W>
struct RowStager {
  typedef Tile<T, DP> Lds;
  static constexpr int kRowsPerLoad = 64 / Lds::kChunks, kLoads = R / (W * kRowsPerLoad), SIZE = R * Lds::kPitch;
  static constexpr int kBytes = 2 * SIZE + 2 * 64 * 4;      // a load of numbers has 64
  static constexpr uint32_t kOutside = 0x80000000u;
  // Starts the loads of rows [first, first + R); `first` is a multiple of R.
  __device__ static __forceinline__ void start(const AttnArgs& p, const SeqTile& t, int kh, lds_char_ptr lds, int first) {
    const int wave = W == 1 ? 0 : uniform((int)threadIdx.x >> 6), rows = t.nq * p.g, token0 = uniform(by_group(p, first));
    const __amdgpu_buffer_rsrc_t q =
        __builtin_amdgcn_make_buffer_rsrc((void*)p.q.row(t.q0 + token0, kh * p.g), 0, kOutside, 0x00020000);
    const __amdgpu_buffer_rsrc_t d =
        __builtin_amdgcn_make_buffer_rsrc((void*)p.dout.row(t.q0 + token0, kh * p.g), 0, kOutside, 0x00020000);
    const int lane = fresh(threadIdx.x) & 63;      // what follows is made here, not kept: registers are short
    // Where the heads in a group divide the rows that lie between two loads of a wavefront, a lane is at the same place of a token's
    // heads with every load, and only the (scalar) token moves.
    if (W * kRowsPerLoad % 16 == 0 && p.g <= W * kRowsPerLoad && (p.g & (p.g - 1)) == 0 && first + R <= rows) {
      const int tokens = by_group(p, W * kRowsPerLoad), r = wave * kRowsPerLoad + lane / Lds::kChunks, token = by_group(p, r);
      const int c = ((lane % Lds::kChunks) ^ Lds::swizzle(r)) * 16, head = r - token * p.g;
      const bool any = c < p.D * (int)sizeof(T);
      const uint32_t whole_q = any ? (uint32_t)(token * (int)p.q.token + head * (int)p.q.head + c) : kOutside;
      const uint32_t whole_d = any ? (uint32_t)(token * (int)p.dout.token + head * (int)p.dout.head + c) : kOutside;
#pragma unroll
      for (int j = 0; j < kLoads; ++j) {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(q, (lds_void_ptr)(lds + (j * W + wave) * 1024), 16, whole_q,
                                                 j * tokens * (int)p.q.token, 0, 0);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(d, (lds_void_ptr)(lds + SIZE + (j * W + wave) * 1024), 16, whole_d,
                                                 j * tokens * (int)p.dout.token, 0, 0);
      }
    } else {
#pragma unroll
      for (int j = 0; j < kLoads; ++j) {
        const int r = (j * W + wave) * kRowsPerLoad + lane / Lds::kChunks, x = first + r;
        const int c = ((lane % Lds::kChunks) ^ Lds::swizzle(r)) * 16;
        const int token = by_group(p, x), head = x - token * p.g;
        const bool any = x < rows && c < p.D * (int)sizeof(T);
        const uint32_t vq = (uint32_t)((token - token0) * (int)p.q.token + head * (int)p.q.head + c);
        const uint32_t vd = (uint32_t)((token - token0) * (int)p.dout.token + head * (int)p.dout.head + c);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(q, (lds_void_ptr)(lds + (j * W + wave) * 1024), 16, any ? vq : kOutside, 0, 0, 0);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(d, (lds_void_ptr)(lds + SIZE + (j * W + wave) * 1024), 16, any ? vd : kOutside, 0, 0, 0);
      }
    }
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      if (W > 1 && wave != which) continue;
      const int left = rows - first < R ? rows - first : R;
      const __amdgpu_buffer_rsrc_t n =
          __builtin_amdgcn_make_buffer_rsrc((void*)((which ? p.delta : p.lse2) + packed_row(p, t, kh, first)), 0, left * 4, 0x00020000);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(n, (lds_void_ptr)(lds + 2 * SIZE + which * 256), 4, lane * 4, 0, 0, 0);
    }
  }
};

// LDS of a workgroup for dk and dv, as KeyLds.
template <class T, int DP, int WK>
struct RowLds {
  static constexpr int kRows = WK == 4 ? 32 : 64, kSlots = WK == 4 && sizeof(T) == 4 ? 1 : 2;
  typedef RowStager<T, DP, kRows, WK == 4 ? 1 : 4> Stage;
  static constexpr int kStages = kSlots * Stage::kBytes, kResults = 32 * (DP * 4 + 16);
  static constexpr int kEach = WK == 4 && kStages > kResults ? kStages : (kResults + 511) / 512 * 512;      // of a wavefront
  static constexpr int kWords = WK == 1 || (WK == 2 && kStages > 4 * kEach) ? kStages : 4 * kEach, kBytes = kWords + 48;
  static_assert(kBytes <= 160 * 1024, "LDS of one CU");
};

// dk and dv: a workgroup has 128 keys, 32 a wavefront, over all rows that see any of them, 64 at a time; or (WK = 2) 64 keys, two
// wavefronts for either half of the 64 rows; or (WK = 4) 32 keys, over steps of 32 rows that the wavefronts take in turn.
// Two accumulators and two resident operands fill a lane's 256 registers, so where in LDS a step reads is computed anew each time.  Bound by
// the matrix cores at the power limit: 2 x 8192 tokens, 32 heads on 8 of 128 channels, no mask, four products in 3.92 ms, 1123
// TFLOP/s, matrix cores busy 0.56 at 1.89 GHz (under the profiler, as above).  Spilled all the same: at 128 channels 9 registers (WK = 4: 4), in fp32
// 100; at 96 channels in fp32 11 to 13.
template <class T, int DW, int WK>
__global__ __launch_bounds__(256, 2) void k_attn_dkdv(const AttnArgs p) {
  constexpr int DP = padded(DW);
  typedef typename FragOf<T>::type Frag;
  typedef Tile<T, DP> Lds;
  typedef RowLds<T, DP, WK> Size;
  typedef typename Size::Stage Stage;
  constexpr int B = 128 / WK, KS = DW / 32, DB = DW / 16, kRows = Size::kRows;
  extern __shared__ char smem[];
  constexpr bool kAlone = WK == 4;      // a wavefront stages rows for itself
  const int wave = uniform((int)threadIdx.x >> 6), tile_wave = wave % (4 / WK);
  const lds_char_ptr lds = (lds_char_ptr)smem + (kAlone ? wave * Size::kEach : 0), words = (lds_char_ptr)smem + Size::kWords;
  const Job job(p);
  const int kh = job.kh;
  SeqTile t;
  const Found found = pick_tile<B>(p, kOfKeys, job.rank, t);
  if (found == kMalformed) {
    poison<T>(p.dk, p.Tk, p.hk, p.D);
    poison<T>(p.dv, p.Tk, p.hk, p.D);
  }
  if (found != kTile) return;
  const int rows = t.nq * p.g, ahead = t.nk - t.nq;
  // the first row that sees the tile's first key, and whole tiles of rows
  const int from = p.causal && t.first > ahead ? (t.first - ahead) * p.g / kRows * kRows : 0;
  const Part part(rows > from ? rows - from : 0, p.splits, job.part, kRows * (kAlone ? 4 : 1));
  // Large tiles go backwards: those that run at a time begin at different rows and end at the same, so they share what the L2 holds from there
  // on (2 x 8192 tokens, 32 heads on 8, 3447 -> 3243 us with dq).  Small ones go forwards (1000 tokens 95, backwards 100 us).
  constexpr int kStep = kRows * (kAlone ? 4 : 1), kBy = kAlone ? kStep : -kStep;
  const int begin = from + part.begin, end = from + part.end;
  int r0 = kAlone ? begin + wave * kRows : begin + (end - begin + kStep - 1) / kStep * kStep - kStep, slot = 0;
  const auto any = [&](int at) { return kAlone ? at < end : at >= begin; };
  if (Size::kSlots == 2 && any(r0)) Stage::start(p, t, kh, lds, r0);
  Frag k[2][KS], v[2][KS];
  f32x4 dk[2][DB], dv[2][DB];
  const auto first_row = [&](int key) { return p.causal && key < t.nk && key > ahead ? (key - ahead) * p.g : 0; };   // that sees it
  int all_from = 0;     // rows from here on see every key of the wavefront
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    const int key = t.first + tile_wave * 32 + n * 16 + (threadIdx.x & 15), at = key < t.nk ? key : t.nk - 1;
#pragma unroll
    for (int d = 0; d < DB; ++d) zero(dk[n][d]), zero(dv[n][d]);
    load_row<T>(p.k.row(t.k0 + at, kh), p.D, k[n]);
    load_row<T>(p.v.row(t.k0 + at, kh), p.D, v[n]);
    all_from = first_row(key) > all_from ? first_row(key) : all_from;
  }
#pragma unroll
  for (int x = 8; x > 0; x >>= 1) {
    const int y = __shfl_xor(all_from, x, 64);
    all_from = y > all_from ? y : all_from;
  }
  all_from = __builtin_amdgcn_readfirstlane(all_from);
  const float scale2 = p.scale * kLog2e;
  const int masked_to = first_row((t.first + B < t.nk ? t.first + B : t.nk) - 1);      // rows from here on see every key of the workgroup
  for (; any(r0); r0 += kBy, slot ^= Size::kSlots == 2) {
    const lds_char_ptr tiles = lds + slot * Stage::kBytes, numbers = tiles + 2 * Stage::SIZE;
    if (Size::kSlots == 1) Stage::start(p, t, kh, lds, r0);
    staged();
    bool odd = r0 < masked_to && (staged_odd<T, Stage::kLoads, kAlone ? 1 : 4>(tiles) || staged_odd<T, Stage::kLoads, kAlone ? 1 : 4>(tiles + Stage::SIZE));
    if (!kAlone) {
      if (r0 < masked_to) tell_odd(words, slot, odd);
      lds_barrier();
      odd = r0 < masked_to && told_odd(words, slot);
    }
    if (Size::kSlots == 2 && any(r0 + kBy)) Stage::start(p, t, kh, lds + (slot ^ 1) * Stage::kBytes, r0 + kBy);
    if (odd) {      // a row's probabilities are NaN where its log-sum-exp is
      typedef __attribute__((address_space(3))) float* lds_f32;
      const uint64_t which = clean_tile<T, DP, kRows, kAlone ? 1 : 4, 2, Stage::SIZE>(tiles, words + 32);
      const int x = kAlone ? threadIdx.x & 63 : threadIdx.x;
      if (x < kRows && (which >> x & 1)) ((lds_f32)numbers)[x] = quiet_nan();
      if (!kAlone) lds_barrier();
    }
#pragma unroll 1
    for (int c = WK == 2 ? wave >> 1 : 0; c < kRows / 32; c += WK) {
      typedef __attribute__((address_space(3))) f32x4* ptr;
      const lds_char_ptr tile = tiles + c * 32 * Lds::kPitch;
      Frag w[2], wd[2];      // probabilities and dS of 32 rows, keys in columns
      f32x4 s[2][2], dp[2][2];     // [keys][rows]
      scores2<Lds, KS, Stage::SIZE>(s, dp, Lds::rows_place(tile, fresh(threadIdx.x)), k, v);      // places are not kept: registers are short
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const lds_char_ptr at = numbers + (fresh(threadIdx.x) >> 4 & 3) * 16 + (c * 32 + b * 16) * 4;
        const f32x4 lse2 = *(ptr)at, delta = *(ptr)(at + 256);
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            s[n][b][i] = __builtin_amdgcn_exp2f(fmaf(s[n][b][i], scale2, -lse2[i]));
            dp[n][b][i] = s[n][b][i] * (dp[n][b][i] - delta[i]);
          }
      }
      if (r0 + c * 32 < all_from) {
        const int lane = fresh(threadIdx.x) & 63, key0 = t.first + tile_wave * 32 + (lane & 15);
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int x = 0; x < 8; ++x) {
            const int row = (x >> 2) * 16 + (lane >> 4) * 4 + (x & 3);
            if (r0 + c * 32 + row < first_row(key0 + n * 16)) s[n][x >> 2][x & 3] = dp[n][x >> 2][x & 3] = 0.f;
          }
      }
#pragma unroll
      for (int n = 0; n < 2; ++n) pack(s[n][0], s[n][1], w[n]), pack(dp[n][0], dp[n][1], wd[n]);
      ready(w);
      ready(wd);
      add_columns2<Lds, DB, Stage::SIZE>(dk, dv, Lds::columns_place(tile, fresh(threadIdx.x)), wd, w);
    }
  }
  settle(dk);
  settle(dv);
  if constexpr (WK == 1) {
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      const int key = t.first + tile_wave * 32 + n * 16 + (threadIdx.x & 15);
      if (key >= t.nk) continue;
      if (p.splits > 1) {
        float* to = partial_row(p, job.part, 2 * p.Tk * p.hk, kh * p.Tk + t.k0 + key);
        store_columns<float>((char*)to, dk[n], 1.f, p.D);
        store_columns<float>((char*)(to + p.Tk * p.hk * p.D), dv[n], 1.f, p.D);
        continue;
      }
      store_columns<T>(p.dk.row(t.k0 + key, kh), dk[n], p.scale, p.D);
      store_columns<T>(p.dv.row(t.k0 + key, kh), dv[n], 1.f, p.D);
    }
  } else {
    const auto share = [&](const Heads& out, int64_t behind, float factor) {
      return [&p, &t, &out, &job, kh, behind, factor](int r, int c0, const auto& x) {
        const int key = t.first + r;
        if (key >= t.nk) return;
        if (p.splits > 1) store_share<float>((char*)(partial_row(p, job.part, 2 * p.Tk * p.hk, kh * p.Tk + t.k0 + key) + behind), c0, x, 1.f, p.D);
        else store_share<T>(out.row(t.k0 + key, kh), c0, x, factor, p.D);
      };
    };
    add_wavefronts<DW, WK>(dk, (lds_char_ptr)smem, Size::kEach, share(p.dk, 0, p.scale));
    add_wavefronts<DW, WK>(dv, (lds_char_ptr)smem, Size::kEach, share(p.dv, p.Tk * p.hk * p.D, 1.f));
  }
}

}  // namespace oapl
