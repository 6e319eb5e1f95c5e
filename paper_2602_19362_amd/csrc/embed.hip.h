// Embedding lookup with scaling, and its gradient.
//
//   out_t = scale E[tok_t],      dE[v] = scale sum over t with tok_t = v of dout_t
//
// Bound by memory.  The gradient's sums have a fixed order: tokens are sorted by id, stably, so by position among equals.  Few of them are sorted
// by counting (k_embed_rank) and summed by the workgroup that a token's rows begin in (k_embed_runs): two launches.  Many are sorted in two
// passes (k_embed_count, k_embed_place twice), and their sorted positions cut into tiles of equal length, so that a frequent token is shared by
// many workgroups (k_embed_sum); what a tile has of a token that reaches over its ends goes into the workspace and is added up by another
// launch, tile by tile (k_embed_join).  dE is cleared beside the sorting, not between reads: memory takes 6.6 TB/s of reads alone, 7.3 of zeros
// and 5.3 of the sums' reads and writes.
//
// 140897 tokens that follow Zipf's law, d = 4096 in bf16, V = 151936 (3.6 GB): counting 6 us, first pass and 0.19 GB of zeros 39,
// second pass and 1.86 GB of zeros 281, sums 343 (1.16 GB in, 0.66 out: 5.3 TB/s), tokens over tiles 23.  1003 of them: places and 2.49 GB of zeros 341, sums 12.
#pragma once

#include "rows.hip.h"

namespace oapl {

// ---------------------------------------------------------------------------------------------------------------- lookup
struct EmbedArgs {
  const void* E;              // [V][d]
  const int32_t* tokens;
  Rows out;
  int64_t T;
  int d, V;
  float scale;
  uint32_t slices;
};

// A wavefront has a token and PIECES times 64 pieces of its row; those of a row follow each other, so that memory is written in order.
// ONCE: results past the caches.  140897 tokens, d = 4096 in bf16, 1 / 2 / 4 pieces: 361 / 308 / 315 us, past the caches 332 / 284 / 300 (1.15 GB
// written, 0.31 of the embedding read: 5.2 TB/s), slices of rows one after the other 462 / 433 / 331 and 424 / 397 / 316.
template <class TE, class T, int W, int PIECES, Form FORM, bool ONCE>
__global__ __launch_bounds__(256) void k_embed_fwd(const EmbedArgs p) {
  const uint32_t unit = (blockIdx.y * gridDim.x + blockIdx.x) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), t = unit / p.slices;
  const int c = (unit % p.slices * PIECES * 64 + (threadIdx.x & 63)) * W;
  if (t >= p.T) return;
  const int32_t v = __builtin_amdgcn_readfirstlane(p.tokens[t]);
  const bool inside = v >= 0 && v < p.V;
  const TE* from = (const TE*)p.E + (int64_t)(inside ? v : 0) * p.d;
  const float scale = inside ? p.scale : quiet_nan();
  Piece<W> x[PIECES];
#pragma unroll
  for (int i = 0; i < PIECES; ++i) x[i] = load_piece<W, FORM>(from, c + i * 64 * W, p.d);
#pragma unroll
  for (int i = 0; i < PIECES; ++i) {
#pragma unroll
    for (int e = 0; e < W; ++e) x[i].v[e] *= scale;
    store_piece<W, FORM, ONCE>(p.out.row<T>(t), c + i * 64 * W, p.d, x[i]);
  }
}

// ---------------------------------------------------------------------------------------------------------------- gradient: sorting
constexpr int kSortThreads = 1024;

// Tokens sorted by id in two passes, each by half of the id's bits; V stands for all ids outside [0, V) and comes last.  A block of keys is
// a workgroup's; `counts` has, of every block, how many keys it has of each digit.
struct SortArgs {
  const int32_t* tokens;
  int32_t *keys[2], *places[2];     // what a pass leaves: ids and their positions
  int32_t* counts[2];               // [blocks][1 << bits]
  uint8_t* present;                 // [V]: whether an id occurs
  int* status;
  float* dE;                        // to be cleared: all of it beside the counting, or its first rows beside the first pass and, of the others,
  bool clear_absent;                // those whose id does not occur, beside the second
  int early;
  int64_t T;
  int V, d, bits, block, blocks;    // keys of a block, and how many of them
};

__device__ __forceinline__ int sort_key(const SortArgs& p, int64_t t) {
  const int32_t v = p.tokens[t];
  return v >= 0 && v < p.V ? v : p.V;
}

// 1024 elements of dE, from 1024 i on, are zero: 4 KB a workgroup, and four workgroups a compute unit, which kClearLds bytes of LDS see to, is the
// order that memory likes best (2.49 GB in a launch of its own 357 us, 16 KB a workgroup 402, 256 KB 400 .. 430; beside the places of 1003 tokens 341; beside the counting of 6000 tokens, eight
// workgroups 431, six 425, four 409).
constexpr int kClearLds = 33 * 1024;
__device__ __forceinline__ void clear_piece(float* dE, int64_t n, int64_t i) {
  const int64_t at = (i * 256 + threadIdx.x) * 4;
  if (at + 4 <= n) {
    store_whole<4>(dE + at, Piece<4>{});
  } else {
    for (int64_t e = at; e < n; ++e) dE[e] = 0.f;
  }
}

// First pass's counts; the second's, and `present`, start at zero.  The workgroups behind clear dE.
__global__ __launch_bounds__(256) void k_embed_count(const SortArgs p) {
  extern __shared__ int32_t count[];
  if ((int)blockIdx.x >= p.blocks || blockIdx.y > 0) {
    clear_piece(p.dE, (int64_t)p.V * p.d, (int64_t)blockIdx.y * gridDim.x + blockIdx.x - p.blocks);
    return;
  }
  const int bins = 1 << p.bits;
  for (int i = threadIdx.x; i < bins; i += 256) count[i] = 0;
  __syncthreads();
  const int64_t from = (int64_t)blockIdx.x * p.block, to = from + p.block < p.T ? from + p.block : p.T;
#pragma unroll 8
  for (int64_t t = from + threadIdx.x; t < to; t += 256) atomicAdd(&count[sort_key(p, t) & (bins - 1)], 1);
  __syncthreads();
  for (int i = threadIdx.x; i < bins; i += 256) {
    p.counts[0][(int64_t)blockIdx.x * bins + i] = count[i];
    p.counts[1][(int64_t)blockIdx.x * bins + i] = 0;
  }
  if (p.clear_absent)
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < p.V; i += (int64_t)p.blocks * 256) p.present[i] = 0;
  if (blockIdx.x == 0 && threadIdx.x < kStatusWords) p.status[threadIdx.x] = 0;
}

// 1024 channels of 16 rows of dE, a wavefront's one each, are zero: of the first p.early rows beside the first pass, of the others, where the row's
// id does not occur, beside the second.
template <int PASS>
__device__ __forceinline__ void clear_rows(const SortArgs& p, int64_t i) {
  const int lane = threadIdx.x & 63, pieces = (p.d + 1023) / 1024;
  const int64_t v = i / pieces * (kSortThreads / 64) + (threadIdx.x >> 6) + (PASS == 0 ? 0 : p.early);
  if (v >= (PASS == 0 ? p.early : p.V) || (PASS == 1 && p.present[v])) return;
  float* row = p.dE + v * p.d;
#pragma unroll
  for (int j = 0; j < 4; ++j) store_piece<4, kAny>(row, (int)(i % pieces) * 1024 + (j * 64 + lane) * 4, p.d, Piece<4>{});
}

// Pass 0 reads tokens, pass 1 what pass 0 left.  A key's place: keys of smaller digits, those of its digit in earlier blocks, in earlier
// wavefronts of this block, and before it in its wavefront.
template <int PASS, int ITEMS>
__global__ __launch_bounds__(kSortThreads) void k_embed_place(const SortArgs p) {
  extern __shared__ int32_t lds[];
  const int bins = 1 << p.bits, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  constexpr int WAVES = kSortThreads / 64;
  if ((int)blockIdx.x >= p.blocks || blockIdx.y > 0) {
    clear_rows<PASS>(p, (int64_t)blockIdx.y * gridDim.x + blockIdx.x - p.blocks);
    return;
  }
  int32_t *mine = lds, *total = lds + WAVES * bins, *earlier = total + bins;
  // mine [WAVES][bins]: first a wavefront's counts, then where its keys of a digit begin
  for (int i = threadIdx.x; i < (WAVES + 2) * bins; i += kSortThreads) lds[i] = 0;
  __syncthreads();
  const int64_t from = ((int64_t)blockIdx.x * WAVES + wave) * 64 * ITEMS;
  int key[ITEMS], rank[ITEMS], first[ITEMS];
  uint64_t same[ITEMS];                      // lanes with the same digit, and the first of them
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const int64_t t = from + i * 64 + lane;
    const bool any = t < p.T;
    key[i] = !any ? 0 : PASS == 0 ? sort_key(p, t) : p.keys[0][t];
    const int digit = PASS == 0 ? key[i] & (bins - 1) : key[i] >> p.bits;
    same[i] = __ballot(any);
    for (int b = 0; b < p.bits; ++b) {
      const uint64_t set = __ballot((digit >> b) & 1);
      same[i] &= (digit >> b) & 1 ? set : ~set;
    }
    const int before = __popcll(same[i] & (((uint64_t)1 << lane) - 1));
    first[i] = any ? __ffsll((unsigned long long)same[i]) - 1 : lane;
    int base = 0;
    if (any && lane == first[i]) base = atomicAdd(&mine[wave * bins + digit], __popcll(same[i]));
    rank[i] = __shfl(base, first[i], 64) + before;
  }
  // keys of every digit, in all blocks and in earlier ones
  const int wide = bins < kSortThreads ? bins : kSortThreads, parts = kSortThreads / wide;
  for (int bin = threadIdx.x & (wide - 1); bin < bins; bin += kSortThreads) {
    int32_t in_all = 0, in_earlier = 0;
#pragma unroll 8
    for (int i = threadIdx.x / wide; i < p.blocks; i += parts) {
      const int32_t n = p.counts[PASS][(int64_t)i * bins + bin];
      in_all += n;
      in_earlier += i < (int)blockIdx.x ? n : 0;
    }
    atomicAdd(&total[bin], in_all);
    atomicAdd(&earlier[bin], in_earlier);
  }
  __syncthreads();
  // where a digit's keys begin: sums over smaller digits, two to a thread
  const int b = threadIdx.x * 2;
  const int32_t n0 = b < bins ? total[b] : 0, n1 = b < bins ? total[b + 1] : 0;
  int32_t up = n0 + n1;
  for (int o = 1; o < 64; o <<= 1) {
    const int32_t below = __shfl_up(up, o, 64);
    if (lane >= o) up += below;
  }
  __shared__ int32_t wave_sums[WAVES];
  if (lane == 63) wave_sums[wave] = up;
  __syncthreads();
  up -= n0 + n1;
  for (int i = 0; i < wave; ++i) up += wave_sums[i];
  if (b < bins) earlier[b] += up, earlier[b + 1] += up + n0;
  __syncthreads();
  for (int i = threadIdx.x; i < bins; i += kSortThreads) {
    int32_t at = earlier[i];
    for (int w = 0; w < WAVES; ++w) {
      const int32_t n = mine[w * bins + i];
      mine[w * bins + i] = at;
      at += n;
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const int64_t t = from + i * 64 + lane;
    const bool any = t < p.T;
    const int digit = PASS == 0 ? key[i] & (bins - 1) : key[i] >> p.bits;
    const int32_t to = mine[wave * bins + digit] + rank[i];
    if (any) {
      p.keys[PASS][to] = key[i];
      p.places[PASS][to] = PASS == 0 ? (int32_t)t : p.places[0][t];
    }
    if constexpr (PASS == 0) {
      // Counts for the second pass.  Lanes that add to the same one as the first of their digit, as those of a frequent token do, add together:
      // 140897 tokens, one in 40 of them the same, V = 151936, each lane for itself / together, us for the whole call: d = 64 94 / 86, 4096 730 / 724.
      const int at = any ? (to / (kSortThreads * ITEMS) << p.bits) + (key[i] >> p.bits) : -1;
      const int with = __shfl(at, first[i], 64);
      const uint64_t together = __ballot(at == with) & same[i];
      if (any && at != with) atomicAdd(&p.counts[1][at], 1);
      if (any && lane == first[i]) atomicAdd(&p.counts[1][at], __popcll(together));
      if (any && lane == first[i] && key[i] == p.V) atomicExch(p.status, kErrTokenRange);
      if (p.clear_absent && any && key[i] < p.V) p.present[key[i]] = 1;
    }
  }
}

// ---------------------------------------------------------------------------------------------------------------- gradient: sums
struct EmbedSumArgs {
  Rows dout;
  const int32_t *keys, *places;     // sorted
  float *dE, *partials;             // partials [tiles][2][d]: of the token that a tile begins in the middle of, and of the one that it leaves
  int64_t T;
  int d, V, tile, tiles, slices;    // slices of 1024 channels
  float scale;
  bool add;                         // to what dE holds
};

// A row's sum into dE.  ONCE: past the caches.
template <Form FORM, bool ONCE = false>
__device__ __forceinline__ void put_row(const EmbedSumArgs& p, int64_t v, int c, Piece<4> sum) {
  float* row = p.dE + v * p.d;
#pragma unroll
  for (int e = 0; e < 4; ++e) sum.v[e] *= p.scale;
  if (p.add) {
    const Piece<4> old = load_piece<4, FORM>(row, c, p.d);
#pragma unroll
    for (int e = 0; e < 4; ++e) sum.v[e] += old.v[e];
  }
  store_piece<4, FORM, ONCE>(row, c, p.d, sum);
}

// Rows of dout whose loads are under way together.  Where fewer are left, the last one is loaded again and left out: a branch around a load keeps
// those after it waiting (140000 tokens, d = 1024, V = 1000 130 us with branches, 102 without; 4000, d = 4096, V = 1544 33 / 26).  Of sorted rows in tiles 16
// (140897 tokens, d = 4096, V = 151936 4 / 8 / 16: 734 / 728 / 723 us).
constexpr int kEmbedRows = 8, kSumRows = 16;

// The sum of `n` of 64 rows, from the i-th on, whose positions a wavefront's lanes have.
template <class T, int ROWS, Form FORM>
__device__ __forceinline__ void add_rows(const EmbedSumArgs& p, Piece<4>& sum, int place, int i, int n, int c) {
  Piece<4> x[ROWS] = {};
#pragma unroll
  for (int u = 0; u < ROWS; ++u)
    x[u] = load_piece<4, FORM>(p.dout.row<T>(__builtin_amdgcn_readlane(place, i + min(u, n - 1))), c, p.d);
#pragma unroll
  for (int u = 0; u < ROWS; ++u)
    if (u < n) {
#pragma unroll
      for (int e = 0; e < 4; ++e) sum.v[e] += x[u].v[e];
    }
}

// A workgroup sums up 1024 channels, four a lane, of a tile's rows; the slices of a tile run side by side.  A wavefront has the ids and
// positions of 64 rows in its lanes, so that its walk over them branches on scalars.  ONCE: rows past the caches, in and out.
template <class T, Form FORM, bool ONCE>
__global__ __launch_bounds__(256) void k_embed_sum(const EmbedSumArgs p) {
  const uint32_t unit = blockIdx.y * gridDim.x + blockIdx.x;
  const int lane = threadIdx.x & 63, tile = unit / p.slices, c = (unit % p.slices * 256 + threadIdx.x) * 4;
  if (tile >= p.tiles || c - lane * 4 >= p.d) return;
  const int from = tile * p.tile, to = from + p.tile < p.T ? from + p.tile : (int)p.T;
  const int first = p.keys[from], last = p.keys[to - 1];
  const bool begun = from > 0 && p.keys[from - 1] == first, open = to < p.T && p.keys[to] == last;
  Piece<4> sum = {};
  for (int base = from; base < to; base += 64) {
    const int n = to - base < 64 ? to - base : 64;
    const int key = lane < n ? p.keys[base + lane] : -1, place = lane < n ? p.places[base + lane] : 0;
    const int after = lane + 1 < n || (lane < n && base + n < to) ? p.keys[base + lane + 1] : -1;
    const uint64_t ends = __ballot(key != after);
    for (int i = 0; i < n; i += kSumRows) {
      Piece<4> x[kSumRows] = {};
#pragma unroll
      for (int u = 0; u < kSumRows; ++u)
        x[u] = load_piece<4, FORM, ONCE>(p.dout.row<T>(__builtin_amdgcn_readlane(place, min(i + u, n - 1))), c, p.d);
#pragma unroll
      for (int u = 0; u < kSumRows; ++u) {
        if (i + u >= n) break;
#pragma unroll
        for (int e = 0; e < 4; ++e) sum.v[e] += x[u].v[e];
        if (!((ends >> (i + u)) & 1)) continue;
        const int v = __builtin_amdgcn_readlane(key, i + u);
        if (begun && v == first) store_piece<4, FORM>(p.partials + (int64_t)tile * 2 * p.d, c, p.d, sum);
        else if (open && v == last) store_piece<4, FORM>(p.partials + ((int64_t)tile * 2 + 1) * p.d, c, p.d, sum);
        else if (v < p.V) put_row<FORM, ONCE>(p, v, c, sum);
        sum = Piece<4>{};
      }
    }
  }
}

// How many of the numbers before i, i - 1 and on, `f` holds for; it holds for none before the first that it does not hold for, and for fewer than
// kMostEqual.  A wavefront asks for 64 of them, and where it holds for all, for every 4096th, every 64th and every one: 8000 equal ids are four
// loads one after the other, not 125 (d = 64, V = 8192: half of 8000 tokens the same 89 us for the whole call with 125, 74 with four; all of
// 140897 140 and 117).
constexpr int kMostEqual = 64 * 64 * 64;
template <class F>
__device__ __forceinline__ int equal_before(int i, F f) {
  const int lane = threadIdx.x & 63;
  const auto steps = [&](int from, int step) {
    const uint64_t not_held = __ballot(!f(from - (lane + 1) * step));
    return not_held ? __ffsll((unsigned long long)not_held) - 1 : 64;
  };
  int n = steps(i, 1);
  if (n < 64) return n;
  n = 0;
#pragma unroll
  for (int step = 4096; step >= 1; step /= 64) n += steps(i - n, step) * step;
  return n;
}

// Tokens that reach over the ends of tiles: where one ends in one of a workgroup's tiles, its wavefronts add up what the tiles have of it,
// equal parts of them each, in their order and in 64 bits.  Tiles and wavefronts of a workgroup 4 and 4 / 4 and 8 / 16 and 8 / 16 and 16, whole call of
// 140897 tokens: 783 / 807 / 804 / 885 us.
// Its loads need no branch: 100000 tokens, d = 64, V = 8192, one id, 296 us with branches, 105 without; one in 21 of V = 1000 60 and 51.
constexpr int kJoinTiles = 4, kJoinParts = 4;

template <Form FORM>
__global__ __launch_bounds__(64 * kJoinParts) void k_embed_join(const EmbedSumArgs p) {
  __shared__ double parts[kJoinParts][4][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = (blockIdx.y * 64 + lane) * 4;
  const int tile0 = blockIdx.x * kJoinTiles;
  const int64_t from = (int64_t)(tile0 + lane) * p.tile, to = from + p.tile < p.T ? from + p.tile : p.T;
  int key = p.V;
  bool here = false;
  if (lane < kJoinTiles && from > 0 && from < p.T) {
    key = p.keys[from];
    here = key < p.V && p.keys[from - 1] == key && !(to < p.T && p.keys[to - 1] == key && p.keys[to] == key);
  }
  for (uint64_t todo = __ballot(here); todo; todo &= todo - 1) {
    const int at = __ffsll((unsigned long long)todo) - 1, v = __builtin_amdgcn_readlane(key, at), tile = tile0 + at;
    // the tile that the token begins in: the last one that does not begin in the middle of it, as `tile` does
    const int begin = tile - equal_before(tile, [&](int t) { return t > 0 && p.keys[(int64_t)t * p.tile - 1] == v; }) - 1;
    const int n = tile - begin + 1, lo = (int)((int64_t)n * wave / kJoinParts), hi = (int)((int64_t)n * (wave + 1) / kJoinParts);
    double sum[4] = {};
#pragma unroll 8
    for (int i = lo; i < hi; ++i) {
      const Piece<4> x = load_piece<4, FORM>(p.partials + ((int64_t)(begin + i) * 2 + (i == 0)) * p.d, c, p.d);
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[e] += (double)x.v[e];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) parts[wave][e][lane] = sum[e];
    __syncthreads();
    if (wave == 0) {
      Piece<4> x;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        double all = parts[0][e][lane];
#pragma unroll
        for (int w = 1; w < kJoinParts; ++w) all += parts[w][e][lane];
        x.v[e] = (float)all;
      }
      put_row<FORM>(p, v, c, x);
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------------------------------------------- gradient: few tokens
constexpr int kFewTokens = 8192, kRankTokens = 8, kRankParts = 256 / kRankTokens;

// Sorting without passes: a token's place is the number of those with smaller ids, and of earlier ones with its own.  A workgroup finds the
// places of eight tokens, each among 32 parts of all (32 tokens and 8 parts, 16 and 16, 8 and 32, of 4096: 14.8 / 10.7 / 9.0 us, of 1501 7.2 / 5.9 / 5.2).  The
// workgroups behind clear dE; the LDS of the others' tokens lets four of them run on a compute unit.
__global__ __launch_bounds__(256) void k_embed_rank(const EmbedSumArgs p, const int32_t* __restrict__ tokens, int32_t* keys, int32_t* places,
                                                    int* status, int sorters) {
  if ((int)blockIdx.x >= sorters || blockIdx.y > 0) {
    clear_piece(p.dE, (int64_t)p.V * p.d, (int64_t)blockIdx.y * gridDim.x + blockIdx.x - sorters);
    return;
  }
  __shared__ int4 all4[kFewTokens / 4];
  __shared__ int ranks[kRankParts][kRankTokens];
  __shared__ int outside;
  int* all = (int*)all4;
  const int T = (int)p.T, padded = (T + 255) / 256 * 256;
  if (threadIdx.x == 0) outside = 0;
  __syncthreads();
#pragma unroll 8
  for (int t = threadIdx.x * 4; t < padded; t += 1024) {
    int4 k = {-1, -1, -1, -1};
    if (t + 4 <= T) {
      __builtin_memcpy(&k, tokens + t, 16);
    } else {
      if (t < T) k.x = tokens[t];
      if (t + 1 < T) k.y = tokens[t + 1];
      if (t + 2 < T) k.z = tokens[t + 2];
    }
    const auto key = [&](int v, int at) {
      if (at >= T) return INT32_MAX;                       // smaller than no id
      if (v >= 0 && v < p.V) return v;
      outside = 1;
      return p.V;
    };
    all4[t / 4] = int4{key(k.x, t), key(k.y, t + 1), key(k.z, t + 2), key(k.w, t + 3)};
  }
  __syncthreads();
  const int t0 = blockIdx.x * kRankTokens, t = t0 + threadIdx.x % kRankTokens, part = threadIdx.x / kRankTokens;
  const int mine = t < T ? all[t] : 0;
  int rank = 0;
  // ids up to and with its own among tokens before, smaller ones among those behind
  const auto count = [&](int from, int to, auto before) {
#pragma unroll 8
    for (int j = from; j < to; ++j) {
      const int4 k = all4[j];
      rank += (k.x < mine + before(4 * j)) + (k.y < mine + before(4 * j + 1)) + (k.z < mine + before(4 * j + 2)) + (k.w < mine + before(4 * j + 3));
    }
  };
  const int each = padded / 4 / kRankParts, from = part * each, to = from + each, own = t0 / 4, behind = own + kRankTokens / 4;
  count(from, min(to, own), [](int) { return 1; });
  count(max(from, own), min(to, behind), [&](int j) { return j < t ? 1 : 0; });
  count(max(from, behind), to, [](int) { return 0; });
  ranks[part][threadIdx.x % kRankTokens] = rank;
  __syncthreads();
  if (part == 0 && t < T) {
#pragma unroll
    for (int i = 1; i < kRankParts; ++i) rank += ranks[i][threadIdx.x];
    keys[rank] = mine;
    places[rank] = t;
  }
  if (blockIdx.x == 0 && threadIdx.x < kStatusWords) status[threadIdx.x] = threadIdx.x == 0 && outside ? kErrTokenRange : 0;
}

// Sums of the sorted rows: a workgroup has 32 of them and 256 channels, each wavefront the tokens that begin among a few; one that goes on
// behind the 32 is shared by the wavefronts, equal parts of its rows each, which are added in their order.  Eight wavefronts / four: 4096 tokens, d = 64,
// V = 1000 17.7 / 22.3 us for the whole call.
constexpr int kRunWaves = 8, kRunRows = 32 / kRunWaves;

template <class T, Form FORM>
__global__ __launch_bounds__(64 * kRunWaves) void k_embed_runs(const EmbedSumArgs p) {
  __shared__ Piece<4> parts[kRunWaves][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = (blockIdx.y * 64 + lane) * 4;
  const int from = blockIdx.x * 32, n = (int)p.T - from < 32 ? (int)p.T - from : 32;
  const int key = lane < n ? p.keys[from + lane] : -1, place = lane < n ? p.places[from + lane] : 0;
  const int before = from + lane > 0 && lane < n ? p.keys[from + lane - 1] : -1;
  const int behind = from + n < p.T ? p.keys[from + n] : -1;
  const uint64_t begins = __ballot(lane < n && key != before);
  const bool on = behind >= 0 && behind == __builtin_amdgcn_readlane(key, n - 1);
  const int last = begins ? 63 - __clzll(begins) : n;          // the last token that begins here
  const uint64_t ours = begins & (((uint64_t)1 << kRunRows) - 1) << (kRunRows * wave), after = begins >> (kRunRows * wave) >> kRunRows;
  // from the first token that begins here to the end of the last one that does not go on behind the 32
  int i = ours ? __ffsll((unsigned long long)ours) - 1 : n, end = after ? kRunRows * (wave + 1) - 1 + __ffsll((unsigned long long)after) : on ? last : n;
  Piece<4> sum = {};
  while (i < end) {
    Piece<4> x[kEmbedRows] = {};
#pragma unroll
    for (int u = 0; u < kEmbedRows; ++u)
      x[u] = load_piece<4, FORM>(p.dout.row<T>(__builtin_amdgcn_readlane(place, min(i + u, end - 1))), c, p.d);
#pragma unroll
    for (int u = 0; u < kEmbedRows; ++u) {
      if (i + u >= end) break;
#pragma unroll
      for (int e = 0; e < 4; ++e) sum.v[e] += x[u].v[e];
      if (i + u + 1 < n && !((begins >> (i + u + 1)) & 1)) continue;
      const int v = __builtin_amdgcn_readlane(key, i + u);
      if (v < p.V) put_row<FORM>(p, v, c, sum);
      sum = Piece<4>{};
    }
    i += kEmbedRows;
  }
  if (!begins || !on || __builtin_amdgcn_readlane(key, last) >= p.V) return;
  const int v = __builtin_amdgcn_readlane(key, last);
  // its last position and one
  end = from + n + equal_before(0, [&](int i) { return from + n - i <= p.T && p.keys[from + n - i - 1] == v; });
  const int begin = from + last, rows = end - begin, lo = begin + rows * wave / kRunWaves, hi = begin + rows * (wave + 1) / kRunWaves;
  sum = Piece<4>{};
  for (int base = lo; base < hi; base += 64) {
    const int at = base + lane < hi ? p.places[base + lane] : 0, here = hi - base < 64 ? hi - base : 64;
    for (int i = 0; i < here; i += kEmbedRows) add_rows<T, kEmbedRows, FORM>(p, sum, at, i, here - i, c);
  }
  parts[wave][lane] = sum;
  __syncthreads();
  if (wave > 0) return;
#pragma unroll
  for (int w = 1; w < kRunWaves; ++w)
#pragma unroll
    for (int e = 0; e < 4; ++e) sum.v[e] += parts[w][lane].v[e];
  put_row<FORM>(p, v, c, sum);
}

}  // namespace oapl
