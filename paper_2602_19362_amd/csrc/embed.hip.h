// Embedding lookup with scaling, and its gradient.
//
//   out_t = scale E[tok_t],      dE[v] = scale sum over t with tok_t = v of dout_t
//
// Bound by memory.  The gradient's sums have a fixed order: tokens are sorted by id (stably, so by position among equals), the sorted
// positions cut into tiles of equal length, so that a frequent token is shared by many workgroups; what a tile has of a token that
// reaches over its ends goes into the workspace and is added up by a second launch, tile by tile.
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
};

// A workgroup takes rows of `out` in turn, a lane eight channels at a time.
template <class TE, class T>
__global__ __launch_bounds__(256) void k_embed_fwd(const EmbedArgs p) {
  const int c = (blockIdx.y * 64 + (threadIdx.x & 63)) * 8;
  if (c >= p.d) return;
  for (int64_t t = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); t < p.T; t += (int64_t)gridDim.x * 4) {
    const int32_t v = p.tokens[t];
    Eight x;
    if (v >= 0 && v < p.V) {
      x = load_piece((const TE*)p.E + (int64_t)v * p.d, c, p.d);
#pragma unroll
      for (int e = 0; e < 8; ++e) x.v[e] *= p.scale;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) x.v[e] = quiet_nan();
    }
    store_piece(p.out.row<T>(t), c, p.d, x);
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
  int64_t T;
  int V, bits, blocks;
};

__device__ __forceinline__ int sort_key(const SortArgs& p, int64_t t) {
  const int32_t v = p.tokens[t];
  return v >= 0 && v < p.V ? v : p.V;
}

// First pass's counts; the second's, and `present`, start at zero.
template <int ITEMS>
__global__ __launch_bounds__(kSortThreads) void k_embed_count(const SortArgs p) {
  extern __shared__ int32_t count[];
  const int bins = 1 << p.bits;
  for (int i = threadIdx.x; i < bins; i += kSortThreads) count[i] = 0;
  __syncthreads();
  const int64_t from = (int64_t)blockIdx.x * kSortThreads * ITEMS;
  for (int i = 0; i < ITEMS; ++i) {
    const int64_t t = from + i * kSortThreads + threadIdx.x;
    if (t < p.T) atomicAdd(&count[sort_key(p, t) & (bins - 1)], 1);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < bins; i += kSortThreads) {
    p.counts[0][(int64_t)blockIdx.x * bins + i] = count[i];
    p.counts[1][(int64_t)blockIdx.x * bins + i] = 0;
  }
  for (int64_t i = (int64_t)blockIdx.x * kSortThreads + threadIdx.x; i < p.V; i += (int64_t)gridDim.x * kSortThreads) p.present[i] = 0;
  if (blockIdx.x == 0 && threadIdx.x < kStatusWords) p.status[threadIdx.x] = 0;
}

// Pass 0 reads tokens, pass 1 what pass 0 left.  A key's place: keys of smaller digits, those of its digit in earlier blocks, in earlier
// wavefronts of this block, and before it in its wavefront.
template <int PASS, int ITEMS>
__global__ __launch_bounds__(kSortThreads) void k_embed_place(const SortArgs p) {
  extern __shared__ int32_t lds[];
  const int bins = 1 << p.bits, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  constexpr int WAVES = kSortThreads / 64;
  int32_t* mine = lds;                       // [WAVES][bins]: first a wavefront's counts, then where its keys of a digit begin
  for (int i = threadIdx.x; i < WAVES * bins; i += kSortThreads) mine[i] = 0;
  __syncthreads();
  const int64_t from = ((int64_t)blockIdx.x * WAVES + wave) * 64 * ITEMS;
  int key[ITEMS], rank[ITEMS];
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const int64_t t = from + i * 64 + lane;
    const bool any = t < p.T;
    key[i] = !any ? 0 : PASS == 0 ? sort_key(p, t) : p.keys[0][t];
    const int digit = PASS == 0 ? key[i] & (bins - 1) : key[i] >> p.bits;
    uint64_t same = __ballot(any);
    for (int b = 0; b < p.bits; ++b) {
      const uint64_t set = __ballot((digit >> b) & 1);
      same &= (digit >> b) & 1 ? set : ~set;
    }
    const int before = __popcll(same & (((uint64_t)1 << lane) - 1)), first = any ? __ffsll((unsigned long long)same) - 1 : lane;
    int base = 0;
    if (any && lane == first) base = atomicAdd(&mine[wave * bins + digit], __popcll(same));
    rank[i] = __shfl(base, first, 64) + before;
  }
  __syncthreads();
  // sums over digits, kSortThreads of them at a time
  __shared__ int32_t wave_sums[WAVES];
  int32_t carry = 0;
  for (int b0 = 0; b0 < bins; b0 += kSortThreads) {
    const int b = b0 + threadIdx.x;
    int32_t total = 0, earlier = 0;
    if (b < bins) {
      const int32_t* column = p.counts[PASS] + b;
#pragma unroll 8
      for (int i = 0; i < p.blocks; ++i) {
        const int32_t n = column[(int64_t)i * bins];
        total += n;
        earlier += i < (int)blockIdx.x ? n : 0;
      }
    }
    int32_t up = total;
    for (int o = 1; o < 64; o <<= 1) {
      const int32_t below = __shfl_up(up, o, 64);
      if (lane >= o) up += below;
    }
    if (lane == 63) wave_sums[wave] = up;
    __syncthreads();
    int32_t smaller = carry + up - total, all = 0;
    for (int i = 0; i < WAVES; ++i) {
      smaller += i < wave ? wave_sums[i] : 0;
      all += wave_sums[i];
    }
    carry += all;
    if (b < bins) {
      int32_t at = smaller + earlier;
      for (int w = 0; w < WAVES; ++w) {
        const int32_t n = mine[w * bins + b];
        mine[w * bins + b] = at;
        at += n;
      }
    }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const int64_t t = from + i * 64 + lane;
    if (t >= p.T) continue;
    const int digit = PASS == 0 ? key[i] & (bins - 1) : key[i] >> p.bits;
    const int32_t to = mine[wave * bins + digit] + rank[i];
    p.keys[PASS][to] = key[i];
    p.places[PASS][to] = PASS == 0 ? (int32_t)t : p.places[0][t];
    if constexpr (PASS == 0) {
      atomicAdd(&p.counts[1][(int64_t)(to / (kSortThreads * ITEMS)) * bins + (key[i] >> p.bits)], 1);
      if (key[i] < p.V) p.present[key[i]] = 1;
      else atomicExch(p.status, kErrTokenRange);
    }
  }
}

// ---------------------------------------------------------------------------------------------------------------- gradient: sums
struct EmbedSumArgs {
  Rows dout;
  const int32_t *keys, *places;     // sorted
  const uint8_t* present;           // nullptr: rows of dE without tokens stay as they are
  float *dE, *partials;             // partials [tiles][2][d]: of the token that a tile begins in the middle of, and of the one that it leaves
  int64_t T;
  int d, V, tile, tiles;
  float scale;
  bool add;                         // to what dE holds
};

__device__ __forceinline__ void put_row(const EmbedSumArgs& p, int key, int c, Eight sum) {
  float* row = p.dE + (int64_t)key * p.d;
#pragma unroll
  for (int e = 0; e < 8; ++e) sum.v[e] *= p.scale;
  if (p.add) {
    const Eight old = load_piece(row, c, p.d);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum.v[e] += old.v[e];
  }
  store_piece(row, c, p.d, sum);
}

// Workgroups below p.tiles sum up a tile's rows (blockIdx.y: 2048 channels), the others clear rows without tokens.
template <class T>
__global__ __launch_bounds__(256) void k_embed_sum(const EmbedSumArgs p) {
  const int c = (blockIdx.y * 256 + threadIdx.x) * 8;
  if (c >= p.d) return;
  if ((int)blockIdx.x >= p.tiles) {
    for (int64_t v = blockIdx.x - p.tiles; v < p.V; v += gridDim.x - p.tiles)
      if (!p.present[v]) store_piece(p.dE + v * p.d, c, p.d, Eight{});
    return;
  }
  const int64_t from = (int64_t)blockIdx.x * p.tile, to = from + p.tile < p.T ? from + p.tile : p.T;
  const bool begun = from > 0 && p.keys[from - 1] == p.keys[from], open = to < p.T && p.keys[to] == p.keys[to - 1];
  const int first = p.keys[from], last = p.keys[to - 1];
  Eight sum = {};
  int key = first;
  for (int64_t i = from; i < to; ++i) {
    const Eight x = load_piece(p.dout.row<T>(p.places[i]), c, p.d);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum.v[e] += x.v[e];
    const int next = i + 1 < to ? p.keys[i + 1] : -1;
    if (next == key) continue;
    if (key < p.V) {
      if (begun && key == first) store_piece(p.partials + (int64_t)blockIdx.x * 2 * p.d, c, p.d, sum);
      else if (open && key == last) store_piece(p.partials + ((int64_t)blockIdx.x * 2 + 1) * p.d, c, p.d, sum);
      else put_row(p, key, c, sum);
    }
    sum = Eight{};
    key = next;
  }
}

// Tokens that reach over the ends of tiles: the tile that one ends in adds up what the tiles have of it, in their order, in 64 bits.
__global__ __launch_bounds__(256) void k_embed_join(const EmbedSumArgs p) {
  const int c = blockIdx.y * 256 + threadIdx.x;
  const int64_t tile = blockIdx.x, from = tile * p.tile, to = from + p.tile < p.T ? from + p.tile : p.T;
  if (from == 0 || c >= p.d) return;
  const int key = p.keys[from];
  if (p.keys[from - 1] != key || key >= p.V) return;                                // begins here
  if (to < p.T && p.keys[to - 1] == key && p.keys[to] == key) return;              // ends further on
  int64_t lo = 0, hi = from;                                                       // its first position
  while (lo < hi) {
    const int64_t mid = (lo + hi) / 2;
    if (p.keys[mid] < key) lo = mid + 1;
    else hi = mid;
  }
  const int64_t begin = lo / p.tile;
  double sum = p.partials[(begin * 2 + 1) * p.d + c];
#pragma unroll 8
  for (int64_t i = begin + 1; i <= tile; ++i) sum += p.partials[i * 2 * p.d + c];
  float* at = p.dE + (int64_t)key * p.d + c;
  *at = (float)sum * p.scale + (p.add ? *at : 0.f);
}

}  // namespace oapl
