// C ABI of the policy's attention: argument checks, workspace plans, launches.  Part of the translation unit of oapl_api.hip.
#pragma once

#include "attention.hip.h"
#include "norm_rope.hip.h"

namespace oapl {

constexpr int64_t kMaxRowBytes = (int64_t)1 << 24;   // between tokens: 64 of them stay within 32-bit offsets
constexpr int64_t kMaxTileRows = ((int64_t)1 << 31) - 1024;

static inline size_t esize(int dtype) { return dtype == OAPL_BF16 ? 2 : 4; }

// A heads argument of n tokens and `heads` heads: 16-byte rows that an offset of 32 bits spans 64 of.  `written` rows must not overlap.
static int check_heads(const oapl_heads* x, int64_t n, int heads, int D, int dtype, bool written) {
  if (!x) return OAPL_ERR_NULL;
  if (n == 0) return OAPL_OK;
  if (!x->data) return OAPL_ERR_NULL;
  const int64_t size = (int64_t)esize(dtype), least = written ? D : 0;
  if (n > 1 && (x->token_stride < least || x->token_stride > kMaxRowBytes / size)) return OAPL_ERR_SHAPE;
  if (heads > 1 && (x->head_stride < least || x->head_stride > ((int64_t)1 << 48))) return OAPL_ERR_SHAPE;
  if ((uintptr_t)x->data % 16 || (n > 1 && x->token_stride * size % 16) || (heads > 1 && x->head_stride * size % 16))
    return OAPL_ERR_ALIGN;
  return OAPL_OK;
}

// The operand that check_heads has accepted.  The stride of a single token or head was not looked at, and nothing is multiplied by it.
static Heads heads_of(const oapl_heads* x, int64_t n, int heads, int dtype) {
  if (!x || n == 0) return Heads{nullptr, 0, 0};
  const int64_t size = (int64_t)esize(dtype);
  return Heads{(char*)x->data, n > 1 ? x->token_stride * size : 0, heads > 1 ? x->head_stride * size : 0};
}

static bool head_counts_ok(int hq, int hk, int D) {
  return hk >= 1 && hq >= hk && hq % hk == 0 && hq <= 65536 && D >= 8 && D <= kMaxHeadDim && D % 8 == 0;
}

static bool workspace_ok(const void* ws, size_t have, size_t need) { return ws && (uintptr_t)ws % 256 == 0 && have >= need; }

// ---------------------------------------------------------------------------------------------------------------- norm, rotation
// Wavefronts that share a token: as many as its heads occupy (four at a time) while tokens alone do not fill the chip.
static int rope_parts(int64_t T, int heads) {
  int64_t parts = 4096 / (T > 0 ? T : 1);
  const int most = (heads + 3) / 4;
  return (int)(parts < 1 ? 1 : parts > most ? most : parts);
}

// Forward: four wavefronts a workgroup, in as many dimensions as it takes: HIP takes fewer than 2^32 threads in one.
static dim3 rope_fwd_grid(int64_t T, int parts) {
  const int64_t n = (T * parts + 3) / 4, most = 1 << 22;
  return n <= most ? dim3((unsigned)n) : dim3((unsigned)most, (unsigned)((n + most - 1) / most));
}

// Workgroups that walk over the tokens backwards, each with sums of the gains' gradients of its own: three a compute unit.  The batch of
// kRopeHeads in 512 / 768 / 1024 / 1536: 124 / 105 / 108 / 113 us (504 MB: 4.8 TB/s, the card's copy 5.1).
static unsigned rope_bwd_grid(int64_t T, int heads) {
  const int64_t n = (T * rope_parts(T, heads) + 3) / 4;
  return (unsigned)(n < 768 ? n : 768);
}

static int rope_args(NormRopeArgs& a, const oapl_heads* q, const oapl_heads* k, const int32_t* positions, const float* cos_sin,
                     const void* q_gain, const void* k_gain, int64_t T, int hq, int hk, int D, int rot, int64_t n_pos, int dtype,
                     float eps) {
  if (dtype != OAPL_F32 && dtype != OAPL_BF16) return OAPL_ERR_DTYPE;
  if (T < 0 || T > kMaxTileRows || hq < 1 || hk < 1 || hq > 65536 || hk > 65536 || D < 8 || D > kMaxHeadDim || D % 8 || rot < 0 ||
      rot > D || rot % 8 || n_pos < 0)
    return OAPL_ERR_SHAPE;
  if (!(eps >= 0.f) || !isfinite(eps)) return OAPL_ERR_BETA;
  if ((q_gain == nullptr) != (k_gain == nullptr)) return OAPL_ERR_NULL;
  if (T > 0 && (!positions || (rot > 0 && n_pos > 0 && !cos_sin))) return OAPL_ERR_NULL;
  if (int rc = check_heads(q, T, hq, D, dtype, false)) return rc;
  if (int rc = check_heads(k, T, hk, D, dtype, false)) return rc;
  if ((uintptr_t)cos_sin % 16 || (uintptr_t)q_gain % 16 || (uintptr_t)k_gain % 16) return OAPL_ERR_ALIGN;
  a = NormRopeArgs{};
  a.q = heads_of(q, T, hq, dtype), a.k = heads_of(k, T, hk, dtype);
  a.positions = positions, a.cos_sin = cos_sin, a.q_gain = q_gain, a.k_gain = k_gain;
  a.T = T, a.n_pos = n_pos, a.hq = hq, a.hk = hk, a.D = D, a.rot = rot, a.eps = eps;
  return OAPL_OK;
}

// ---------------------------------------------------------------------------------------------------------------- attention
// What a call of average sequences is cut into; nothing more is known here of them.  Microseconds below: equal lengths, causal, bf16 and 128
// channels where nothing else is said, as replayed graphs on one MI355X; of backward, both kernels together with the other one's cut fixed.
struct AttnPlan {
  bool few = false, few_dq = false, few_dkdv = false;      // tiles of 32 rows (keys) whose wavefronts share the steps
  bool two = false, two_dq = false, two_dkdv = false;      // tiles of 64 rows (keys) whose wavefronts share each step's keys (rows)
  int fwd = 1, dq = 1, dkdv = 1;       // workgroups that share a tile's steps
  size_t off_lse2 = 0, off_delta = 0, off_sums = 0, off_partials = 0, total = 0;
};

// At most `want` workgroups in all, with at least `least` steps each.
static int attn_splits(int64_t want, int64_t steps, int64_t least) {
  return (int)std::max<int64_t>(1, std::min<int64_t>({want, steps / least, 64}));
}

static void attn_cut(AttnPlan& p, int64_t Tq, int64_t Tk, int n_seq, int g, int hk, int D, bool f32, bool causal) {
  const int64_t seqs = std::max(n_seq, 1), rows = Tq * g;
  const auto tiles = [&](int64_t n, int64_t b) { return std::max<int64_t>(1, (n + seqs * b - 1) / (seqs * b)) * seqs * hk; };
  // Forward: tiles of 32 rows for few rows, and where they are one round of workgroups (up to 133 KB of LDS: one a compute unit, of 64 channels
  // two) however many; two rounds where walks are long and end apart.  32 / 64 / 128 rows a tile: 300 tokens, 32 on 8 (304 small tiles of 9 steps)
  // 15 / 13 / 16; 1200, 8 heads (304 of 37) 18 / 25 / 39, without a mask 30 / 25; 2 of 500, 16 on 8 (512 of 15) 19 / 17 / 22; 1000, 16 on 8 (504 of 31) 23 / 24 / 35; 1000, 32 on 8
  // (1000) 41 / 26 / 35.  64 channels: 300, 32 on 8 (304) 8 / 10 / 12; 2 of 500, 16 on 8 (512) 10 / 13 / 17; 600, 32 on 8 (600) 15 / 14 / 18; 8 of 200, 16
  // on 8 (832) 14 / 10 / 11.  Equal walks, each at its best split, 32 / 128: 16 sequences of 64 rows over 2000 keys, 8 key heads (256) 29 / 34, of 96
  // rows (384) 52 / 38.
  // fp32 products take nine times as long, and what small tiles cost is hidden behind them for longer: 80 channels, 4 of 400 tokens, 6 on 2
  // (304) 25 / 50; 64 channels, 2 of 1000, 16 on 8 (1008) 57 / 85; 4 of 2000, 8 on 2 (2000) 354 / 381; 4 of 4000, 8 heads (4000) 1252 / 1111.
  const int64_t t32 = tiles(rows, 32), t64 = tiles(rows, 64), t128 = tiles(rows, 128), steps = Tk / seqs / 32;
  p.few = rows <= seqs * 32 || t32 <= (f32 ? 2048 : D <= 64 ? 512 : 256) || (causal && t32 <= 512 && steps >= 30 && 2 * Tq > Tk);
  // ... in parts of the keys.  Small tiles, parts that fill the round: one token over 4096 / 32768 keys, 8 key heads, 1 part 35 / 236, 8
  // parts 13 / 40, 16 parts 12 / 31; 8 over 32768, 1 part 389, 4 189, 8 199; 24 over 4096 (192 tiles), 1 part 83, 2 94.  Short parts cost more
  // to put together than they save: 4 x 32 rows over 2000 keys, 4 parts 16, 8 parts (of two steps) 19.
  // Large ones where few tiles have long walks: 8000 tokens, 4 heads on one (250 tiles of 250 steps), 1 part 217, 4 90; 1000 tokens, 32 on 8
  // (256 of 31), 1 part 35.5, 2 37.5.
  p.fwd = p.few ? attn_splits(256 / t32, steps / 4, 3) : attn_splits(1024 / t128, steps, 32);
  // Tiles of 64 rows halve a walk: where they are one round (two workgroups a compute unit) or large ones few, of long walks, and their keys are
  // not split.  64 / 128 rows: 600 tokens, 32 on 8 (304 tiles of 64 rows) 19 / 24; 1000 (504) 26 / 36; 1500 (752 of 46 steps) 40 / 51; 2500 (1256)
  // 85 / 81; 4 of 300 (608 of 9) 24 / 18; 4 of 1000, 16 on 8 (1008) 43 / 40; 64 of 30, 8 heads (512 of either size) 12 / 9.  64 channels: 13 of up to
  // 400, 14 on 2 (572 large ones) 12 / 15; 2500, 32 on 8 (632) 46 / 57; 64 of 60, 8 heads (512) 8.9 / 9.3; 4000, 32 on 8 (1000) 95 / 95.
  p.two = !f32 && !p.few && p.fwd == 1 && (D <= 64 ? t128 <= 768 : (t64 <= 512 && t64 > t128) || (t128 <= 400 && steps >= 24));
  // dq: tiles of 32 rows up to two rounds.  32 rows / 128 rows, each at its best split: 64 channels, 1000 tokens, 6 heads (192 small tiles)
  // 48 / 55; 1200, 8 heads (304) 46 / 52; 300, 32 on 8 (304) 79 / 78; 4 of 1000, 4 on one (500) 187 / 193; 4800, 8 on 2 (1200) 278 / 241;
  // 1000, 32 on 8 (1000) 213 / 199.  fp32, the other kernel by the rules: 80 channels, 4 of 400, 6 on 2 (304) 85 / 91; 64 channels, 2 of 1000, 16 on 8
  // (1008) 187 / 204; 8 of 600, 8 on 2 (1200) 491 / 444.
  p.few_dq = t32 <= (f32 ? 1024 : 512);
  // ... in parts of the keys.  Small tiles: 16 rows over 4096 keys (2 of 32 steps), 1 part 50, 4 30, 8 25; 64 rows over 1024 (8 of 8), 1
  // part 28, 2 27; 2000 tokens, one head (63 of 15), 1 part 57, 2 52; 192 of 7, 1 part 48, 2 51.  Large ones: 9000, 4 on one (282 of 140), 1
  // part 456, 2 373, 3 355; 1000, 32 on 8 (256 of 15), 1 part 199, 2 200; 2500, 32 on 8 (632 of 39), 1 part 460, 2 491.
  p.dq = p.few_dq ? attn_splits(256 / t32, steps / 4, 4) : attn_splits(900 / t128, steps / 2, 24);
  // ... of 64 rows where large ones are few rounds and not cut, as forward.  64 / 128 rows: 600 tokens, 32 on 8 (152 large tiles of 9 steps) 61 / 63;
  // 1000 (256) 89 / 95; 1500 (376) 123 / 130; 2500 (632) 235 / 223; 4 of 300 (320 of 4) 55 / 48.  64 channels: 13 of up to 400, 14 on 2 (572) 44 / 46;
  // 4 of 1000, 16 on 8 (512) 80 / 79, 32 channels 52 / 57; 4000, 32 on 8 (1000) 286 / 286.
  p.two_dq = !f32 && !p.few_dq && p.dq == 1 && t128 <= (D <= 64 ? 640 : 400) && (D <= 64 || steps >= 16);
  // dk, dv: tiles of 32 keys where they are few (a workgroup of 128 channels has a compute unit's LDS for itself, of 64 channels half of it) and
  // their walks, in steps of 64 rows, short; their wavefronts have a SIMD each, which saves time there and costs rate.  32 / 64 / 128 keys, each at
  // its best split: 300 tokens, 32 on 8 (80 small tiles of 18 steps) 39 / 44 / 48; 4 of 300 (320 of 18) 48 / 59 / 64; 1000 (256 of 62) 83 / 78 / 87; 1500
  // (376 of 93) 129 / 119 / 135; 16 of 200, 16 on 8 (896 of 6) 64 / 48 / 54; 4 of 1000, 16 on 8 (1024 of 31) 126 / 102 / 116.  64 channels: 13 of up
  // to 400, 14 on 2 (338 of 43) 37 / 44 / 47; 4 of 1000, 16 on 8 (1024 of 31) 68 / 75 / 78; 64 of up to 120, 8 heads (2048 of one) 32 / 24 / 25.
  // fp32, 32 / 128: 80 channels, 4 of 400, 6 on 2 (104 of 18) 86 / 98; 64 channels, 8 of 1000, 8 heads (2048 of 15) 339 / 356; 4 of 2000, 8 on 2
  // (504 of 125) 1637 / 1578; 96 channels, 8000, 8 on 2 (500 of 500) 3537 / 3360; 4 of 4000, 8 heads (4000 of 62) 6268 / 5790.
  const int64_t small = tiles(Tk, 32), work = small * std::max<int64_t>(1, rows / seqs / 64);
  p.few_dkdv = f32 ? work <= 256 * 128 : D <= 64 ? small <= 1024 && work <= 256 * 128 : small <= 400 && work <= 256 * 64;
  // Tiles of 64 keys halve the longest walks, which end a call of few rounds, and read rows twice as often.  64 / 128 keys, each at its best
  // split: 2500, 32 on 8 (160 large tiles) 226 / 233; 4000, 8 on one (32) 189 / 201; 4000, 32 on 8 (256) 492 / 486; 3 of 2500 (480) 561 / 600;
  // 8192 (512) 1779 / 1766; 12000 (752) 3737 / 3640; 8 of up to 4096 (1072) 1330 / 1267.  64 channels: 2500, 32 on 8 142 / 157; 8 of up to 4096
  // 760 / 799; 2 of 8192, 32 on 8 (1024) 1954 / 1891; 32 channels 1284 / 1266 and 512 / 519.  fp32: 4 of 2000, 8 on 2 (128) 1627 / 1582.
  p.two_dkdv = !f32 && tiles(Tk, 128) <= (D <= 64 ? 1152 : 512);
  // ... in parts of the rows.  32 keys: to fill a round, or two with longer parts: 300 tokens, 4 on one (10 of 18), 1 part 43, 4 34, 8 32; 80 of 18,
  // 1 part 42, 2 39, 4 45; 600, 32 on 8 (152 of 37), 1 part 61, 2 54, 3 57; 1500, 8 on 2 (94 of 93), 1 part 108, 4 64, 8 78; 256 of 62, 1 part
  // 89, 2 83, 3 90; 320 of 18, 1 part 48, 2 70; fp32, 304 of 37, 1 part 453, 2 431, 4 471.  64 keys, two workgroups a compute unit: 2500, 32 on
  // 8 (320 small tiles of 156), 1 part 318, 3 226, 4 242; 1500 (188 of 93), 1 part 189, 3 119, 4 123; 4000, 8 on one (63 of 500), 1 part 776, 8
  // 198, 16 189; 3 of 2500 (960 of 156), 1 part 561, 2 622; 4 of 1000, 16 on 8 (512 of 31), 1 part 102, 2 121.  128 keys in fp32: 4 of 2000, 8 on 2 (128
  // of 125), 1 part 3126, 4 1581, 8 1626.
  p.dkdv = p.few_dkdv   ? std::max(attn_splits((f32 ? 512 : 256) / small, rows / seqs / 128, 1), attn_splits(512 / small, rows / seqs / 128, 4))
           : p.two_dkdv ? attn_splits(1024 / tiles(Tk, 64), rows / seqs / 64, 24)
                        : attn_splits((511 + tiles(Tk, 128)) / tiles(Tk, 128), rows / seqs / 64, 4);
}

// A launch of so many tiles in so many parts has fewer than 2^32 threads, which is what HIP takes in a dimension of a grid.
static bool attn_launches(const AttnPlan& p, int64_t rows, int64_t Tk, int n_seq, int hk, bool bwd) {
  const auto fits = [&](int64_t n, bool few, bool two, int parts) {
    const int64_t tiles = few ? tile_ids<32>(n, n_seq) : two ? tile_ids<64>(n, n_seq) : tile_ids<128>(n, n_seq);
    return tiles * hk * parts < (int64_t)1 << 24;
  };
  return bwd ? fits(rows, p.few_dq, p.two_dq, p.dq) && fits(Tk, p.few_dkdv, p.two_dkdv, p.dkdv) : fits(rows, p.few, p.two, p.fwd);
}

static bool attn_plan(AttnPlan& p, int64_t Tq, int64_t Tk, int n_seq, int hq, int hk, int D, int dtype, bool causal, bool bwd) {
  if (dtype != OAPL_F32 && dtype != OAPL_BF16) return false;
  if (!head_counts_ok(hq, hk, D) || Tq < 0 || Tk < 0 || n_seq < 0 || (n_seq == 0 && (Tq || Tk)) || Tk > kMaxTileRows ||
      Tq > kMaxTileRows / hq || n_seq > (1 << 24))
    return false;
  const int g = hq / hk;
  attn_cut(p, Tq, Tk, n_seq, g, hk, D, dtype == OAPL_F32, causal);
  if (!attn_launches(p, Tq * g, Tk, n_seq, hk, bwd)) return false;
  size_t at = kStatusWords * sizeof(int);
  const auto take = [&](int64_t floats) {
    const size_t was = at;
    at += (size_t)round_up(floats * (int64_t)sizeof(float), 256);
    return was;
  };
  if (bwd) {
    p.off_lse2 = take(Tq * hq), p.off_delta = take(Tq * hq);
    p.off_partials = take(std::max(p.dq > 1 ? p.dq * Tq * hq * D : 0, p.dkdv > 1 ? p.dkdv * 2 * Tk * hk * D : 0));
  } else if (p.fwd > 1) {
    p.off_sums = take(2 * p.fwd * Tq * hq), p.off_partials = take(p.fwd * Tq * hq * D);
  }
  p.total = at;
  return true;
}

static int attn_args(AttnArgs& a, const oapl_heads* q, const oapl_heads* k, const oapl_heads* v, const int64_t* q_offsets,
                     const int64_t* k_offsets, int64_t Tq, int64_t Tk, int n_seq, int hq, int hk, int D, int dtype, int causal,
                     float scale) {
  if (!isfinite(scale * kLog2e)) return OAPL_ERR_BETA;      // what the kernels multiply by
  if (n_seq > 0 && (!q_offsets || !k_offsets)) return OAPL_ERR_NULL;
  if (int rc = check_heads(q, Tq, hq, D, dtype, false)) return rc;
  if (int rc = check_heads(k, Tk, hk, D, dtype, false)) return rc;
  if (int rc = check_heads(v, Tk, hk, D, dtype, false)) return rc;
  a = AttnArgs{};
  a.q = heads_of(q, Tq, hq, dtype), a.k = heads_of(k, Tk, hk, dtype), a.v = heads_of(v, Tk, hk, dtype);
  a.q_offsets = q_offsets, a.k_offsets = k_offsets;
  a.Tq = Tq, a.Tk = Tk, a.n_seq = n_seq, a.hq = hq, a.hk = hk, a.g = hq / hk, a.D = D, a.causal = causal != 0, a.scale = scale;
  // floor(2^(31 + s) / g) + 1 with 2^s >= g: exact for numbers below 2^31
  int s = 0;
  while ((1 << s) < a.g) ++s;
  a.g_shift = 31 + s;
  a.g_mul = (uint32_t)((((uint64_t)1 << a.g_shift) / (uint64_t)a.g) + 1);
  return OAPL_OK;
}

// Heads of up to 32, 64, 96 and 128 channels have kernels of their own; channels behind D are zeros.
template <class T, class F>
static int by_width(int D, F&& launch) {
  if (D <= 32) return launch((T*)nullptr, std::integral_constant<int, 32>{});
  if (D <= 64) return launch((T*)nullptr, std::integral_constant<int, 64>{});
  if (D <= 96) return launch((T*)nullptr, std::integral_constant<int, 96>{});
  return launch((T*)nullptr, std::integral_constant<int, 128>{});
}
template <class F>
static int by_type(int dtype, int D, F&& launch) {
  return dtype == OAPL_BF16 ? by_width<bf16_t>(D, launch) : by_width<float>(D, launch);
}

template <auto kernel, int lds>
static int launch_attn(int64_t tiles, const AttnArgs& a, hipStream_t st) {
  static const bool ready = allow_big_lds(kernel, lds);
  if (!ready) return OAPL_ERR_HIP;
  kernel<<<(unsigned)(tiles * a.splits), 256, lds, st>>>(a);
  OAPL_LAUNCH_CHECK();
  return OAPL_OK;
}

// What goes before either pass: the status of no sequences (nothing else is launched), the offsets of many.
static int launch_attn_begin(const AttnArgs& a, hipStream_t st) {
  if (a.n_seq == 0) k_fill_i32<<<1, 64, 0, st>>>(a.status, kStatusWords, 0);
  else if (a.n_seq > kLookedAt) k_attn_check<<<1, 1024, 0, st>>>(a);
  else return OAPL_OK;
  OAPL_LAUNCH_CHECK();
  return OAPL_OK;
}

template <class T, int DW>
static int launch_attn_fwd(AttnArgs a, const AttnPlan& p, hipStream_t st) {
  a.splits = p.fwd;
  const int64_t rows = a.Tq * a.g;
  constexpr int DP = padded(DW);
  const auto fwd = [&](auto wk) {
    constexpr int WK = wk, B = 128 / WK;
    return launch_attn<k_attn_fwd<T, DW, WK>, KeyLds<T, DP, WK, fwd_keys<WK>>::kBytes>(tile_ids<B>(rows, a.n_seq) * a.hk, a, st);
  };
  int rc;
  if constexpr (sizeof(T) == 2) {
    rc = p.few ? fwd(std::integral_constant<int, 4>{}) : p.two ? fwd(std::integral_constant<int, 2>{}) : fwd(std::integral_constant<int, 1>{});
  } else {
    rc = p.few ? fwd(std::integral_constant<int, 4>{}) : fwd(std::integral_constant<int, 1>{});
  }
  if (rc != OAPL_OK || p.fwd == 1 || a.Tq == 0) return rc;
  k_attn_join<T><<<grid1d(a.Tq * a.hq, 8), 256, 0, st>>>(a);
  OAPL_LAUNCH_CHECK();
  return OAPL_OK;
}

template <class T, int DW>
static int launch_attn_bwd(AttnArgs a, const AttnPlan& p, hipStream_t st) {
  constexpr int DP = padded(DW);
  a.splits = p.dq;
  const int64_t rows = a.Tq * a.g;
  const auto dq = [&](auto wk) {
    constexpr int WK = wk, B = 128 / WK;
    return launch_attn<k_attn_dq<T, DW, WK>, KeyLds<T, DP, WK, dq_keys<WK>>::kBytes>(tile_ids<B>(rows, a.n_seq) * a.hk, a, st);
  };
  int rc;
  if constexpr (sizeof(T) == 2) {
    rc = p.few_dq ? dq(std::integral_constant<int, 4>{}) : p.two_dq ? dq(std::integral_constant<int, 2>{}) : dq(std::integral_constant<int, 1>{});
  } else {
    rc = p.few_dq ? dq(std::integral_constant<int, 4>{}) : dq(std::integral_constant<int, 1>{});
  }
  if (rc != OAPL_OK) return rc;
  if (p.dq > 1 && a.Tq > 0) {
    const GradSum sum{a.dq, a.partials, a.scale};
    k_attn_add<T><<<grid1d(a.Tq * a.hq, 8), 256, 0, st>>>(a, sum, sum, a.Tq * a.hq * a.D, a.Tq, a.g);
    OAPL_LAUNCH_CHECK();
  }
  a.splits = p.dkdv;
  const auto dkdv = [&](auto wk) {
    constexpr int WK = wk, B = 128 / WK;
    return launch_attn<k_attn_dkdv<T, DW, WK>, RowLds<T, DP, WK>::kBytes>(tile_ids<B>(a.Tk, a.n_seq) * a.hk, a, st);
  };
  if constexpr (sizeof(T) == 2) {
    rc = p.few_dkdv ? dkdv(std::integral_constant<int, 4>{}) : p.two_dkdv ? dkdv(std::integral_constant<int, 2>{}) : dkdv(std::integral_constant<int, 1>{});
  } else {
    rc = p.few_dkdv ? dkdv(std::integral_constant<int, 4>{}) : dkdv(std::integral_constant<int, 1>{});
  }
  if (rc != OAPL_OK) return rc;
  if (p.dkdv > 1 && a.Tk > 0) {
    const int64_t one = a.Tk * a.hk * a.D;
    const GradSum dk{a.dk, a.partials, a.scale}, dv{a.dv, a.partials + one, 1.f};
    k_attn_add<T><<<dim3(grid1d(a.Tk * a.hk, 8), 2), 256, 0, st>>>(a, dk, dv, 2 * one, a.Tk, 1);
    OAPL_LAUNCH_CHECK();
  }
  return OAPL_OK;
}

}  // namespace oapl

using namespace oapl;

extern "C" {

int32_t oapl_qk_norm_rope_fwd(const oapl_heads* q, const oapl_heads* k, const oapl_heads* v, const int32_t* positions,
                              const float* cos_sin, const void* q_gain, const void* k_gain, const int64_t* rows, int64_t T,
                              int32_t n_q_heads, int32_t n_k_heads, int32_t head_dim, int32_t rot_dim, int64_t n_positions,
                              int64_t n_rows, int32_t dtype, float eps, const oapl_heads* q_out, const oapl_heads* k_out,
                              const oapl_heads* v_out, void* stream) {
  NormRopeArgs a;
  if (int rc = rope_args(a, q, k, positions, cos_sin, q_gain, k_gain, T, n_q_heads, n_k_heads, head_dim, rot_dim, n_positions,
                         dtype, eps))
    return rc;
  if (rows && n_rows < 0) return OAPL_ERR_SHAPE;
  if ((v == nullptr) != (v_out == nullptr)) return OAPL_ERR_NULL;
  const int64_t out_rows = rows ? n_rows : T;
  if (int rc = check_heads(q_out, T, n_q_heads, head_dim, dtype, true)) return rc;
  if (int rc = check_heads(k_out, out_rows, n_k_heads, head_dim, dtype, true)) return rc;
  if (v) {
    if (int rc = check_heads(v, T, n_k_heads, head_dim, dtype, false)) return rc;
    if (int rc = check_heads(v_out, out_rows, n_k_heads, head_dim, dtype, true)) return rc;
  }
  if (T == 0) return OAPL_OK;
  a.v = heads_of(v, T, n_k_heads, dtype);
  a.q_out = heads_of(q_out, T, n_q_heads, dtype), a.k_out = heads_of(k_out, out_rows, n_k_heads, dtype);
  a.v_out = heads_of(v_out, out_rows, n_k_heads, dtype);
  a.rows = rows, a.n_rows = n_rows;
  a.parts = rope_parts(T, n_q_heads + n_k_heads * (v ? 2 : 1));
  const dim3 grid = rope_fwd_grid(T, a.parts);
  if (dtype == OAPL_BF16) k_qk_norm_rope_fwd<bf16_t><<<grid, 256, 0, (hipStream_t)stream>>>(a);
  else k_qk_norm_rope_fwd<float><<<grid, 256, 0, (hipStream_t)stream>>>(a);
  OAPL_LAUNCH_CHECK();
  return OAPL_OK;
}

size_t oapl_qk_norm_rope_workspace_bytes(int64_t T, int32_t n_q_heads, int32_t n_k_heads, int32_t head_dim) {
  if (T < 0 || T > kMaxTileRows || n_q_heads < 1 || n_k_heads < 1 || n_q_heads > 65536 || n_k_heads > 65536 || head_dim < 8 ||
      head_dim > kMaxHeadDim || head_dim % 8)
    return 0;
  return (size_t)round_up((int64_t)rope_bwd_grid(T, n_q_heads + n_k_heads) * 2 * head_dim * (int64_t)sizeof(float) + 1, 256);
}

int32_t oapl_qk_norm_rope_bwd(const oapl_heads* q, const oapl_heads* k, const oapl_heads* dq_out, const oapl_heads* dk_out,
                              const int32_t* positions, const float* cos_sin, const void* q_gain, const void* k_gain, int64_t T,
                              int32_t n_q_heads, int32_t n_k_heads, int32_t head_dim, int32_t rot_dim, int64_t n_positions,
                              int32_t dtype, float eps, const oapl_heads* dq, const oapl_heads* dk, float* dq_gain, float* dk_gain,
                              void* workspace, size_t workspace_bytes, void* stream) {
  NormRopeArgs a;
  if (int rc = rope_args(a, q, k, positions, cos_sin, q_gain, k_gain, T, n_q_heads, n_k_heads, head_dim, rot_dim, n_positions,
                         dtype, eps))
    return rc;
  if (int rc = check_heads(dq_out, T, n_q_heads, head_dim, dtype, false)) return rc;
  if (int rc = check_heads(dk_out, T, n_k_heads, head_dim, dtype, false)) return rc;
  if (int rc = check_heads(dq, T, n_q_heads, head_dim, dtype, true)) return rc;
  if (int rc = check_heads(dk, T, n_k_heads, head_dim, dtype, true)) return rc;
  if (q_gain && (!dq_gain || !dk_gain)) return OAPL_ERR_NULL;
  if (q_gain &&
      !workspace_ok(workspace, workspace_bytes, oapl_qk_norm_rope_workspace_bytes(T, n_q_heads, n_k_heads, head_dim)))
    return OAPL_ERR_WORKSPACE;
  a.q_out = heads_of(dq_out, T, n_q_heads, dtype), a.k_out = heads_of(dk_out, T, n_k_heads, dtype);
  a.dq = heads_of(dq, T, n_q_heads, dtype), a.dk = heads_of(dk, T, n_k_heads, dtype);
  a.partials = q_gain ? (float*)workspace : nullptr;
  a.parts = rope_parts(T, n_q_heads + n_k_heads);
  const unsigned grid = rope_bwd_grid(T, n_q_heads + n_k_heads);
  hipStream_t st = (hipStream_t)stream;
  if (T > 0) {
    if (dtype == OAPL_BF16) k_qk_norm_rope_bwd<bf16_t><<<grid, 256, 0, st>>>(a);
    else k_qk_norm_rope_bwd<float><<<grid, 256, 0, st>>>(a);
    OAPL_LAUNCH_CHECK();
  }
  if (q_gain) {
    k_gain_grads<<<grid1d(2 * head_dim, 16), 1024, 0, st>>>(a.partials, (int)grid, head_dim, dq_gain, dk_gain);
    OAPL_LAUNCH_CHECK();
  }
  return OAPL_OK;
}

size_t oapl_attention_workspace_bytes(int64_t Tq, int64_t Tk, int32_t n_seq, int32_t n_q_heads, int32_t n_k_heads,
                                      int32_t head_dim, int32_t dtype, int32_t with_backward) {
  size_t most = 0;      // of either mask
  for (const bool causal : {false, true}) {
    AttnPlan p;
    if (!attn_plan(p, Tq, Tk, n_seq, n_q_heads, n_k_heads, head_dim, dtype, causal, with_backward != 0)) return 0;
    most = std::max(most, p.total);
  }
  return most;
}

int32_t oapl_attention_fwd(const oapl_heads* q, const oapl_heads* k, const oapl_heads* v, const int64_t* q_offsets,
                           const int64_t* k_offsets, const int64_t* k_used, int64_t Tq, int64_t Tk, int32_t n_seq,
                           int32_t n_q_heads, int32_t n_k_heads, int32_t head_dim, int32_t dtype, int32_t causal, float scale,
                           const oapl_heads* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  if (dtype != OAPL_F32 && dtype != OAPL_BF16) return OAPL_ERR_DTYPE;
  AttnPlan p;
  if (!attn_plan(p, Tq, Tk, n_seq, n_q_heads, n_k_heads, head_dim, dtype, causal != 0, false)) return OAPL_ERR_SHAPE;
  AttnArgs a;
  if (int rc = attn_args(a, q, k, v, q_offsets, k_offsets, Tq, Tk, n_seq, n_q_heads, n_k_heads, head_dim, dtype, causal, scale))
    return rc;
  if (int rc = check_heads(out, Tq, n_q_heads, head_dim, dtype, true)) return rc;
  if (!workspace_ok(workspace, workspace_bytes, p.total)) return OAPL_ERR_WORKSPACE;
  hipStream_t st = (hipStream_t)stream;
  a.o = heads_of(out, Tq, n_q_heads, dtype);
  a.lse = lse;
  a.k_used = k_used;
  a.status = (int*)workspace;
  a.part_sums = (float*)((char*)workspace + p.off_sums);
  a.partials = (float*)((char*)workspace + p.off_partials);
  if (int rc = launch_attn_begin(a, st)) return rc;
  if (n_seq == 0) return OAPL_OK;
  return by_type(dtype, head_dim, [&](auto* t, auto dp) {
    return launch_attn_fwd<std::remove_pointer_t<decltype(t)>, decltype(dp)::value>(a, p, st);
  });
}

int32_t oapl_attention_bwd(const oapl_heads* q, const oapl_heads* k, const oapl_heads* v, const oapl_heads* out, const float* lse,
                           const oapl_heads* dout, const int64_t* q_offsets, const int64_t* k_offsets, int64_t Tq, int64_t Tk,
                           int32_t n_seq, int32_t n_q_heads, int32_t n_k_heads, int32_t head_dim, int32_t dtype, int32_t causal,
                           float scale, const oapl_heads* dq, const oapl_heads* dk, const oapl_heads* dv, void* workspace,
                           size_t workspace_bytes, void* stream) {
  if (dtype != OAPL_F32 && dtype != OAPL_BF16) return OAPL_ERR_DTYPE;
  AttnPlan p;
  if (!attn_plan(p, Tq, Tk, n_seq, n_q_heads, n_k_heads, head_dim, dtype, causal != 0, true)) return OAPL_ERR_SHAPE;
  AttnArgs a;
  if (int rc = attn_args(a, q, k, v, q_offsets, k_offsets, Tq, Tk, n_seq, n_q_heads, n_k_heads, head_dim, dtype, causal, scale))
    return rc;
  if (Tq > 0 && !lse) return OAPL_ERR_NULL;
  if (int rc = check_heads(out, Tq, n_q_heads, head_dim, dtype, false)) return rc;
  if (int rc = check_heads(dout, Tq, n_q_heads, head_dim, dtype, false)) return rc;
  if (int rc = check_heads(dq, Tq, n_q_heads, head_dim, dtype, true)) return rc;
  if (int rc = check_heads(dk, Tk, n_k_heads, head_dim, dtype, true)) return rc;
  if (int rc = check_heads(dv, Tk, n_k_heads, head_dim, dtype, true)) return rc;
  if (!workspace_ok(workspace, workspace_bytes, p.total)) return OAPL_ERR_WORKSPACE;
  hipStream_t st = (hipStream_t)stream;
  a.o = heads_of(out, Tq, n_q_heads, dtype), a.dout = heads_of(dout, Tq, n_q_heads, dtype);
  // RowStager's offsets: 64 tokens and the heads of a group within 31 bits
  if (a.g > 1 && std::max(a.q.head, a.dout.head) > ((int64_t)1 << 30) / (a.g - 1)) return OAPL_ERR_SHAPE;
  a.dq = heads_of(dq, Tq, n_q_heads, dtype), a.dk = heads_of(dk, Tk, n_k_heads, dtype), a.dv = heads_of(dv, Tk, n_k_heads, dtype);
  a.lse = const_cast<float*>(lse);
  a.lse2 = (float*)((char*)workspace + p.off_lse2);
  a.delta = (float*)((char*)workspace + p.off_delta);
  a.partials = (float*)((char*)workspace + p.off_partials);
  a.status = (int*)workspace;
  if (int rc = launch_attn_begin(a, st)) return rc;
  if (n_seq == 0) return OAPL_OK;
  return by_type(dtype, head_dim, [&](auto* t, auto dp) {
    return launch_attn_bwd<std::remove_pointer_t<decltype(t)>, decltype(dp)::value>(a, p, st);
  });
}

}  // extern "C"
