// C ABI of what lies around the policy's blocks: embedding, residual stream and norms, clipping.  Part of the translation unit of
// oapl_api.hip.
#pragma once

#include <memory>
#include <new>

#include "clip.hip.h"
#include "embed.hip.h"
#include "residual_norm.hip.h"

namespace oapl {

constexpr int64_t kMaxRows = 65535 * 256;              // the head's limit
constexpr int64_t kMaxElements = (int64_t)1 << 42;     // of all tensors of a call: 2^31 chunks
constexpr int kMaxNormWidth = 16384;                   // 1024 lanes with two pieces of a row each

// A rows argument of n rows of d channels.  The stride of a single row is not looked at.  `written` rows must not overlap.
static int check_rows(const oapl_rows* x, int64_t n, int64_t d, bool written) {
  if (!x) return OAPL_ERR_NULL;
  if (n == 0) return OAPL_OK;
  if (!x->data) return OAPL_ERR_NULL;
  if (n > 1 && (x->row_stride < (written ? d : 0) || x->row_stride > ((int64_t)1 << 46) / (n - 1))) return OAPL_ERR_SHAPE;
  return OAPL_OK;
}
static Rows rows_of(const oapl_rows* x, int64_t n, int dtype) {
  if (!x || n == 0) return Rows{nullptr, 0};
  return Rows{(char*)x->data, n > 1 ? x->row_stride * (int64_t)esize(dtype) : 0};
}
static bool dtype_ok(int dtype) { return dtype == OAPL_F32 || dtype == OAPL_BF16; }
// An address that elements of this type may have.
static bool element_aligned(const void* p, int dtype) { return (uintptr_t)p % esize(dtype) == 0; }

// ---------------------------------------------------------------------------------------------------------------- embedding
struct EmbedPlan {
  bool few = false;
  int bits = 1, items = 1, blocks = 1, tile = 1, tiles = 0;
  size_t off_keys[2], off_places[2], off_counts[2], off_present = 0, off_partials = 0, total = 0;
};

static bool embed_sizes_ok(int64_t T, int d, int V) {
  return T >= 0 && T <= kMaxRows && d >= 1 && d <= (1 << 21) && V >= 1 && V <= (1 << 21) && T * d <= (int64_t)1 << 40;
}

static bool embed_plan(EmbedPlan& p, int64_t T, int d, int V) {
  if (!embed_sizes_ok(T, d, V)) return false;
  p.total = kStatusWords * sizeof(int);
  const auto take = [&](int64_t bytes) {
    const size_t was = p.total;
    p.total += (size_t)round_up(bytes, 256);
    return was;
  };
  p.off_keys[1] = take(T * 4), p.off_places[1] = take(T * 4);
  // Counting / sorting, us for the whole call in bf16: d = 64, V = 1000 8000 tokens 24 / 33; d = 512 8000 28 / 34; d = 1024 8000 30 / 36; d = 4096,
  // V = 1544 4000 25 / 40, 6000 34 / 45.  With a token in half of the places, whose rows one workgroup a slice reads: d = 64 4000 37 / 34, 8000 74 / 36;
  // d = 1024 8000 95 / 42; d = 4096 4000 54 / 40, 6000 82 / 44.
  p.few = T <= (d <= 512 ? kFewTokens : kFewTokens / 2);
  if (p.few) return true;
  while (((int64_t)1 << (2 * p.bits)) <= V) ++p.bits;      // ids 0 .. V
  p.items = T <= 128 * kSortThreads * 2 ? 2 : 8;
  p.blocks = (int)std::max<int64_t>(1, (T + (int64_t)kSortThreads * p.items - 1) / (kSortThreads * p.items));
  // By the wavefronts that a row's channels take, all rows together.  16 / 32 / 64 rows a tile, us for the whole call in bf16: d = 4096: V = 1544
  // 10000 tokens 55 / 51 / 51, 20000 82 / 77 / 75, V = 151936 140897 762 / 731 / 723; d = 1024, V = 8192 40000 62 / 59 / 61, 80000 92 / 88 / 87; d = 64,
  // V = 151936 50000 47 / 50 / 54, 140000 67 / 65 / 67, V = 8192 400000 144 / 129 / 125.
  constexpr int64_t small = 1 << 18;
  p.tile = T * ((d + 255) / 256) <= small ? 32 : 64;
  static_assert(kMaxRows / 64 < kMostEqual && small / 32 < kMostEqual && kFewTokens < kMostEqual, "a token's rows and tiles are found by equal_before");
  p.tiles = (int)((T + p.tile - 1) / p.tile);
  p.off_keys[0] = take(T * 4), p.off_places[0] = take(T * 4);
  for (int i = 0; i < 2; ++i) p.off_counts[i] = take(((int64_t)p.blocks << p.bits) * 4);
  p.off_present = take(V);
  p.off_partials = take((int64_t)p.tiles * 2 * d * 4);
  return true;
}

// So many workgroups, and what is missing to whole rows of `most`: HIP takes fewer than 2^32 threads in a dimension.
static dim3 wide_grid(int64_t n, int64_t most) {
  return dim3((unsigned)std::min(n, most), (unsigned)((n + most - 1) / most));
}

// k_embed_sum's: a workgroup for every tile and 1024 channels, which are 2^24 of them and more at the ends of the sizes.  Rows of 2^20, so that
// calls of 2^36 elements of dout have more than one.
static dim3 embed_sum_grid(const EmbedPlan& p, int d) { return wide_grid((int64_t)p.tiles * grid1d(d, 1024), 1 << 20); }

// f(true or false as a type).
template <class F>
static void by_truth(bool x, F f) {
  if (x) f(std::true_type{});
  else f(std::false_type{});
}

// f(how rows of d channels lie in pieces of W, as a type).  NARROW: d may be smaller than W.
template <int W, bool NARROW, class F>
static void by_form(int d, F f) {
  if (d % W == 0) return f(std::integral_constant<Form, kWhole>{});
  if constexpr (NARROW)
    if (d < W) return f(std::integral_constant<Form, kAny>{});
  f(std::integral_constant<Form, kRagged>{});
}

// Accesses of so many bytes go past the caches: the memory-side one holds 256 MiB.
static bool past_caches(int64_t bytes) { return bytes > (int64_t)256 << 20; }

template <class TE, class T>
static int launch_embed_fwd(EmbedArgs a, hipStream_t st) {
  constexpr int W = sizeof(TE) + sizeof(T) == 4 ? 8 : 4;
  const auto launch = [&](auto pieces, auto form, auto once) {
    constexpr int PIECES = pieces;
    constexpr Form FORM = form;
    constexpr bool ONCE = once;
    a.slices = grid1d(a.d, 64 * W * PIECES);
    k_embed_fwd<TE, T, W, PIECES, FORM, ONCE><<<wide_grid((a.T * a.slices + 3) / 4, 1 << 23), 256, 0, st>>>(a);
  };
  by_form<W, true>(a.d, [&](auto form) {
    by_truth(past_caches(a.T * a.d * (int64_t)sizeof(T)), [&](auto once) {
      // 140000 rows of 256 channels in bf16, one piece a wavefront / two: 27 / 35 us; 20000 of 520 9.5 / 9.1
      if (a.d <= 64 * W) launch(std::integral_constant<int, 1>{}, form, once);
      else launch(std::integral_constant<int, 2>{}, form, once);
    });
  });
  OAPL_LAUNCH_CHECK();
  return OAPL_OK;
}

template <int ITEMS>
static int launch_embed_sort(const SortArgs& a, hipStream_t st) {
  const int bins = 1 << a.bits, bytes = (kSortThreads / 64 + 2) * bins * 4;
  if (bytes > 48 * 1024 && (!allow_big_lds(k_embed_place<0, ITEMS>, bytes) || !allow_big_lds(k_embed_place<1, ITEMS>, bytes)))
    return OAPL_ERR_HIP;
  const int64_t all = a.dE && !a.clear_absent ? ((int64_t)a.V * a.d + 1023) / 1024 : 0;
  k_embed_count<<<wide_grid(a.blocks + all, 1 << 23), 256, std::max(bins * 4, kClearLds), st>>>(a);
  OAPL_LAUNCH_CHECK();
  const auto clears = [&](int rows) { return a.dE && a.clear_absent ? (int64_t)grid1d(rows, kSortThreads / 64) * grid1d(a.d, 1024) : 0; };
  k_embed_place<0, ITEMS><<<wide_grid(a.blocks + clears(a.early), 1 << 21), kSortThreads, bytes, st>>>(a);
  OAPL_LAUNCH_CHECK();
  k_embed_place<1, ITEMS><<<wide_grid(a.blocks + clears(a.V - a.early), 1 << 21), kSortThreads, bytes, st>>>(a);
  OAPL_LAUNCH_CHECK();
  return OAPL_OK;
}

// ---------------------------------------------------------------------------------------------------------------- residual stream
// How a row of d channels is held, W in a piece: f(lanes of a row, or 0 for a workgroup's; lanes of a workgroup at most; pieces a lane).  Eight
// channels a lane, 16 where there are no more lanes: 16411 rows of 4096 in bf16 with 8 / 16 / 32 / 64 forward 92 / 97 / 107 / 158 us (workgroups
// that take row after row 101 .. 111), 3000 of 8192 36 / 40 / 47 / 66, 8000 of 4096 in fp32 97 / 102 / 121 / 164.  A workgroup has as many lanes as the
// row has pieces for, in wavefronts: with 1024 lanes, and branches around the loads, 6007 rows of 5120 took 110 us backwards instead of 83 and 51
// forward instead of 45 (the two were not timed apart).
template <int W, class F>
static void by_width(int d, F f) {
  constexpr std::integral_constant<int, 8 / W> eight{};
  constexpr std::integral_constant<int, 0> workgroup{};
  if (d <= 16 * 8) return f(std::integral_constant<int, 16>{}, std::integral_constant<int, 256>{}, eight);
  if (d <= 64 * 8) return f(std::integral_constant<int, 64>{}, std::integral_constant<int, 256>{}, eight);
  if (d <= 512 * 8) return f(workgroup, std::integral_constant<int, 512>{}, eight);
  if (d <= 768 * 8) return f(workgroup, std::integral_constant<int, 768>{}, eight);
  if (d <= 1024 * 8) return f(workgroup, std::integral_constant<int, 1024>{}, eight);
  return f(workgroup, std::integral_constant<int, 1024>{}, std::integral_constant<int, 16 / W>{});
}
// Lanes of a workgroup, and the rows they hold.
static int norm_lanes(int d) { return d <= 512 ? 256 : (int)round_up((d + (d <= 8192 ? 8 : 16) - 1) / (d <= 8192 ? 8 : 16), 64); }
static int norm_rows(int d) { return d <= 128 ? 16 : d <= 512 ? 4 : 1; }
static int64_t norm_workgroups(int64_t T, int d) { return (T + norm_rows(d) - 1) / norm_rows(d); }

// f(null pointer to the residual stream's type, ... to the block's).
template <class F>
static int by_types(int x_dtype, int dtype, F f) {
  if (x_dtype == OAPL_BF16) return f((bf16_t*)nullptr, (bf16_t*)nullptr);
  if (dtype == OAPL_BF16) return f((float*)nullptr, (bf16_t*)nullptr);
  return f((float*)nullptr, (float*)nullptr);
}

// Backwards every workgroup has sums of its own, and as many rows as any other or one more.  Workgroups of 512 / 768 / 1024 lanes a compute unit, 16411 rows in
// bf16: d = 4096 154 / 174 / 165 us, 2048 81 / 87 / 89 (256 lanes: 124), 1024 45.8 / 46.7 / 47.0 (70), 512 23.2 / 23.5 / 23.8 (31).
// Few rows, the kernels alone (calls in a graph), these / as few as leave the most rows of a workgroup as they are / 512 / 256 workgroups, us: d = 768 in fp32 500
// rows 12.1 / 12.1 / 12.1 / 10.8, 900 13.6 / 13.6 / 12.8 / 15.0, 1501 15.5 / 14.8 / 15.2 / 19.2, 2000 16.6 / 17.1 / 17.4 / 22.8, 4000 22.2 / 22.9 / 25.8 / 37.6; bf16 2048 700 rows 13.6 / 13.0 /
// 13.6 / 13.5, 1501 17.1 / 18.2 / 16.8 / 19.3, 4000 27.3 / 27.7 / 26.8 / 35.7, 512 3000 10.5 / 11.4 / 10.4 / 11.2.
static unsigned norm_bwd_grid(int64_t T, int d) {
  return (unsigned)std::min<int64_t>(norm_workgroups(T, d), std::max(256, 256 * 512 / norm_lanes(d)));
}

// In 32 bits a workgroup adds up so many rows one after the other and no more: more tokens are several launches, each with sums of its own, which
// are added in 64 bits.  Equal rows of 129 channels, 8192 of them one after the other: off by up to 2017 roundings.  One launch / several, bf16:
// 300000 tokens, d = 4096 2837 / 2652 us, 600000 5573 / 5282, 2000000, d = 520 3779 / 3739.
constexpr int kNormChain = 1024;
struct NormParts {
  int n;
  int64_t rows;      // of one
};
static NormParts norm_bwd_parts(int64_t T, int d) {
  const int64_t workgroups = norm_workgroups(T, d), at_once = std::max<int64_t>(1, (int64_t)norm_bwd_grid(T, d) * kNormChain);
  const int64_t n = std::max<int64_t>(1, (workgroups + at_once - 1) / at_once);
  return {(int)n, (workgroups + n - 1) / n * norm_rows(d)};
}

static int residual_norm_args(ResidualNormArgs& a, const oapl_rows* x, const oapl_rows* y, const void* y_gain, const oapl_rows* gate,
                              int gate_per_token, const void* gain, int64_t T, int d, int x_dtype, int dtype, float scale, float eps) {
  if (!dtype_ok(x_dtype) || !dtype_ok(dtype) || (x_dtype == OAPL_BF16 && dtype == OAPL_F32)) return OAPL_ERR_DTYPE;
  if (T < 0 || T > kMaxRows || d < 1 || d > kMaxNormWidth) return OAPL_ERR_SHAPE;
  if (!(eps >= 0.f) || !isfinite(eps) || !isfinite(scale)) return OAPL_ERR_BETA;
  if (!y && !gain) return OAPL_ERR_NULL;
  if (!y && (y_gain || gate)) return OAPL_ERR_NULL;
  if (int rc = check_rows(x, T, d, false)) return rc;
  if (int rc = y ? check_rows(y, T, d, false) : OAPL_OK) return rc;
  if (int rc = gate ? check_rows(gate, gate_per_token ? T : 1, d, false) : OAPL_OK) return rc;
  if ((T > 0 && !element_aligned(x->data, x_dtype)) || (y && T > 0 && !element_aligned(y->data, dtype)) ||
      (gate && !element_aligned(gate->data, dtype)) || !element_aligned(gain, dtype) || !element_aligned(y_gain, dtype))
    return OAPL_ERR_ALIGN;
  a = ResidualNormArgs{};
  a.x = rows_of(x, T, x_dtype), a.y = rows_of(y, T, dtype);
  a.gate = rows_of(gate, gate_per_token ? T : 1, dtype);
  a.gain = gain, a.y_gain = y_gain;
  a.T = T, a.d = d, a.scale = scale, a.eps = eps;
  return OAPL_OK;
}

// Rows that a call writes, or gradients that it reads.
static int take_rows(Rows& to, const oapl_rows* x, int64_t T, int d, int dtype, bool written) {
  if (int rc = check_rows(x, T, d, written)) return rc;
  if (T > 0 && !element_aligned(x->data, dtype)) return OAPL_ERR_ALIGN;
  to = rows_of(x, T, dtype);
  return OAPL_OK;
}

// ---------------------------------------------------------------------------------------------------------------- clipping
struct ClipPlan {
  int chunk = 0, launches = 0;
  int64_t elements = 0;
  bool large = false;              // a launch for the norm between
  bool load_once = false, store_once = false;
};

// The tensors' memory: what is written overlaps nothing but what it is the result of.
static int check_overlaps(const oapl_tensor* tensors, int n) {
  struct Span { uintptr_t from, to; bool written; };
  const std::unique_ptr<Span[]> spans(new (std::nothrow) Span[2 * (size_t)n + 1]);
  if (!spans) return OAPL_ERR_HIP;
  Span* end = spans.get();
  for (int i = 0; i < n; ++i) {
    const uintptr_t bytes = (uintptr_t)tensors[i].n * esize(tensors[i].dtype), data = (uintptr_t)tensors[i].data, out = (uintptr_t)tensors[i].out;
    if (bytes == 0) continue;
    *end++ = {out, out + bytes, true};
    if (out != data) *end++ = {data, data + bytes, false};
  }
  std::sort(spans.get(), end, [](const Span& a, const Span& b) { return a.from < b.from; });
  uintptr_t read = 0, written = 0;       // how far what came before reaches
  for (const Span* s = spans.get(); s < end; ++s) {
    if (s->from < written || (s->written && s->from < read)) return OAPL_ERR_SHAPE;
    (s->written ? written : read) = std::max(s->written ? written : read, s->to);
  }
  return OAPL_OK;
}

static int clip_plan(ClipPlan& p, const oapl_tensor* tensors, int n, bool written) {
  if (n < 0 || n > (1 << 20)) return OAPL_ERR_SHAPE;
  if (n > 0 && !tensors) return OAPL_ERR_NULL;
  int64_t read = 0, apart = 0;
  for (int i = 0; i < n; ++i) {
    const oapl_tensor& t = tensors[i];
    if (!dtype_ok(t.dtype)) return OAPL_ERR_DTYPE;
    if (t.n < 0 || t.n > kMaxElements - p.elements) return OAPL_ERR_SHAPE;
    p.elements += t.n;
    read += t.n * (int64_t)esize(t.dtype);
    if (t.out != t.data) apart += t.n * (int64_t)esize(t.dtype);
    if (t.n == 0) continue;
    if (!t.data || (written && !t.out)) return OAPL_ERR_NULL;
    if (!element_aligned(t.data, t.dtype) || (written && !element_aligned(t.out, t.dtype))) return OAPL_ERR_ALIGN;
  }
  // Small sets are a launch for the squares and one for the scaling, whose workgroups all add up the sums; of larger ones a workgroup has one
  // chunk, so that memory sees them in order, and the norm is a launch of its own.  Chunks of 2048 / 4096 / 8192 / 16384 elements: 98 tensors of
  // 6.3 GB 3351 / 3352 / 3412 / 3462 us (workgroups that take chunk after chunk 3906), of 1.9 GB 1347 / 1253 / 1285 / 1316.
  p.large = p.elements > ((int64_t)16 << 20);
  p.chunk = p.large ? 4096 : 2048;
  // What the caches cannot hold goes past them: 6.3 GB 3352 -> 3247 us with loads and stores of the scaling, 3239 with the loads for the squares,
  // 3205 with all; 135 MB into other tensors 191 -> 162 with the stores.
  p.load_once = past_caches(read), p.store_once = past_caches(read + (written ? apart : 0));
  p.launches = (n + kClipTensors - 1) / kClipTensors;
  return OAPL_OK;
}

// One launch for every kClipTensors tensors, the last ones first where `back`: f(arguments).
template <class F>
static int clip_batches(const ClipPlan& p, const oapl_tensor* tensors, int n, bool back, ClipArgs& a, F f) {
  a.chunk = p.chunk;
  for (int k = 0; k < p.launches; ++k) {
    const int batch = back ? p.launches - 1 - k : k, at = batch * kClipTensors;
    a.count = std::min(kClipTensors, n - at);
    a.mine = batch * kClipGrid;
    a.chunks = 0;
    for (int i = 0; i < a.count; ++i) {
      const oapl_tensor& t = tensors[at + i];
      a.t[i] = ClipTensor{t.data, t.out, t.n, a.chunks, t.dtype == OAPL_BF16};
      a.chunks += (uint32_t)((t.n + p.chunk - 1) / p.chunk);
    }
    f(a);
    OAPL_LAUNCH_CHECK();
  }
  return OAPL_OK;
}

static int clip_squares(const ClipPlan& p, const oapl_tensor* tensors, int n, void* workspace, ClipArgs& a, hipStream_t st) {
  a.sum = (double*)workspace;
  // one launch: as many sums as workgroups; more of them: as many each as there may be
  a.sums = p.launches * kClipGrid;
  return clip_batches(p, tensors, n, false, a, [&](ClipArgs& b) {
    if (p.launches == 1) b.sums = (int)std::min<int64_t>(kClipGrid, std::max(b.chunks, 1u));
    const int grid = p.launches == 1 ? b.sums : kClipGrid;
    if (p.load_once) k_grad_squares<true><<<grid, 256, 0, st>>>(b);
    else k_grad_squares<false><<<grid, 256, 0, st>>>(b);
  });
}

}  // namespace oapl

using namespace oapl;

extern "C" {

int32_t oapl_embed_fwd(const void* E, const int32_t* tokens, int64_t T, int32_t d, int32_t V, int32_t dtype, int32_t out_dtype,
                       float scale, const oapl_rows* out, void* stream) {
  if (!dtype_ok(dtype) || !dtype_ok(out_dtype)) return OAPL_ERR_DTYPE;
  if (!embed_sizes_ok(T, d, V)) return OAPL_ERR_SHAPE;
  if (!isfinite(scale)) return OAPL_ERR_BETA;
  if (T > 0 && (!E || !tokens)) return OAPL_ERR_NULL;
  if (!element_aligned(E, dtype) || (uintptr_t)tokens % sizeof(int32_t)) return OAPL_ERR_ALIGN;
  EmbedArgs a{E, tokens, {}, T, d, V, scale};
  if (int rc = take_rows(a.out, out, T, d, out_dtype, true)) return rc;
  if (T == 0) return OAPL_OK;
  hipStream_t st = (hipStream_t)stream;
  if (dtype == OAPL_BF16 && out_dtype == OAPL_BF16) return launch_embed_fwd<bf16_t, bf16_t>(a, st);
  if (dtype == OAPL_BF16) return launch_embed_fwd<bf16_t, float>(a, st);
  if (out_dtype == OAPL_BF16) return launch_embed_fwd<float, bf16_t>(a, st);
  return launch_embed_fwd<float, float>(a, st);
}

size_t oapl_embed_workspace_bytes(int64_t T, int32_t d, int32_t V) {
  EmbedPlan p;
  return embed_plan(p, T, d, V) ? p.total : 0;
}

int32_t oapl_embed_bwd(const oapl_rows* dout, const int32_t* tokens, int64_t T, int32_t d, int32_t V, int32_t dtype, float scale,
                       int32_t accumulate, float* dE, void* workspace, size_t workspace_bytes, void* stream) {
  if (!dtype_ok(dtype)) return OAPL_ERR_DTYPE;
  EmbedPlan p;
  if (!embed_plan(p, T, d, V)) return OAPL_ERR_SHAPE;
  if (!isfinite(scale)) return OAPL_ERR_BETA;
  if (!dE || (T > 0 && !tokens)) return OAPL_ERR_NULL;
  EmbedSumArgs a = {};
  if (int rc = take_rows(a.dout, dout, T, d, dtype, false)) return rc;
  if (!element_aligned(dE, OAPL_F32) || (uintptr_t)tokens % sizeof(int32_t)) return OAPL_ERR_ALIGN;
  if (!workspace_ok(workspace, workspace_bytes, p.total)) return OAPL_ERR_WORKSPACE;
  hipStream_t st = (hipStream_t)stream;
  char* ws = (char*)workspace;
  a.dE = dE, a.T = T, a.d = d, a.V = V, a.scale = scale, a.add = accumulate != 0;
  int32_t* const keys = (int32_t*)(ws + p.off_keys[1]), * const places = (int32_t*)(ws + p.off_places[1]);
  a.keys = keys, a.places = places;
  if (p.few) {
    const int sorters = (int)std::max<int64_t>(1, (T + kRankTokens - 1) / kRankTokens);
    const int64_t clear = accumulate ? 0 : ((int64_t)V * d + 1023) / 1024;
    k_embed_rank<<<wide_grid(sorters + clear, 1 << 23), 256, 0, st>>>(a, tokens, keys, places, (int*)ws, sorters);
    OAPL_LAUNCH_CHECK();
    if (T == 0) return OAPL_OK;
    const dim3 runs(grid1d(T, 32), grid1d(d, 256));
    by_form<4, true>(d, [&](auto form) {
      constexpr Form FORM = form;
      if (dtype == OAPL_BF16) k_embed_runs<bf16_t, FORM><<<runs, 64 * kRunWaves, 0, st>>>(a);
      else k_embed_runs<float, FORM><<<runs, 64 * kRunWaves, 0, st>>>(a);
    });
    OAPL_LAUNCH_CHECK();
    return OAPL_OK;
  }
  SortArgs s = {};
  s.tokens = tokens;
  s.keys[0] = (int32_t*)(ws + p.off_keys[0]), s.places[0] = (int32_t*)(ws + p.off_places[0]);
  s.keys[1] = keys, s.places[1] = places;
  for (int i = 0; i < 2; ++i) s.counts[i] = (int32_t*)(ws + p.off_counts[i]);
  s.present = (uint8_t*)(ws + p.off_present), s.status = (int*)ws;
  s.dE = accumulate ? nullptr : dE;
  s.T = T, s.V = V, s.d = d, s.bits = p.bits, s.block = kSortThreads * p.items, s.blocks = p.blocks;
  // Rows without tokens alone are cleared where that leaves out enough: 140897 tokens, d = 4096, V = 151936 774 us, all rows 833; 50000, d = 1024
  // 176, 182; 16000, d = 4096 482, 472; d = 256 (rows of 1 KB) 50000 92, 73.
  s.clear_absent = d >= 1024 && 8 * T >= V;
  // ... after what the first pass leaves time for: 140897 tokens, d = 4096, V = 151936 with 0 / 64 / 128 / 224 MB of it 742 / 737 / 731 / 725 us,
  // 140000, d = 1024 249 / 245 / 241 / 237; 12000, d = 4096, V = 8192 (134 MB in all) 73.7, with all of it 76.
  s.early = (int)std::min<int64_t>(V / 4, 192000000 / (4 * (int64_t)d));
  if (int rc = p.items == 2 ? launch_embed_sort<2>(s, st) : launch_embed_sort<8>(s, st)) return rc;
  a.partials = (float*)(ws + p.off_partials);
  a.tile = p.tile, a.tiles = p.tiles, a.slices = (int)grid1d(d, 1024);
  const dim3 grid = embed_sum_grid(p, d);
  // Beyond 64 MiB rows, in and out, go past the caches, us in bf16: 140897 tokens, d = 4096 (1.15 GB) 758 -> 723, 40000, d = 2048, V = 151936
  // 300 -> 286; d = 4096: V = 1000 15000 (123 MB) 66 -> 62, V = 1544 10000 (82 MB) 51 -> 52; d = 2048, V = 8192 10000 (41 MB) 46 -> 48.
  const bool once = T * d * (int64_t)esize(dtype) > (int64_t)64 << 20;
  by_form<4, true>(d, [&](auto form) {
    by_truth(once, [&](auto past) {
      constexpr Form FORM = form;
      constexpr bool ONCE = past;
      if (dtype == OAPL_BF16) k_embed_sum<bf16_t, FORM, ONCE><<<grid, 256, 0, st>>>(a);
      else k_embed_sum<float, FORM, ONCE><<<grid, 256, 0, st>>>(a);
    });
  });
  OAPL_LAUNCH_CHECK();
  by_form<4, true>(d, [&](auto form) {
    constexpr Form FORM = form;
    k_embed_join<FORM><<<dim3(grid1d(p.tiles, kJoinTiles), grid1d(d, 256)), 64 * kJoinParts, 0, st>>>(a);
  });
  OAPL_LAUNCH_CHECK();
  return OAPL_OK;
}

int32_t oapl_residual_norm_fwd(const oapl_rows* x, const oapl_rows* y, const void* y_gain, const oapl_rows* gate, int32_t gate_per_token,
                               const void* gain, int64_t T, int32_t d, int32_t x_dtype, int32_t dtype, float scale, float eps,
                               const oapl_rows* x_out, const oapl_rows* out, void* stream) {
  ResidualNormArgs a;
  if (int rc = residual_norm_args(a, x, y, y_gain, gate, gate_per_token, gain, T, d, x_dtype, dtype, scale, eps)) return rc;
  if ((y == nullptr) != (x_out == nullptr) || (gain == nullptr) != (out == nullptr)) return OAPL_ERR_NULL;
  if (int rc = x_out ? take_rows(a.x_out, x_out, T, d, x_dtype, true) : OAPL_OK) return rc;
  if (int rc = out ? take_rows(a.out, out, T, d, dtype, true) : OAPL_OK) return rc;
  if (T == 0) return OAPL_OK;
  by_types(x_dtype, dtype, [&](auto* tx, auto* t) {
    typedef std::remove_pointer_t<decltype(tx)> TX;
    typedef std::remove_pointer_t<decltype(t)> TY;
    constexpr int W = sizeof(TX) == 2 ? 8 : 4;
    by_width<W>(d, [&](auto lanes, auto most, auto pieces) {
      by_form<W, decltype(lanes)::value == 16>(d, [&](auto form) {
        constexpr int LANES = lanes, MOST = most, PIECES = pieces;
        constexpr Form FORM = form;
        k_residual_norm_fwd<TX, TY, W, LANES, MOST, PIECES, FORM>
            <<<wide_grid(norm_workgroups(T, d), 1 << 21), norm_lanes(d), 0, (hipStream_t)stream>>>(a);
      });
    });
    return 0;
  });
  OAPL_LAUNCH_CHECK();
  return OAPL_OK;
}

size_t oapl_residual_norm_workspace_bytes(int64_t T, int32_t d) {
  if (T < 0 || T > kMaxRows || d < 1 || d > kMaxNormWidth) return 0;
  return (size_t)round_up((int64_t)norm_bwd_parts(T, d).n * norm_bwd_grid(T, d) * 2 * d * (int64_t)sizeof(float) + 1, 256);
}

int32_t oapl_residual_norm_bwd(const oapl_rows* x, const oapl_rows* y, const void* y_gain, const oapl_rows* gate, int32_t gate_per_token,
                               const void* gain, const oapl_rows* dx_out, const oapl_rows* dout, int64_t T, int32_t d, int32_t x_dtype,
                               int32_t dtype, float scale, float eps, const oapl_rows* dx, const oapl_rows* dy, float* dgain,
                               float* dy_gain, const oapl_rows* dgate_rows, float* dgate, void* workspace, size_t workspace_bytes,
                               void* stream) {
  ResidualNormArgs a;
  if (int rc = residual_norm_args(a, x, y, y_gain, gate, gate_per_token, gain, T, d, x_dtype, dtype, scale, eps)) return rc;
  if ((gain == nullptr) != (dout == nullptr) || (y == nullptr) != (dy == nullptr) || (gain && !dgain) || (y_gain && !dy_gain)) return OAPL_ERR_NULL;
  const bool shared = gate && !gate_per_token;
  if ((gate && gate_per_token && !dgate_rows) || (shared && !dgate)) return OAPL_ERR_NULL;
  if (int rc = dx_out ? take_rows(a.x_out, dx_out, T, d, x_dtype, false) : OAPL_OK) return rc;
  if (int rc = dout ? take_rows(a.out, dout, T, d, dtype, false) : OAPL_OK) return rc;
  if (int rc = take_rows(a.dx, dx, T, d, x_dtype, true)) return rc;
  if (int rc = dy ? take_rows(a.dy, dy, T, d, dtype, true) : OAPL_OK) return rc;
  if (int rc = gate && gate_per_token ? take_rows(a.dgate, dgate_rows, T, d, dtype, true) : OAPL_OK) return rc;
  if (!element_aligned(dgain, OAPL_F32) || !element_aligned(dy_gain, OAPL_F32) || !element_aligned(dgate, OAPL_F32)) return OAPL_ERR_ALIGN;
  const bool sums = gain || y_gain || shared;
  if (sums && !workspace_ok(workspace, workspace_bytes, oapl_residual_norm_workspace_bytes(T, d))) return OAPL_ERR_WORKSPACE;
  a.partials = sums ? (float*)workspace : nullptr;
  hipStream_t st = (hipStream_t)stream;
  const unsigned grid = norm_bwd_grid(T, d);
  const NormParts parts = sums ? norm_bwd_parts(T, d) : NormParts{1, T};
  return by_types(x_dtype, dtype, [&](auto* tx, auto* t) -> int {
    typedef std::remove_pointer_t<decltype(tx)> TX;
    typedef std::remove_pointer_t<decltype(t)> TY;
    for (int i = 0; i < parts.n && T > 0; ++i) {
      ResidualNormArgs b = a;
      for (Rows* rows : {&b.x, &b.y, &b.gate, &b.x_out, &b.out, &b.dx, &b.dy, &b.dgate})
        if (rows->p) rows->p += i * parts.rows * rows->stride;
      if (sums) b.partials += (int64_t)i * grid * 2 * d;
      b.T = std::min(parts.rows, T - i * parts.rows);
      constexpr int W = sizeof(TX) == 2 ? 8 : 4;
      by_width<W>(d, [&](auto lanes, auto most, auto pieces) {
        by_form<W, decltype(lanes)::value == 16>(d, [&](auto form) {
          constexpr int LANES = lanes, MOST = most, PIECES = pieces;
          constexpr Form FORM = form;
          k_residual_norm_bwd<TX, TY, W, LANES, MOST, PIECES, FORM><<<grid, norm_lanes(d), 0, st>>>(b);
        });
      });
      OAPL_LAUNCH_CHECK();
    }
    if (sums) {
      k_norm_gain_grads<TY><<<grid1d(2 * d, 16), 1024, 0, st>>>(a.partials, parts.n * (int)grid, d,
                                                               shared ? (const TY*)gate->data : nullptr, (const TY*)y_gain,
                                                               gain ? dgain : nullptr, y_gain ? dy_gain : nullptr, shared ? dgate : nullptr);
      OAPL_LAUNCH_CHECK();
    }
    return OAPL_OK;
  });
}

size_t oapl_clip_workspace_bytes(int32_t n_tensors) {
  if (n_tensors < 0 || n_tensors > (1 << 20)) return 0;
  return (size_t)std::max(1, (n_tensors + kClipTensors - 1) / kClipTensors) * kClipGrid * sizeof(double);
}

int32_t oapl_grad_norm(const oapl_tensor* tensors, int32_t n_tensors, float* norm, void* workspace, size_t workspace_bytes,
                       void* stream) {
  ClipPlan p;
  if (int rc = clip_plan(p, tensors, n_tensors, false)) return rc;
  if (!norm) return OAPL_ERR_NULL;
  if (!element_aligned(norm, OAPL_F32)) return OAPL_ERR_ALIGN;
  if (!workspace_ok(workspace, workspace_bytes, oapl_clip_workspace_bytes(n_tensors))) return OAPL_ERR_WORKSPACE;
  hipStream_t st = (hipStream_t)stream;
  ClipArgs a = {};
  if (int rc = clip_squares(p, tensors, n_tensors, workspace, a, st)) return rc;
  a.norm_out = norm;
  k_grad_norm<<<1, 256, 0, st>>>(a);
  OAPL_LAUNCH_CHECK();
  return OAPL_OK;
}

int32_t oapl_clip_grads(const oapl_tensor* tensors, int32_t n_tensors, float max_norm, const float* norm_given, float* norm_out,
                        void* workspace, size_t workspace_bytes, void* stream) {
  ClipPlan p;
  if (int rc = clip_plan(p, tensors, n_tensors, true)) return rc;
  if (!(max_norm >= 0.f) || !isfinite(max_norm)) return OAPL_ERR_BETA;
  if ((norm_given == nullptr) == (norm_out == nullptr)) return OAPL_ERR_NULL;
  if (!element_aligned(norm_given, OAPL_F32) || !element_aligned(norm_out, OAPL_F32)) return OAPL_ERR_ALIGN;
  if (int rc = check_overlaps(tensors, n_tensors)) return rc;
  if (!norm_given && !workspace_ok(workspace, workspace_bytes, oapl_clip_workspace_bytes(n_tensors))) return OAPL_ERR_WORKSPACE;
  hipStream_t st = (hipStream_t)stream;
  ClipArgs a = {};
  a.max_norm = max_norm, a.norm = norm_given;
  if (!norm_given) {
    if (int rc = clip_squares(p, tensors, n_tensors, workspace, a, st)) return rc;
    a.norm_out = norm_out;
    if (p.large || p.launches != 1) {
      // the norm once, for workgroups that have little else to do
      k_grad_norm<<<1, 256, 0, st>>>(a);
      OAPL_LAUNCH_CHECK();
      a.norm = norm_out, a.norm_out = nullptr;
    }
  }
  return clip_batches(p, tensors, n_tensors, true, a, [&](const ClipArgs& b) {
    if (b.chunks == 0 && !b.norm_out) return;
    const dim3 grid = wide_grid(std::max<int64_t>(1, b.chunks), 1 << 23);
    if (p.load_once) k_grad_scale<true, true><<<grid, 256, 0, st>>>(b);
    else if (p.store_once) k_grad_scale<false, true><<<grid, 256, 0, st>>>(b);
    else k_grad_scale<false, false><<<grid, 256, 0, st>>>(b);
  });
}

}  // extern "C"
