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
constexpr int kMaxNormWidth = 16384;                   // 1024 lanes with two pieces of a row each

// A rows argument of n rows of d channels.  The stride of a single row is not looked at.  `written` rows must not overlap.
static int check_rows(const oapl_rows* x, int64_t n, int64_t d, bool written) {
  if (!x) return OAPL_ERR_NULL;
  if (n == 0) return OAPL_OK;
  if (!x->data) return OAPL_ERR_NULL;
  if (n > 1 && (x->row_stride < (written ? d : 0) || x->row_stride > ((int64_t)1 << 40))) return OAPL_ERR_SHAPE;
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
  int bits = 1, items = 1, blocks = 1, tile = 1, tiles = 0;
  size_t off_keys[2], off_places[2], off_counts[2], off_present = 0, off_partials = 0, total = 0;
};

static bool embed_sizes_ok(int64_t T, int d, int V) {
  return T >= 0 && T <= kMaxRows && d >= 1 && d <= (1 << 21) && V >= 1 && V <= (1 << 21);
}

static bool embed_plan(EmbedPlan& p, int64_t T, int d, int V) {
  if (!embed_sizes_ok(T, d, V)) return false;
  while (((int64_t)1 << (2 * p.bits)) <= V) ++p.bits;      // ids 0 .. V
  p.items = T <= 128 * kSortThreads * 2 ? 2 : 8;
  p.blocks = (int)std::max<int64_t>(1, (T + (int64_t)kSortThreads * p.items - 1) / (kSortThreads * p.items));
  p.tile = 64;
  p.tiles = (int)((T + p.tile - 1) / p.tile);
  size_t at = kStatusWords * sizeof(int);
  const auto take = [&](int64_t bytes) {
    const size_t was = at;
    at += (size_t)round_up(bytes, 256);
    return was;
  };
  for (int i = 0; i < 2; ++i) {
    p.off_keys[i] = take(T * 4), p.off_places[i] = take(T * 4);
    p.off_counts[i] = take(((int64_t)p.blocks << p.bits) * 4);
  }
  p.off_present = take(V);
  p.off_partials = take((int64_t)p.tiles * 2 * d * 4);
  p.total = at;
  return true;
}

template <int ITEMS>
static int launch_embed_sort(const SortArgs& a, hipStream_t st) {
  const int bins = 1 << a.bits, bytes = kSortThreads / 64 * bins * 4;
  if (bytes > 48 * 1024 && (!allow_big_lds(k_embed_place<0, ITEMS>, bytes) || !allow_big_lds(k_embed_place<1, ITEMS>, bytes)))
    return OAPL_ERR_HIP;
  k_embed_count<ITEMS><<<a.blocks, kSortThreads, bins * 4, st>>>(a);
  OAPL_LAUNCH_CHECK();
  k_embed_place<0, ITEMS><<<a.blocks, kSortThreads, bytes, st>>>(a);
  OAPL_LAUNCH_CHECK();
  k_embed_place<1, ITEMS><<<a.blocks, kSortThreads, bytes, st>>>(a);
  OAPL_LAUNCH_CHECK();
  return OAPL_OK;
}

// ---------------------------------------------------------------------------------------------------------------- residual stream
// How the lanes of a workgroup divide rows of d channels; f(threads of a row, pieces of eight channels a thread).
template <class F>
static int by_width(int d, F f) {
  if (d <= 512) return f(std::integral_constant<int, 64>{}, std::integral_constant<int, 1>{});
  if (d <= 1024) return f(std::integral_constant<int, 64>{}, std::integral_constant<int, 2>{});
  if (d <= 2048) return f(std::integral_constant<int, 256>{}, std::integral_constant<int, 1>{});
  if (d <= 4096) return f(std::integral_constant<int, 256>{}, std::integral_constant<int, 2>{});
  if (d <= 8192) return f(std::integral_constant<int, 512>{}, std::integral_constant<int, 2>{});
  return f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 2>{});
}
static int norm_rows_of_a_workgroup(int d) { return d <= 1024 ? 4 : 1; }

// f(null pointer to the residual stream's type, ... to the block's).
template <class F>
static int by_types(int x_dtype, int dtype, F f) {
  if (x_dtype == OAPL_BF16) return f((bf16_t*)nullptr, (bf16_t*)nullptr);
  if (dtype == OAPL_BF16) return f((float*)nullptr, (bf16_t*)nullptr);
  return f((float*)nullptr, (float*)nullptr);
}

static unsigned norm_fwd_grid(int64_t T, int d) {
  return (unsigned)std::min<int64_t>((T + norm_rows_of_a_workgroup(d) - 1) / norm_rows_of_a_workgroup(d), 1 << 16);
}
// Backwards every workgroup has sums of its own.
static unsigned norm_bwd_grid(int64_t T, int d) {
  return (unsigned)std::min<int64_t>((T + norm_rows_of_a_workgroup(d) - 1) / norm_rows_of_a_workgroup(d), 512);
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
static int clip_launches(int64_t n) { return (int)((n + kClipTensors - 1) / kClipTensors); }

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

static int check_tensors(const oapl_tensor* tensors, int n, bool written) {
  if (n < 0 || n > (1 << 20)) return OAPL_ERR_SHAPE;
  if (n > 0 && !tensors) return OAPL_ERR_NULL;
  int64_t chunks = 0;
  for (int i = 0; i < n; ++i) {
    const oapl_tensor& t = tensors[i];
    if (!dtype_ok(t.dtype)) return OAPL_ERR_DTYPE;
    if (t.n < 0 || t.n > (int64_t)1 << 44) return OAPL_ERR_SHAPE;
    chunks += (t.n + kClipChunk - 1) / kClipChunk;
    if (chunks >= (int64_t)1 << 31) return OAPL_ERR_SHAPE;
    if (t.n == 0) continue;
    if (!t.data || (written && !t.out)) return OAPL_ERR_NULL;
    if (!element_aligned(t.data, t.dtype) || (written && !element_aligned(t.out, t.dtype))) return OAPL_ERR_ALIGN;
  }
  return OAPL_OK;
}

// One launch for every kClipTensors tensors; f(arguments, workgroups).
template <class F>
static int clip_batches(const oapl_tensor* tensors, int n, ClipArgs& a, F f) {
  for (int at = 0; at < n; at += kClipTensors) {
    a.count = std::min(kClipTensors, n - at);
    int64_t chunks = 0;
    for (int i = 0; i < a.count; ++i) {
      const oapl_tensor& t = tensors[at + i];
      a.t[i] = ClipTensor{t.data, t.out, t.n, (uint32_t)chunks, t.dtype};
      chunks += (t.n + kClipChunk - 1) / kClipChunk;
    }
    a.chunks = (uint32_t)chunks;
    a.mine = at / kClipTensors * kClipGrid;
    if (int rc = f(a, kClipGrid)) return rc;
  }
  return OAPL_OK;
}

static int clip_squares(const oapl_tensor* tensors, int n, ClipArgs& a, hipStream_t st) {
  return clip_batches(tensors, n, a, [&](const ClipArgs& b, int grid) -> int {
    k_grad_squares<<<grid, 256, 0, st>>>(b);
    OAPL_LAUNCH_CHECK();
    return OAPL_OK;
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
  if (!element_aligned(E, dtype)) return OAPL_ERR_ALIGN;
  EmbedArgs a{E, tokens, {}, T, d, V, scale};
  if (int rc = take_rows(a.out, out, T, d, out_dtype, true)) return rc;
  if (T == 0) return OAPL_OK;
  const dim3 grid((unsigned)std::min<int64_t>((T + 3) / 4, 1 << 16), grid1d(d, 512));
  hipStream_t st = (hipStream_t)stream;
  if (dtype == OAPL_BF16 && out_dtype == OAPL_BF16) k_embed_fwd<bf16_t, bf16_t><<<grid, 256, 0, st>>>(a);
  else if (dtype == OAPL_BF16) k_embed_fwd<bf16_t, float><<<grid, 256, 0, st>>>(a);
  else if (out_dtype == OAPL_BF16) k_embed_fwd<float, bf16_t><<<grid, 256, 0, st>>>(a);
  else k_embed_fwd<float, float><<<grid, 256, 0, st>>>(a);
  OAPL_LAUNCH_CHECK();
  return OAPL_OK;
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
  if (!element_aligned(dE, OAPL_F32)) return OAPL_ERR_ALIGN;
  if (!workspace_ok(workspace, workspace_bytes, p.total)) return OAPL_ERR_WORKSPACE;
  hipStream_t st = (hipStream_t)stream;
  char* ws = (char*)workspace;
  SortArgs s = {};
  s.tokens = tokens;
  for (int i = 0; i < 2; ++i) {
    s.keys[i] = (int32_t*)(ws + p.off_keys[i]), s.places[i] = (int32_t*)(ws + p.off_places[i]);
    s.counts[i] = (int32_t*)(ws + p.off_counts[i]);
  }
  s.present = (uint8_t*)(ws + p.off_present), s.status = (int*)ws;
  s.T = T, s.V = V, s.bits = p.bits, s.blocks = p.blocks;
  if (int rc = p.items == 2 ? launch_embed_sort<2>(s, st) : launch_embed_sort<8>(s, st)) return rc;
  a.keys = s.keys[1], a.places = s.places[1], a.present = s.present;
  a.dE = dE, a.partials = (float*)(ws + p.off_partials);
  a.T = T, a.d = d, a.V = V, a.tile = p.tile, a.tiles = p.tiles, a.scale = scale, a.add = accumulate != 0;
  const unsigned fill = accumulate ? 0 : (unsigned)std::min(V, 4096);
  if (p.tiles + fill > 0) {
    const dim3 grid(p.tiles + fill, grid1d(d, 2048));
    if (dtype == OAPL_BF16) k_embed_sum<bf16_t><<<grid, 256, 0, st>>>(a);
    else k_embed_sum<float><<<grid, 256, 0, st>>>(a);
    OAPL_LAUNCH_CHECK();
  }
  if (p.tiles > 1) {
    k_embed_join<<<dim3(p.tiles, grid1d(d, 256)), 256, 0, st>>>(a);
    OAPL_LAUNCH_CHECK();
  }
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
    return by_width(d, [&](auto threads, auto pieces) {
      constexpr int THREADS = threads, PIECES = pieces;
      k_residual_norm_fwd<std::remove_pointer_t<decltype(tx)>, std::remove_pointer_t<decltype(t)>, THREADS, PIECES>
          <<<norm_fwd_grid(T, d), std::max(256, THREADS), 0, (hipStream_t)stream>>>(a);
      return 0;
    });
  });
  OAPL_LAUNCH_CHECK();
  return OAPL_OK;
}

size_t oapl_residual_norm_workspace_bytes(int64_t T, int32_t d) {
  if (T < 0 || T > kMaxRows || d < 1 || d > kMaxNormWidth) return 0;
  return (size_t)round_up((int64_t)norm_bwd_grid(T, d) * norm_rows_of_a_workgroup(d) * 2 * d * (int64_t)sizeof(float) + 1, 256);
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
  return by_types(x_dtype, dtype, [&](auto* tx, auto* t) -> int {
    typedef std::remove_pointer_t<decltype(tx)> TX;
    typedef std::remove_pointer_t<decltype(t)> TY;
    if (T > 0) {
      by_width(d, [&](auto threads, auto pieces) {
        constexpr int THREADS = threads, PIECES = pieces;
        k_residual_norm_bwd<TX, TY, THREADS, PIECES><<<grid, std::max(256, THREADS), 0, st>>>(a);
        return 0;
      });
      OAPL_LAUNCH_CHECK();
    }
    if (sums) {
      k_norm_gain_grads<TY><<<grid1d(2 * d, 16), 1024, 0, st>>>(a.partials, (int)grid * norm_rows_of_a_workgroup(d), d,
                                                               shared ? (const TY*)gate->data : nullptr, (const TY*)y_gain,
                                                               gain ? dgain : nullptr, y_gain ? dy_gain : nullptr, shared ? dgate : nullptr);
      OAPL_LAUNCH_CHECK();
    }
    return OAPL_OK;
  });
}

size_t oapl_clip_workspace_bytes(int32_t n_tensors) {
  if (n_tensors < 0 || n_tensors > (1 << 20)) return 0;
  return (size_t)std::max(1, clip_launches(n_tensors)) * kClipGrid * sizeof(double);
}

int32_t oapl_grad_norm(const oapl_tensor* tensors, int32_t n_tensors, float* norm, void* workspace, size_t workspace_bytes,
                       void* stream) {
  if (int rc = check_tensors(tensors, n_tensors, false)) return rc;
  if (!norm) return OAPL_ERR_NULL;
  if (!element_aligned(norm, OAPL_F32)) return OAPL_ERR_ALIGN;
  if (!workspace_ok(workspace, workspace_bytes, oapl_clip_workspace_bytes(n_tensors))) return OAPL_ERR_WORKSPACE;
  hipStream_t st = (hipStream_t)stream;
  ClipArgs a = {};
  a.sum = (double*)workspace, a.sums = clip_launches(n_tensors) * kClipGrid;
  if (int rc = clip_squares(tensors, n_tensors, a, st)) return rc;
  a.norm_out = norm;
  k_grad_norm<<<1, 256, 0, st>>>(a);
  OAPL_LAUNCH_CHECK();
  return OAPL_OK;
}

int32_t oapl_clip_grads(const oapl_tensor* tensors, int32_t n_tensors, float max_norm, const float* norm_given, float* norm_out,
                        void* workspace, size_t workspace_bytes, void* stream) {
  if (int rc = check_tensors(tensors, n_tensors, true)) return rc;
  if (!(max_norm >= 0.f) || !isfinite(max_norm)) return OAPL_ERR_BETA;
  if ((norm_given == nullptr) == (norm_out == nullptr)) return OAPL_ERR_NULL;
  if (!element_aligned(norm_given, OAPL_F32) || !element_aligned(norm_out, OAPL_F32)) return OAPL_ERR_ALIGN;
  if (int rc = check_overlaps(tensors, n_tensors)) return rc;
  if (!norm_given && !workspace_ok(workspace, workspace_bytes, oapl_clip_workspace_bytes(n_tensors))) return OAPL_ERR_WORKSPACE;
  hipStream_t st = (hipStream_t)stream;
  ClipArgs a = {};
  a.max_norm = max_norm, a.norm = norm_given;
  if (!norm_given) {
    if (n_tensors == 0) return oapl_grad_norm(tensors, 0, norm_out, workspace, workspace_bytes, stream);
    a.sum = (double*)workspace, a.sums = clip_launches(n_tensors) * kClipGrid;
    if (int rc = clip_squares(tensors, n_tensors, a, st)) return rc;
  }
  a.norm_out = norm_out;
  return clip_batches(tensors, n_tensors, a, [&](const ClipArgs& b, int grid) -> int {
    k_grad_scale<<<grid, 256, 0, st>>>(b);
    OAPL_LAUNCH_CHECK();
    return OAPL_OK;
  });
}

}  // extern "C"
