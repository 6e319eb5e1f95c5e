// Host-side sanitizer driver of the embedding, residual-norm and clipping entry points: argument checks, plans and grids over sizes, strides and
// numbers at the ends of their types, compiled for the host alone with AddressSanitizer and UndefinedBehaviorSanitizer.  Every call below is a
// pure host query or fails a host-side check (at the latest, for want of an output or a workspace); nothing is launched.
#include <climits>
#include <cstdint>
#include <cstdio>
#include <cstdlib>

#include "../../paper_2602_19362_amd/csrc/oapl_api.hip"

#define CHECK(cond)                                         \
  do {                                                      \
    if (!(cond)) {                                          \
      std::printf("FAILED line %d: %s\n", __LINE__, #cond); \
      std::exit(1);                                         \
    }                                                       \
  } while (0)

static bool fits(dim3 g, int64_t threads) { return g.x * threads < ((int64_t)1 << 32) && g.y < 65536; }

int main() {
  void* one = (void*)(uintptr_t)256;      // aligned, never dereferenced
  float* f = (float*)one;
  const int32_t* tokens = (const int32_t*)one;
  const int64_t counts[] = {INT64_MIN, -1, 0, 1, 31, 4096, 4097, 6144, 6145, 8192, 8193, 262144, 262145, (int64_t)65535 * 256, (int64_t)65535 * 256 + 1, INT64_MAX};
  const int32_t widths[] = {INT_MIN, -1, 0, 1, 7, 128, 512, 513, 1024, 2048, 2049, 8192, 16384, 16385, 1 << 21, (1 << 21) + 1, INT_MAX};
  const int64_t strides[] = {INT64_MIN, -8, 0, 8, 16384, (int64_t)1 << 40, ((int64_t)1 << 40) + 1, INT64_MAX};
  long plans = 0, calls = 0;

  for (int64_t T : counts)
    for (int32_t d : widths)
      for (int32_t V : widths) {
        EmbedPlan p;
        const bool good = embed_plan(p, T, d, V);
        CHECK(good == (T >= 0 && T <= (int64_t)65535 * 256 && d >= 1 && d <= 1 << 21 && V >= 1 && V <= 1 << 21 && T * d <= (int64_t)1 << 40));
        CHECK(oapl_embed_workspace_bytes(T, d, V) == (good ? p.total : 0) && (!good || p.total % 256 == 0));
        ++plans;
        // counting holds all ids in a workgroup's LDS
        CHECK(!good || !p.few || T <= kFewTokens);
        if (!good || p.few) continue;
        // ids 0 .. V have two digits; blocks and tiles hold all tokens; a workgroup's counts fit the LDS
        CHECK(((int64_t)1 << (2 * p.bits)) > V && p.bits <= 11 && (kSortThreads / 64 + 2) * (4 << p.bits) <= 150 * 1024);
        CHECK((int64_t)p.blocks * kSortThreads * p.items >= T && (int64_t)p.tiles * p.tile >= T && (int64_t)(p.tiles - 1) * p.tile < T);
        CHECK((int64_t)p.tiles * 256 * grid1d(d, 1024) < ((int64_t)1 << 32));
        // the lookup's wavefronts are counted in 32 bits
        CHECK(T * grid1d(d, 256) < ((int64_t)1 << 32) - (1 << 23) * 4);
      }
  for (int64_t n : {(int64_t)1, (int64_t)(1 << 23), (int64_t)(1 << 23) + 1, (int64_t)1 << 32, ((int64_t)1 << 38) - 1}) {
    const dim3 g = wide_grid(n, 1 << 23), h = wide_grid(n, 1 << 21);
    CHECK(fits(g, 256) && (int64_t)g.x * g.y >= n && (int64_t)g.x * (g.y - 1) < n);
    CHECK(h.x * (int64_t)1024 < ((int64_t)1 << 32) && (int64_t)h.x * h.y >= n);
  }
  for (int64_t T : counts)
    for (int32_t d : widths) {
      const size_t bytes = oapl_residual_norm_workspace_bytes(T, d);
      const bool good = T >= 0 && T <= (int64_t)65535 * 256 && d >= 1 && d <= 16384;
      CHECK(good == (bytes > 0) && bytes % 256 == 0);
      ++plans;
      if (!good) continue;
      CHECK(norm_lanes(d) * 16 >= d && norm_workgroups(T, d) * norm_rows(d) >= T && fits(wide_grid(std::max<int64_t>(1, norm_workgroups(T, d)), 1 << 21), norm_lanes(d)));
      CHECK(norm_bwd_grid(T, d) <= 1024 && bytes >= (size_t)norm_bwd_grid(T, d) * 2 * d * 4);
    }

  for (int64_t stride : strides)
    for (int64_t T : {(int64_t)0, (int64_t)1, (int64_t)5, (int64_t)65535 * 256})
      for (int32_t d : {1, 8, 16384})
        for (int dtype = 0; dtype < 2; ++dtype) {
          const oapl_rows x{one, stride}, plain{one, 16384};
          for (const oapl_rows* a : {&x, &plain})
            for (const oapl_rows* b : {&x, &plain}) {
              CHECK(oapl_embed_bwd(a, tokens, T, d, 100, dtype, 1.f, 0, f, nullptr, 0, nullptr) != OAPL_OK);
              CHECK(oapl_embed_fwd(one, tokens, T, d, 100, dtype, dtype, 1.f, nullptr, nullptr) != OAPL_OK);
              CHECK(oapl_residual_norm_fwd(a, b, one, b, 1, one, T, d, dtype, dtype, 1.f, 1e-6f, a, nullptr, nullptr) != OAPL_OK);
              CHECK(oapl_residual_norm_bwd(a, b, one, b, 1, one, a, b, T, d, dtype, dtype, 1.f, 1e-6f, a, b, f, f, b, f, nullptr, 0, nullptr) != OAPL_OK);
              calls += 4;
            }
        }
  const float numbers[] = {-1.f, __builtin_inff(), -__builtin_inff(), __builtin_nanf("")};
  const oapl_rows x{one, 64};
  for (float bad : numbers) {
    CHECK(oapl_residual_norm_fwd(&x, nullptr, nullptr, nullptr, 0, one, 4, 64, 1, 1, 1.f, bad, nullptr, &x, nullptr) == OAPL_ERR_BETA);
    oapl_tensor t{one, one, 4, 0};
    CHECK(oapl_clip_grads(&t, 1, bad, nullptr, f, one, 1 << 20, nullptr) == OAPL_ERR_BETA);
  }

  // lists of tensors: counts, sizes and addresses at the ends of their types
  for (int64_t n : {INT64_MIN, (int64_t)-1, ((int64_t)1 << 42) + 1, INT64_MAX}) {
    oapl_tensor t[2] = {{one, one, 5, 0}, {one, one, n, 1}};
    CHECK(oapl_grad_norm(t, 2, f, one, 1 << 20, nullptr) == OAPL_ERR_SHAPE && oapl_clip_grads(t, 2, 1.f, nullptr, f, one, 1 << 20, nullptr) == OAPL_ERR_SHAPE);
  }
  for (int32_t n : {INT_MIN, -1, (1 << 20) + 1, INT_MAX}) CHECK(oapl_grad_norm(nullptr, n, f, one, 1 << 20, nullptr) == OAPL_ERR_SHAPE && oapl_clip_workspace_bytes(n) == 0);
  for (int32_t n : {0, 1, 112, 113, 1 << 20}) CHECK(oapl_clip_workspace_bytes(n) >= (size_t)((n + kClipTensors - 1) / kClipTensors) * kClipGrid * 8);
  {
    const int n = 1000;
    std::vector<oapl_tensor> many(n);
    for (int i = 0; i < n; ++i) many[i] = {(void*)(uintptr_t)(4096 + 64 * i), (void*)(uintptr_t)(4096 + 64 * i), i % 17, i & 1};
    ClipPlan p;
    CHECK(clip_plan(p, many.data(), n, true) == OAPL_OK && p.launches == 9 && check_overlaps(many.data(), n) == OAPL_OK);
    many[7].out = (void*)(uintptr_t)(4096 + 64 * 900 + 4), many[7].n = 1, many[900].n = 9;
    CHECK(check_overlaps(many.data(), n) == OAPL_ERR_SHAPE);
    many[7].n = 0;      // nothing is written
    CHECK(check_overlaps(many.data(), n) == OAPL_OK);
  }
  std::printf("host sanitizer driver: %ld plans, %ld calls, all checks passed\n", plans, calls);
  return 0;
}
