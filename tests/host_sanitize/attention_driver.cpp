// Host-side sanitizer driver of the attention entry points: argument checks, plans and grids over sizes, strides and numbers at the ends of
// their types, compiled for the host alone with AddressSanitizer and UndefinedBehaviorSanitizer.  Every call below is a pure host query or
// fails a host-side check (at the latest, for want of a workspace); nothing is launched.
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

int main() {
  void* one = (void*)(uintptr_t)256;      // aligned, never dereferenced
  float* f = (float*)one;
  const int64_t* off = (const int64_t*)one;
  const int64_t counts[] = {INT64_MIN, -1, 0, 1, 31, 33, 4096, (int64_t)1 << 24, (int64_t)1 << 26, ((int64_t)1 << 31) - 1024, (int64_t)1 << 31, (int64_t)1 << 40, INT64_MAX};
  const int32_t seqs[] = {INT_MIN, -1, 0, 1, 64, 129, 1 << 20, (1 << 24) - 1, 1 << 24, (1 << 24) + 1, INT_MAX};
  const int32_t heads[][2] = {{1, 1}, {32, 8}, {65536, 1}, {65536, 65536}, {65537, 1}, {7, 2}, {0, 0}, {INT_MAX, 1}, {INT_MAX, INT_MAX}, {-4, -2}};
  const int64_t strides[] = {INT64_MIN, -8, 0, 8, 128, (int64_t)1 << 22, (int64_t)1 << 24, (int64_t)1 << 48, ((int64_t)1 << 48) + 8, INT64_MAX - 7};
  long plans = 0, calls = 0;

  for (int64_t Tq : counts)
    for (int64_t Tk : counts)
      for (int32_t n : seqs)
        for (const auto& h : heads)
          for (int32_t D : {8, 80, 128, 136, INT_MIN})
            for (int dtype = 0; dtype < 3; ++dtype)
              for (int bwd = 0; bwd < 2; ++bwd) {
                const size_t bytes = oapl_attention_workspace_bytes(Tq, Tk, n, h[0], h[1], D, dtype, bwd);
                const bool possible = Tq >= 0 && Tk >= 0 && n >= 0 && h[1] >= 1 && h[0] % h[1] == 0 && D >= 8 && D <= 128 && dtype < 2;
                CHECK(possible || bytes == 0);
                CHECK(bytes % 256 == 0);
                ++plans;
              }
  for (int64_t T : counts)
    for (const auto& h : heads)
      for (int32_t D : {8, 128, 132, INT_MAX}) {
        CHECK(oapl_qk_norm_rope_workspace_bytes(T, h[0], h[1], D) % 256 == 0);
        ++plans;
      }

  // strides at the ends of their range, with one token or head (whose stride is not looked at) and more
  for (int64_t token : strides)
    for (int64_t head : strides)
      for (int64_t T : {(int64_t)0, (int64_t)1, (int64_t)5, ((int64_t)1 << 31) - 1024})
        for (const auto& h : heads)
          for (int dtype = 0; dtype < 2; ++dtype) {
            const oapl_heads x{one, token, head}, plain{one, (int64_t)65536 * 64, 64};
            for (const oapl_heads* q : {&x, &plain})
              for (const oapl_heads* k : {&x, &plain}) {
                CHECK(oapl_attention_fwd(q, k, k, off, off, nullptr, T, T, 1, h[0], h[1], 64, dtype, 1, 0.1f, q, f, nullptr, 0, nullptr) != OAPL_OK);
                CHECK(oapl_attention_bwd(q, k, k, q, f, q, off, off, T, T, 1, h[0], h[1], 64, dtype, 1, 0.1f, q, k, k, nullptr, 0, nullptr) != OAPL_OK);
                CHECK(oapl_qk_norm_rope_bwd(q, k, q, k, (const int32_t*)one, f, one, one, T, h[0], h[1], 64, 64, 10, dtype, 1e-6f, q, k, f, f, nullptr, 0,
                                            nullptr) != OAPL_OK);
                // (rows without a number of rows: refused behind the inputs' checks)
                CHECK(oapl_qk_norm_rope_fwd(q, k, nullptr, (const int32_t*)one, f, one, one, off, T, h[0], h[1], 64, 64, 10, INT64_MIN, dtype, 1e-6f, q, k,
                                            nullptr, nullptr) != OAPL_OK);
                calls += 4;
              }
          }
  for (float scale : {3.4e38f, -3.4e38f, 2.4e38f, __builtin_inff(), -__builtin_inff(), __builtin_nanf("")}) {
    const oapl_heads x{one, 128, 64};
    CHECK(oapl_attention_fwd(&x, &x, &x, off, off, nullptr, 4, 4, 1, 2, 2, 64, 1, 1, scale, &x, f, nullptr, 0, nullptr) == OAPL_ERR_BETA);
  }
  // grids
  for (int64_t T : {(int64_t)1, (int64_t)1 << 26, ((int64_t)1 << 31) - 1024})
    for (int h : {2, 40, 131072}) {
      const dim3 g = rope_fwd_grid(T, rope_parts(T, h));
      CHECK((int64_t)g.x * 256 < ((int64_t)1 << 32) && g.y < 65536 && (int64_t)g.x * g.y * 4 >= T);
      CHECK(rope_bwd_grid(T, h) <= 768);
    }
  std::printf("host sanitizer driver: %ld plans, %ld calls, all checks passed\n", plans, calls);
  return 0;
}
