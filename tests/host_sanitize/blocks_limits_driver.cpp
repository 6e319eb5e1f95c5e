// Launches of the gradients of embedding and residual norm at the ends of the sizes that they take, compiled for the host alone with AddressSanitizer and
// UndefinedBehaviorSanitizer: a dimension of a launch has fewer than 2^32 threads, and the other ones fewer than 2^16 workgroups.  Nothing is launched.
#include <cstdint>
#include <cstdio>
#include <cstdlib>

#include "../../paper_2602_19362_amd/csrc/oapl_api.hip"

#define CHECK(cond)                                                                         \
  do {                                                                                      \
    if (!(cond)) {                                                                          \
      std::printf("FAILED line %d: %s (T = %ld, d = %d)\n", __LINE__, #cond, (long)T, d);   \
      std::exit(1);                                                                         \
    }                                                                                       \
  } while (0)

static bool fits(dim3 g, int64_t threads) { return g.x * threads < ((int64_t)1 << 32) && g.y < 65536 && g.z == 1; }

int main() {
  long plans = 0;
  // powers of two and their neighbours, and the most tokens and channels that go together
  const int64_t most = (int64_t)65535 * 256, elements = (int64_t)1 << 40;
  std::vector<int64_t> counts{most - 1, most};
  for (int i = 0; i < 24; ++i)
    for (int64_t T : {((int64_t)1 << i) - 1, (int64_t)1 << i, ((int64_t)1 << i) + 1})
      if (T <= most) counts.push_back(T);
  for (int64_t T : counts) {
    std::vector<int> widths{1 << 21};
    for (int i = 0; i <= 21; ++i)
      for (int d : {(1 << i) - 1, 1 << i, (1 << i) + 1}) widths.push_back(d);
    if (T > 0) widths.push_back((int)std::min<int64_t>(elements / T, 1 << 21));
    for (int d : widths) {
      EmbedPlan p;
      if (!embed_plan(p, T, d, 9)) continue;
      ++plans;
      if (p.few) {
        CHECK(fits(dim3(grid1d(T, 32), grid1d(d, 256)), 64 * kRunWaves));
        continue;
      }
      // a token may have all of the tiles, which one search goes through
      CHECK(p.tiles < kMostEqual);
      const dim3 sum = embed_sum_grid(p, d);
      const int64_t units = (int64_t)p.tiles * grid1d(d, 1024);
      CHECK(fits(sum, 256) && (int64_t)sum.x * sum.y >= units && (int64_t)sum.x * (sum.y - 1) < units);
      CHECK(fits(dim3(grid1d(p.tiles, kJoinTiles), grid1d(d, 256)), 64 * kJoinParts));
      // units and what is missing to whole rows of them are counted in 32 bits
      CHECK((int64_t)sum.x * sum.y < (int64_t)1 << 31);
    }
  }
  for (int64_t T : counts)
    for (int d : {1, 127, 128, 129, 512, 513, 1024, 4096, 4097, 8192, 8193, 16384}) {
      const NormParts parts = norm_bwd_parts(T, d);
      const int64_t grid = norm_bwd_grid(T, d), slots = grid * norm_rows(d);
      ++plans;
      // parts hold all rows, none is empty, and a lane has no more than the chain's rows of one
      CHECK(parts.n >= 1 && parts.n * parts.rows >= T && (T == 0 || (parts.n - 1) * parts.rows < T) && parts.rows % norm_rows(d) == 0);
      CHECK(parts.rows <= slots * 1024);
      CHECK(oapl_residual_norm_workspace_bytes(T, d) >= (size_t)(parts.n * grid * 2 * d * 4));
    }
  std::printf("launches of %ld plans, all checks passed\n", plans);
  return 0;
}
