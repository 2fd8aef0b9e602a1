// Host code of exact attention under the sanitizers: every bucket table, workspace sizes over the range of sizes
// (the launch rules run in them), and calls that are refused before any device work.
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <vector>

#include "mca.h"

#define CHECK(x)                                                    \
  do {                                                              \
    if (!(x)) {                                                     \
      std::printf("line %d: %s: %s\n", __LINE__, #x, mca_last_error()); \
      return 1;                                                     \
    }                                                               \
  } while (0)

static int64_t pick(uint64_t& s, std::initializer_list<int64_t> of) {
  s = s * 6364136223846793005ull + 1442695040888963407ull;
  return of.begin()[(s >> 33) % of.size()];
}

int main() {
  std::vector<int32_t> out(513);
  int tables = 0;
  for (int both = 0; both < 2; ++both)
    for (int buckets = 0; buckets <= 130; ++buckets)
      for (int top : {1, 2, 3, 20, 64, 100, 128, 255, 256, 257}) {
        const mca_status st = mca_relative_buckets(buckets, top, both, out.data());
        CHECK(st == MCA_OK || st == MCA_ERR_INVALID_ARGUMENT);
        if (st != MCA_OK) continue;
        ++tables;
        const int n = both ? buckets / 2 : buckets;
        CHECK(out[top] == 0 && out[0] == n - 1);
        for (int r = 1; r <= 2 * top; ++r) CHECK(out[r] >= 0 && out[r] < buckets);
        for (int r = 1; r <= top; ++r) CHECK(out[r] <= out[r - 1]);
      }
  CHECK(tables > 500);

  uint64_t seed = 1;
  int sized = 0;
  for (int k = 0; k < 20000; ++k) {
    mca_exact_desc d;
    std::memset(&d, 0, sizeof d);
    d.batch = pick(seed, {1, 2, 7, 64, 1000, 1 << 20, 1 << 24});
    d.q_len = pick(seed, {1, 2, 31, 32, 33, 128, 129, 1000, 4096, 1 << 20, 1 << 24});
    d.kv_len = pick(seed, {1, 2, 31, 32, 33, 128, 129, 1000, 16384, 1 << 20, 1 << 24});
    d.kv_heads = pick(seed, {1, 2, 3, 12, 16});
    d.heads = d.kv_heads * pick(seed, {1, 1, 2, 4, 64});
    d.d_head = 64;
    d.dtype = (int32_t)pick(seed, {MCA_F32, MCA_BF16});
    d.causal = (int32_t)pick(seed, {0, 1});
    d.window = pick(seed, {0, 0, 2, 256, 1 << 25});
    d.scale = 0.125;
    if (pick(seed, {0, 1})) {
      d.bias_table = reinterpret_cast<const void*>(uintptr_t(1) << 20);
      d.bias_buckets = (int32_t)pick(seed, {4, 8, 32, 128});
      d.bias_max_distance = (int32_t)pick(seed, {40, 128, 256});
      d.bias_bidirectional = (int32_t)pick(seed, {0, 1});
    }
    for (int backward = 0; backward < 2; ++backward) {
      size_t bytes = 0;
      const mca_status st = mca_exact_workspace_size(&d, backward, &bytes);
      CHECK(st == MCA_OK || st == MCA_ERR_INVALID_ARGUMENT);
      if (st != MCA_OK) continue;
      ++sized;
      // the statistics of the rows, parts of which there are never more than a few per CU, the bias' parts
      const double rows = 8.0 * d.batch * d.heads * d.q_len + 256;
      CHECK((double)bytes <= rows + 1e9 + 4.0 * d.bias_buckets * d.heads * 8.0 * (1100 + (double)d.batch * (d.kv_len / 32 + 1)));
    }
    // null operands and operands of one memory
    CHECK(mca_exact_attention_forward(&d, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, 0, nullptr) != MCA_OK);
    mca_rows t = {reinterpret_cast<void*>(uintptr_t(1) << 30), 0, d.heads * 64};
    float* lse = reinterpret_cast<float*>(uintptr_t(1) << 29);
    CHECK(mca_exact_attention_backward(&d, &t, &t, &t, &t, &t, lse, &t, &t, &t, nullptr, reinterpret_cast<void*>(uintptr_t(1) << 28),
                                       ~size_t(0), nullptr) != MCA_OK);
  }
  CHECK(sized > 5000);
  std::printf("all exact checks passed: %d tables, %d sizes\n", tables, sized);
  return 0;
}
