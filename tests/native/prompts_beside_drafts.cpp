// Prompts that share a prefix while other requests of the batch draft: the plan (batch.hpp) weighs the shared keys as precisely as without the drafts.
//
// usage: prompts_beside_drafts   (prints "plans ok")
#include <cstdio>
#include <vector>

#include "../../paper_2510_02758_amd/csrc/batch.hpp"

#define CHECK(cond, ...)                                                \
  do {                                                                  \
    if (!(cond)) {                                                      \
      fprintf(stderr, "%s:%d: %s failed: ", __FILE__, __LINE__, #cond); \
      fprintf(stderr, __VA_ARGS__);                                     \
      fprintf(stderr, "\n");                                            \
      return false;                                                     \
    }                                                                   \
  } while (0)

// `n` requests behind `prefix` tokens with `q` new ones each; which[i % size] says whether request i drafts.
static bool plan(int32_t D, int n, int32_t prefix, int32_t q, const std::vector<uint8_t>& which, bool drafts, int* shared, int* fine) {
  const int32_t H = 8, G = 4, B = 16;
  const kvswap::BatchShape s = kvswap::batch_shape(H, D, B, 1 << 20, 256, false, drafts);
  std::vector<int32_t> off{0}, ids, len, ql;
  std::vector<uint8_t> trees;
  int next = prefix / B;
  for (int i = 0; i < n; i++) {
    for (int k = 0; k < prefix / B; k++) ids.push_back(k);
    for (int k = 0; k < (q + 100 + B - 1) / B; k++) ids.push_back(next++);
    off.push_back((int32_t)ids.size());
    len.push_back(prefix + q + 100);
    ql.push_back(q);
    trees.push_back(which[(size_t)i % which.size()]);
  }
  kvswap::BatchPlan p;
  CHECK(p.set(n, off.data(), ids.data(), len.data(), ql.data(), G * H, s, drafts ? trees.data() : nullptr) == KV_OK, "refused");
  *shared = *fine = 0;
  for (size_t i = (size_t)p.big_first; i < p.items.size(); i++) {
    const kvswap::AttnItem& it = p.items[i];
    if (it.k1 > prefix) continue;
    *shared += it.rows > q * G;  // (rows of several requests)
    *fine += it.rows > q * G && it.fine;
  }
  return true;
}

static bool all() {
  struct {
    int n;
    int32_t prefix, q;
  } const batches[] = {{40, 4096, 10}, {2, 65536, 20}, {3, 65536, 12}, {40, 8192, 16}};
  for (int32_t D : {64, 128})
    for (const auto& b : batches) {
      int shared, fine;
      if (!plan(D, b.n, b.prefix, b.q, {0}, false, &shared, &fine)) return false;
      CHECK(shared == fine, "%d requests behind %d, without drafts: %d of %d shares", b.n, b.prefix, fine, shared);
      const bool shares = shared > 0;
      for (const std::vector<uint8_t>& which : {std::vector<uint8_t>{0}, {0, 1}, {1, 0}, {1, 1, 0}}) {
        if ((int)which.size() > b.n) continue;  // (the batch has no prompt then)
        if (!plan(D, b.n, b.prefix, b.q, which, true, &shared, &fine)) return false;
        CHECK(shared == fine, "%d requests behind %d, %zu kinds: %d of %d shares", b.n, b.prefix, which.size(), fine, shared);
      }
      CHECK(shares || D == 64, "nothing is shared");
    }
  // drafts alone, of many rows: in one term
  int shared, fine;
  if (!plan(128, 40, 4096, 10, {1}, true, &shared, &fine)) return false;
  CHECK(shared > 0 && fine == 0, "%d of %d", fine, shared);
  return true;
}

int main() {
  if (!all()) return 1;
  printf("plans ok\n");
  return 0;
}
