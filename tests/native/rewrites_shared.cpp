// BatchPlan::rewrites_shared against a plain count, over random batches whose blocks repeat within a request, between requests that are
// rewritten and between these and others, asked several times with other bounds.  Prints "checks ok" and how many reached a shared block.
#include <cstdio>
#include <cstdlib>
#include <map>
#include <random>

#include "../../paper_2510_02758_amd/csrc/batch.hpp"

int main() {
  long asked = 0, shared = 0;
  for (int seed = 0; seed < 3000; seed++) {
    std::mt19937 rng(seed);
    auto pick = [&](int lo, int hi) { return lo + (int)(rng() % (unsigned)(hi - lo + 1)); };
    const int B = pick(1, 5), N = pick(60, 400), n = pick(0, 6);
    std::vector<int32_t> off{0}, ids, len, q;
    int fresh = 0;
    for (int i = 0; i < n; i++) {
      const int tokens = pick(0, 40);
      for (int k = 0; k < (tokens + B - 1) / B; k++) ids.push_back(pick(0, 30) && fresh < N ? fresh++ : pick(0, N - 1));
      if (i && pick(0, 2) == 0)  // begins as the one before
        for (size_t k = 0; k < 3 && (size_t)off[i] + k < ids.size() && off[i - 1] + (int)k < off[i]; k++) ids[off[i] + k] = ids[off[i - 1] + k];
      off.push_back((int32_t)ids.size());
      len.push_back(tokens);
      q.push_back(std::min(tokens, pick(0, 1)));
    }
    kvswap::BatchPlan p;
    if (p.set(n, off.data(), ids.data(), len.data(), q.data(), 2, kvswap::batch_shape(1, 64, B, N, 256, false)) != KV_OK) return 1;
    std::map<int, int> times;
    for (int32_t id : ids) times[id]++;
    for (int turn = 0; turn < 4; turn++) {
      const int keep = pick(0, 40), first = pick(0, keep) / B, blocks = (keep + B - 1) / B;
      bool want = false;
      for (int i = 0; i < n; i++)
        for (int k = first; len[i] > keep && k < blocks; k++) want = want || times[ids[off[i] + k]] > 1;
      if (p.rewrites_shared(keep, first, blocks) != want) {
        std::printf("FAILED seed %d turn %d: want %d\n", seed, turn, want);
        return 1;
      }
      asked++;
      shared += want;
    }
  }
  std::printf("checks ok: %ld of %ld reach a shared block\n", shared, asked);
  return shared > 1000 && shared < asked - 1000 ? 0 : 1;
}
