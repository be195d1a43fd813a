// Batches with drafted trees that are padded to a fixed number of requests: the plan (batch.hpp) shares out the real requests' keys among workgroups as it
// does without the padding.
//
// usage: padded_drafts   (prints "plans ok")
#include <cstdio>
#include <vector>

#include "../../paper_2510_02758_amd/csrc/batch.hpp"

#define CHECK(cond, ...)                                                        \
  do {                                                                          \
    if (!(cond)) {                                                              \
      fprintf(stderr, "%s:%d: %s failed: ", __FILE__, __LINE__, #cond);         \
      fprintf(stderr, __VA_ARGS__);                                             \
      fprintf(stderr, "\n");                                                    \
      return false;                                                             \
    }                                                                           \
  } while (0)

// Keys of the workgroup of row tiles that has most, and workgroups with keys.
struct Shares {
  int64_t longest = 0, busy = 0, keys = 0;
};
static Shares shares(const std::vector<int32_t>& wgs, const kvswap::BatchPlan& p) {
  Shares s;
  for (size_t w = 0; w + 1 < wgs.size(); w++) {
    int64_t keys = 0;
    for (int32_t i = wgs[w]; i < wgs[w + 1]; i++) keys += p.items[i].k1 - p.items[i].k0;
    s.longest = std::max(s.longest, keys);
    s.busy += keys > 0;
    s.keys += keys;
  }
  return s;
}

// `n` requests of `tokens` tokens with `q` drafts, and `padded` of none with one row each: behind the others, in front of them, or between them.
static bool plan(int32_t B, int32_t D, int32_t H, int32_t G, int n, int32_t tokens, int32_t q, int padded, int where, Shares* rows, Shares* bigs) {
  const kvswap::BatchShape s = kvswap::batch_shape(H, D, B, 1 << 20, 256, false, true);
  std::vector<int32_t> off{0}, ids, len, ql;
  int real = 0, none = 0, next = 0;
  while (real < n || none < padded) {
    const bool pad = real == n || (none < padded && (where == 0 ? false : where == 1 ? true : (int64_t)none * n <= (int64_t)real * padded));
    if (pad)
      none++;
    else
      real++;
    for (int k = 0; !pad && k < (tokens + B - 1) / B; k++) ids.push_back(next++);
    off.push_back((int32_t)ids.size());
    len.push_back(pad ? 0 : tokens);
    ql.push_back(pad ? 1 : q);
  }
  std::vector<uint8_t> trees(len.size(), 1);
  kvswap::BatchPlan p;
  CHECK(p.set((int32_t)len.size(), off.data(), ids.data(), len.data(), ql.data(), G * H, s, trees.data()) == KV_OK, "refused");
  *rows = shares(p.wg_items, p);
  *bigs = shares(p.wg_big, p);
  CHECK(rows->keys + bigs->keys == (int64_t)n * tokens * ((int64_t)q * G > s.row_tile ? ((int64_t)q * G + s.big_tile - 1) / s.big_tile : 1), "%ld keys",
        (long)(rows->keys + bigs->keys));
  return true;
}

static bool all() {
  for (int32_t B : {16, 128})
    for (int32_t q : {4, 24})  // (row tiles, big ones)
      for (int32_t D : {64, 128})
        for (int n : {1, 8, 100})
          for (int padded : {1, 100, 128, 300, 1000})
            for (int where : {0, 1, 2}) {
              Shares rows, bigs, rows0, bigs0;
              if (!plan(B, D, 8, 4, n, 16000, q, 0, 0, &rows0, &bigs0) || !plan(B, D, 8, 4, n, 16000, q, padded, where, &rows, &bigs)) return false;
              // a padded request may end a workgroup early, which has the others take a little more, but never twice as much
              CHECK(rows.longest <= rows0.longest * 3 / 2 && bigs.longest <= bigs0.longest * 3 / 2,
                    "B %d, D %d, %d requests with %d drafts, %d padded (%d): %ld and %ld keys at most, %ld and %ld without", B, D, n, q, padded, where,
                    (long)rows.longest, (long)bigs.longest, (long)rows0.longest, (long)bigs0.longest);
              CHECK(rows.busy * 3 >= rows0.busy * 2 && bigs.busy * 3 >= bigs0.busy * 2, "%d padded (%d): %ld and %ld workgroups have keys, %ld and %ld without", padded,
                    where, (long)rows.busy, (long)bigs.busy, (long)rows0.busy, (long)bigs0.busy);
            }
  return true;
}

int main() {
  if (!all()) return 1;
  printf("plans ok\n");
  return 0;
}
