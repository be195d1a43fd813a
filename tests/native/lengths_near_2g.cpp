// The plan of batches whose requests have nearly as many tokens as 32 bits count (batch.hpp): positions a little behind the last token are computed on the
// way, by the plan and by the kernels, so lengths that leave no room for these are refused.
//
// usage: lengths_near_2g   (prints "lengths ok")
#include <cstdio>
#include <vector>

#include "../../paper_2510_02758_amd/csrc/batch.hpp"

#define CHECK(cond)                                              \
  do {                                                           \
    if (!(cond)) {                                               \
      fprintf(stderr, "%s:%d: %s\n", __FILE__, __LINE__, #cond); \
      return 1;                                                  \
    }                                                            \
  } while (0)

int main() {
  const int32_t B = 1 << 20;
  kvswap::BatchShape s;
  s.B = B;
  s.N = 1 << 12;
  std::vector<int32_t> ids(2048);
  for (int32_t k = 0; k < 2048; k++) ids[k] = k;
  const int32_t off[2] = {0, 2048};
  const uint8_t tree = 1;
  for (int32_t q : {1, 40})
    for (const uint8_t* trees : {(const uint8_t*)nullptr, &tree})
      for (int32_t len : {INT32_MAX, INT32_MAX - 16, INT32_MAX - 100, INT32_MAX - 1023, INT32_MAX - 1024, INT32_MAX / 2}) {
        kvswap::BatchPlan p;
        const int rc = p.set(1, off, ids.data(), &len, &q, 1, s, trees);
        CHECK(rc == (len > INT32_MAX - 1024 ? KV_EINVAL : KV_OK));
        if (rc) continue;
        int64_t keys = 0;
        for (const kvswap::AttnItem& it : p.items) {
          CHECK(it.k0 >= 0 && it.k1 > it.k0 && it.k1 <= len && it.clear >= it.k0 && it.clear <= it.k1);
          keys += it.k1 - it.k0;
        }
        CHECK(keys == len && p.cached == len);
      }
  printf("lengths ok\n");
  return 0;
}
