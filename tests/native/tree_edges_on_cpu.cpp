// The operators' kernels for drafted trees (sources unchanged, lane by lane) where their batches and values have edges: rows of no tree and weights, padded
// requests and paths, scales far apart.
//
// usage: tree_edges_on_cpu NAME   (one of the checks in main; prints "ok")
#include "mock_device.h"

#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <limits>
#include <string>
#include <vector>

#undef __shared__
#define __shared__ static  // one workgroup at a time, its lanes share it

#include "pool_view.hpp"
#include "attn.hpp"
#include "attn_sum.hip.inc"
#include "append.hip.inc"
#include "tree.hip.inc"

#define CHECK(cond)                                                 \
  do {                                                              \
    if (!(cond)) {                                                  \
      std::printf("FAILED %s:%d: %s\n", __FILE__, __LINE__, #cond); \
      std::exit(1);                                                 \
    }                                                               \
  } while (0)

namespace {

constexpr float kInf = std::numeric_limits<float>::infinity(), kNan = std::numeric_limits<float>::quiet_NaN();

// A row that sees nothing gives no weight, whatever its products with the keys are: of a query of zeros and a key that is not finite they are NaN.
void weights_of_rows_that_see_nothing() {
  const int keys = 40, G = 2, tokens = 3, rows = tokens * G, score_row = 48;
  const kvswap::ScoreItem item{0, 0, keys, 0, score_row, 0, 0, rows};
  const int32_t q_first[2] = {0, tokens};
  std::vector<float> scores((size_t)rows * score_row), lse((size_t)tokens * G), weights((size_t)keys, 1.f), want((size_t)keys, 1.f);
  for (int r = 0; r < rows; r++) {
    const bool none = r / G == 1;  // the second token is in no tree
    lse[r] = none ? -kInf : 0.25f * r;
    for (int x = 0; x < score_row; x++) {
      float& s = scores[(size_t)r * score_row + x];
      s = none ? (x % 3 == 0 ? kNan : x % 3 == 1 ? kInf : 0.f) : x == 7 ? -kInf : 0.125f * (x - r);
      if (!none && x < keys) want[x] += exp2f(fmaf(s, 0.5f, -lse[r] * 1.4426950408889634f));
    }
  }
  SumArgs a{&item, q_first, scores.data(), 0, lse.data(), G, weights.data(), 0, 0, 0.5f, 1, G};
  mockhip::run_grid(dim3(1), dim3(256), 16, [&] { kv_attn_sum_kernel(a); });
  for (int x = 0; x < keys; x++) CHECK(std::fabs(weights[x] - want[x]) <= 1e-5f * want[x]);
}

}  // namespace

int main(int, char** argv) {
  const std::string name = argv[1];
  if (name == "weights_of_rows_that_see_nothing") weights_of_rows_that_see_nothing();
  else return 2;
  std::printf("ok\n");
  return 0;
}
