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

// A padded batch: requests that draft, one that has nothing cached and one row, one without rows, and one whose new tokens are no tree.  What was in `path`
// goes from every row of a tree, and from no other.
void paths_of_padded_trees() {
  kvswap::BatchShape s;
  s.B = 4;
  s.H = 1;
  s.N = 64;
  const int n = 5, most = 6;
  const int32_t off[n + 1] = {0, 3, 3, 6, 9, 9}, ids[9] = {1, 2, 3, 4, 5, 6, 7, 8, 9}, len[n] = {10, 0, 9, 12, 0}, ql[n] = {4, 1, 0, 3, 1};
  const uint8_t trees[n] = {1, 1, 1, 0, 1};
  kvswap::BatchPlan p;
  CHECK(p.set(n, off, ids, len, ql, 1, s, trees) == KV_OK && p.T == 9);
  const int32_t parents[9] = {-1, 0, 1, -2, -1, 7, 7, 7, -2};
  std::vector<int32_t> parent(9), position(9), limit = p.tok_limit, tokens(9, 5), chosen(9, 5), count(n, -9), next(n, -9), path((size_t)n * most, -9);
  std::vector<uint32_t> bits((size_t)p.tree_words);
  TreeArgs t{p.tree_reqs.data(), parents, (p.tree_units + 255) / 256, parent.data(), position.data(), limit.data(), bits.data()};
  mockhip::run_grid(dim3((unsigned)(n * t.chunks)), dim3(256), 16, [&] { kv_tree_kernel(t); });
  AcceptArgs a{};
  a.reqs = p.tree_reqs.data();
  a.parent = parent.data();
  a.tokens = tokens.data();
  a.chosen = chosen.data();
  a.q_first = p.q_first.data();
  a.len = p.len.data();
  a.off = p.off.data();
  a.table = p.ids.data();
  a.count = count.data();
  a.path = path.data();
  a.next = next.data();
  a.path_stride = most;
  a.n = n;
  a.H = 1;
  a.B = s.B;
  a.row = 16;
  a.groups = a.cols = a.vecs = 1;
  mockhip::run_grid(dim3((unsigned)n), dim3(256), 16, [&] { kv_accept_kernel<u32x4, false, 1>(a); });
  CHECK((count == std::vector<int32_t>{3, 0, 0, 3, 0}) && (next == std::vector<int32_t>{5, -1, -1, 5, -1}));
  const std::vector<int32_t> want[n] = {{0, 1, 2, -1, -9, -9}, {-1, -9, -9, -9, -9, -9}, {-9, -9, -9, -9, -9, -9}, {-9, -9, -9, -9, -9, -9}, {-1, -9, -9, -9, -9, -9}};
  for (int i = 0; i < n; i++)
    for (int k = 0; k < most; k++) CHECK(path[i * most + k] == want[i][k]);
}

}  // namespace

int main(int, char** argv) {
  const std::string name = argv[1];
  if (name == "weights_of_rows_that_see_nothing") weights_of_rows_that_see_nothing();
  else if (name == "paths_of_padded_trees") paths_of_padded_trees();
  else return 2;
  std::printf("ok\n");
  return 0;
}
