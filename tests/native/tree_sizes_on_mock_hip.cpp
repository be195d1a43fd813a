// Sizes of drafted batches that no launch could have, on the stand-in HIP runtime: they are refused before anything is computed from them.
//
// usage: tree_sizes_on_mock_hip   (prints "ok")
#define main checks_of_trees_host
#include "trees_host_on_mock_hip.cpp"
#undef main

int main() {
  World w(1, 1, 64, 16, 1 << 12);
  const int32_t n = 40000;
  std::vector<int32_t> off((size_t)n + 1, 0), ids(64, 0), len((size_t)n, 0), q((size_t)n, 0), trees((size_t)n, 0);
  for (size_t i = 1; i < off.size(); i++) off[i] = 64;
  const int32_t* parents = (const int32_t*)kSomewhere;
  auto set = [&] { return kv_batch_set_trees(w.b, n, off.data(), ids.data(), len.data(), q.data(), 1, trees.data(), parents, w.s[0]); };
  len[0] = 1000;
  q[0] = 10;
  trees[0] = 1;
  CHECK(set() == KV_OK && launched.size() == 1);
  // workgroups of such trees, times the requests, are more than 63 bits count
  for (int32_t rows : {INT32_MAX, INT32_MAX - 126, 1 << 30, KV_TREE_MAX + 1, -1, INT32_MIN}) {
    q[0] = rows;
    for (int32_t tokens : {1000, INT32_MAX}) {
      len[0] = tokens;
      CHECK(set() == KV_EINVAL && launched.size() == 1);
    }
  }
  // neither are as many rows that follow one another; what was set stays
  trees[0] = 0;
  q[0] = INT32_MAX;
  CHECK(set() == KV_EINVAL && launched.size() == 1);
  kv_batch_info info{};
  info.struct_size = sizeof(info);
  CHECK(kv_batch_query(w.b, &info) == KV_OK && info.rows == 10);
  std::printf("ok\n");
  return 0;
}
