// The host side of drafted trees (kvops.hip, unchanged) on the stand-in HIP runtime: captures and replays, the order between streams, sizes of launches,
// calls that fail half-way.  Kernels are not run; a launch is an operation in its stream that notes that it ran.
//
// usage: trees_host_on_mock_hip NAME   (one of the checks in main; prints "ok")
#include "mock_device.h"

#include <cstdio>
#include <cstdlib>
#include <string>

struct Launched {
  std::string args;
  dim3 grid, block;
  int32_t groups, cols, layers;
  const void *parents, *count;
  bool ran;
};
static std::vector<Launched> launched;

#undef hipLaunchKernelGGL
#define hipLaunchKernelGGL(kern, grid, block, lds_bytes, stream, ...) record((grid), (block), (stream), __VA_ARGS__)
template <class Args, class... More>
void record(dim3 grid, dim3 block, hipStream_t st, const Args& a, const More&...);

#include "kvops.hip"

template <class Args, class... More>
void record(dim3 grid, dim3 block, hipStream_t st, const Args& a, const More&...) {
  const size_t at = launched.size();
  launched.push_back({"", grid, block, 0, 0, 0, nullptr, nullptr, false});
  if constexpr (std::is_same_v<Args, TreeArgs>) {
    launched[at].args = "tree";
    launched[at].parents = a.given;
  }
  if constexpr (std::is_same_v<Args, AcceptArgs>) {
    launched[at].args = "accept";
    launched[at].groups = a.groups;
    launched[at].cols = a.cols;
    launched[at].layers = a.layers;
    launched[at].count = a.count;
  }
  mockhip::enqueue(st, [at] { launched[at].ran = true; });
}

static long attended = 0, with_trees = 0;
template <typename E>
void launch_attn(bool, const AttnArgs& a, const kvswap::BatchPlan&, hipStream_t) {
  attended++;
  with_trees += a.sight && a.bits;
}
template <typename E>
void launch_join(const JoinArgs&, const kvswap::BatchPlan&, hipStream_t) {}
template <typename E>
void launch_weights(bool, const WeightArgs&, int, hipStream_t) {}
template void launch_attn<__bf16>(bool, const AttnArgs&, const kvswap::BatchPlan&, hipStream_t);
template void launch_attn<_Float16>(bool, const AttnArgs&, const kvswap::BatchPlan&, hipStream_t);
template void launch_join<__bf16>(const JoinArgs&, const kvswap::BatchPlan&, hipStream_t);
template void launch_join<_Float16>(const JoinArgs&, const kvswap::BatchPlan&, hipStream_t);
template void launch_weights<__bf16>(bool, const WeightArgs&, int, hipStream_t);
template void launch_weights<_Float16>(bool, const WeightArgs&, int, hipStream_t);

struct kv_pool {
  kvswap::PoolView v;
  int last_hip = 0;
};
namespace kvswap {
int pool_view(kv_pool* p, PoolView* out) { return *out = p->v, KV_OK; }
int pool_usable(kv_pool*) { return KV_OK; }
void pool_hip_error(kv_pool* p, int code) { p->last_hip = code; }
int pool_may_rewrite(kv_pool*, int32_t, const uint64_t*) { return KV_OK; }
long rewritten = 0;
std::vector<int32_t> unchanged;
void pool_rewritten(kv_pool*, int32_t n, const uint64_t*, const int32_t* u) { rewritten++, unchanged.assign(u, u + n); }
}  // namespace kvswap

#define CHECK(cond)                                                      \
  do {                                                                   \
    if (!(cond)) {                                                       \
      std::printf("FAILED %s:%d: %s\n", __FILE__, __LINE__, #cond);      \
      std::exit(1);                                                      \
    }                                                                    \
  } while (0)

namespace {

char* const kSomewhere = (char*)(uintptr_t)4096;  // stands for device memory that nothing here touches

struct World {
  kv_pool pool;
  hipStream_t s[3];
  kv_batch* b = nullptr;
  explicit World(int32_t L = 2, int32_t H = 2, int32_t D = 128, int32_t B = 16, int64_t N = 1 << 20) {
    mockhip::reset(1);
    const int64_t chunk = (int64_t)B * H * D * 2;
    pool.v = kvswap::PoolView{L, H, D, B, KV_BF16, N, kSomewhere, 2 * N * chunk, N * chunk, chunk, nullptr, 0, 0, 0, false, false, 256};
    for (hipStream_t& x : s) {
      CHECK(hipStreamCreateWithFlags(&x, hipStreamNonBlocking) == hipSuccess);
      all_streams.push_back(x);
    }
    mockhip::set_policy(mockhip::kLazy, nullptr);  // nothing runs before somebody waits for it
    CHECK(kv_batch_create(&pool, &b) == KV_OK);
    launched.clear();
  }
  // n requests of `tokens` tokens in blocks of their own, the last q of them a tree (not: they follow one another)
  int set(hipStream_t st, int32_t n, int32_t tokens, int32_t q, bool trees = true) {
    std::vector<int32_t> off{0}, ids, len, ql;
    for (int32_t i = 0; i < n; i++) {
      for (int32_t k = 0; k < (tokens + pool.v.B - 1) / pool.v.B; k++) ids.push_back((int32_t)(ids.size() % pool.v.N));
      off.push_back((int32_t)ids.size());
      len.push_back(tokens);
      ql.push_back(q);
    }
    return trees ? kv_batch_set_trees(b, n, off.data(), ids.data(), len.data(), ql.data(), pool.v.H, nullptr, (const int32_t*)kSomewhere, st)
                 : kv_batch_set(b, n, off.data(), ids.data(), len.data(), ql.data(), pool.v.H, st);
  }
  int attn(hipStream_t st) {
    kv_attn_args a{};
    a.struct_size = sizeof(a);
    a.io_dtype = KV_BF16;
    a.scale = 1.f;
    a.q = a.out = kSomewhere;
    return kv_attn(b, &a, st);
  }
  int accept(hipStream_t st, int32_t layers, const uint64_t* req_ids = nullptr) {
    kv_accept_args a{};
    a.struct_size = sizeof(a);
    a.num_layers = layers;
    a.tokens = a.chosen = (const int32_t*)kSomewhere;
    a.count = a.path = a.next = (int32_t*)kSomewhere;
    a.path_cap = KV_TREE_MAX;
    a.req_ids = req_ids;
    return kv_accept(b, &a, st);
  }
  ~World() {
    for (hipStream_t x : s) CHECK(hipStreamSynchronize(x) == hipSuccess);
    if (b) CHECK(kv_batch_destroy(b) == KV_OK);
    for (hipStream_t x : s) CHECK(hipStreamDestroy(x) == hipSuccess);
    all_streams.clear();
  }
};

// A batch's trees are worked out where it is set, once, and forgotten when it is set without.
void trees_of_a_batch() {
  World w;
  CHECK(w.set(w.s[0], 3, 40, 8) == KV_OK && launched.size() == 1 && launched[0].args == "tree" && launched[0].parents == kSomewhere);
  CHECK(w.attn(w.s[0]) == KV_OK && attended == 1 && with_trees == 1);
  CHECK(w.set(w.s[0], 3, 40, 8, false) == KV_OK && launched.size() == 1);
  CHECK(w.attn(w.s[0]) == KV_OK && attended == 2 && with_trees == 1);
  CHECK(w.set(w.s[0], 0, 0, 0) == KV_OK && launched.size() == 1);  // no requests
  CHECK(w.set(w.s[0], 3, 40, 0) == KV_OK && launched.size() == 1); // no rows
}

// As kv_batch_set: not in a capture, and behind replays of what was captured before.
void captures_and_replays() {
  World w;
  CHECK(w.set(w.s[0], 3, 40, 8) == KV_OK);
  CHECK(hipStreamSynchronize(w.s[0]) == hipSuccess);
  mockhip::begin_capture(w.s[0]);
  CHECK(w.set(w.s[0], 3, 40, 8) == KV_EINVAL && launched.size() == 1);
  const uint64_t ids[3] = {5, 6, 7};
  CHECK(w.accept(w.s[0], 2, ids) == KV_EINVAL && kvswap::rewritten == 0 && launched.size() == 1);
  CHECK(w.accept(w.s[0], 2) == KV_OK && launched.size() == 2 && launched[1].args == "accept");
  const mockhip::Graph g = mockhip::end_capture();
  launched[1].ran = false;
  mockhip::replay(w.s[1], g);
  const long waits = device_waits;
  CHECK(!launched[1].ran && w.set(w.s[0], 3, 40, 8) == KV_OK);
  CHECK(device_waits == waits + 1 && launched[1].ran);  // the replay is over before what it reads is replaced
  CHECK(w.accept(w.s[0], 2, ids) == KV_OK && kvswap::rewritten == 1);
  CHECK((kvswap::unchanged == std::vector<int32_t>{2, 2, 2}));  // tokens 33 .. may be written, in the third block
  // another stream's call comes behind the batch's own
  CHECK(w.set(w.s[0], 3, 40, 8) == KV_OK && w.accept(w.s[2], 2) == KV_OK);
  const size_t last = launched.size() - 1;
  CHECK(hipStreamSynchronize(w.s[2]) == hipSuccess && launched[last].ran && launched[last - 1].ran);
}

// Every plane of every request has its workgroup, and no launch more than the chip holds at a time but for one each.
void launches_of_an_acceptance() {
  for (int32_t L : {1, 2, 80})
    for (int32_t n : {1, 7, 300, 3000}) {
      World w(L, 8, 128, 16, 1 << 20);
      CHECK(w.set(w.s[0], n, 40, 8) == KV_OK && w.accept(w.s[0], L) == KV_OK);
      const Launched& l = launched.back();
      CHECK(l.cols == 1 && l.layers == L && l.groups >= 1 && l.groups <= 2 * L && (int64_t)l.grid.x == (int64_t)n * l.groups);
      CHECK(l.groups == 1 || l.grid.x <= 8u * 256);
      CHECK(w.accept(w.s[0], 0) == KV_OK && launched.back().grid.x == (unsigned)n && launched.back().layers == 0);
    }
  World without(2, 8, 128, 16, 1 << 20);
  CHECK(without.set(without.s[0], 5, 40, 8, false) == KV_OK && without.accept(without.s[0], 2) == KV_OK && launched.back().layers == 0);
  // rows of several workgroups
  World wide(2, 71, 256, 2, 1 << 16);
  CHECK(wide.set(wide.s[0], 5, 40, 8) == KV_OK && wide.accept(wide.s[0], 2) == KV_OK && launched.back().cols == (71 * 256 * 2 / 16 + 255) / 256);
}

// The largest trees of as many requests as a launch can have; one more is refused, and the batch stays as it was.
void launches_of_large_trees() {
  World w(1, 1, 64, 16, 1 << 12);
  // (a request of 1024 rows in 34 words each: 136 workgroups)
  const int32_t most = ((1 << 24) - 1) / 136;
  std::vector<int32_t> off((size_t)most + 2, 0), q((size_t)most + 1, 0), len((size_t)most + 1, 0), trees((size_t)most + 1, 0);
  std::vector<int32_t> ids(64);
  for (int k = 0; k < 64; k++) ids[k] = k;
  for (size_t i = 1; i < off.size(); i++) off[i] = 64;
  len[0] = 1024;
  q[0] = 1024;
  trees[0] = 1;
  const int32_t* parents = (const int32_t*)kSomewhere;
  CHECK(kv_batch_set_trees(w.b, most, off.data(), ids.data(), len.data(), q.data(), 1, trees.data(), parents, w.s[0]) == KV_OK);
  CHECK(launched.size() == 1 && (uint64_t)launched[0].grid.x * 256 < 1ull << 32);
  CHECK(kv_batch_set_trees(w.b, most + 1, off.data(), ids.data(), len.data(), q.data(), 1, trees.data(), parents, w.s[0]) == KV_EINVAL);
  kv_batch_info info{};
  info.struct_size = sizeof(info);
  CHECK(kv_batch_query(w.b, &info) == KV_OK && info.rows == 1024 && launched.size() == 1);
}

}  // namespace

int main(int, char** argv) {
  const std::string name = argv[1];
  if (name == "trees_of_a_batch") trees_of_a_batch();
  else if (name == "captures_and_replays") captures_and_replays();
  else if (name == "launches_of_an_acceptance") launches_of_an_acceptance();
  else if (name == "launches_of_large_trees") launches_of_large_trees();
  else return 2;
  std::printf("ok\n");
  return 0;
}
