// The host side of the operators on the pool's contents (kvops.hip, unchanged) on the stand-in HIP runtime: order between calls, captures and
// replays, workspaces, launches.  Kernels are not run; a launch is an operation in its stream that notes what it would have read.
//
// usage: ops_on_mock_hip NAME   (one of the checks in main; prints "ok")
#include "mock_device.h"

#include <cstdio>
#include <string>

struct Launched {
  std::string kernel;
  dim3 grid, block;
  const void *turns, *pool, *kept;
  int32_t first_len;  // the batch's first length, as the launch found it in the tables when it ran (evictions)
  bool ran;
};
static std::vector<Launched> launched;

#undef hipLaunchKernelGGL
#define hipLaunchKernelGGL(kern, grid, block, lds_bytes, stream, ...) record(#kern, (grid), (block), (stream), __VA_ARGS__)
template <class Args, class... More>
void record(const char* kernel, dim3 grid, dim3 block, hipStream_t st, const Args& a, const More&...);

#include "kvops.hip"

template <class Args, class... More>
void record(const char* kernel, dim3 grid, dim3 block, hipStream_t st, const Args& a, const More&...) {
  const size_t at = launched.size();
  launched.push_back({kernel, grid, block, nullptr, nullptr, nullptr, -1, false});
  const int32_t* len = nullptr;
  if constexpr (std::is_same_v<Args, EvictArgs>) {
    launched[at].turns = a.turns;
    launched[at].pool = a.pool;
    launched[at].kept = a.kept;
    len = a.len;
  }
  mockhip::enqueue(st, [at, len] {
    launched[at].ran = true;
    if (len) launched[at].first_len = len[0];
  });
}

// The attention's tiles are in files of their own.
static std::vector<int32_t> tables_seen;
template <typename E>
void launch_attn(bool, const AttnArgs& a, const kvswap::BatchPlan&, hipStream_t st) {
  const int32_t* table = a.table;
  mockhip::enqueue(st, [table] { tables_seen.push_back(table[0]); });
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

// A pool handle as far as the operators look at one.
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
void pool_rewritten(kv_pool*, int32_t, const uint64_t*, const int32_t*) { rewritten++; }
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
  }
  // n requests of `tokens` tokens in blocks of their own, from block `first` on
  int set(hipStream_t st, int32_t n, int32_t tokens, int32_t first = 0) {
    std::vector<int32_t> off{0}, ids, len, q;
    for (int32_t i = 0; i < n; i++) {
      for (int32_t k = 0; k < (tokens + pool.v.B - 1) / pool.v.B; k++) ids.push_back(first + (int32_t)ids.size());
      off.push_back((int32_t)ids.size());
      len.push_back(tokens);
      q.push_back(1);
    }
    return kv_batch_set(b, n, off.data(), ids.data(), len.data(), q.data(), pool.v.H, st);
  }
  int attn(hipStream_t st, bool weights = false) {
    kv_attn_args a{};
    a.struct_size = sizeof(a);
    a.io_dtype = KV_BF16;
    a.scale = 1.f;
    a.q = a.out = kSomewhere;
    if (weights) {
      a.weights = (float*)kSomewhere;
      a.weights_cap = 1 << 30;
    }
    return kv_attn(b, &a, st);
  }
  int append(hipStream_t st) {
    kv_append_args a{};
    a.struct_size = sizeof(a);
    a.io_dtype = KV_BF16;
    a.k = a.v = kSomewhere;
    return kv_append(b, &a, st);
  }
  int evict(hipStream_t st, int32_t keep, const uint64_t* req_ids = nullptr) {
    kv_evict_args a{};
    a.struct_size = sizeof(a);
    a.num_layers = pool.v.L;
    a.keep = keep;
    a.weights = (const float*)kSomewhere;
    a.kept = (int32_t*)kSomewhere;
    a.weights_cap = 1 << 30;
    a.req_ids = req_ids;
    return kv_evict(b, &a, st);
  }
  ~World() {
    for (hipStream_t x : s) CHECK(hipStreamSynchronize(x) == hipSuccess);
    if (b) CHECK(kv_batch_destroy(b) == KV_OK);
    for (hipStream_t x : s) CHECK(hipStreamDestroy(x) == hipSuccess);
    all_streams.clear();
  }
};

// A replay that is under way on another stream reads the tables it was captured with: a new batch, or the end of this one, comes after it.
void replay_then_set() {
  World w;
  CHECK(w.set(w.s[0], 3, 40, 100) == KV_OK);
  CHECK(hipStreamSynchronize(w.s[0]) == hipSuccess);
  mockhip::begin_capture(w.s[0]);
  CHECK(w.attn(w.s[0]) == KV_OK);
  const mockhip::Graph g = mockhip::end_capture();
  mockhip::replay(w.s[1], g);
  mockhip::replay(w.s[1], g);
  CHECK(tables_seen.empty());
  CHECK(w.set(w.s[0], 3, 40, 500) == KV_OK);
  CHECK(hipStreamSynchronize(w.s[0]) == hipSuccess);  // the new tables are there
  CHECK(hipStreamSynchronize(w.s[1]) == hipSuccess);
  CHECK((tables_seen == std::vector<int32_t>{100, 100}));
  // without a capture since, nothing waits for the device
  CHECK(device_waits == 1 && w.attn(w.s[0]) == KV_OK && w.set(w.s[0], 3, 40, 900) == KV_OK && device_waits == 1);
  mockhip::begin_capture(w.s[0]);
  CHECK(w.attn(w.s[0]) == KV_OK);
  const mockhip::Graph g2 = mockhip::end_capture();
  CHECK(hipStreamSynchronize(w.s[0]) == hipSuccess);
  tables_seen.clear();
  mockhip::replay(w.s[2], g2);
  CHECK(kv_batch_destroy(w.b) == KV_OK);
  w.b = nullptr;
  CHECK((tables_seen == std::vector<int32_t>{900}));
}

// Tickets are for direct calls alone, also once there is room for them.
void captures_draw_no_tickets() {
  World w;
  CHECK(w.set(w.s[0], 2, 4000) == KV_OK);
  CHECK(w.evict(w.s[0], 2000) == KV_OK);
  CHECK(launched.size() == 2 && launched[1].turns);
  mockhip::begin_capture(w.s[0]);
  CHECK(w.evict(w.s[0], 2000) == KV_OK);
  mockhip::end_capture();
  CHECK(launched.size() == 4 && !launched[2].turns && !launched[3].turns && launched[3].grid.x == 2u * 2 * 2 * 2);
  CHECK(w.evict(w.s[0], 2000) == KV_OK);
  CHECK(launched.size() == 6 && launched[5].turns);
}

// An error that another part of the program has left behind is none of the call's: an eviction would stop between its two launches.
void an_earlier_error() {
  World w;
  auto leave_error = [] { CHECK(hipFree(kSomewhere) != hipSuccess); };
  CHECK(w.set(w.s[0], 2, 4000) == KV_OK);
  leave_error();
  CHECK(w.append(w.s[0]) == KV_OK);
  leave_error();
  CHECK(w.attn(w.s[0], true) == KV_OK);
  leave_error();
  launched.clear();
  CHECK(w.evict(w.s[0], 2000) == KV_OK && launched.size() == 2);
  mockhip::fail_after(1, hipErrorInvalidValue);  // (an injected failure: the launch's own)
  CHECK(w.append(w.s[0]) == KV_EHIP && w.pool.last_hip == hipErrorInvalidValue);
}

// Calls allocate nothing but the first room that one of them wants, free nothing, and do not wait: kv_batch_set grows what has been wanted.
void room_is_grown_by_set() {
  World w;
  auto calls = [&] { return mockhip::resource_calls(); };
  CHECK(w.set(w.s[0], 2, 300) == KV_OK);
  const long waits = mockhip::host_waits();
  long before = calls();
  CHECK(w.attn(w.s[0], true) == KV_OK && calls() == before + 1);
  CHECK(w.evict(w.s[0], 140) == KV_OK && launched.back().turns && calls() == before + 2);
  CHECK(w.attn(w.s[0], true) == KV_OK && w.evict(w.s[0], 140) == KV_OK && calls() == before + 2 && mockhip::host_waits() == waits);
  CHECK(w.set(w.s[0], 9, 9000) == KV_OK);
  const long waits_then = mockhip::host_waits();
  before = calls();
  CHECK(w.attn(w.s[0], true) == KV_OK && w.evict(w.s[0], 5000) == KV_OK && launched.back().turns);
  CHECK(calls() == before && mockhip::host_waits() == waits_then);
  // a first call in a capture takes nothing; the first one outside does
  World other;
  CHECK(other.set(other.s[0], 2, 300) == KV_OK);
  before = calls();
  mockhip::begin_capture(other.s[0]);
  CHECK(other.attn(other.s[0], true) == KV_OK && other.evict(other.s[0], 140) == KV_OK && calls() == before);
  mockhip::end_capture();
  CHECK(other.attn(other.s[0], true) == KV_OK && other.evict(other.s[0], 140) == KV_OK && calls() == before + 2);
}

// A kv_batch_set that fails on the device's side leaves a batch without requests, whose calls do nothing; the next one is good.
void set_that_fails() {
  for (int n = 1;; n++) {
    World w;
    CHECK(w.set(w.s[0], 2, 300, 7) == KV_OK && w.attn(w.s[0], true) == KV_OK && w.evict(w.s[1], 140) == KV_OK);
    CHECK(hipStreamSynchronize(w.s[0]) == hipSuccess && hipStreamSynchronize(w.s[1]) == hipSuccess);
    mockhip::fail_after(n, hipErrorInvalidValue);
    const int rc = w.set(w.s[2], 40, 9000, 7);
    const bool fired = mockhip::failure_fired();
    mockhip::fail_after(0, 0);
    if (!fired) {
      CHECK(rc == KV_OK && n > 4);
      return;
    }
    CHECK(rc == KV_EHIP && w.pool.last_hip == hipErrorInvalidValue);
    tables_seen.clear();
    launched.clear();
    kv_batch_info info{sizeof(kv_batch_info)};
    CHECK(kv_batch_query(w.b, &info) == KV_OK && info.rows == 0 && info.cached_tokens == 0);
    CHECK(w.attn(w.s[0], true) == KV_OK && w.append(w.s[0]) == KV_OK && w.evict(w.s[0], 140) == KV_OK && launched.empty());
    CHECK(w.set(w.s[0], 2, 300, 9) == KV_OK && w.attn(w.s[0], true) == KV_OK && w.evict(w.s[0], 140) == KV_OK && launched.size() >= 2);
    CHECK(hipStreamSynchronize(w.s[0]) == hipSuccess && (tables_seen == std::vector<int32_t>{9}));
  }
}

// Host copies go stale when an eviction's call says so, which a replay cannot: none is captured with requests.
void captured_evictions_have_no_requests() {
  World w;
  const uint64_t ids[2] = {5, 6};
  CHECK(w.set(w.s[0], 2, 300) == KV_OK && w.evict(w.s[0], 140, ids) == KV_OK && kvswap::rewritten == 1);
  const size_t before = launched.size();
  mockhip::begin_capture(w.s[0]);
  CHECK(w.evict(w.s[0], 140, ids) == KV_EINVAL && launched.size() == before && kvswap::rewritten == 1);
  CHECK(w.evict(w.s[0], 140) == KV_OK && launched.size() == before + 2);
  mockhip::end_capture();
}

// A launch has fewer than 2^32 lanes; an eviction that needs more goes through its layers in parts, each selected and moved.
void launches_of_a_large_eviction() {
  World w(80, 8, 128, 16, 1 << 20);
  const int32_t n = 512, keep = 4000;
  CHECK(w.set(w.s[0], n, 5000) == KV_OK && w.evict(w.s[0], keep) == KV_OK);
  const int64_t chunks = (keep + 127) / 128;  // 32 KB of rows of 256 bytes
  int64_t moved = 0, layer = 0;
  CHECK(launched.size() >= 4 && launched.size() % 2 == 0);
  for (size_t i = 0; i < launched.size(); i += 2) {
    for (size_t j = i; j < i + 2; j++) {
      CHECK((uint64_t)launched[j].grid.x * launched[j].block.x < 1ull << 32);
      CHECK(launched[j].pool == kSomewhere + layer * w.pool.v.ls && launched[j].kept == (const int32_t*)kSomewhere);
    }
    CHECK(launched[i + 1].grid.x == launched[i].grid.x * 2 * chunks && launched[i + 1].turns);
    moved += launched[i + 1].grid.x;
    layer += launched[i].grid.x / (n * 8);
  }
  CHECK(layer == 80 && moved == 80 * n * 8 * 2 * chunks);
  // more heads than a launch can have: refused, nothing launched
  World many(1, 1 << 15, 8, 2, 1 << 10);
  launched.clear();
  CHECK(many.set(many.s[0], 300, 2) == KV_OK && many.evict(many.s[0], 1) == KV_EINVAL && launched.empty());
}

// The kernels' angles of far positions: products that wrap around are taken without a sign (run under the sanitizer; no lane sees another's).
void far_positions() {
  uint16_t k[8] = {}, v[8] = {}, pool[2 * 8] = {};
  const int64_t turns[4] = {(int64_t)1 << 61, 123456789012345678, -1, INT64_MIN};
  for (const int32_t pos : {2000000000, -2000000000, INT32_MIN, 0}) {
    const kvswap::TokenPlace place{0, 0, pos, 0};
    AppendArgs a{};
    a.k = (const char*)k;
    a.v = (const char*)v;
    a.turns = turns;
    a.positions = pos ? &pos : nullptr;
    a.places = &place;
    a.pool = (char*)pool;
    a.vk = sizeof(pool) / 2;
    a.magnitude = 1;
    a.rot = a.D = 8;
    a.H = a.chunks = a.pairs = a.units = a.interleaved = 1;
    mockhip::run_grid(dim3(1), dim3(256), 0, [&] { kv_append_kernel<__bf16, false>(a); });
    mockhip::run_grid(dim3(1), dim3(256), 0, [&] { kv_append_wide_kernel<__bf16, false>(a); });
  }
}

}  // namespace

int main(int, char** argv) {
  const std::string name = argv[1];
  if (name == "replay_then_set") replay_then_set();
  else if (name == "captures_draw_no_tickets") captures_draw_no_tickets();
  else if (name == "an_earlier_error") an_earlier_error();
  else if (name == "launches_of_a_large_eviction") launches_of_a_large_eviction();
  else if (name == "room_is_grown_by_set") room_is_grown_by_set();
  else if (name == "far_positions") far_positions();
  else if (name == "set_that_fails") set_that_fails();
  else if (name == "captured_evictions_have_no_requests") captured_evictions_have_no_requests();
  else return 2;
  std::printf("ok\n");
  return 0;
}
