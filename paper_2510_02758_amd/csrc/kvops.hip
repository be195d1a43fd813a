// C ABI of the operators on the pool's contents (declared in include/kvswap.h): the batch, rotary append, attention, eviction, accepted drafts.
// Host side of each call: check everything, then a few launches on the caller's stream: one for kv_append and kv_accept, two for kv_evict (two for
// each part of its layers where all of them need more workgroups than a launch can have), for kv_attn one or two for the tiles, one for their join
// and up to two for the weights.  Nothing waits on the host outside kv_batch_create, kv_batch_set and kv_batch_destroy, and nothing is
// allocated there but the first room for kept products and for the order of moves, when they are first needed.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstring>
#include <mutex>
#include <new>
#include <stdexcept>
#include <type_traits>
#include <utility>
#include <vector>

#include "pool_view.hpp"
#include "attn.hpp"

#include "attn_sum.hip.inc"
#include "append.hip.inc"
#include "evict.hip.inc"
#include "tree.hip.inc"

using kvswap::AttnItem;
using kvswap::BatchPlan;
using kvswap::PoolView;
using kvswap::ScoreItem;
using kvswap::TokenPlace;
using kvswap::WeightItem;

struct kv_batch {
  kv_pool* pool = nullptr;
  PoolView v{};
  BatchPlan plan;
  int32_t max_len = 0;

  // Device copy of the plan, one allocation that grows; `up` are the two pinned buffers that it is uploaded from in turn.
  char* mem = nullptr;
  size_t mem_cap = 0;
  char* up[2] = {nullptr, nullptr};
  size_t up_cap[2] = {0, 0};
  hipEvent_t up_ev[2] = {nullptr, nullptr};
  bool up_busy[2] = {false, false};
  int turn = 0;
  const int32_t *wg_items = nullptr, *wg_big = nullptr, *wreqs = nullptr, *table = nullptr, *off = nullptr, *len = nullptr, *q_first = nullptr, *limit = nullptr, *lists = nullptr,
                *join_off = nullptr, *join = nullptr;
  const AttnItem* items = nullptr;
  const WeightItem *witems = nullptr, *wrest = nullptr;
  const ScoreItem* sitems = nullptr;
  const TokenPlace* places = nullptr;
  const kvswap::TreeReq* tree_reqs = nullptr;
  const kvswap::TreeSight* tree_sight = nullptr;
  int32_t max_tree = 0;  // rows of the largest tree

  // Partial results and, for callers that want weights without lse, the lse.
  char* ws = nullptr;
  size_t ws_cap = 0;
  float *part_o = nullptr, *lse = nullptr;
  float2* part_ml = nullptr;
  // Drafted trees: parents that can be relied on, positions by depth, what the rows see.
  int32_t *parent = nullptr, *position = nullptr;
  uint32_t* bits = nullptr;

  // Products of row tiles that the weights are computed from, and tickets of an eviction's chunks.  The first call that wants one of them takes it
  // (not in a capture); from then on kv_batch_set sees to it that there is room for its batch.
  struct Room {
    char* at = nullptr;
    size_t cap = 0;
    bool wanted = false;
  } scores, turns;

  // The stream of the newest work; another stream's call waits for what is on it.
  bool used = false;
  hipStream_t last = nullptr;
  hipEvent_t ev = nullptr;
  bool captured = false;  // a capture has taken calls since the batch was set: replays may be under way on any stream
};

namespace {

int fail(kv_batch* b, hipError_t e) {
  kvswap::pool_hip_error(b->pool, (int)e);
  return KV_EHIP;
}
#define OPCHK(b, expr)                       \
  do {                                       \
    hipError_t e_ = (expr);                  \
    if (e_ != hipSuccess) return fail(b, e_); \
  } while (0)

int caught() noexcept {
  try {
    throw;
  } catch (const std::bad_alloc&) {
    return KV_ENOMEM;
  } catch (const std::length_error&) {
    return KV_ENOMEM;
  } catch (...) {
    return KV_EINVAL;
  }
}

bool is_capturing(hipStream_t st) {
  hipStreamCaptureStatus s = hipStreamCaptureStatusNone;
  return hipStreamIsCapturing(st, &s) != hipSuccess || s != hipStreamCaptureStatusNone;
}

// While it lives, calls that wait do not invalidate a capture that another thread is at (in the global mode).
struct Relaxed {
  hipStreamCaptureMode mode = hipStreamCaptureModeRelaxed;
  const bool changed = hipThreadExchangeStreamCaptureMode(&mode) == hipSuccess;
  ~Relaxed() {
    if (changed) (void)hipThreadExchangeStreamCaptureMode(&mode);
  }
};

// Room of `need` bytes that nobody uses; none if there is not that much memory.
void take(kv_batch::Room& r, size_t need) {
  if (hipMalloc((void**)&r.at, need + need / 4) == hipSuccess) {
    r.cap = need + need / 4;
  } else {
    (void)hipGetLastError();
    r.at = nullptr;
  }
}

// In a call: is there room?  Only the first call of all may take some: kv_batch_set has grown what has been wanted before as far as it could.
bool has_room(kv_batch::Room& r, size_t need, hipStream_t st) {
  const bool first = !r.wanted;
  r.wanted = true;
  if (need <= r.cap) return true;
  if (is_capturing(st)) {
    r.wanted = !first || r.at;  // (the next call that is not captured is the first)
    return false;
  }
  if (!first) return false;
  Relaxed relaxed;
  take(r, need);
  return need <= r.cap;
}

// Room for the batch's kept products.
size_t scores_need(const kv_batch* b) { return (size_t)b->plan.scores * b->v.H * 4; }

// Bytes of an element of the pool, and rows of a chunk of an eviction's moves (0: moves are not made in chunks).
int32_t elem(const PoolView& v) { return v.dtype == KV_FP8_E4M3 ? 1 : 2; }
constexpr int kMoveUnroll = 8;
int32_t chunk_rows(const PoolView& v) {
  const int32_t bytes = v.D * elem(v), most = bytes % 16 ? 0 : std::min(kMoveRows, kMoveUnroll * (256 / (bytes / 16)));
  return v.has_scale ? most / v.B * v.B : most;
}

// Room for the tickets of any eviction of this batch.
size_t turns_need(const kv_batch* b) {
  const int32_t rows = chunk_rows(b->v);
  return rows ? (size_t)b->v.L * b->plan.n * b->v.H * 2 * (2 + (size_t)b->max_len / rows) * 4 : 0;
}

// Puts `st` behind the batch's work on another stream.  The checks behind the launches read the thread's last HIP error, which any earlier
// call of the application may have left behind (an event query that said "not ready" is enough): it is cleared first.
int order(kv_batch* b, hipStream_t st) {
  const bool capturing = is_capturing(st);
  if (b->used && b->last != st) {
    if (capturing || is_capturing(b->last)) return KV_EINVAL;
    OPCHK(b, hipEventRecord(b->ev, b->last));
    OPCHK(b, hipStreamWaitEvent(st, b->ev, 0));
  }
  b->used = true;
  b->last = st;
  b->captured = b->captured || capturing;
  (void)hipGetLastError();
  return KV_OK;
}

// Waits for replays of captured calls, which may be on any stream, before what they read is changed or freed.
int settle(kv_batch* b) {
  if (!b->captured) return KV_OK;
  OPCHK(b, hipDeviceSynchronize());
  b->captured = false;
  return KV_OK;
}

int drain(kv_batch* b) {
  if (b->used) OPCHK(b, hipStreamSynchronize(b->last));
  return KV_OK;
}

// Workgroups of 256 lanes that one launch may have: its lanes are counted in 32 bits.
constexpr int64_t kMostWgs = (1 << 24) - 1;

size_t padded(size_t bytes) { return (bytes + 63) / 64 * 64; }

// x / B by a product for 0 <= x < 2^31.
DivBy division(int32_t B) {
  int sh = 0;
  while ((1ll << sh) < B) sh++;
  return {sh ? (uint32_t)(((1ull << (31 + sh)) + B - 1) / B) : 0, (uint32_t)(sh ? sh - 1 : 32)};
}

KvSide side(const kv_batch* b, int32_t layer) {
  const PoolView& v = b->v;
  KvSide s{};
  const int e = elem(v);
  s.k = v.pool + layer * v.ls;
  s.vk = v.ks;
  s.bs = v.bs;
  s.ks = v.scale ? v.scale + layer * v.sls : nullptr;
  s.vks = v.sks;
  s.sbs = v.sbs;
  s.row = v.H * v.D * e;
  s.head = v.D * e;
  s.D = v.D;
  s.B = v.B;
  s.by_b = division(v.B);
  return s;
}

bool io_fits(const PoolView& v, int32_t io) { return io == (v.dtype == KV_FP8_E4M3 ? (io == KV_F16 ? KV_F16 : KV_BF16) : v.dtype); }

bool aligned(const void* p, const int64_t* strides, int bytes) {
  const int el = bytes / 2;
  return (uintptr_t)p % bytes == 0 && strides[0] % el == 0 && strides[1] % el == 0;
}

}  // namespace

extern "C" {

int kv_batch_create(kv_pool* p, kv_batch** out) try {
  if (!p || !out) return KV_EINVAL;
  *out = nullptr;
  PoolView v;
  int rc = kvswap::pool_view(p, &v);
  if (rc) return rc;
  if (v.D % 8 || v.D > 256 || (v.D > 128 && v.D % 16)) return KV_EINVAL;
  kv_batch* b = new (std::nothrow) kv_batch;
  if (!b) return KV_ENOMEM;
  b->pool = p;
  b->v = v;
  if (!v.plan_only) {
    hipEvent_t* all[3] = {&b->ev, &b->up_ev[0], &b->up_ev[1]};
    for (hipEvent_t* e : all) {
      const hipError_t er = hipEventCreateWithFlags(e, hipEventDisableTiming);
      if (er != hipSuccess) {
        kvswap::pool_hip_error(p, (int)er);
        (void)kv_batch_destroy(b);
        return KV_EHIP;
      }
    }
  }
  *out = b;
  return KV_OK;
}
catch (...) {
  return caught();
}

int kv_batch_destroy(kv_batch* b) try {
  if (!b) return KV_EINVAL;
  int rc = KV_OK;
  if (!b->v.plan_only) {  // (the pool may be gone: it is not touched)
    Relaxed relaxed;
    if (b->captured ? hipDeviceSynchronize() != hipSuccess : b->used && hipStreamSynchronize(b->last) != hipSuccess) rc = KV_EHIP;
    for (hipEvent_t e : {b->ev, b->up_ev[0], b->up_ev[1]})
      if (e) (void)hipEventDestroy(e);
    for (char* u : b->up)
      if (u) (void)hipHostFree(u);
    if (b->mem) (void)hipFree(b->mem);
    if (b->ws) (void)hipFree(b->ws);
    if (b->scores.at) (void)hipFree(b->scores.at);
    if (b->turns.at) (void)hipFree(b->turns.at);
  }
  delete b;
  return rc;
}
catch (...) {
  return caught();
}

}  // extern "C"

namespace {

// `trees`: null without drafted ones; else of each request, whether its new tokens are one.
int set_batch(kv_batch* b, int32_t n, const int32_t* offsets, const int32_t* block_ids, const int32_t* num_tokens, const int32_t* q_lens,
              int32_t num_q_heads, const uint8_t* trees, const int32_t* parents, void* stream) {
  int rc = kvswap::pool_usable(b->pool);
  if (rc) return rc;
  hipStream_t st = (hipStream_t)stream;
  if (!b->v.plan_only && (is_capturing(st) || (b->used && b->last != st && is_capturing(b->last)))) return KV_EINVAL;
  BatchPlan& pl = b->plan;
  Relaxed relaxed;
  rc = settle(b);
  if (rc) {
    pl.n = pl.T = 0;
    return rc;
  }
  rc = pl.set(n, offsets, block_ids, num_tokens, q_lens, num_q_heads,
              kvswap::batch_shape(b->v.H, b->v.D, b->v.B, b->v.N, b->v.cus, b->v.dtype == KV_FP8_E4M3, trees != nullptr), trees);
  if (rc) return rc;
  b->max_len = b->max_tree = 0;
  for (int32_t i = 0; i < pl.n; i++) b->max_len = std::max(b->max_len, pl.len[i]);
  for (int32_t i = 0; i < pl.n; i++)
    if (pl.is_tree(i)) b->max_tree = std::max(b->max_tree, pl.q_len[i]);
  if (b->v.plan_only) return KV_OK;
  // a failure from here on leaves a batch that describes nothing: the device does not have what the plan says
  struct Undo {
    BatchPlan* pl;
    ~Undo() {
      if (pl) pl->n = pl->T = 0;
    }
  } undo{&pl};
  rc = order(b, st);
  if (rc) return rc;

  struct Part {
    const void* from;
    size_t bytes;
    const void** at;
  };
#define VEC(x, to) Part{(x).data(), (x).size() * sizeof((x)[0]), (const void**)&(to)}
  const Part parts[] = {VEC(pl.items, b->items),     VEC(pl.wg_items, b->wg_items),   VEC(pl.wg_big, b->wg_big),       VEC(pl.witems, b->witems),
                        VEC(pl.wrest, b->wrest),     VEC(pl.sitems, b->sitems),       VEC(pl.wreqs, b->wreqs),         VEC(pl.ids, b->table),
                        VEC(pl.off, b->off),         VEC(pl.len, b->len),             VEC(pl.q_first, b->q_first),     VEC(pl.places, b->places),
                        VEC(pl.tok_limit, b->limit), VEC(pl.lists, b->lists),         VEC(pl.join_off, b->join_off),   VEC(pl.join, b->join),
                        VEC(pl.tree_reqs, b->tree_reqs), VEC(pl.tree_sight, b->tree_sight)};
#undef VEC
  size_t need = 0;
  for (const Part& p : parts) need += padded(p.bytes);
  const int H = b->v.H;
  const size_t prows = (size_t)pl.partial_rows * H, lse_n = (size_t)pl.T * H * pl.G;
  const size_t tree_rows = pl.tree.empty() ? 0 : padded((size_t)pl.T * 4);
  const size_t ws_need = padded(prows * b->v.D * 4) + padded(prows * sizeof(float2)) + padded(lse_n * 4) + 2 * tree_rows + padded((size_t)pl.tree_words * 4);
  const int k = b->turn;
  if (need > b->mem_cap) {
    rc = drain(b);
    if (rc) return rc;
    if (b->mem) OPCHK(b, hipFree(b->mem));
    b->mem = nullptr;
    b->mem_cap = 0;
    OPCHK(b, hipMalloc((void**)&b->mem, need + need / 2));
    b->mem_cap = need + need / 2;
  }
  if (ws_need > b->ws_cap) {
    rc = drain(b);
    if (rc) return rc;
    if (b->ws) OPCHK(b, hipFree(b->ws));
    b->ws = nullptr;
    b->ws_cap = 0;
    OPCHK(b, hipMalloc((void**)&b->ws, ws_need + ws_need / 2));
    b->ws_cap = ws_need + ws_need / 2;
  }
  const std::pair<kv_batch::Room*, size_t> rooms[2] = {{&b->scores, scores_need(b)}, {&b->turns, turns_need(b)}};
  for (auto [room, room_need] : rooms)
    if (room->wanted && room_need > room->cap) {
      rc = drain(b);
      if (rc) return rc;
      if (room->at) OPCHK(b, hipFree(room->at));
      *room = {nullptr, 0, true};
      take(*room, room_need);
    }
  if (b->up_busy[k]) OPCHK(b, hipEventSynchronize(b->up_ev[k]));
  b->up_busy[k] = false;
  if (need > b->up_cap[k]) {
    if (b->up[k]) OPCHK(b, hipHostFree(b->up[k]));
    b->up[k] = nullptr;
    b->up_cap[k] = 0;
    OPCHK(b, hipHostMalloc((void**)&b->up[k], need + need / 2, hipHostMallocDefault));
    b->up_cap[k] = need + need / 2;
  }
  size_t at = 0;
  for (const Part& p : parts) {
    if (p.bytes) std::memcpy(b->up[k] + at, p.from, p.bytes);
    *p.at = b->mem + at;
    at += padded(p.bytes);
  }
  char* room = b->ws;
  auto next = [&](size_t bytes) { return std::exchange(room, room + padded(bytes)); };
  b->part_o = (float*)next(prows * b->v.D * 4);
  b->part_ml = (float2*)next(prows * sizeof(float2));
  b->lse = (float*)next(lse_n * 4);
  b->parent = (int32_t*)next(tree_rows);
  b->position = (int32_t*)next(tree_rows);
  b->bits = (uint32_t*)next((size_t)pl.tree_words * 4);
  if (at) {
    OPCHK(b, hipMemcpyAsync(b->mem, b->up[k], at, hipMemcpyHostToDevice, st));
    OPCHK(b, hipEventRecord(b->up_ev[k], st));
    b->up_busy[k] = true;
    b->turn = 1 - k;
  }
  if (!pl.tree.empty() && pl.T) {
    const TreeArgs t{b->tree_reqs, parents, (pl.tree_units + 255) / 256, b->parent, b->position, (int32_t*)b->limit, b->bits};
    hipLaunchKernelGGL(kv_tree_kernel, dim3((unsigned)(pl.n * t.chunks)), dim3(256), 0, st, t);
    OPCHK(b, hipGetLastError());
  }
  undo.pl = nullptr;
  return KV_OK;
}

}  // namespace

extern "C" {

int kv_batch_set(kv_batch* b, int32_t n, const int32_t* offsets, const int32_t* block_ids, const int32_t* num_tokens, const int32_t* q_lens,
                 int32_t num_q_heads, void* stream) try {
  if (!b) return KV_EINVAL;
  return set_batch(b, n, offsets, block_ids, num_tokens, q_lens, num_q_heads, nullptr, nullptr, stream);
}
catch (...) {
  return caught();
}

int kv_batch_set_trees(kv_batch* b, int32_t n, const int32_t* offsets, const int32_t* block_ids, const int32_t* num_tokens, const int32_t* q_lens,
                       int32_t num_q_heads, const int32_t* trees, const int32_t* parents, void* stream) try {
  if (!b || n < 0 || (n && !q_lens)) return KV_EINVAL;
  std::vector<uint8_t> which((size_t)n);
  bool rows = false;
  int64_t units = 0;
  for (int32_t i = 0; i < n; i++) {
    which[i] = !trees || trees[i];
    if (q_lens[i] < 0 || (which[i] && q_lens[i] > KV_TREE_MAX)) return KV_EINVAL;
    rows = rows || (which[i] && q_lens[i] > 0);
    // (as many workgroups as the request that needs most; more than a launch may have: refused)
    units = std::max<int64_t>(units, which[i] ? (int64_t)q_lens[i] * ((q_lens[i] + 126ll) / 64 * 2) : q_lens[i]);
  }
  if (rows && !parents) return KV_EINVAL;
  if ((units + 255) / 256 * n > kMostWgs) return KV_EINVAL;
  return set_batch(b, n, offsets, block_ids, num_tokens, q_lens, num_q_heads, n ? which.data() : nullptr, parents, stream);
}
catch (...) {
  return caught();
}

int kv_batch_query(const kv_batch* b, kv_batch_info* out) {
  if (!b || !out || out->struct_size != sizeof(kv_batch_info)) return KV_EINVAL;
  const BatchPlan& pl = b->plan;
  const bool some = pl.n > 0;
  out->rows = pl.T;
  out->items = some ? (int32_t)pl.items.size() : 0;
  out->partial_rows = some ? pl.partial_rows : 0;
  out->cached_tokens = some ? pl.cached : 0;
  out->read_tokens = some ? pl.read : 0;
  return KV_OK;
}

int kv_rope_freqs(int32_t rot, double base, int32_t kind, double factor, double trained, double low, double high, int64_t* turns,
                  float* magnitude) {
  if (rot <= 0 || rot % 2 || rot > 256 || !(base > 1.0) || !std::isfinite(base) || !turns || !magnitude) return KV_EINVAL;
  if (kind < KV_ROPE_PLAIN || kind > KV_ROPE_YARN) return KV_EINVAL;
  if (kind != KV_ROPE_PLAIN && (!(factor >= 1.0) || !std::isfinite(factor))) return KV_EINVAL;
  if ((kind == KV_ROPE_PARTS || kind == KV_ROPE_YARN) && (!(trained > 0.0) || !std::isfinite(trained) || !(low > 0.0) || !(high > low) || !std::isfinite(high)))
    return KV_EINVAL;
  const double two_pi = 6.283185307179586476925286766559;
  if (kind == KV_ROPE_BASE) base *= rot > 2 ? std::pow(factor, (double)rot / (rot - 2)) : factor;
  double lo_index = 0, hi_index = 1;
  if (kind == KV_ROPE_YARN) {
    // the (fractional) index of the pair that turns `times` times within the trained length
    auto index = [&](double times) { return rot * std::log(trained / (times * two_pi)) / (2 * std::log(base)); };
    lo_index = std::fmax(0.0, std::floor(index(high)));
    hi_index = std::fmin(rot - 1.0, std::ceil(index(low)));
    if (hi_index <= lo_index) hi_index = lo_index + 0.001;
  }
  for (int j = 0; j < rot / 2; j++) {
    double f = std::pow(base, -2.0 * j / rot) / two_pi;
    double stretched = 0;  // share of the frequency that is divided by factor
    if (kind == KV_ROPE_LINEAR) stretched = 1;
    if (kind == KV_ROPE_PARTS) stretched = 1 - std::fmin(1.0, std::fmax(0.0, (trained * f - low) / (high - low)));
    if (kind == KV_ROPE_YARN) stretched = std::fmin(1.0, std::fmax(0.0, (j - lo_index) / (hi_index - lo_index)));
    if (stretched > 0) f = stretched * f / factor + (1 - stretched) * f;
    // below 1/2 turn (base^0 / 2 pi is 0.16): the product fits a signed word
    turns[j] = (int64_t)std::llround(std::ldexp(f, 64));
  }
  *magnitude = kind == KV_ROPE_YARN ? (float)(0.1 * std::log(factor) + 1.0) : 1.0f;
  return KV_OK;
}

}  // extern "C"

namespace {

// axes 0: positions have one, and every pair is turned by it.
int append(kv_batch* b, const kv_append_args* a, int32_t axes, const int32_t* pair_axes, int64_t positions_stride, void* stream) {
  int rc = kvswap::pool_usable(b->pool);
  if (rc) return rc;
  const PoolView& v = b->v;
  const BatchPlan& pl = b->plan;
  if (a->layer < 0 || a->layer >= v.L || !io_fits(v, a->io_dtype) || a->rot < 0 || a->rot > v.D || a->rot % 2) return KV_EINVAL;
  uint32_t packed[8] = {};
  if (axes) {
    if (axes < 0 || axes > KV_MOST_AXES || (a->rot && !pair_axes)) return KV_EINVAL;
    for (int32_t j = 0; j < a->rot / 2; j++) {
      if (pair_axes[j] < 0 || pair_axes[j] >= axes) return KV_EINVAL;
      packed[j / 16] |= (uint32_t)pair_axes[j] << j % 16 * 2;
    }
  }
  const bool scaled = v.has_scale;
  if (scaled != (a->k_scale != nullptr) || scaled != (a->v_scale != nullptr)) return KV_EINVAL;
  if (pl.T == 0 || pl.n == 0) return KV_OK;
  if (!a->k || !a->v || (a->q != nullptr) != (a->q_out != nullptr) || (a->rot && !a->turns) || (axes && a->rot && !a->positions)) return KV_EINVAL;
  if (v.plan_only) return KV_OK;
  hipStream_t st = (hipStream_t)stream;
  rc = order(b, st);
  if (rc) return rc;
  AppendArgs k{};
  k.q = (const char*)a->q;
  k.k = (const char*)a->k;
  k.v = (const char*)a->v;
  k.q_out = (char*)a->q_out;
  for (int i = 0; i < 2; i++) {
    k.qs[i] = a->q_strides[i];
    k.ks[i] = a->k_strides[i];
    k.vs[i] = a->v_strides[i];
    k.qos[i] = a->q_out_strides[i];
  }
  k.turns = a->turns;
  k.positions = a->positions ? a->positions : pl.tree.empty() ? nullptr : b->position;
  k.axis_stride = positions_stride;
  std::memcpy(k.axis, packed, sizeof packed);
  k.k_scale = a->k_scale;
  k.v_scale = a->v_scale;
  k.places = b->places;
  k.pool = v.pool + a->layer * v.ls;
  k.vk = v.ks;
  k.bs = v.bs;
  k.scale = v.scale ? v.scale + a->layer * v.sls : nullptr;
  k.svk = v.sks;
  k.sbs = v.sbs;
  k.magnitude = a->magnitude;
  k.rot = a->rot;
  k.H = v.H;
  k.Hq = a->q ? v.H * pl.G : 0;
  k.D = v.D;
  k.interleaved = a->interleaved;
  const bool fp8 = v.dtype == KV_FP8_E4M3, f16 = a->io_dtype == KV_F16;
  const bool wide = a->rot % (a->interleaved ? 8 : 16) == 0 && aligned(a->k, a->k_strides, 16) && aligned(a->v, a->v_strides, 16) &&
                    (!a->q || (aligned(a->q, a->q_strides, 16) && aligned(a->q_out, a->q_out_strides, 16)));
  if (wide) {
    k.pairs = a->rot / (a->interleaved ? 8 : 16);
    k.units = k.pairs + (v.D - a->rot) / 8;
    k.chunks = ((k.Hq + v.H) * k.units + v.H * (v.D / 8) + 255) / 256;
  }
  k.T = pl.T;
  auto go = [&](auto kern, int64_t wgs) { hipLaunchKernelGGL(kern, dim3((unsigned)wgs), dim3(256), 0, st, k); };
  const int64_t all = (int64_t)pl.T * k.chunks;
  auto any = [&](auto e, auto p, auto x) {
    using E = decltype(e);
    constexpr bool P = decltype(p)::value, X = decltype(x)::value;
    if (!wide)
      go(kv_append_kernel<E, P, X>, pl.T);
    else if (all <= kAppendMany * v.cus)
      go(kv_append_wide_kernel<E, P, X, 1>, all);
    else
      go(kv_append_wide_kernel<E, P, X, 2>, (int64_t)(pl.T + 1) / 2 * k.chunks);
  };
  auto typed = [&](auto p, auto x) { f16 ? any(_Float16(), p, x) : any(__bf16(), p, x); };
  auto stored = [&](auto x) { fp8 ? typed(std::true_type(), x) : typed(std::false_type(), x); };
  axes ? stored(std::true_type()) : stored(std::false_type());
  OPCHK(b, hipGetLastError());
  return KV_OK;
}

}  // namespace

extern "C" {

int kv_append(kv_batch* b, const kv_append_args* a, void* stream) try {
  if (!b || !a || a->struct_size != sizeof(kv_append_args)) return KV_EINVAL;
  return append(b, a, 0, nullptr, 0, stream);
}
catch (...) {
  return caught();
}

int kv_append_axes(kv_batch* b, const kv_append_args* a, int32_t axes, const int32_t* pair_axes, int64_t positions_stride, void* stream) try {
  if (!b || !a || a->struct_size != sizeof(kv_append_args) || axes < 1) return KV_EINVAL;
  return append(b, a, axes, pair_axes, positions_stride, stream);
}
catch (...) {
  return caught();
}

int kv_attn(kv_batch* b, const kv_attn_args* a, void* stream) try {
  if (!b || !a || a->struct_size != sizeof(kv_attn_args)) return KV_EINVAL;
  int rc = kvswap::pool_usable(b->pool);
  if (rc) return rc;
  const PoolView& v = b->v;
  const BatchPlan& pl = b->plan;
  if (a->layer < 0 || a->layer >= v.L || !io_fits(v, a->io_dtype) || !std::isfinite(a->scale)) return KV_EINVAL;
  if (a->weights && a->weights_cap < b->max_len) return KV_EINVAL;
  if (pl.T == 0 || pl.n == 0) return KV_OK;
  if (!a->q || !a->out) return KV_EINVAL;
  if (v.plan_only) return KV_OK;
  hipStream_t st = (hipStream_t)stream;
  rc = order(b, st);
  if (rc) return rc;
  AttnArgs k{};
  k.kv = side(b, a->layer);
  k.items = b->items;
  k.wg_items = b->wg_items;
  k.wg_big = b->wg_big;
  k.lists = b->lists;
  k.limit = b->limit;
  k.table = b->table;
  k.q = (const char*)a->q;
  k.out = (char*)a->out;
  k.q_ts = a->q_strides[0];
  k.q_hs = a->q_strides[1];
  k.o_ts = a->out_strides[0];
  k.o_hs = a->out_strides[1];
  k.lse = a->lse;
  k.lse_ts = a->lse_stride;
  if (a->weights && !a->lse) {
    k.lse = b->lse;
    k.lse_ts = (int64_t)v.H * pl.G;
  }
  k.part_o = b->part_o;
  k.part_ml = b->part_ml;
  // a scale of next to nothing rather than none: what is masked has to stay below everything
  k.scale2 = (float)std::max(std::fabs((double)a->scale) * 1.4426950408889634, 1e-30);
  k.flip = a->scale < 0;
  k.H = v.H;
  k.G = pl.G;
  k.hw = pl.heads;
  k.q_vec = aligned(a->q, a->q_strides, 16);
  k.o_vec = aligned(a->out, a->out_strides, 8);
  const bool keeps = a->weights && pl.scores && has_room(b->scores, scores_need(b), st);
  if (keeps) {
    k.scores = (float*)b->scores.at;
    k.scores_head = pl.scores;
  }
  const bool fp8 = v.dtype == KV_FP8_E4M3, f16 = a->io_dtype == KV_F16, trees = !pl.tree.empty();
  if (trees) {
    k.sight = b->tree_sight;
    k.bits = b->bits;
  }
  f16 ? launch_attn<_Float16>(fp8, k, pl, st) : launch_attn<__bf16>(fp8, k, pl, st);
  OPCHK(b, hipGetLastError());
  if (pl.partial_rows) {
    JoinArgs j{b->join_off, b->join, b->part_o, b->part_ml, k.out, k.o_ts, k.o_hs, k.lse, k.lse_ts, v.H, pl.G, v.D, trees ? b->limit : nullptr};
    f16 ? launch_join<_Float16>(j, pl, st) : launch_join<__bf16>(j, pl, st);
    OPCHK(b, hipGetLastError());
  }
  if (a->weights && keeps) {
    const SumArgs s{b->sitems, b->q_first, k.scores, k.scores_head, k.lse, k.lse_ts, a->weights, a->weights_strides[0], a->weights_strides[1], k.scale2, v.H, pl.G};
    hipLaunchKernelGGL(kv_attn_sum_kernel, dim3((unsigned)pl.sitems.size() * v.H), dim3(256), 0, st, s);
    OPCHK(b, hipGetLastError());
  }
  const std::vector<WeightItem>& again = keeps ? pl.wrest : pl.witems;
  if (a->weights && !again.empty()) {
    WeightArgs w{k, keeps ? b->wrest : b->witems, b->q_first, b->wreqs, k.lse, k.lse_ts, a->weights, a->weights_strides[0], a->weights_strides[1],
                 division(pl.G)};
    f16 ? launch_weights<_Float16>(fp8, w, (int)again.size(), st) : launch_weights<__bf16>(fp8, w, (int)again.size(), st);
    OPCHK(b, hipGetLastError());
  }
  return KV_OK;
}
catch (...) {
  return caught();
}

int kv_evict(kv_batch* b, const kv_evict_args* a, void* stream) try {
  if (!b || !a || a->struct_size != sizeof(kv_evict_args)) return KV_EINVAL;
  int rc = kvswap::pool_usable(b->pool);
  if (rc) return rc;
  const PoolView& v = b->v;
  BatchPlan& pl = b->plan;
  if (a->layer < 0 || a->num_layers < 0 || a->layer > v.L - a->num_layers) return KV_EINVAL;
  if (a->keep_first < 0 || a->keep_last < 0 || (int64_t)a->keep_first + a->keep_last > a->keep) return KV_EINVAL;
  if (pl.n == 0 || a->num_layers == 0) return KV_OK;
  if (!a->weights || !a->kept || a->weights_cap < b->max_len) return KV_EINVAL;
  const int32_t fixed_blocks = a->keep_first / v.B, keep_blocks = (int32_t)(((int64_t)a->keep + v.B - 1) / v.B);
  if ((int64_t)pl.n * v.H * 2 > kMostWgs) return KV_EINVAL;
  const bool crowded = b->max_len > a->keep;
  if (crowded && pl.rewrites_shared(a->keep, fixed_blocks, keep_blocks)) return KV_EDUP;
  std::vector<int32_t> unchanged;
  if (a->req_ids) {
    // what becomes of host copies is settled now: a replay would come after copies that have been made since
    if (!v.plan_only && is_capturing((hipStream_t)stream)) return KV_EINVAL;
    rc = kvswap::pool_may_rewrite(b->pool, pl.n, a->req_ids);
    if (rc) return rc;
    for (int32_t i = 0; i < pl.n; i++) unchanged.push_back(pl.len[i] > a->keep ? fixed_blocks : -1);
  }
  if (!v.plan_only) {
    hipStream_t st = (hipStream_t)stream;
    rc = order(b, st);
    if (rc) return rc;
    EvictArgs k{};
    k.w = a->weights;
    k.w_out = a->weights_out ? a->weights_out : (float*)a->weights;
    for (int i = 0; i < 3; i++) {
      k.ws[i] = a->weights_strides[i];
      k.ks[i] = a->kept_strides[i];
    }
    k.kept = a->kept;
    k.len = b->len;
    k.off = b->off;
    k.table = b->table;
    k.n = pl.n;
    k.H = v.H;
    k.keep = a->keep;
    k.first = a->keep_first;
    k.last = a->keep_last;
    k.pool = v.pool + a->layer * v.ls;
    k.ls = v.ls;
    k.vk = v.ks;
    k.bs = v.bs;
    k.scale = v.scale ? v.scale + a->layer * v.sls : nullptr;
    k.sls = v.sls;
    k.svk = v.sks;
    k.sbs = v.sbs;
    k.D = v.D;
    k.B = v.B;
    k.e = elem(v);
    k.group = v.B >= 64 ? v.B : 64 / v.B * v.B;
    k.first_tok = fixed_blocks * v.B;
    // chunks of the move
    constexpr int kU = kMoveUnroll;
    k.rows = chunk_rows(v);
    const int64_t heads_layer = (int64_t)pl.n * v.H;
    bool apart = crowded && k.rows > 0;
    if (apart) {
      k.chunks = std::max(1, (a->keep - k.first_tok + k.rows - 1) / k.rows);
      if (k.chunks > 1) {
        // No tickets in a capture: two launches that drew from the same ones at a time would leave chunks out and wait for these, and when a
        // replay runs is not known here.
        apart = heads_layer * 2 * k.chunks <= kMostWgs && !is_capturing(st) && has_room(b->turns, turns_need(b), st);
        if (apart) k.turns = (int32_t*)b->turns.at;
      }
    }
    // Lanes of a row's workgroup: 256; more where a few rows are longer than these have registers for; a wavefront, which waits for no
    // other, where there are rows enough to fill the chip with and one has the registers.  With the few moves that keeping 8 tokens needs,
    // 64 / 256 / 1024 lanes: 2048 rows of 300 to 500 tokens 25 / 35 / 131 us, 64 such 16 / 15 / 22, 160 rows of 1790 to 7026 94 / 42 / 25, 8192 of
    // 5000 to 8000 490 / 494 / 585.
    const bool many = a->num_layers * heads_layer > 4 * v.cus;
    // as many layers at a time as one launch may have workgroups for
    const int32_t layers = (int32_t)std::min<int64_t>(a->num_layers, std::max<int64_t>(1, kMostWgs / (heads_layer * 2 * (apart ? k.chunks : 1))));
    for (int32_t done = 0; done < a->num_layers; done += layers) {
      const unsigned heads = (unsigned)(std::min(layers, a->num_layers - done) * heads_layer);
      auto select = [&](auto kern, int lanes) { hipLaunchKernelGGL(kern, dim3(heads), dim3(lanes), 0, st, k); };
      if (many && b->max_len <= 64 * kSelectEach)
        select(kv_evict_select_kernel<64>, 64);
      else if (!many && b->max_len > 256 * kSelectEach)
        select(kv_evict_select_kernel<1024>, 1024);
      else
        select(kv_evict_select_kernel<256>, 256);
      OPCHK(b, hipGetLastError());
      if (crowded) {
        auto go = [&](auto kern, unsigned grid) { hipLaunchKernelGGL(kern, dim3(grid), dim3(256), 0, st, k); };
        if (apart)
          v.scale ? go(kv_evict_move_kernel<true, kU>, heads * 2 * k.chunks) : go(kv_evict_move_kernel<false, kU>, heads * 2 * k.chunks);
        else
          v.scale ? go(kv_evict_move_alone_kernel<true>, heads * 2) : go(kv_evict_move_alone_kernel<false>, heads * 2);
        OPCHK(b, hipGetLastError());
      }
      k.w += layers * k.ws[0];
      k.w_out += layers * k.ws[0];
      k.kept += layers * k.ks[0];
      k.pool += layers * k.ls;
      if (k.scale) k.scale += layers * k.sls;
    }
  }
  if (a->req_ids) kvswap::pool_rewritten(b->pool, pl.n, a->req_ids, unchanged.data());
  return KV_OK;
}
catch (...) {
  return caught();
}

int kv_accept(kv_batch* b, const kv_accept_args* a, void* stream) try {
  if (!b || !a || a->struct_size != sizeof(kv_accept_args)) return KV_EINVAL;
  int rc = kvswap::pool_usable(b->pool);
  if (rc) return rc;
  const PoolView& v = b->v;
  const BatchPlan& pl = b->plan;
  if (a->layer < 0 || a->num_layers < 0 || a->layer > v.L - a->num_layers) return KV_EINVAL;
  if (pl.n == 0) return KV_OK;
  if (!a->count || !a->next || (pl.T && !a->chosen)) return KV_EINVAL;
  if (b->max_tree && (!a->tokens || !a->path || a->path_cap < b->max_tree)) return KV_EINVAL;
  if (a->weights && a->weights_cap < b->max_len) return KV_EINVAL;
  if (a->num_layers && !pl.tree.empty() && pl.tree_tails_shared) return KV_EDUP;
  const int bytes = v.H * v.D * elem(v), vec = bytes % 16 || (v.has_scale && v.D % 16) ? 8 : 16;
  AcceptArgs k{};
  k.cols = (bytes / vec + 255) / 256;
  k.vecs = (bytes / vec + k.cols - 1) / k.cols;
  if ((int64_t)pl.n * k.cols > kMostWgs) return KV_EINVAL;
  std::vector<int32_t> unchanged;
  if (a->req_ids) {
    if (!v.plan_only && is_capturing((hipStream_t)stream)) return KV_EINVAL;
    rc = kvswap::pool_may_rewrite(b->pool, pl.n, a->req_ids);
    if (rc) return rc;
    // the first new token stays where it is
    for (int32_t i = 0; i < pl.n; i++) unchanged.push_back(pl.is_tree(i) && pl.q_len[i] > 1 ? (pl.len[i] - pl.q_len[i] + 1) / v.B : -1);
  }
  if (!v.plan_only) {
    hipStream_t st = (hipStream_t)stream;
    rc = order(b, st);
    if (rc) return rc;
    const bool trees = !pl.tree.empty();
    k.reqs = trees ? b->tree_reqs : nullptr;
    k.parent = b->parent;
    k.tokens = a->tokens;
    k.chosen = a->chosen;
    k.q_first = b->q_first;
    k.len = b->len;
    k.off = b->off;
    k.table = b->table;
    k.count = a->count;
    k.path = a->path;
    k.next = a->next;
    k.path_stride = a->path_stride;
    k.n = pl.n;
    k.H = v.H;
    k.B = v.B;
    k.pool = v.pool + a->layer * v.ls;
    k.ls = v.ls;
    k.vk = v.ks;
    k.bs = v.bs;
    k.row = bytes;
    k.scale = v.scale ? v.scale + a->layer * v.sls : nullptr;
    k.sls = v.sls;
    k.svk = v.sks;
    k.sbs = v.sbs;
    k.head = v.D * elem(v);
    k.weights = a->weights;
    for (int i = 0; i < 3; i++) k.ws[i] = a->weights_strides[i];
    k.layers = trees ? a->num_layers : 0;
    // as many workgroups as fit the chip at a time (8 a CU) share the planes; without trees, or without layers, the counts alone
    const int64_t each = (int64_t)pl.n * k.cols;
    k.groups = (int32_t)std::max<int64_t>(1, std::min<int64_t>(2 * k.layers, 8 * v.cus / each));
    auto go = [&](auto kern) { hipLaunchKernelGGL(kern, dim3((unsigned)(each * k.groups)), dim3(256), 0, st, k); };
    // a workgroup that has one plane takes eight rows of it at a time, one that has more four of two
    auto any = [&](auto scaled, auto q) {
      constexpr bool S = decltype(scaled)::value;
      constexpr int Q = decltype(q)::value;
      vec == 16 ? go(kv_accept_kernel<u32x4, S, Q>) : go(kv_accept_kernel<u32x2, S, Q>);
    };
    const std::integral_constant<int, 1> one;
    const std::integral_constant<int, 2> two;
    if (k.groups >= 2 * k.layers)
      v.scale ? any(std::true_type(), one) : any(std::false_type(), one);
    else
      v.scale ? any(std::true_type(), two) : any(std::false_type(), two);
    OPCHK(b, hipGetLastError());
  }
  if (a->req_ids) kvswap::pool_rewritten(b->pool, pl.n, a->req_ids, unchanged.data());
  return KV_OK;
}
catch (...) {
  return caught();
}

}  // extern "C"
