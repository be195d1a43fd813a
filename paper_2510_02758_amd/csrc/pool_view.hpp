// What the operators on the pool's contents (kvops.hip) need of a pool handle (kvswap.hip): its geometry, where to leave a HIP error,
// and the bookkeeping of host copies, which an eviction makes stale.
#pragma once

#include <cstdint>

#include "planner.hpp"

namespace kvswap {

struct PoolView {
  int32_t L, H, D, B, dtype;
  int64_t N;
  char* pool;
  int64_t ls, ks, bs;  // bytes
  float* scale;        // null: no scales
  int64_t sls, sks, sbs;  // words
  bool has_scale, plan_only;
  int cus;
};

// KV_EHIP on a handle on which an earlier call failed half-way.
int pool_view(kv_pool* p, PoolView* out);
int pool_usable(kv_pool* p);
void pool_hip_error(kv_pool* p, int code);
// May these requests' blocks be rewritten (none of them is swapped out; unknown ones are fine)?
int pool_may_rewrite(kv_pool* p, int32_t n, const uint64_t* ids);
// Request ids[i] keeps its first `unchanged[i]` blocks as they are: of its host copy no more than that stays valid, and its entry in the
// write queue goes.  A negative number: nothing of it changes.
void pool_rewritten(kv_pool* p, int32_t n, const uint64_t* ids, const int32_t* unchanged);

}  // namespace kvswap
