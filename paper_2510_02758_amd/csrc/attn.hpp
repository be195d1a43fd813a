// What the attention's host side (kvops.hip) and its kernels (attn.hip.inc) have in common.  The kernels are built once for either
// 16-bit type, in files of their own (attn_bf16.hip, attn_f16.hip).
#pragma once

#include <hip/hip_runtime.h>

#include "batch.hpp"

using kvswap::big_tile;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

struct DivBy {
  uint32_t mul, shift;
};
__device__ __forceinline__ uint32_t div_by(const DivBy& d, uint32_t x) {
  return d.shift >= 32 ? x : (uint32_t)(((uint64_t)x * d.mul) >> 32) >> d.shift;
}

struct KvSide {
  const char* k;   // keys of the layer
  int64_t vk;      // from a key to its value, bytes
  int64_t bs;      // block stride, bytes
  const float* ks; // scales of the layer's keys, null without
  int64_t vks, sbs;
  int32_t row;     // bytes from a token's head to the next token's: H * D * e
  int32_t head;    // bytes of a head: D * e
  int32_t D, B;
  DivBy by_b;
};

__device__ __forceinline__ uint32_t div_by_b(const KvSide& s, uint32_t x) { return div_by(s.by_b, x); }

struct AttnArgs {
  KvSide kv;
  const kvswap::AttnItem* items;
  const int32_t *wg_items, *wg_big;  // where each workgroup's items begin, of row tiles and of big ones
  const int32_t *lists, *limit, *table;
  const char* q;
  char* out;
  int64_t q_ts, q_hs, o_ts, o_hs;  // elements
  float* lse;
  int64_t lse_ts;
  float* part_o;
  float2* part_ml;
  float scale2;  // |scale| * log2(e), not 0
  int32_t flip;  // the scale is negative: queries change sign
  int32_t H, G, q_vec;
  int32_t o_vec;
  float* scores;         // null: the products of row tiles are not kept
  int64_t scores_head;   // of one KV head
  int32_t hw;  // heads of a workgroup of row tiles (1, 2 or 4): its wavefronts take one each, and 4 / hw share a head's keys
  const kvswap::TreeSight* sight;  // null: no request's new tokens are a drafted tree
  const uint32_t* bits;
};

// What a tile's rows see of its keys: all, those in front of each row's limit, or what a tree's bits say.
enum Sees { kAll = 0, kUpTo = 1, kTree = 2 };

template <typename E>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  typedef E E2 __attribute__((ext_vector_type(2)));
  E2 v = {(E)a, (E)b};
  return __builtin_bit_cast(uint32_t, v);
}

struct JoinArgs {
  const int32_t *join_off, *join;
  const float* part_o;
  const float2* part_ml;
  char* out;
  int64_t o_ts, o_hs;
  float* lse;
  int64_t lse_ts;
  int32_t H, G, D;
  const int32_t* limit;  // of a batch with drafted trees: 0 is a row that is in none
};

// kv_attn_join_few_kernel: lanes of a row, workgroups of a token, and of a launch (0: it would have more lanes than 32 bits count).
constexpr int join_few_stride(int D) { return D <= 64 ? 16 : D <= 128 ? 32 : 64; }
constexpr int64_t join_few_chunks(int64_t heads, int D) { return (heads * join_few_stride(D) + 255) / 256; }
constexpr int64_t join_few_wgs(int64_t T, int64_t heads, int D) {
  return T * join_few_chunks(heads, D) <= UINT32_MAX / 256 ? T * join_few_chunks(heads, D) : 0;
}

struct WeightArgs {
  AttnArgs a;
  const kvswap::WeightItem* items;
  const int32_t *q_first, *reqs;
  const float* lse;
  int64_t lse_ts;
  float* weights;
  int64_t w_rs, w_hs;
  DivBy by_g;
};

struct SumArgs {
  const kvswap::ScoreItem* items;
  const int32_t* q_first;
  const float* scores;
  int64_t scores_head;
  const float* lse;
  int64_t lse_ts;
  float* weights;
  int64_t w_rs, w_hs;
  float scale2;
  int32_t H, G;
};

// Enqueue the batch's tiles, the join of its partial results, its weight items.  E: the type of the products.
template <typename E>
void launch_attn(bool fp8, const AttnArgs& a, const kvswap::BatchPlan& pl, hipStream_t st);
template <typename E>
void launch_join(const JoinArgs& j, const kvswap::BatchPlan& pl, hipStream_t st);
template <typename E>
void launch_weights(bool fp8, const WeightArgs& w, int items, hipStream_t st);
// The two for batches with drafted trees, whose kernels are built in files of their own (attn_tree_bf16.hip, attn_tree_f16.hip); the others call them.
template <typename E>
void launch_tree_attn(bool fp8, const AttnArgs& a, const kvswap::BatchPlan& pl, hipStream_t st);
template <typename E>
void launch_tree_weights(bool fp8, const WeightArgs& w, int items, hipStream_t st);
