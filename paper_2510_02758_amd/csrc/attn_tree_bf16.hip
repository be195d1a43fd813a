// The attention's kernels for batches with drafted trees, with products of bf16 elements (and fp8 ones widened to them).
#include <algorithm>
#include <type_traits>

#include "attn.hpp"

#include "attn.hip.inc"

template void launch_tree_attn<__bf16>(bool, const AttnArgs&, const kvswap::BatchPlan&, hipStream_t);
template void launch_tree_weights<__bf16>(bool, const WeightArgs&, int, hipStream_t);
