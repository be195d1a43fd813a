// The attention's kernels with products of bf16 elements (and fp8 ones widened to them).
#include <algorithm>
#include <type_traits>

#include "attn.hpp"

#include "attn.hip.inc"

extern template void launch_tree_attn<__bf16>(bool, const AttnArgs&, const kvswap::BatchPlan&, hipStream_t);
extern template void launch_tree_weights<__bf16>(bool, const WeightArgs&, int, hipStream_t);

template void launch_attn<__bf16>(bool, const AttnArgs&, const kvswap::BatchPlan&, hipStream_t);
template void launch_join<__bf16>(const JoinArgs&, const kvswap::BatchPlan&, hipStream_t);
template void launch_weights<__bf16>(bool, const WeightArgs&, int, hipStream_t);
