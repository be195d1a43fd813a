// The attention's kernels with products of f16 elements (and fp8 ones widened to them).
#include <algorithm>
#include <type_traits>

#include "attn.hpp"

#include "attn.hip.inc"

extern template void launch_tree_attn<_Float16>(bool, const AttnArgs&, const kvswap::BatchPlan&, hipStream_t);
extern template void launch_tree_weights<_Float16>(bool, const WeightArgs&, int, hipStream_t);

template void launch_attn<_Float16>(bool, const AttnArgs&, const kvswap::BatchPlan&, hipStream_t);
template void launch_join<_Float16>(const JoinArgs&, const kvswap::BatchPlan&, hipStream_t);
template void launch_weights<_Float16>(bool, const WeightArgs&, int, hipStream_t);
