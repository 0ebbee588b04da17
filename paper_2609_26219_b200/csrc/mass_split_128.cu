#include "mass_split_launch.cuh"

namespace patchkv {
template cudaError_t launch_weigh<128>(const AttentionParams&, const WeightParams&, const WeighPlan&, int, int, cudaStream_t);
}
