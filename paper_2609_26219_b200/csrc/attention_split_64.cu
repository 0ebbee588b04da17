#include "attention_split_launch.cuh"

namespace patchkv {
template cudaError_t launch_split<64>(const AttentionParams&, const SplitPlan&, int, int, cudaStream_t);
}
