#include "attention_split_launch.cuh"

namespace patchkv {
template cudaError_t launch_split<128>(const AttentionParams&, const SplitPlan&, int, int, cudaStream_t);
}
