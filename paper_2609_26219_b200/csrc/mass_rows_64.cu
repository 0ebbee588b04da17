#include "mass_rows_launch.cuh"

namespace patchkv {
template cudaError_t launch_weigh_rows<64>(const AttentionParams&, const WeightParams&, WeighRowsPlan, cudaStream_t);
}
