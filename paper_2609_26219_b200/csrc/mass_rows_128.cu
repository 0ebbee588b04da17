#include "mass_rows_launch.cuh"

namespace patchkv {
template cudaError_t launch_weigh_rows<128>(const AttentionParams&, const WeightParams&, WeighRowsPlan, cudaStream_t);
}
