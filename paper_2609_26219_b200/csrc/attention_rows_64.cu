#include "attention_rows_launch.cuh"

namespace patchkv {
template cudaError_t launch_rows<64>(const AttentionParams&, const RowsPlan&, cudaStream_t);
}
