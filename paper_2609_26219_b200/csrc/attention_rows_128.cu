#include "attention_rows_launch.cuh"

namespace patchkv {
template cudaError_t launch_rows<128>(const AttentionParams&, const RowsPlan&, cudaStream_t);
}
