// Launches of the kernels of mass_split.cuh for one head dimension; a translation unit per dimension (mass_split_64.cu, mass_split_128.cu).
#pragma once

#include <algorithm>

#include "attention_launch.cuh"
#include "mass_split.cuh"

namespace patchkv {

template <int KF, int D, int NC>
struct WeighShape {
    static constexpr int kWarps = split_warps(KF == FMT_BF16, NC);
    static constexpr int kBytes = kTile * ((KF == FMT_BF16 ? 2 * D : KF == FMT_INT8 ? D : D / 2) + 24) + 64;
    // (8 x 64k tokens of 4-bit pages, 8 columns: 119.9, 120.3 and 135.9 us with rings of 4, 6 and 10 stages)
    static constexpr int kFit = 212 * 1024 / (kWarps * kBytes), kStages = kFit > 4 ? 4 : kFit;
    static_assert(kStages >= 2, "the ring needs two stages");
};

template <int KF, int D, int NC, bool G32>
cudaError_t launch_weigh_one(const AttentionParams& p, const WeighPlan& pl, int groups, cudaStream_t stream) {
    using S = WeighShape<KF, D, NC>;
    constexpr int smem = WeighKernel<KF, D, NC, S::kStages, S::kWarps, G32>::kSmemK;
    auto kernel = weigh_split_kernel<KF, D, NC, S::kStages, S::kWarps, G32>;
    static std::atomic<uint64_t> allowed{0};
    const cudaError_t e = allow_smem((const void*)kernel, smem, &allowed);
    if (e != cudaSuccess) return e;
    return launch_pdl(kernel, dim3(pl.s.max_items, groups), dim3(S::kWarps * 32), smem, stream, p, pl);
}
template <int D, int NC>
cudaError_t launch_weigh_columns(const AttentionParams& p, const WeightParams& m, const WeighPlan& pl, int groups, cudaStream_t s) {
    const int kf = k_format(p.c.tag);
    cudaError_t e;
    if (kf == FMT_BF16) e = launch_weigh_one<FMT_BF16, D, NC, true>(p, pl, groups, s);
    else if (kf == FMT_INT8) e = p.c.G == 32 ? launch_weigh_one<FMT_INT8, D, NC, true>(p, pl, groups, s) : launch_weigh_one<FMT_INT8, D, NC, false>(p, pl, groups, s);
    else e = p.c.G == 32 ? launch_weigh_one<FMT_INT4, D, NC, true>(p, pl, groups, s) : launch_weigh_one<FMT_INT4, D, NC, false>(p, pl, groups, s);
    if (e != cudaSuccess) return e;
    const int blocks = (p.b.max_kv_len + kWeighTokens - 1) / kWeighTokens, ctas = std::max(1, 4 * 148 / p.b.n_seqs);
    return launch_pdl(weigh_join_kernel<NC>, dim3(std::min(blocks, ctas), p.b.n_seqs), dim3(kWeighThreads), 0, s, p, m, pl);
}
template <int D>
cudaError_t launch_weigh(const AttentionParams& p, const WeightParams& m, const WeighPlan& pl, int nc, int groups, cudaStream_t s) {
    return nc == 1 ? launch_weigh_columns<D, 1>(p, m, pl, groups, s) : nc == 2 ? launch_weigh_columns<D, 2>(p, m, pl, groups, s)
                                                                               : launch_weigh_columns<D, 4>(p, m, pl, groups, s);
}

}  // namespace patchkv
