// Launches of the split kernels (attention_split.cuh) for one head dimension.  A translation unit per dimension instantiates them
// (attention_split_64.cu, attention_split_128.cu), so that they compile side by side.
#pragma once

#include "attention_launch.cuh"
#include "attention_split.cuh"

namespace patchkv {

template <int KF, int VF, int D, int NC>
struct SplitShape {
    static constexpr int kWarps = split_warps(KF == FMT_BF16, NC);
    static constexpr int kBytes = kTile * ((KF == FMT_BF16 ? 2 * D : KF == FMT_INT8 ? D : D / 2) + (VF == FMT_BF16 ? 2 * D : VF == FMT_INT8 ? D : D / 2) + 32) + 256;
    static constexpr int kFit = 220 * 1024 / (kWarps * kBytes);
    static constexpr int kStages = kFit > 4 ? 4 : kFit;
    static_assert(kStages >= 2, "the ring needs two stages");
};

template <int KF, int VF, int D, int NC, bool G32>
cudaError_t launch_split_one(const AttentionParams& p, const SplitPlan& pl, int groups, cudaStream_t stream) {
    using S = SplitShape<KF, VF, D, NC>;
    using K = SplitKernel<KF, VF, D, NC, S::kStages, S::kWarps, G32>;
    constexpr int smem = K::kSmem > K::kMerge ? K::kSmem : K::kMerge;
    auto kernel = attention_split_kernel<KF, VF, D, NC, S::kStages, S::kWarps, G32>;
    static std::atomic<uint64_t> allowed{0};
    cudaError_t e = allow_smem((const void*)kernel, smem, &allowed);
    if (e != cudaSuccess) return e;
    e = launch_pdl(kernel, dim3(pl.max_items, groups), dim3(S::kWarps * 32), smem, stream, p, pl);
    if (e != cudaSuccess || pl.target == 0) return e;
    const dim3 grid(p.b.n_seqs, p.c.H, (NC == 1 ? 2 : 2 * NC) * (D / 16) / 4);
    if (pl.max_items > 16 * p.b.n_seqs) return launch_pdl(attention_join_kernel<KF == FMT_BF16, D, NC, 16>, grid, dim3(512), 0, stream, p, pl);
    return launch_pdl(attention_join_kernel<KF == FMT_BF16, D, NC, 4>, grid, dim3(128), 0, stream, p, pl);
}
template <int D, int NC, bool G32>
cudaError_t launch_split_tag(const AttentionParams& p, const SplitPlan& pl, int groups, cudaStream_t s) {
    switch (p.c.tag) {
        case PATCHKV_TAG_INT8: return launch_split_one<FMT_INT8, FMT_INT8, D, NC, G32>(p, pl, groups, s);
        case PATCHKV_TAG_INT4: return launch_split_one<FMT_INT8, FMT_INT4, D, NC, G32>(p, pl, groups, s);
        default: return launch_split_one<FMT_INT4, FMT_INT4, D, NC, G32>(p, pl, groups, s);
    }
}
template <int D, int NC>
cudaError_t launch_split_group(const AttentionParams& p, const SplitPlan& pl, int groups, cudaStream_t s) {
    if (p.c.tag == PATCHKV_TAG_BF16) return launch_split_one<FMT_BF16, FMT_BF16, D, NC, true>(p, pl, groups, s);
    return p.c.G == 32 ? launch_split_tag<D, NC, true>(p, pl, groups, s) : launch_split_tag<D, NC, false>(p, pl, groups, s);
}
template <int D>
cudaError_t launch_split(const AttentionParams& p, const SplitPlan& pl, int nc, int groups, cudaStream_t s) {
    return nc == 1 ? launch_split_group<D, 1>(p, pl, groups, s) : nc == 2 ? launch_split_group<D, 2>(p, pl, groups, s) : launch_split_group<D, 4>(p, pl, groups, s);
}

}  // namespace patchkv
