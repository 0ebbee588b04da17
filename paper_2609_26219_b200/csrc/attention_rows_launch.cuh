// Launches of the row kernels (attention_rows.cuh) for one head dimension.  A translation unit per dimension instantiates them
// (attention_rows_64.cu, attention_rows_128.cu), so that they compile side by side.
#pragma once

#include <algorithm>

#include "attention_launch.cuh"
#include "attention_rows.cuh"

namespace patchkv {

template <int KF, int VF, int D, bool IMAGE, bool ONE, bool FINE>
cudaError_t launch_rows_kernel(const AttentionParams& p, const RowsPlan& pl, cudaStream_t stream) {
    auto kernel = attention_rows_kernel<KF, VF, D, IMAGE, ONE, FINE>;
    static std::atomic<uint64_t> allowed{0};
    const cudaError_t e = allow_smem((const void*)kernel, RowsSmem<D>::kLaunch, &allowed);
    if (e != cudaSuccess) return e;
    return launch_pdl(kernel, dim3(pl.tiles * p.c.H * p.b.n_seqs * pl.splits), dim3(rows_threads(IMAGE)), RowsSmem<D>::kLaunch, stream, p, pl);
}
template <int KF, int VF, int D, bool FINE>
cudaError_t launch_rows_one(const AttentionParams& p, const RowsPlan& pl, cudaStream_t stream) {
    cudaError_t e;
    if (pl.images) {
        e = launch_pdl(attention_image_kernel<KF, VF, D, FINE>, dim3(pl.steps, p.c.H, p.b.n_seqs), dim3(kImageThreads), 0, stream, p, pl);
        if (e != cudaSuccess) return e;
        constexpr int F = KF == FMT_BF16 ? FMT_BF16 : FMT_INT8;
        e = launch_rows_kernel<F, F, D, true, false, FINE>(p, pl, stream);
    } else if ((long long)std::min(p.b.max_rows, p.b.n_rows) * p.share <= kRowTile) {
        e = launch_rows_kernel<KF, VF, D, false, true, FINE>(p, pl, stream);
    } else {
        e = launch_rows_kernel<KF, VF, D, false, false, FINE>(p, pl, stream);
    }
    if (e != cudaSuccess || pl.splits == 1) return e;
    const long long vectors = (long long)std::min(p.b.max_rows, p.b.n_rows) * p.Hq;          // of a sequence at most
    return launch_pdl(attention_rows_join_kernel<D>, dim3((unsigned)((vectors + 3) / 4), p.b.n_seqs), dim3(128), 0, stream, p, pl);
}
template <int KF, int VF, int D>
cudaError_t launch_rows_type(const AttentionParams& p, const RowsPlan& pl, cudaStream_t s) {
    return p.f16 ? launch_rows_one<KF, VF, D, true>(p, pl, s) : launch_rows_one<KF, VF, D, false>(p, pl, s);
}
template <int D>
cudaError_t launch_rows(const AttentionParams& p, const RowsPlan& pl, cudaStream_t s) {
    switch (p.c.tag) {
        case PATCHKV_TAG_BF16: return launch_rows_one<FMT_BF16, FMT_BF16, D, false>(p, pl, s);
        case PATCHKV_TAG_INT8: return launch_rows_type<FMT_INT8, FMT_INT8, D>(p, pl, s);
        case PATCHKV_TAG_INT4: return launch_rows_type<FMT_INT8, FMT_INT4, D>(p, pl, s);
        default: return launch_rows_type<FMT_INT4, FMT_INT4, D>(p, pl, s);
    }
}

}  // namespace patchkv
