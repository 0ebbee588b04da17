// Launches of the kernels of mass_rows.cuh for one head dimension; a translation unit per dimension (mass_rows_64.cu, mass_rows_128.cu).
#pragma once

#include <algorithm>

#include "attention_launch.cuh"
#include "mass_rows.cuh"

namespace patchkv {

template <int KF, int D, bool IMAGE, bool ONE, bool COLUMNS>
cudaError_t launch_weigh_rows_kernel(const AttentionParams& p, const WeighRowsPlan& pl, cudaStream_t stream) {
    auto kernel = weigh_rows_kernel<KF, D, IMAGE, ONE, COLUMNS>;
    static std::atomic<uint64_t> allowed{0};
    const cudaError_t e = allow_smem((const void*)kernel, WeighSmem<D>::kLaunch, &allowed);
    if (e != cudaSuccess) return e;
    const long long items = (long long)pl.chunk_tiles * p.c.H * p.b.n_seqs * pl.splits;
    return launch_pdl(kernel, dim3((unsigned)std::min(items, 148ll)), dim3(weigh_threads(IMAGE)), WeighSmem<D>::kLaunch, stream, p, pl);
}
template <int KF, int D, bool IMAGE, bool ONE>
cudaError_t launch_weigh_rows_passes(const AttentionParams& p, const WeightParams& m, WeighRowsPlan pl, cudaStream_t stream) {
    const int chunk = pl.chunk_tiles;
    pl.chunk = 0;
    pl.chunk_tiles = pl.tiles;
    cudaError_t e = launch_weigh_rows_kernel<KF, D, IMAGE, ONE, false>(p, pl, stream);
    for (int at = 0; e == cudaSuccess && at < pl.tiles; at += chunk) {
        pl.chunk = at;
        pl.chunk_tiles = std::min(chunk, pl.tiles - at);
        pl.last = at + chunk >= pl.tiles;
        e = launch_weigh_rows_kernel<KF, D, IMAGE, ONE, true>(p, pl, stream);
        if (e != cudaSuccess) break;
        cudaLaunchConfig_t cfg;
        memset(&cfg, 0, sizeof(cfg));
        const unsigned steps = (p.b.max_kv_len + kRowTile - 1) / kRowTile;
        const unsigned ctas = pl.chunk_tiles > kWeighJoin / 128 && (long long)steps * p.b.n_seqs * kWeighJoinCtas <= 2 * 148 ? kWeighJoinCtas : 1;
        cfg.gridDim = dim3(steps, p.b.n_seqs, ctas); cfg.blockDim = dim3(128 * std::min(pl.chunk_tiles, kWeighJoin / 128)); cfg.stream = stream;
        cudaLaunchAttribute attr[2];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = 1; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = ctas;
        attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[1].val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = attr; cfg.numAttrs = 2;
        e = cudaLaunchKernelEx(&cfg, weigh_rows_join_kernel, p, m, pl);
    }
    return e;
}
template <int KF, int D>
cudaError_t launch_weigh_rows_format(const AttentionParams& p, const WeightParams& m, const WeighRowsPlan& pl, cudaStream_t s) {
    if constexpr (KF != FMT_BF16)
        if (pl.images) {
            const cudaError_t e = launch_pdl(weigh_image_kernel<KF, D>, dim3(pl.steps, p.c.H, p.b.n_seqs), dim3(kImageThreads), 0, s, p, pl);
            return e != cudaSuccess ? e : launch_weigh_rows_passes<FMT_INT8, D, true, false>(p, m, pl, s);
        }
    return pl.one ? launch_weigh_rows_passes<KF, D, false, true>(p, m, pl, s) : launch_weigh_rows_passes<KF, D, false, false>(p, m, pl, s);
}
template <int D>
cudaError_t launch_weigh_rows(const AttentionParams& p, const WeightParams& m, WeighRowsPlan pl, cudaStream_t s) {
    switch (k_format(p.c.tag)) {
        case FMT_BF16: return launch_weigh_rows_format<FMT_BF16, D>(p, m, pl, s);
        case FMT_INT8: return launch_weigh_rows_format<FMT_INT8, D>(p, m, pl, s);
        default: return launch_weigh_rows_format<FMT_INT4, D>(p, m, pl, s);
    }
}

}  // namespace patchkv
