// Attention weight from few query columns (up to 16 (row, query head) pairs per KV head): the keys are split over the grid and read once.
//
// A weight is known only when the sum over the whole row is, so it takes two passes.  The first is the split attention kernel's
// without its values: it leaves the logits, in fp32, and of each piece the column's sums.  The second adds the pieces' sums
// up and, a token at a time, the weights of all heads and rows.  For 4-bit keys and 8 columns a logit written and read back costs 64 bytes
// for a token and head where reading the keys again costs 72 and turning their codes into operands twice as well.
// One CTA an SM: two of 64 registers a thread took 130 us where one of 128 takes 120 (8 x 64k tokens of 4-bit pages, 8 KV heads of 128, 64
// query heads; now 115 in all, 85 of them this pass: 302 MB of keys and scales read and 134 MB of logits written, 5.1 TB/s).  Neither
// is full: the instructions, some 225 for 16 tokens of a head and 8 columns, take 63 % of the issue slots.  The workspace holds the logits: 4 bytes
// for each row, query head and token that the row's sequence may have.
// Sums run in an order that the arguments fix: no atomics.
#pragma once

#include "attention_split.cuh"
#include "mass.cuh"

namespace patchkv {

struct WeighPlan {
    SplitPlan s;                // its target, items and head layout; partial and item_stride are not used
    float* logits;              // [sequence][KV head][cols][tokens]: log2 of the weights but for their sums; -infinity where a row sees none
    float2* sums;               // [item][KV head][4 * NC]: reference and sum of a column over the piece
    int32_t tokens;             // of a sequence in `logits`: 16 for each virtual tile
    int32_t cols;               // columns of a KV head in `logits`
};
template <int D>
cudaError_t launch_weigh(const AttentionParams& p, const WeightParams& m, const WeighPlan& pl, int nc, int groups, cudaStream_t s);

// Sums need no 16-bit weights here: a reference is moved only when fp32 runs short.
constexpr float kWeighTop = 60.0f;

template <int KF, int D, int NC, int STAGES, int WARPS, bool G32>
struct WeighKernel : SplitKernel<KF, KF, D, NC, STAGES, WARPS, G32> {
    using B = SplitKernel<KF, KF, D, NC, STAGES, WARPS, G32>;
    static constexpr int kScalesAt = kTile * B::kKStride, kStageK = kScalesAt + (B::kPool ? 0 : kTile * 8);
    static constexpr int kSmemK = WARPS * (STAGES * kStageK + B::kCold);

    __device__ __forceinline__ WeighKernel(const AttentionParams& p_) : B(p_) {}

    // SplitKernel::fetch without the values.
    __device__ __forceinline__ void fetch_keys(uint32_t base, long long at, uint32_t row0, bool whole, bool present, int t0) {
        constexpr int kc = B::kKRow / 16;
        const CacheDev& c = this->p.c;
        const int lane = this->lane;
        const uint32_t dst = base + (lane / kc) * B::kKStride + (lane % kc) * 16;
        if constexpr (B::kPool) {
            const uint8_t* k = reinterpret_cast<const uint8_t*>(c.k) + at + (lane % kc) * 16;
#pragma unroll
            for (int i = 0; i < kTile * kc / 32; i++) {
                const int tok = lane / kc + i * (32 / kc);
                const bool live = whole || (present && t0 + tok <= min(this->hi_pos(), this->kv() - 1) && sees(this->p, this->lo_pos(), t0 + tok));
                cp16(dst + i * (32 / kc) * B::kKStride, k + (live ? 2 * tok * c.stride_token : 0), live);
            }
        } else {
            const uint8_t* pg = c.base + at;
            const uint8_t* ks = pg + (row0 * B::kKRow + this->k_off);
#pragma unroll
            for (int i = 0; i < kTile * kc / 32; i++) cp16(dst + i * (32 / kc) * B::kKStride, ks + i * (32 / kc) * B::kKRow * c.H, present);
            if (lane < 16) {
                const uint8_t* sc = pg + (row0 * (uint32_t)this->scales_per_row() * 2 + this->s_off);
                const int tok = t0 + lane;
                const bool live = whole || (present && tok <= min(this->hi_pos(), this->kv() - 1) && sees(this->p, this->lo_pos(), tok));
                if (D == 128 && G32) cp_small<8>(base + kScalesAt + lane * 8, sc, live);
                else cp_small<4>(base + kScalesAt + lane * 8, reinterpret_cast<const uint8_t*>(reinterpret_cast<uintptr_t>(sc) & ~(uintptr_t)3), live);
            }
        }
    }

    // The logits of a tile's tokens g and g + 8, as in SplitKernel::tile.
    __device__ __forceinline__ void logits(uint32_t base, uint32_t row0, float (&x)[NC][2]) {
        constexpr int NT = B::NT;
        const int lane = this->lane, g = this->g, t = this->t;
        if constexpr (B::kPool) {
            float y[NT][4];
#pragma unroll
            for (int nt = 0; nt < NT; nt++)
#pragma unroll
                for (int i = 0; i < 4; i++) y[nt][i] = 0.0f;
            const uint32_t a = base + ((lane & 7) + (lane & 8)) * B::kKStride + (lane >> 4) * 16;
#pragma unroll
            for (int k = 0; k < B::kMT; k++) {
                uint32_t r[4];
                ldmatrix4(r, a + 32 * k);
#pragma unroll
                for (int nt = 0; nt < NT; nt++) mma_bf16(y[nt], r[0], r[1], r[2], r[3], this->qf[nt][k][0], this->qf[nt][k][1]);
            }
#pragma unroll
            for (int c = 0; c < NC; c++) { x[c][0] = y[c >> 1][c & 1]; x[c][1] = y[c >> 1][2 + (c & 1)]; }
        } else {
            uint32_t odd_a = 0, odd_b = 0;
            if (!G32 && this->p.c.G == D) {                                // which half of the word a lone scale is
                odd_a = (row0 + g * this->p.c.H) & 1;
                odd_b = (row0 + (g + 8) * this->p.c.H) & 1;
            }
            const uint2 sa = lds64(base + kScalesAt + 8 * g), sb = lds64(base + kScalesAt + 8 * (g + 8));
            const uint32_t ra = base + g * B::kKStride + 4 * t, rb = ra + 8 * B::kKStride;
#pragma unroll
            for (int j = 0; j < B::kChunks; j++) {
                float y[NT][4];
                uint32_t wa, wb;
                if constexpr (B::kK4) { wa = lds32(ra + 16 * j); wb = lds32(rb + 16 * j); }
#pragma unroll
                for (int m = 0; m < 2; m++) {
                    uint32_t a0, a1, a2, a3;
                    if constexpr (B::kK4) {
                        a0 = and_xor<0x000F000Fu>(wa, this->flip0); a1 = and_xor<0x000F000Fu>(wb, this->flip0);
                        a2 = and_xor<0x00F000F0u>(wa, this->flip1); a3 = and_xor<0x00F000F0u>(wb, this->flip1);
                        if (m == 0) { wa >>= 8; wb >>= 8; }
                    } else {
                        wa = lds32(ra + 32 * j + 16 * m) ^ 0x80808080u;
                        wb = lds32(rb + 32 * j + 16 * m) ^ 0x80808080u;
                        a0 = __byte_perm(wa, 0, 0x4140); a1 = __byte_perm(wb, 0, 0x4140);
                        a2 = __byte_perm(wa, 0, 0x4342); a3 = __byte_perm(wb, 0, 0x4342);
                    }
#pragma unroll
                    for (int q = 0; q < NT; q++) {
                        if (m == 0) mma_f16(y[q], a0, a1, a2, a3, this->qf[q][2 * j][0], this->qf[q][2 * j][1], this->bias[q][j][0], this->bias[q][j][1]);
                        else mma_f16(y[q], a0, a1, a2, a3, this->qf[q][2 * j + 1][0], this->qf[q][2 * j + 1][1]);
                    }
                }
                const float fa = this->chunk_scale(sa, j, odd_a), fb = this->chunk_scale(sb, j, odd_b);
#pragma unroll
                for (int c = 0; c < NC; c++) {
                    const float ya = y[c >> 1][c & 1], yb = y[c >> 1][2 + (c & 1)];
                    x[c][0] = j ? fmaf(ya, fa, x[c][0]) : ya * fa;
                    x[c][1] = j ? fmaf(yb, fb, x[c][1]) : yb * fb;
                }
            }
        }
#pragma unroll
        for (int c = 0; c < NC; c++) { x[c][0] = finite_low(x[c][0] * this->factor[c]); x[c][1] = finite_low(x[c][1] * this->factor[c]); }
    }
    // -infinity stands for a token that the row does not see; one that it sees, of an infinite key or query, has the weight that its
    // row's sum gives it (NaN where that is NaN).  A row that has no other logits keeps its first reference: weigh_join_kernel makes its sum NaN.
    __device__ __forceinline__ static float finite_low(float x) {
        float y;
        asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(x), "f"(kNoMax));
        return y;
    }
};

template <int KF, int D, int NC, int STAGES, int WARPS, bool G32>
__global__ void __launch_bounds__(WARPS * 32, 1) weigh_split_kernel(const __grid_constant__ AttentionParams p, const __grid_constant__ WeighPlan pl) {
    using K = WeighKernel<KF, D, NC, STAGES, WARPS, G32>;
    extern __shared__ __align__(16) uint8_t smem[];
    pdl_trigger();
    pdl_wait();
    const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    __shared__ Item found;
    __shared__ float2 merge[WARPS][4 * NC];
    if (warp == 0) {
        const Item x = find_item(p, pl.s, blockIdx.x);
        if (lane == 0) found = x;
    }
    __syncthreads();
    const Item it = found;
    if (!it.ok) return;
    const int heads = 1 << pl.s.heads_log2, local = warp & (heads - 1), sub = warp >> pl.s.heads_log2, head = blockIdx.y * heads + local;
    const bool live = head < p.c.H;
    const int cols = min(it.rows * p.share, 4 * NC);
    K k(p);
    k.start(lane, smem_u32(smem) + warp * STAGES * K::kStageK, smem_u32(smem) + WARPS * STAGES * K::kStageK + warp * K::kCold);
    if (live) {
        k.ask_queries(it.first, cols, head, pl.s.share_magic);
        const int step = 1 << pl.s.per_head_log2, n = it.begin + sub < it.end ? (it.end - it.begin - sub + step - 1) >> pl.s.per_head_log2 : 0;
        uint32_t* cold = reinterpret_cast<uint32_t*>(smem + WARPS * STAGES * K::kStageK + warp * K::kCold);
        if (lane == 0) {
            const TileRange range = tile_range(p, it.kv, it.lo, it.hi);
            const uint64_t table = reinterpret_cast<uint64_t>(p.b.block_table + (long long)it.seq * p.b.table_stride);
            cold[0] = it.kv; cold[1] = it.lo; cold[2] = it.hi;
            cold[3] = it.begin + sub; cold[4] = pl.s.per_head_log2; cold[5] = range.sink_tiles; cold[6] = range.first;
            cold[7] = it.least;
            cold[8] = (uint32_t)table; cold[9] = (uint32_t)(table >> 32);
        }
        if (lane < 4 * NC) cold[12 + lane] = lane < cols ? row_position(p.b, it.seq, it.first + (int)(lane * pl.s.share_magic >> 16)) : -1;
        __syncwarp();
        struct Place { long long at; uint32_t row0, flags; };        // of a tile: flags bit 0 whole, bit 1 has a page
        auto place_of = [&](int i) {
            Place o = {0, 0, 0};
            if (i < n && k.some_row_sees(k.first_token(i))) {
                const int t0 = k.first_token(i), lp = div_page(p.c, t0), slot0 = t0 - lp * p.c.P;
                const int pg = *(k.table() + lp);
                o.row0 = (uint32_t)slot0 * p.c.H + head;
                if (pg < 0 || pg >= p.c.n_pages) {
                    latch(p.status);
                } else {
                    o.at = K::kPool ? 2 * ((long long)pg * p.c.stride_page + (long long)slot0 * p.c.stride_token + (long long)head * p.c.stride_head)
                                    : (long long)pg * p.c.stride_page;
                    const int lo = k.lo_whole(), hi = k.hi_pos();
                    o.flags = t0 + kTile - 1 <= min(lo, k.kv() - 1) && (p.window == 0 || hi - t0 < p.window || t0 + kTile <= p.sinks) ? 3 : 2;
                }
            }
            return o;
        };
        Place here = place_of(lane);
        uint32_t whole = 0, present = 0, odd = 0;            // bit j: flags (and row0 & 1) of the tile fetched j ago
        uint32_t fetch_base = k.ring, base = k.ring;
        auto fetch = [&](int i) {
            const uint32_t flags = __shfl_sync(0xFFFFFFFFu, here.flags, i & 31), row0 = __shfl_sync(0xFFFFFFFFu, here.row0, i & 31);
            const long long at = __shfl_sync(0xFFFFFFFFu, here.at, i & 31);
            if (i < n) {
                if (flags & 1) k.fetch_keys(fetch_base, at, row0, true, true, 0);
                else k.fetch_keys(fetch_base, at, row0, false, flags >> 1, k.first_token(i));
            }
            cp_commit();
            if ((i & 31) == 31) here = place_of(i + 1 + lane);
            whole = whole << 1 | (flags & 1);
            present = present << 1 | flags >> 1;
            if (!G32) odd = odd << 1 | (row0 & 1);
            fetch_base = fetch_base == k.ring + (STAGES - 1) * K::kStageK ? k.ring : fetch_base + K::kStageK;
        };
#pragma unroll 1
        for (int i = 0; i < STAGES - 1; i++) fetch(i);
        k.load_queries();
        // The lane's columns in the logits; tokens of a tile lie together.
        float* to[NC];
        bool mine[NC];
#pragma unroll
        for (int c = 0; c < NC; c++) {
            const int col = column_of(c, k.t);
            mine[c] = col < cols;
            to[c] = pl.logits + (((long long)it.seq * p.c.H + head) * pl.cols + (mine[c] ? col : 0)) * pl.tokens + (long long)(it.begin + sub) * kTile + k.g;
        }
#pragma unroll 1
        for (int i = 0; i < n; i++) {
            fetch(i + STAGES - 1);
            cp_wait<STAGES - 1>();
            __syncwarp();
            const bool w = whole >> (STAGES - 1) & 1, there = present >> (STAGES - 1) & 1;
            float x[NC][2];
            k.logits(base, odd >> (STAGES - 1) & 1, x);
            if (!w) {
                const int t0 = k.first_token(i);
#pragma unroll
                for (int c = 0; c < NC; c++)
#pragma unroll
                    for (int e = 0; e < 2; e++) {
                        const int tok = t0 + k.g + 8 * e, ps = k.pos(c);
                        if (!(there && tok <= ps && tok < k.kv() && sees(p, ps, tok))) x[c][e] = -INFINITY;
                    }
            }
#pragma unroll
            for (int c = 0; c < NC; c++) {
                if (mine[c]) { to[c][0] = x[c][0]; to[c][8] = x[c][1]; }
                to[c] += kTile << pl.s.per_head_log2;
            }
            float most = kNoMax;
#pragma unroll
            for (int c = 0; c < NC; c++) most = fmaxf(most, fmaxf(x[c][0], x[c][1]) - k.ref[c]);
            if (__any_sync(0xFFFFFFFFu, most > kWeighTop)) {
#pragma unroll
                for (int c = 0; c < NC; c++) {
                    float m = fmaxf(x[c][0], x[c][1]);
                    m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 4));
                    m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 8));
                    m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 16));
                    if (m > k.ref[c] + kWeighTop) {
                        k.sum[c] *= fast_exp2(k.ref[c] - m);
                        k.ref[c] = m;
                    }
                }
            }
#pragma unroll
            for (int c = 0; c < NC; c++) k.sum[c] += fast_exp2(x[c][0] - k.ref[c]) + fast_exp2(x[c][1] - k.ref[c]);
            __syncwarp();                                    // the stage may be filled again
            base = base == k.ring + (STAGES - 1) * K::kStageK ? k.ring : base + K::kStageK;
        }
        cp_wait<0>();
    }
    if (it.split == 0 && blockIdx.y == 0 && threadIdx.x == 0) {
        pl.s.items[2 * it.seq] = it.first_item;
        pl.s.items[2 * it.seq + 1] = it.splits;
    }
#pragma unroll
    for (int c = 0; c < NC; c++) {
        k.sum[c] += __shfl_xor_sync(0xFFFFFFFFu, k.sum[c], 4);
        k.sum[c] += __shfl_xor_sync(0xFFFFFFFFu, k.sum[c], 8);
        k.sum[c] += __shfl_xor_sync(0xFFFFFFFFu, k.sum[c], 16);
        if (lane < 4) merge[warp][column_of(c, lane)] = make_float2(k.ref[c], k.sum[c]);
    }
    __syncthreads();
    if (!live || sub != 0 || lane >= 4 * NC) return;
    float m = kNoMax, l = 0.0f;
    for (int w = local; w < WARPS; w += heads) m = fmaxf(m, merge[w][lane].x);
    for (int w = local; w < WARPS; w += heads) l = fmaf(fast_exp2(merge[w][lane].x - m), merge[w][lane].y, l);
    pl.sums[((long long)blockIdx.x * p.c.H + head) * (4 * NC) + lane] = make_float2(m, l);
}

// Second pass (grid: CTAs of a sequence, sequence): a CTA takes every gridDim.x-th 256 tokens, a thread four tokens and a quarter of the columns.
// Bound by the latency of reading the logits (134 MB in 31 us, some of it from L2; captured 3.2 TB/s of DRAM, warps waiting on loads); the
// columns' sums are found once a CTA, so there are no more of those than fill the SMs (four an SM: 114.5 us a call, six 118.3, three 116.9).  A thread has eight logits of each token on their way (144 us a call with one, 131 with
// eight, 143 with sixteen, when it was made).
constexpr int kWeighTokens = 256, kWeighThreads = 256, kWeighColumns = 256;
template <int NC>
__global__ void __launch_bounds__(kWeighThreads, 4) weigh_join_kernel(const __grid_constant__ AttentionParams p, const __grid_constant__ WeightParams m,
                                                                   const __grid_constant__ WeighPlan pl) {
    __shared__ float2 column[kWeighColumns];                 // log2 of a column's sum, and its place in the logits (a whole number's bits)
    __shared__ float2 pieces_of[kWeighThreads];
    __shared__ float4 part[3][kWeighTokens / 4];
    pdl_trigger();
    pdl_wait();
    const int s = gridDim.y - 1 - blockIdx.y;                 // the last sequences' logits are still in L2 (129.5 for 130.9 us)
    int first, kv, rows, lo, hi, least;
    if (!sequence_rows(p, s, &first, &kv, &rows) || (int)blockIdx.x * kWeighTokens >= kv) return;
    const int quad = threadIdx.x & (kWeighTokens / 4 - 1), part_of = threadIdx.x / (kWeighTokens / 4);
    position_range(p, s, first, rows, &lo, &hi, &least);
    const TileRange range = tile_range(p, kv, lo, hi);
    const int all = rows == 0 ? 0 : min(min(rows, p.b.max_rows) * p.share, 4 * NC);
    const int item0 = all ? pl.s.items[2 * s] : 0, pieces = all ? pl.s.items[2 * s + 1] : 0, columns = p.c.H * all;
    const float* logits = pl.logits + (long long)s * p.c.H * pl.cols * pl.tokens;
    // log2 of the sums of columns j0 .. j0 + n - 1: several threads share a column's pieces.
    auto sums_of = [&](int j0, int n) {
        const int shares = kWeighThreads / n, j = (int)threadIdx.x % n, share = (int)threadIdx.x / n;
        const int h = (j0 + j) / all, c = (j0 + j) - h * all;
        float top = kNoMax, sum = 0.0f;
        if (share < shares) {
            const float2* ml = pl.sums + ((long long)item0 * p.c.H + h) * (4 * NC) + c;
#pragma unroll 4
            for (int i = share; i < pieces; i += shares) {
                const float2 z = ml[(long long)i * p.c.H * (4 * NC)];
                const float to = fmaxf(top, z.x);
                sum = fmaf(sum, fast_exp2(top - to), z.y * fast_exp2(z.x - to));
                top = to;
            }
        }
        __syncthreads();                                     // nobody reads the columns before any more
        pieces_of[threadIdx.x] = make_float2(top, sum);
        __syncthreads();
        if (threadIdx.x < n) {
            for (int i = 1; i < shares; i++) {
                const float2 z = pieces_of[i * n + j];
                const float to = fmaxf(top, z.x);
                sum = fmaf(sum, fast_exp2(top - to), z.y * fast_exp2(z.x - to));
                top = to;
            }
            const float total = sum == 0.0f ? INFINITY : top == kNoMax ? __uint_as_float(0x7FC00000u) : top + log2f(sum);
            column[j] = make_float2(total, __int_as_float(h * pl.cols + c));
        }
        __syncthreads();
    };
    if (columns > 0 && columns <= kWeighColumns) sums_of(0, columns);
#pragma unroll 1
    for (int t0 = blockIdx.x * kWeighTokens; t0 < kv; t0 += gridDim.x * kWeighTokens) {
        // the place of this thread's tokens in the logits
        const int tile = (t0 + 4 * quad) / kTile, v = tile < range.sink_tiles ? tile : tile - range.first + range.sink_tiles;
        const bool seen = tile < range.sink_tiles || (tile >= range.first && v < range.count);
        const float* from = logits + (long long)v * kTile + (4 * quad & (kTile - 1));
        float4 y = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 1
        for (int j0 = 0; j0 < columns; j0 += kWeighColumns) {
            const int n = min(columns - j0, kWeighColumns);
            if (columns > kWeighColumns) sums_of(j0, n);
            if (!seen) continue;
            // (a token that the row does not see has no weight, whatever the row's sum is)
            auto weight = [](float x, float total) { return x == -INFINITY ? 0.0f : fast_exp2(x - total); };
            constexpr int kAtOnce = 8;
#pragma unroll 1
            for (int j = part_of; j < n; j += 4 * kAtOnce) {
                float4 x[kAtOnce];
#pragma unroll
                for (int i = 0; i < kAtOnce; i++)
                    if (j + 4 * i < n) x[i] = *reinterpret_cast<const float4*>(from + (long long)__float_as_int(column[j + 4 * i].y) * pl.tokens);
#pragma unroll
                for (int i = 0; i < kAtOnce; i++)
                    if (j + 4 * i < n) {
                        const float total = column[j + 4 * i].x;
                        y.x += weight(x[i].x, total);
                        y.y += weight(x[i].y, total);
                        y.z += weight(x[i].z, total);
                        y.w += weight(x[i].w, total);
                    }
            }
        }
        if (part_of) part[part_of - 1][quad] = y;
        __syncthreads();
        if (!part_of) {
#pragma unroll
            for (int i = 0; i < 3; i++) {
                const float4 z = part[i][quad];
                y.x += z.x; y.y += z.y; y.z += z.z; y.w += z.w;
            }
            const int t = t0 + 4 * quad;
            if (t < kv) store_mass(p, m, s, t, y.x);
            if (t + 1 < kv) store_mass(p, m, s, t + 1, y.y);
            if (t + 2 < kv) store_mass(p, m, s, t + 2, y.z);
            if (t + 3 < kv) store_mass(p, m, s, t + 3, y.w);
        }
        __syncthreads();
    }
}

}  // namespace patchkv
