// Attention weight from many query vectors, on the 5th-generation tensor cores.
//
// As in the row kernel of the attention a CTA takes one KV head and up to 256 query vectors of it, in one or two tiles of 128, and walks
// the keys in steps of 128 tokens.  It does so twice, since a weight is known only when the sum over its row is:
//   first pass    S = Q K^T, a lane of TMEM per query vector; a thread adds up 2^(S - ref) over the tokens of its row
//   second pass   S = K Q^T, a lane per token; a thread adds up 2^(S - log2 of the row's sum) over the vectors of the CTA
// In both the sum runs along a thread's own lane, so nothing is exchanged, and nothing comes behind the sums: the products of the next
// steps run while a step is added up.  Four warpgroups do that, two (a pair) for each tile, half of the columns each, with two places
// in TMEM for each pair; with one tile of vectors the pairs take turns at the steps.  (Two warpgroups, a tile each, were as fast in
// the first pass, where the exponential unit is the bound.)  The second pass leaves a number for each token, head and CTA, which
// the last kernel adds up in an order that the arguments fix.
// Keys as operands: bf16 as they are, quantised ones as the sum of two fp16 matrices (22 bits), for two products per 16 channels.  One fp16 matrix alone would put a logit 2^-12 of its terms off and the masses 1e-4.  With many tiles of vectors the operands are
// laid out in the workspace first (images), as for the attention; else each CTA makes them from the pages, eight warps of it.
// A step of two tiles takes 1024 cycles of products (quantised 2048) and 2048 cycles of the exponential unit.  8192 rows of 32 query heads over
// 8192 tokens, 8 KV heads of 128 channels: 459 and 478 us for the passes on quantised pages (1.2 PFLOP/s each, both matrices counted, at the
// 1.67 GHz that the power limit leaves), 15 for the images, 15 for the last sum; 740 us in all on a bf16 pool.  Few rows are bound by the
// way to the first product and by the keys' bytes: 32 rows over 32k tokens of a pool 22 and 25 us (67 MB each), 58 in all.
#pragma once

#include <cooperative_groups.h>

#include "attention_rows.cuh"
#include "mass.cuh"

namespace patchkv {

struct WeighRowsPlan {
    float2* sums;               // [split][n_rows * Hq]: reference and sum of a vector over a piece of the tokens
    int4* ranges;               // [sequence][tile]: sink steps, first step and count of the steps that a CTA's rows see
    float* partial;             // [sequence][KV head][tile of the chunk][tokens]: what a CTA's vectors give to a token
    int32_t tiles, splits;      // CTAs along the vectors of a sequence, and along the tokens
    int32_t chunk, chunk_tiles; // the second pass: first tile, and number of tiles, of this launch
    int32_t one;                // no sequence has more than 128 vectors
    int32_t tokens;             // of a tile in `partial`: 128 for each of its steps
    uint8_t* images;            // [sequence][step][KV head]: the matrix of K and what it leaves of K; null: no images
    uint32_t* meta;             // of each image: 4 words of absent tokens, 4 unused
    int32_t steps;              // of a sequence in the two
    double* acc;                // [sequence][max_kv_len]: the chunks before; null: only one
    int32_t last;               // the last chunk
};
template <int D>
cudaError_t launch_weigh_rows(const AttentionParams& p, const WeightParams& m, WeighRowsPlan pl, cudaStream_t s);

constexpr int kWeighConsumers = 512, kWeighProducers = 256;
__host__ __device__ constexpr int weigh_issuer(bool image) { return kWeighConsumers + (image ? 32 : kWeighProducers); }
__host__ __device__ constexpr int weigh_threads(bool image) { return weigh_issuer(image) + 64; }        // and the warp that finds the work

// A piece of work: up to 256 vectors of a KV head and some of the tokens that they see.
struct WeighItem {
    int32_t ok;                 // 0: there is no more work
    int32_t seq, head, tile, split, first, kv, m0, m_end, tiles;
    int32_t lo, least, hi;      // smallest position not below 0, smallest and largest of the rows
    TileRange range;
    int32_t begin, end;         // its steps of the range
};
struct WeighBars {
    uint64_t item_full[2], item_empty[2];
    uint64_t q_ready[2];                                            // [tile] the queries are there, and what goes with them
    uint64_t q_free;                                                // the products of an item are done
    uint64_t mate_done[2];                                          // [pair] its other warpgroups are through with an item
    uint64_t second_done;                                           // first pass: so is the whole of the second pair, with an item of two tiles
    uint64_t s_full[2][2], s_empty[2][2], k_full[4], k_empty[4];    // [pair][place in TMEM]; stages of the ring of keys
    uint64_t part_full[4][4];                                       // second pass: [warpgroup][unit mod 4] its sum is there
    uint64_t drained;
    alignas(16) uint32_t absent[8][8];                              // per step (mod 8): tokens whose page is out of range
    WeighItem item[2];
    float factor[256];                                              // of the vectors' logits
    int32_t pos[256];
    alignas(16) float scale[256], low[256];                         // second pass: the factors again, and -log2 of the vectors' sums
    float2 sums[4][kRowTile];                                       // first pass: [warpgroup] reference and sum
    float part[4][4][kRowTile];                                     // second pass: [unit mod 4][warpgroup]
    uint32_t tmem;
    int32_t abort;
};
template <int D>
struct WeighSmem {
    static constexpr int kBytes = RowsSmem<D>::kBars + (int)sizeof(WeighBars) + 1024;
    static constexpr int kLaunch = kBytes > 120 * 1024 ? kBytes : 120 * 1024;       // one CTA per SM: it takes all of TMEM
};
static_assert(WeighSmem<128>::kLaunch <= 227 * 1024, "shared memory");

// 2^y of a pair, as RowsKernel::exp2_pair with one more term (2.1e-7).
__device__ __forceinline__ void weigh_exp2_pair(f32x2 y2, float& a, float& b) {
    float u, v;
    unpack2(y2, u, v);
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(u) : "f"(-127.0f));
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(v) : "f"(-127.0f));
    asm("min.NaN.f32 %0, %0, %1;" : "+f"(u) : "f"(126.0f));
    asm("min.NaN.f32 %0, %0, %1;" : "+f"(v) : "f"(126.0f));
    const f32x2 y = pack2(u, v), magic = pack2(12582912.0f, 12582912.0f);       // 1.5 * 2^23
    const f32x2 t = add2(y, magic), f = sub2(y, sub2(t, magic));
    f32x2 e = fma2(f, pack2(0.001327647129073739f, 0.001327647129073739f), pack2(0.009675541892647743f, 0.009675541892647743f));
    e = fma2(e, f, pack2(0.05550713092088699f, 0.05550713092088699f));
    e = fma2(e, f, pack2(0.24022120237350464f, 0.24022120237350464f));
    e = fma2(e, f, pack2(0.6931469440460205f, 0.6931469440460205f));
    e = fma2(e, f, pack2(1.0000001192092896f, 1.0000001192092896f));
    float n0, n1;
    unpack2(t, n0, n1);
    unpack2(mul2(e, pack2(__uint_as_float((__float_as_uint(n0) << 23) + 0x3F800000u), __uint_as_float((__float_as_uint(n1) << 23) + 0x3F800000u))), a, b);
}
// KF: format of the keys; IMAGE: they come as images (KF = FMT_INT8 stands for those).  ONE: no sequence has more than one tile of vectors.
// COLUMNS: the second pass.  A CTA stays on its SM and takes one item after the other: setting one up (12 us of 40 when every
// item was a CTA of its own) goes on under the products of the one before, but for the queries, which have one place.  Counters run through
// all items: g steps, u the units (steps of a tile) of a pair.
template <int KF, int D, bool IMAGE, bool ONE, bool COLUMNS>
struct WeighRows {
    static constexpr bool FINE = KF != FMT_BF16, kPool = KF == FMT_BF16;
    using B = RowsKernel<KF, KF, D, IMAGE, FINE>;
    using S = RowsSmem<D>;
    static constexpr int kStages = FINE ? 2 : 4, kPer = D / 32, kTok = 32 / kPer;
    static constexpr uint32_t kStage = (FINE ? 2 : 1) * S::kMat;
    const AttentionParams& p;
    const WeighRowsPlan& pl;
    WeighBars& w;
    const uint32_t smem;
    WeighItem it;
    int last;                                                       // a step up to this token needs no mask

    __device__ __forceinline__ WeighRows(const AttentionParams& p_, const WeighRowsPlan& pl_, WeighBars& w_, uint32_t smem_) : p(p_), pl(pl_), w(w_), smem(smem_) {}
    // A wait of a whole warp: all of its lanes go on, or none.
    __device__ __forceinline__ bool wait(uint64_t* bar, uint32_t parity) { return __all_sync(0xFFFFFFFFu, mbar_wait(bar, parity, &w.abort)); }
    __device__ __forceinline__ void arrive(uint64_t* bar) {
        __syncwarp();
        if ((threadIdx.x & 31) == 0) mbar_arrive(bar);
    }
    __device__ __forceinline__ static uint32_t turn(int n) { return (uint32_t)(n / kStages) & 1u; }
    __device__ __forceinline__ uint32_t key_stage(int n) const { return smem + S::kK + (n % kStages) * kStage; }
    // Seen by some row (or by none): only then does a token's slot take part.  The same exactly, for what counts as an error.
    __device__ __forceinline__ bool any_sees(int t) const { return t <= min(it.hi, it.kv - 1) && sees(p, it.lo, t); }
    __device__ __forceinline__ bool really_seen(int t) const {
        return any_sees(t) && (!p.b.pos || p.window == 0 || some_row_sees(p, it.first + it.m0 / p.share, it.first + (it.m_end - 1) / p.share, t));
    }
    __device__ __forceinline__ bool whole(int t0) const { return whole_step(p, last, it.hi, t0); }
    __device__ __forceinline__ int steps() const { return it.end - it.begin; }

    // The k-th item, into registers; false when there is none, or after an abort.
    __device__ __forceinline__ bool next(int k) {
        if (!wait(&w.item_full[k & 1], (k >> 1) & 1)) return false;
        it = w.item[k & 1];
        arrive(&w.item_empty[k & 1]);
        last = min(it.least, it.kv - 1);
        return it.ok != 0;
    }

    // ---- the warp that finds the items: in order of the CTAs, and back again, the last rows (the most tokens) of all heads first
    __device__ __forceinline__ void find_items() {
        const int lane = threadIdx.x & 31;
        const long long total = (long long)pl.chunk_tiles * p.c.H * p.b.n_seqs * pl.splits;
        int k = 0;
        for (long long round = 0;; round++) {
            const long long at = round * gridDim.x + (round & 1 ? gridDim.x - 1 - blockIdx.x : blockIdx.x);
            const bool more = round * gridDim.x < total;
            if (more && at >= total) continue;
            WeighItem x;
            x.ok = 0;
            if (more) {
                long long id = at;
                x.split = (int)(id % pl.splits); id /= pl.splits;
                x.head = (int)(id % p.c.H); id /= p.c.H;
                x.seq = (int)(id % p.b.n_seqs);
                x.tile = pl.chunk_tiles - 1 - (int)(id / p.b.n_seqs);
                int rows;
                const bool ordered = sequence_rows(p, x.seq, &x.first, &x.kv, &rows);
                if (lane == 0 && (!ordered || rows > p.b.max_rows || p.b.kv_len[x.seq] > x.kv)) latch(p.status);
                if (!ordered) continue;
                x.m0 = (pl.chunk + x.tile) * 2 * kRowTile;
                x.m_end = min(min(rows, p.b.max_rows) * p.share, x.m0 + 2 * kRowTile);
                if (x.m0 >= x.m_end) continue;
                x.tiles = !ONE && x.m_end - x.m0 > kRowTile ? 2 : 1;
                // positions of the rows (one below 0 sees nothing: no window need reach back for it)
                uint32_t low = 0x7FFFFFFFu;
                int least = 0x7FFFFFFF, most = -1;
                for (int r = x.m0 / p.share + lane; r <= (x.m_end - 1) / p.share; r += 32) {
                    const int pos = row_position(p.b, x.seq, x.first + r);
                    low = min(low, (uint32_t)pos);
                    least = min(least, pos);
                    most = max(most, pos);
                }
                x.lo = (int)__reduce_min_sync(0xFFFFFFFFu, low);
                x.least = __reduce_min_sync(0xFFFFFFFFu, least);
                x.hi = __reduce_max_sync(0xFFFFFFFFu, most);
                x.range = step_range(p, x.kv, x.lo, x.hi);
                x.begin = (int)((long long)x.range.count * x.split / pl.splits);
                x.end = (int)((long long)x.range.count * (x.split + 1) / pl.splits);
                x.ok = 1;
                if (!COLUMNS && x.head == 0 && x.split == 0 && lane == 0)
                    pl.ranges[(long long)x.seq * pl.tiles + pl.chunk + x.tile] = make_int4(x.range.sink_tiles, x.range.first, x.range.count, 0);
            }
            if (!wait(&w.item_empty[k & 1], ((k >> 1) & 1) ^ 1)) return;
            if (lane == 0) w.item[k & 1] = x;
            arrive(&w.item_full[k & 1]);
            k++;
            if (!more) return;
        }
    }

    // ---- the warps that bring the keys
    __device__ __forceinline__ void fetch_images() {
        int n = 0;
        bool good = true;
        for (int k = 0; good && next(k); k++)
            for (int j = it.begin; j < it.end; j++) {
                const int st = n % kStages;
                const long long at = ((long long)it.seq * pl.steps + it.range.tile(j)) * p.c.H + it.head;
                if (!wait(&w.k_empty[st], turn(n) ^ 1)) { good = false; break; }
                if (elect_lane()) {
                    mbar_arrive_expect_tx(&w.k_full[st], kStage + 32);
                    bulk_g2s_at(key_stage(n), pl.images + at * kStage, kStage, &w.k_full[st]);
                    bulk_g2s_at(smem_u32(w.absent[n & 7]), pl.meta + at * 8, 32, &w.k_full[st]);
                }
                __syncwarp();
                n++;
            }
        // The last copies (after an abort they may have no reader) must have landed before the CTA goes.
        for (int back = 1; back <= kStages && back <= n; back++)
            for (uint32_t i = 0; i < kWaitLimit && !mbar_try_wait(&w.k_full[(n - back) % kStages], turn(n - back)); i++) __nanosleep(40);
    }
    // Sixteen tokens a warp, kPer lanes to a token.
    struct Pages { int page, t0; };
    __device__ __forceinline__ Pages pages_of(int j, int warp) const {
        Pages g = {-1, 0};
        if (j >= it.end) return g;
        g.t0 = it.range.tile(j) * kRowTile;
        const int t = g.t0 + 16 * warp;
        if (t >= it.kv) return g;
        const int pg = p.b.block_table[(long long)it.seq * p.b.table_stride + div_page(p.c, t)];
        if (pg >= 0 && pg < p.c.n_pages) g.page = pg;
        return g;
    }
    // Address of the thread's token (quantised: its page, and its row in *row); live: some row sees it and it has a page.
    __device__ __forceinline__ long long token_at(const Pages& g, int tok, uint32_t* row, bool* live) const {
        const int t = g.t0 + tok, slot = t - div_page(p.c, t) * p.c.P;
        *live = g.page >= 0 && any_sees(t);
        *row = (uint32_t)slot * p.c.H + it.head;
        if (!*live) return 0;
        return (long long)g.page * p.c.stride_page + (kPool ? (long long)slot * p.c.stride_token + (long long)it.head * p.c.stride_head : 0ll);
    }
    // Notes the warp's tokens that some row sees but that have no page.
    __device__ __forceinline__ void note(const Pages& g, int warp, int n) {
        const int lane = threadIdx.x & 31;
        const uint32_t gone = __ballot_sync(0xFFFFFFFFu, lane < 16 && g.page < 0 && any_sees(g.t0 + 16 * warp + lane));
        if (gone >> lane & 1u && really_seen(g.t0 + 16 * warp + lane)) latch(p.status);
        if (lane == 0) reinterpret_cast<uint16_t*>(w.absent[n & 7])[warp] = (uint16_t)gone;
    }
    __device__ __forceinline__ void load_keys(const Pages& g, int tok, int c, uint32_t (&code)[8], uint32_t& scale) const {
        uint32_t row;
        bool live;
        const uint8_t* pg = p.c.base + token_at(g, tok, &row, &live);
#pragma unroll
        for (int i = 0; i < 8; i++) code[i] = 0;
        scale = 0;
        if (!live) return;
        const uint8_t* codes = pg + row * (KF == FMT_INT8 ? D : D / 2) + c * (KF == FMT_INT8 ? 32 : 16);
        const uint4 a = *reinterpret_cast<const uint4*>(codes);
        code[0] = a.x; code[1] = a.y; code[2] = a.z; code[3] = a.w;
        if (KF == FMT_INT8) {
            const uint4 b = *reinterpret_cast<const uint4*>(codes + 16);
            code[4] = b.x; code[5] = b.y; code[6] = b.z; code[7] = b.w;
        }
        scale = *reinterpret_cast<const uint16_t*>(pg + (row * (D / p.c.G) + c * 32 / p.c.G) * 2 + p.c.k_scales);
    }
    __device__ __forceinline__ void produce(B& b, int warp) {
        constexpr int kPass = 16 / kTok;                            // tokens of a thread
        const int lane = threadIdx.x & 31, c = lane % kPer, tok0 = 16 * warp + lane / kPer;
        uint32_t m0, m1;
        asm volatile("mov.b32 %0, 0x64086408;" : "=r"(m0));
        asm volatile("mov.b32 %0, 0x64806480;" : "=r"(m1));
        int n = 0, told = 0;                                        // steps, and those that have been reported
        for (int k = 0; next(k); k++) {
            Pages now = pages_of(it.begin, warp), after = pages_of(it.begin + 1, warp);
            uint32_t code[kPool ? 1 : kPass][8], scale[kPool ? 1 : kPass];
            if constexpr (!kPool)
#pragma unroll
                for (int i = 0; i < kPass; i++) load_keys(now, tok0 + i * kTok, c, code[i], scale[i]);
#pragma unroll 1
            for (int j = it.begin; j < it.end; j++, n++) {
                if (!wait(&w.k_empty[n % kStages], turn(n) ^ 1)) return;
                note(now, warp, n);
                if constexpr (kPool) {
#pragma unroll
                    for (int i = 0; i < kPass; i++) {
                        uint32_t row;
                        bool live;
                        const uint16_t* x = p.c.k + token_at(now, tok0 + i * kTok, &row, &live) + 8 * c;
#pragma unroll
                        for (int q = 0; q < 4; q++)                 // chunks kPer apart: a row's lanes read a contiguous run
                            cp16(key_stage(n) + swizzled(tok0 + i * kTok, q * kPer + c), live ? x + 8 * q * kPer : p.c.k, live);
                    }
                    cp_commit();
                    if (told <= n - 2) {                            // two steps behind
                        cp_wait<2>();
                        fence_async_smem();
                        mbar_arrive(&w.k_full[told++ % kStages]);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < kPass; i++) {
                        b.template store_operands<KF, true>(key_stage(n), tok0 + i * kTok, c, code[i], scale[i], m0, m1);
                        load_keys(after, tok0 + i * kTok, c, code[i], scale[i]);
                    }
                    fence_async_smem();
                    mbar_arrive(&w.k_full[n % kStages]);
                }
                now = after;
                after = pages_of(j + 2, warp);
            }
            if constexpr (kPool) {                                  // the next item may be long in coming
                cp_wait<0>();
                fence_async_smem();
                while (told < n) mbar_arrive(&w.k_full[told++ % kStages]);
            }
        }
    }

    // ---- the warp that issues the products.  Step j of tile i goes to pair i, or with one tile to pair j & 1.
    __device__ __forceinline__ void issue(uint32_t tmem) {
        constexpr uint32_t kDesc = instr_desc(KF == FMT_BF16, false, kRowTile), kMat16 = S::kMat >> 4;
        const uint64_t q_desc = smem_desc(smem + S::kQ, 16), k_desc = smem_desc(smem + S::kK, 16);
        int g = 0, units[2] = {0, 0}, uses[2] = {0, 0};             // steps; units of the pairs; items of the tiles' queries
        for (int k = 0; next(k); k++) {
            for (int i = 0; i < it.tiles; i++) {
                if (!wait(&w.q_ready[i], uses[i] & 1)) return;
                uses[i]++;
            }
            // The steps of an item of one tile go to the first pair alone.  The second may not have read the last steps' `absent` of the
            // item before, which the producers, eight steps on, write over.  (In the second pass the first pair waits for its sums.)
            if (!COLUMNS && !ONE && it.tiles == 1 && uses[1] > 0 && !wait(&w.second_done, (uses[1] - 1) & 1)) return;
            const int n = steps();
#pragma unroll 1
            for (int j = 0; j < n; j++, g++) {
                const int st = g % kStages;
                if (!wait(&w.k_full[st], turn(g))) return;
#pragma unroll 1
                for (int i = 0; i < it.tiles; i++) {
                    const int pair = ONE ? j & 1 : i, u = pair ? units[1]++ : units[0]++;
                    if (!wait(&w.s_empty[pair][u & 1], ((u >> 1) & 1) ^ 1)) return;
                    tc_after();
                    const uint64_t q = q_desc + i * kMat16, key = k_desc + st * (kStage >> 4);
                    const uint32_t d = tmem + (2 * pair + (u & 1)) * kRowTile;
                    if (elect_lane()) {
#pragma unroll
                        for (int x = 0; x < D / 16; x++) {          // 16 channels: 32 bytes inside a 128-byte row, then the next half
                            const uint32_t o = (x >> 2) * (kRowTile * 8) + (x & 3) * 2;
                            tc_mma_ss(d, COLUMNS ? key + o : q + o, COLUMNS ? q + o : key + o, kDesc, x != 0);
                            if (FINE) tc_mma_ss(d, COLUMNS ? key + o + kMat16 : q + o, COLUMNS ? q + o : key + o + kMat16, kDesc, true);
                        }
                        tc_commit(&w.s_full[pair][u & 1]);
                        if (i == it.tiles - 1) tc_commit(&w.k_empty[st]);
                    }
                    __syncwarp();
                }
            }
            if (elect_lane()) tc_commit(&w.q_free);
            __syncwarp();
        }
    }

    // ---- the warpgroups: pair wg >> 1, columns 64 (wg & 1) .. + 63 of a place
    // Of 16 pairs of exponentials, those that are computed instead of left to the exponential unit (0 .. 16).  With 0, 2, 4 and 6 of them 8192
    // rows over 8192 tokens (32 query heads) take 950, 1000, 1015 and 1060 us on 8-bit keys, and 749, 738, 760 and 810 us on bf16 keys.
    static constexpr int kOnFma = FINE ? 0 : 2;
    __device__ __forceinline__ static void exp2_both(int c, f32x2 y, float& a, float& b) {
        if (c * kOnFma % 16 < kOnFma) {
            weigh_exp2_pair(y, a, b);
        } else {
            unpack2(y, a, b);
            a = fast_exp2(a);
            b = fast_exp2(b);
        }
    }
    __device__ __forceinline__ static void add_row(const float (&x)[32], f32x2 factor2, f32x2 ref2, f32x2 (&total)[2]) {
#pragma unroll
        for (int c = 0; c < 16; c++) {
            float a, b;
            exp2_both(c, fma2(pack2(x[2 * c], x[2 * c + 1]), factor2, ref2), a, b);
            total[c & 1] = add2(total[c & 1], pack2(a, b));
        }
    }
    __device__ __forceinline__ long long vector_index(int m) const {
        return (long long)(it.first + m / p.share) * p.Hq + it.head * p.share + m % p.share;
    }
    __device__ __forceinline__ void release(int pair, int u) {
        tc_before();
        arrive(&w.s_empty[pair][u & 1]);
    }
    // Queries into shared memory, their factors and positions: a tile by the first warpgroup of a pair; the others wait for them.
    // `k` items have been before, `uses` of them with this tile.
    __device__ __forceinline__ bool queries(B& b, int wg, int i, int k, int uses) {
        const int r = threadIdx.x & 127;
        if (wg == 2 * i) {
            if (k > 0 && !wait(&w.q_free, (k - 1) & 1)) return false;
            const int m = it.m0 + 128 * i + r;
            const bool live = m < it.m_end;
            // Behind the last vector the second pass has the item's first again, with the weight 0: zeros times an infinite key would be NaN.
            const int from = COLUMNS ? it.m0 : 0, row = it.first + (live ? m : from) / p.share, hq = it.head * p.share + (live ? m : from) % p.share;
            w.pos[128 * i + r] = live ? max(-1, row_position(p.b, it.seq, row)) : -1;
            float factor = b.load_query(i, r, COLUMNS || live, row, hq);
            w.factor[128 * i + r] = factor;
            if (COLUMNS) {
                // -log2 of the row's sum; NaN where all of its logits are minus infinity, minus infinity for a row that sees nothing and for
                // vectors behind the last
                float low = -INFINITY;
                if (live) {
                    const long long vec = vector_index(m), step = (long long)p.b.n_rows * p.Hq;
                    float top = kNoMax, sum = 0.0f;
#pragma unroll 8
                    for (int q = 0; q < pl.splits; q++) top = fmaxf(top, pl.sums[q * step + vec].x);
#pragma unroll 8
                    for (int q = 0; q < pl.splits; q++) {
                        const float2 z = pl.sums[q * step + vec];
                        sum = fmaf(z.y, fast_exp2(z.x - top), sum);
                    }
                    if (sum != 0.0f) low = -(top + log2f(sum));
                    else if (sees_some(p, w.pos[128 * i + r], it.kv)) low = __uint_as_float(0x7FC00000u);
                }
                if (factor != factor) factor = p.scale_log2;        // (of zeros)
                w.scale[128 * i + r] = factor;
                w.low[128 * i + r] = low;
            }
            fence_async_smem();
            arrive(&w.q_ready[i]);
        }
        return wait(&w.q_ready[i], uses & 1);
    }

    // The sums of a step's 64 columns of the row.
    __device__ __forceinline__ static void add_step(uint32_t s_at, f32x2 factor2, float ref, f32x2 (&total)[2]) {
        const f32x2 ref2 = pack2(-ref, -ref);
        total[0] = total[1] = pack2(0.0f, 0.0f);
#pragma unroll
        for (int q = 0; q < 2; q++) {
            float x[32];
            tc_ld32(x, s_at + 32 * q);
            tc_wait_ld();
            add_row(x, factor2, ref2, total);
        }
    }
    // The reference at the largest logit so far, and the sums brought to it.
    __device__ __forceinline__ static void move_reference(uint32_t s_at, float factor, float& ref, f32x2 (&sum2)[2]) {
        float y = ref;
#pragma unroll 1
        for (int q = 0; q < 4; q++) {
            uint32_t x[16];
            tc_ld16(x, s_at + 16 * q);
            tc_wait_ld();
#pragma unroll
            for (int c = 0; c < 16; c++) y = fmaxf(y, __uint_as_float(x[c]) * factor);
        }
        const float keep = fast_exp2(ref - y);
        ref = y;
        sum2[0] = mul2(sum2[0], pack2(keep, keep));
        sum2[1] = mul2(sum2[1], pack2(keep, keep));
    }

    // First pass: a thread per query vector.
    __device__ __forceinline__ void rows(B& b, int wg, uint32_t tmem) {
        const int pair = wg >> 1, half = wg & 1, i = ONE ? 0 : pair, r = threadIdx.x & 127;
        const bool leader = ONE ? wg == 0 : half == 0;              // puts the sums of a vector together
        const uint32_t at = tmem + ((uint32_t)((threadIdx.x >> 5) & 3) << 21) + 64 * half;
        int g = 0, u = 0, uses = 0;
        for (int k = 0; next(k); k++) {
            const int n = steps();
            if (i >= it.tiles) { g += n; continue; }
            if (!queries(b, wg, i, k, uses)) return;
            const int m = it.m0 + 128 * i + r, pos = w.pos[128 * i + r], kv = it.kv;
            float factor = w.factor[128 * i + r];
            const bool broken = factor != factor;
            if (broken) factor = 1.0f;
            if (factor == 0.0f) factor = 1.17549435e-38f;           // a mask is minus infinity over the factor
            float ref = kNoMax;
            f32x2 sum2[2] = {pack2(0.0f, 0.0f), pack2(0.0f, 0.0f)};
            const f32x2 factor2 = pack2(factor, factor);
            bool start = true;
#pragma unroll 1
            for (int j = ONE ? pair : 0; j < n; u++, j += ONE ? 2 : 1) {
                const int t0 = it.range.tile(it.begin + j) * kRowTile;
                const uint32_t s_at = at + (2 * pair + (u & 1)) * kRowTile;
                if (!wait(&w.s_full[pair][u & 1], (u >> 1) & 1)) return;
                tc_after();
                const uint4 absent = lds128(smem_u32(w.absent[(g + j) & 7]));
                const bool gaps = (absent.x | absent.y | absent.z | absent.w) != 0;
                if (gaps || !whole(t0)) {                           // what a row does not see becomes minus infinity, in TMEM
                    if (IMAGE && gaps && !half) latch_absent(t0, absent);
                    const int x0 = 64 * half, hi = min(pos, kv - 1) - t0, lo = p.window > 0 ? max(pos - p.window + 1, 0) - t0 : -t0, s = p.sinks - t0;
                    const uint32_t none = factor < 0.0f ? 0x7F800000u : 0xFF800000u;
#pragma unroll 1
                    for (int q = 0; q < 4; q++) {
                        const uint32_t gone = (half ? (q < 2 ? absent.z : absent.w) : (q < 2 ? absent.x : absent.y)) >> (16 * (q & 1));
                        const uint32_t in = B::seen(x0 + 16 * q, lo, hi, s, gone);
                        uint32_t x[16];
                        tc_ld16(x, s_at + 16 * q);
                        tc_wait_ld();
#pragma unroll
                        for (int c = 0; c < 16; c++) x[c] = in >> c & 1u ? x[c] : none;
                        tc_st16(s_at + 16 * q, x);
                    }
                    tc_wait_st();
                }
                // Against the reference as it stands, a row's largest logit in the first step it had tokens in; where the sum shows that it has
                // become too small (fp32 has room for logits 60 above it) the largest is looked for again and the step done once more.
                if (start) move_reference(s_at, factor, ref, sum2);
                start = false;
                f32x2 total[2];
                add_step(s_at, factor2, ref, total);
                float a, c;
                unpack2(add2(total[0], total[1]), a, c);
                if (__any_sync(0xFFFFFFFFu, a + c > 1.0e18f)) {
                    move_reference(s_at, factor, ref, sum2);
                    add_step(s_at, factor2, ref, total);
                }
                sum2[0] = add2(sum2[0], total[0]);              // (step by step: a long row's 32-bit sum rounds less often)
                sum2[1] = add2(sum2[1], total[1]);
                release(pair, u);
            }
            g += n;
            float sum, odd;
            unpack2(add2(sum2[0], sum2[1]), sum, odd);
            sum += odd;
            if (broken && sum != 0.0f) sum = __uint_as_float(0x7FC00000u);
            if (!leader) {
                w.sums[wg][r] = make_float2(ref, sum);
                arrive(&w.mate_done[ONE ? 0 : pair]);
            } else {
                if (!wait(&w.mate_done[ONE ? 0 : pair], uses & 1)) return;
                for (int q = wg + 1; q < (ONE ? 4 : wg + 2); q++) {
                    const float2 z = w.sums[q][r];
                    const float to = fmaxf(ref, z.x);
                    sum = fmaf(sum, fast_exp2(ref - to), z.y * fast_exp2(z.x - to));
                    ref = to;
                }
                if (m < it.m_end) pl.sums[(long long)it.split * p.b.n_rows * p.Hq + vector_index(m)] = make_float2(ref, sum);
                if (!ONE && pair == 1) arrive(&w.second_done);
            }
            uses++;
        }
    }
    // Tokens on pages out of range count when some row sees them (with images nobody has looked at that yet).
    __device__ __forceinline__ void latch_absent(int t0, const uint4& absent) const {
        const int lane = threadIdx.x & 31;
        const uint32_t gone[4] = {absent.x, absent.y, absent.z, absent.w};
#pragma unroll
        for (int q = 0; q < 4; q++)
            if (gone[q] >> lane & 1u && really_seen(t0 + 32 * q + lane)) latch(p.status);
    }

    // Second pass: a thread per token, the vectors of a tile along its lane; `in`: the vectors that see it, where not all do.  Where all vectors
    // have one factor (bf16 pages, fp16 queries) half as much is read along the way.
    template <bool MASK, bool EVEN>
    __device__ __forceinline__ void add_column(const float (&x)[32], int first, uint32_t in, f32x2 factor2, f32x2 (&total)[2]) const {
#pragma unroll
        for (int c = 0; c < 16; c += 2) {
            const uint4 low = lds128(smem_u32(w.low + first + 2 * c));
            uint4 f = make_uint4(0, 0, 0, 0);
            if (!EVEN) f = lds128(smem_u32(w.scale + first + 2 * c));
#pragma unroll
            for (int e = 0; e < 2; e++) {
                const f32x2 l = e ? pack2(__uint_as_float(low.z), __uint_as_float(low.w)) : pack2(__uint_as_float(low.x), __uint_as_float(low.y));
                const f32x2 s = EVEN ? factor2 : e ? pack2(__uint_as_float(f.z), __uint_as_float(f.w)) : pack2(__uint_as_float(f.x), __uint_as_float(f.y));
                float a, b;
                exp2_both(c + e, fma2(pack2(x[2 * (c + e)], x[2 * (c + e) + 1]), s, l), a, b);
                if (MASK) {
                    a = in >> (2 * (c + e)) & 1u ? a : 0.0f;
                    b = in >> (2 * (c + e) + 1) & 1u ? b : 0.0f;
                }
                total[e] = add2(total[e], pack2(a, b));
            }
        }
    }
    template <bool MASK, bool EVEN>
    __device__ __forceinline__ float column_sum(uint32_t s_at, int first, unsigned long long in) const {
        f32x2 total[2] = {pack2(0.0f, 0.0f), pack2(0.0f, 0.0f)};
        const f32x2 factor2 = pack2(p.scale_log2, p.scale_log2);
#pragma unroll
        for (int q = 0; q < 2; q++) {
            float x[32];
            tc_ld32(x, s_at + 32 * q);
            tc_wait_ld();
            add_column<MASK, EVEN>(x, first + 32 * q, (uint32_t)(in >> (32 * q)), factor2, total);
        }
        float a, b;
        unpack2(add2(total[0], total[1]), a, b);
        return a + b;
    }
    // Which of 64 vectors from number `first` of the item see token t.  A row's vectors lie together.
    __device__ __forceinline__ unsigned long long seeing(int first, int t) const {
        unsigned long long in = 0;
        const int share = p.share;
        int left = share - (it.m0 + first) % share;                 // of the row's vectors, from this one on
#pragma unroll 1
        for (int c = 0; c < 64; c += left, left = share) {
            const int pos = w.pos[first + c];
            if (t <= pos && sees(p, pos, t)) in |= (left < 64 ? (1ull << left) - 1ull : ~0ull) << c;
        }
        return in;
    }
    __device__ __forceinline__ void columns(B& b, int wg, uint32_t tmem) {
        const int pair = wg >> 1, half = wg & 1, i = ONE ? 0 : pair, r = threadIdx.x & 127, from = 128 * i + 64 * half;
        const bool leader = ONE ? half == 0 : wg == 0;              // adds up the other warpgroups' sums of a step, one step later
        const uint32_t at = tmem + ((uint32_t)((threadIdx.x >> 5) & 3) << 21) + 64 * half;
        int g = 0, u = 0, uses = 0;
        for (int k = 0; next(k); k++) {
            const int n = steps();
            if (i >= it.tiles) { g += n; continue; }
            if (!queries(b, wg, i, k, uses)) return;
            const int kv = it.kv;
            float* out = pl.partial + (((long long)it.seq * p.c.H + it.head) * pl.chunk_tiles + it.tile) * pl.tokens + (long long)it.begin * kRowTile + r;
            float sum = 0.0f;
            int before = -1;                                        // step whose sum the leader still has: unit u - 1
            auto finish = [&]() {
                const int v = u - 1;
                for (int q = wg + 1; q < (ONE ? wg + 2 : 2 * it.tiles); q++) {
                    // (pair 1 has had its own number of units: one for each step of the items with two tiles)
                    const int x = q < 2 || ONE ? v : u2 - 1;
                    if (!wait(&w.part_full[q][x & 3], (x >> 2) & 1)) return false;
                    sum += w.part[x & 3][q][r];
                }
                out[(long long)before * kRowTile] = sum;
                return true;
            };
#pragma unroll 1
            for (int j = ONE ? pair : 0; j < n; u++, j += ONE ? 2 : 1) {
                const int t0 = it.range.tile(it.begin + j) * kRowTile, t = t0 + r;
                const uint32_t s_at = at + (2 * pair + (u & 1)) * kRowTile;
                if (leader && before >= 0 && !finish()) return;
                if (it.tiles == 2) u2++;
                if (!wait(&w.s_full[pair][u & 1], (u >> 1) & 1)) return;
                tc_after();
                const uint4 absent = lds128(smem_u32(w.absent[(g + j) & 7]));
                const bool gaps = (absent.x | absent.y | absent.z | absent.w) != 0;
                if (gaps || !whole(t0)) {
                    const uint32_t word = r < 32 ? absent.x : r < 64 ? absent.y : r < 96 ? absent.z : absent.w;
                    const bool there = t < kv && !(word >> (r & 31) & 1u);
                    sum = column_sum<true, kPool>(s_at, from, there ? seeing(from, t) : 0ull);
                } else if (kPool || p.f16) {
                    sum = column_sum<false, true>(s_at, from, 0ull);
                } else {
                    sum = column_sum<false, false>(s_at, from, 0ull);
                }
                release(pair, u);
                if (leader) {
                    before = j;
                } else {
                    w.part[u & 3][wg][r] = sum;
                    arrive(&w.part_full[wg][u & 3]);
                }
            }
            g += n;
            if (leader && before >= 0 && !finish()) return;
            // The first warpgroup of a pair writes the next item's numbers over this one's.
            if (wg != 2 * i) arrive(&w.mate_done[ONE ? 0 : pair]);
            else if (!wait(&w.mate_done[ONE ? 0 : pair], uses & 1)) return;
            uses++;
        }
    }
    int u2 = 0;                                                     // second pass: units of pair 1, as the leader counts them
};

template <int KF, int D, bool IMAGE, bool ONE, bool COLUMNS>
__global__ void __launch_bounds__(weigh_threads(IMAGE), 1) weigh_rows_kernel(const __grid_constant__ AttentionParams p, const __grid_constant__ WeighRowsPlan pl) {
    using K = WeighRows<KF, D, IMAGE, ONE, COLUMNS>;
    constexpr int kIssuer = weigh_issuer(IMAGE) / 32;
    extern __shared__ uint8_t raw[];
    const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u;
    WeighBars& bars = *reinterpret_cast<WeighBars*>(raw + (base - smem_u32(raw)) + RowsSmem<D>::kBars);
    pdl_trigger();
    const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x >> 5, 0);
    if (threadIdx.x == 0) {
        for (int i = 0; i < 2; i++) {
            mbar_init(&bars.item_full[i], 1);
            mbar_init(&bars.item_empty[i], weigh_threads(IMAGE) / 32 - 1);      // all warps but the one that finds the items
            mbar_init(&bars.q_ready[i], 4);
            mbar_init(&bars.mate_done[i], ONE ? 12 : 4);
            for (int k = 0; k < 2; k++) { mbar_init(&bars.s_full[i][k], 1); mbar_init(&bars.s_empty[i][k], 8); }
        }
        for (int i = 0; i < 4; i++) {
            mbar_init(&bars.k_full[i], IMAGE ? 1 : kWeighProducers);
            mbar_init(&bars.k_empty[i], 1);
            for (int k = 0; k < 4; k++) mbar_init(&bars.part_full[i][k], 4);
        }
        mbar_init(&bars.q_free, 1);
        mbar_init(&bars.second_done, 4);
        mbar_init(&bars.drained, 1);
        bars.abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kIssuer) tc_alloc(&bars.tmem, 512);
    tc_before();
    __syncthreads();
    tc_after();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(&bars.tmem);
    pdl_wait();
    K k(p, pl, bars, base);
    // The attention's helpers that need no barriers: queries and operands.
    RowsBars unused;
    typename K::B b(p, unused);
    b.smem = base;
    if (warp < kWeighConsumers / 32) {
        if (COLUMNS) k.columns(b, warp >> 2, tmem);
        else k.rows(b, warp >> 2, tmem);
    } else if (warp < kIssuer) {
        if constexpr (IMAGE) {
            k.fetch_images();
        } else {
            k.produce(b, warp - kWeighConsumers / 32);
            cp_wait<0>();
        }
    } else if (warp == kIssuer) {
        k.issue(tmem);
        if (__any_sync(0xFFFFFFFFu, *reinterpret_cast<volatile int32_t*>(&bars.abort))) {      // what was issued must have ended before TMEM goes
            if (elect_lane()) tc_commit(&bars.drained);
            __syncwarp();
            for (uint32_t i = 0; i < kWaitLimit && !mbar_try_wait(&bars.drained, 0); i++) __nanosleep(40);
        }
    } else {
        k.find_items();
    }
    __syncwarp();
    tc_before();
    __syncthreads();
    tc_after();
    if (warp == kIssuer) tc_free(tmem, 512);
    if (threadIdx.x == 0 && bars.abort) atomicCAS(p.status, 0, (int)PATCHKV_E_TIMEOUT);
}

// Images of the two matrices of a step's keys (grid: step, KV head, sequence), as attention_image_kernel lays them out.
template <int KF, int D>
__global__ void __launch_bounds__(kImageThreads) weigh_image_kernel(const __grid_constant__ AttentionParams p, const __grid_constant__ WeighRowsPlan pl) {
    using S = RowsSmem<D>;
    constexpr int kPer = D / 32, kTokens = kImageThreads / kPer;        // 32 channels a thread; tokens per pass
    __shared__ uint32_t meta[8];
    pdl_trigger();
    pdl_wait();
    const int step = blockIdx.x, head = blockIdx.y, seq = blockIdx.z, t0 = step * kRowTile;
    int first, kv, rows, lo = 0, hi;
    if (!sequence_rows(p, seq, &first, &kv, &rows) || rows == 0) return;
    hi = kv - 1;
    if (!p.b.pos) {                                             // the last positions: what no row sees needs no image
        const int a = p.b.kv_len[seq] - rows;
        lo = max(-1, a);
        hi = a + min(rows, p.b.max_rows) - 1;
    }
    const TileRange range = step_range(p, kv, p.b.pos ? 0 : lo, hi);
    if (t0 > min(hi, kv - 1) || (!p.b.pos && step >= range.sink_tiles && step < range.first)) return;
    if (threadIdx.x < 8) meta[threadIdx.x] = 0;
    __syncthreads();
    const int c = threadIdx.x % kPer;
    uint8_t* image = pl.images + (((long long)seq * pl.steps + step) * p.c.H + head) * (2 * S::kMat);
#pragma unroll
    for (int i = 0; i < kRowTile / kTokens; i++) {
        const int tok = threadIdx.x / kPer + i * kTokens, t = t0 + tok;
        int page = -1, slot = 0;
        if (t < kv) {
            const int lp = div_page(p.c, t);
            slot = t - lp * p.c.P;
            page = p.b.block_table[(long long)seq * p.b.table_stride + lp];
            if (page < 0 || page >= p.c.n_pages) {
                page = -1;
                if (c == 0) atomicOr(&meta[tok >> 5], 1u << (tok & 31));
            }
        }
        uint4 a[4], b[4];
        if (page < 0) {
#pragma unroll
            for (int q = 0; q < 4; q++) a[q] = b[q] = make_uint4(0, 0, 0, 0);
        } else {
            const uint8_t* pg = p.c.base + (long long)page * p.c.stride_page;
            const uint32_t row = (uint32_t)slot * p.c.H + head, sc = (row * (D / p.c.G) + c * 32 / p.c.G) * 2;
            uint32_t s = *reinterpret_cast<const uint16_t*>(pg + p.c.k_scales + sc);
            s |= s << 16;
            image_operands<KF>(a, b, pg + row * (KF == FMT_INT8 ? D : D / 2), c, s, 0x64086408u, 0x64806480u);
        }
#pragma unroll
        for (int q = 0; q < 4; q++) {
            *reinterpret_cast<uint4*>(image + swizzled(tok, 4 * c + q)) = a[q];
            *reinterpret_cast<uint4*>(image + S::kMat + swizzled(tok, 4 * c + q)) = b[q];
        }
    }
    __syncthreads();
    if (threadIdx.x < 8) pl.meta[(((long long)seq * pl.steps + step) * p.c.H + head) * 8 + threadIdx.x] = meta[threadIdx.x];
}

// The sum over heads and tiles of vectors (grid: step of 128 tokens, sequence, CTA of a cluster): a thread per token, the cluster's groups of 128 threads
// (no more than there are tiles: 58 us for 62 with one tile) share the tiles, and its first CTA adds up (distributed shared memory): with
// one CTA a step, and half of the SMs idle, 8192 rows over 8192 tokens of a pool take 761 us instead of 743 in all.  64 bits: tens of
// thousands of numbers are added one by one.
constexpr int kWeighJoin = 1024, kWeighJoinCtas = 4;
static __global__ void __launch_bounds__(kWeighJoin) weigh_rows_join_kernel(const __grid_constant__ AttentionParams p, const __grid_constant__ WeightParams m,
                                                                            const __grid_constant__ WeighRowsPlan pl) {
    __shared__ double part[kWeighJoin], whole[kWeighJoinCtas][kRowTile];
    cooperative_groups::cluster_group cluster = cooperative_groups::this_cluster();
    const int rank = (int)cluster.block_rank(), ctas = (int)cluster.num_blocks();
    pdl_trigger();
    cluster.barrier_arrive();
    pdl_wait();
    const int s = blockIdx.y, step = blockIdx.x, r = threadIdx.x & 127, group = threadIdx.x >> 7, groups = blockDim.x >> 7;
    int first, kv, rows;
    const bool ordered = sequence_rows(p, s, &first, &kv, &rows) && step * kRowTile < kv;
    double sum = 0.0;
    if (ordered) {
        const int tiles = (min(rows, p.b.max_rows) * p.share + 2 * kRowTile - 1) / (2 * kRowTile), end = min(tiles, pl.chunk + pl.chunk_tiles);
        for (int tile = pl.chunk + group + groups * rank; tile < end; tile += groups * ctas) {
            const int4 range = pl.ranges[(long long)s * pl.tiles + tile];
            const int v = step < range.x ? step : step - range.y + range.x;
            if (!(step < range.x || (step >= range.y && v < range.z))) continue;
            const float* from = pl.partial + ((long long)s * p.c.H * pl.chunk_tiles + tile - pl.chunk) * pl.tokens + (long long)v * kRowTile + r;
            float heads = 0.0f;
#pragma unroll 8
            for (int h = 0; h < p.c.H; h++) heads += from[(long long)h * pl.chunk_tiles * pl.tokens];
            sum += heads;
        }
    }
    part[threadIdx.x] = sum;
    __syncthreads();
    cluster.barrier_wait();                                     // the first CTA is there to be written to
    if (group == 0) {
        for (int i = 1; i < groups; i++) sum += part[i * 128 + r];
        cluster.map_shared_rank(&whole[0][0], 0)[rank * kRowTile + r] = sum;
    }
    cluster.sync();
    const int t = step * kRowTile + r;
    if (rank != 0 || group != 0 || !ordered || t >= kv) return;
    for (int i = 1; i < ctas; i++) sum += whole[i][r];
    double* acc = pl.acc ? pl.acc + (long long)s * p.b.max_kv_len + t : nullptr;
    if (acc && pl.chunk) sum += *acc;
    if (pl.last) store_mass(p, m, s, t, (float)sum);
    else *acc = sum;
}

}  // namespace patchkv
