// Attention weight from many query vectors, on the 5th-generation tensor cores.
//
// As in the row kernel of the attention a CTA takes one KV head and up to 256 query vectors of it, in one or two tiles of 128, and walks
// the keys in steps of 128 tokens.  It does so twice, since a weight is known only when the sum over its row is:
//   first pass    S = Q K^T, a lane of TMEM per query vector; a thread adds up 2^(S - ref) over the tokens of its row
//   second pass   S = K Q^T, a lane per token; a thread adds up 2^(S - log2 of the row's sum) over the vectors of the CTA
// In both the sum runs along a thread's own lane, so nothing is exchanged, and nothing comes behind the sums: the products of the next
// steps run while a step is added up.  Four warpgroups do that, two (a pair) for each tile, half of the columns each, with two places
// in TMEM for each pair; with one tile of vectors the pairs take turns at the steps.  (Two warpgroups, a tile each, took 3000 cycles a step:
// two warps a scheduler do not hide one another's latencies.)  The second pass leaves a number for each token, head and CTA, which
// the last kernel adds up in an order that the arguments fix.
// Keys are operands without a rounding: bf16 as they are, quantised ones as the sum of two fp16 matrices (22 bits), for two products per
// 16 channels.  One fp16 matrix alone would put a logit 2^-12 of its terms off and the masses 1e-4.  With many tiles of vectors the operands are
// laid out in the workspace first (images), as for the attention; else each CTA makes them from the pages, eight warps of it.
// A step of two tiles takes 1024 cycles of products (quantised 2048) and as many exponentials as 2048 cycles of the exponential unit, of which
// a part is computed on the fma pipe instead.
#pragma once

#include "attention_rows.cuh"
#include "mass.cuh"

namespace patchkv {

struct WeighRowsPlan {
    float2* sums;               // [slot][n_rows * Hq]: reference and sum of a vector over some of the tokens
    int4* ranges;               // [sequence][tile]: sink steps, first step and count of the steps that a CTA's rows see
    float* partial;             // [sequence][KV head][tile of the chunk][tokens]: what a CTA's vectors give to a token
    int32_t tiles, splits;      // CTAs along the vectors of a sequence, and along the tokens
    int32_t slots;              // entries of a vector in `sums`
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
__host__ __device__ constexpr int weigh_slots(bool one) { return one ? 4 : 2; }     // sums of a vector and a piece: a warpgroup each
__host__ __device__ constexpr int weigh_threads(bool image) { return weigh_issuer(image) + 32; }

struct WeighBars {
    RowsBars r;
    uint64_t s_full[2][2], s_empty[2][2], k_full[4], k_empty[4];    // [pair][place in TMEM]; stages of the ring of keys
    uint64_t part_full[2][4];                                       // second pass: [pair][step mod 4] the other warpgroups' sums are there
    alignas(16) uint32_t absent[8][8];                              // per step (mod 8)
    float factor[256];                                              // of the vectors' logits
    int32_t pos[256];
    alignas(16) float4 column[128];                                 // second pass: of two vectors their factors and -log2 of their sums
    float part[4][3][kRowTile];                                     // [step mod 4][warpgroup 1 .. 3]
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
// The threads of the four warpgroups.
__device__ __forceinline__ void sync_consumers() { asm volatile("bar.sync 1, %0;" ::"n"(kWeighConsumers) : "memory"); }

// KF: format of the keys; IMAGE: they come as images (KF = FMT_INT8 stands for those).  ONE: no sequence has more than one tile of vectors.
// COLUMNS: the second pass.
template <int KF, int D, bool IMAGE, bool ONE, bool COLUMNS>
struct WeighRows : RowsKernel<KF, KF, D, IMAGE, KF != FMT_BF16> {
    static constexpr bool FINE = KF != FMT_BF16;
    using B = RowsKernel<KF, KF, D, IMAGE, FINE>;
    using S = RowsSmem<D>;
    static constexpr int kStages = FINE ? 2 : 4;
    static constexpr uint32_t kStage = (FINE ? 2 : 1) * S::kMat;
    WeighBars& w;

    __device__ __forceinline__ WeighRows(const AttentionParams& p_, WeighBars& b) : B(p_, b.r), w(b) {}
    __device__ __forceinline__ static uint32_t turn(int n) { return (uint32_t)(n / kStages) & 1u; }
    __device__ __forceinline__ uint32_t key_stage(int n) const { return this->smem + S::kK + (n % kStages) * kStage; }

    // ---- the warps that bring the keys
    __device__ __forceinline__ void fetch_images(const WeighRowsPlan& pl) {
        int n = 0;
        for (int j = this->begin; j < this->end; j++, n++) {
            const int st = n % kStages;
            const long long at = ((long long)this->seq * pl.steps + this->range.tile(j)) * this->p.c.H + this->head;
            if (!this->wait_warp(&w.k_empty[st], turn(n) ^ 1)) break;
            if (elect_lane()) {
                mbar_arrive_expect_tx(&w.k_full[st], kStage + 32);
                bulk_g2s_at(key_stage(n), pl.images + at * kStage, kStage, &w.k_full[st]);
                bulk_g2s_at(smem_u32(w.absent[n & 7]), pl.meta + at * 8, 32, &w.k_full[st]);
            }
            __syncwarp();
        }
        // The last copies (after an abort they may have no reader) must have landed before the CTA goes.
        for (int back = 1; back <= kStages && back <= n; back++)
            for (uint32_t i = 0; i < kWaitLimit && !mbar_try_wait(&w.k_full[(n - back) % kStages], turn(n - back)); i++) __nanosleep(40);
    }
    __device__ __forceinline__ void produce(int warp) {
        constexpr int TOK = 16, kPass = TOK / B::kTok;              // tokens of a warp, and passes over them
        using Pages = typename B::Pages;
        const int lane = threadIdx.x & 31, c = lane % B::kPer, tok0 = TOK * warp + lane / B::kPer;
        uint32_t m0, m1;
        asm volatile("mov.b32 %0, 0x64086408;" : "=r"(m0));
        asm volatile("mov.b32 %0, 0x64806480;" : "=r"(m1));
        const int begin = this->begin, end = this->end;
        if (begin >= end) return;
        auto pages_of = [&](int j) { return Pages{this->page_of(j, TOK * warp), j < end ? this->range.tile(j) * kRowTile : 0}; };
        auto note = [&](const Pages& g, int n) {                    // tokens that some row sees but that have no page
            const uint32_t gone = this->template missing<TOK>(g, warp);
            if (lane == 0) reinterpret_cast<uint16_t*>(w.absent[n & 7])[warp] = (uint16_t)gone;
        };
        Pages now = pages_of(begin), next = pages_of(begin + 1);
        if constexpr (KF == FMT_BF16) {
            int n = 0;
#pragma unroll 1
            for (int j = begin; j < end; j++, n++) {
                if (!this->wait_warp(&w.k_empty[n % kStages], turn(n) ^ 1)) return;
                note(now, n);
#pragma unroll
                for (int i = 0; i < kPass; i++) {
                    uint32_t row;
                    bool live;
                    const uint16_t* x = this->p.c.k + this->template token_at<TOK>(now, tok0 + i * B::kTok, &row, &live) + 8 * c;
#pragma unroll
                    for (int q = 0; q < 4; q++)                     // chunks kPer apart: a row's lanes read a contiguous run
                        cp16(key_stage(n) + swizzled(tok0 + i * B::kTok, q * B::kPer + c), live ? x + 8 * q * B::kPer : this->p.c.k, live);
                }
                cp_commit();
                if (n >= 2) {
                    cp_wait<2>();
                    fence_async_smem();
                    mbar_arrive(&w.k_full[(n - 2) % kStages]);
                }
                now = next;
                next = pages_of(j + 2);
            }
            cp_wait<0>();
            fence_async_smem();
            if (n >= 2) mbar_arrive(&w.k_full[(n - 2) % kStages]);
            mbar_arrive(&w.k_full[(n - 1) % kStages]);
        } else {
            uint32_t code[kPass][8], scale[kPass];
#pragma unroll
            for (int i = 0; i < kPass; i++) this->template load_piece<KF, TOK>(now, tok0 + i * B::kTok, c, false, code[i], scale[i]);
            int n = 0;
#pragma unroll 1
            for (int j = begin; j < end; j++, n++) {
                if (!this->wait_warp(&w.k_empty[n % kStages], turn(n) ^ 1)) return;
                note(now, n);
#pragma unroll
                for (int i = 0; i < kPass; i++) {
                    this->template store_operands<KF, true>(key_stage(n), tok0 + i * B::kTok, c, code[i], scale[i], m0, m1);
                    this->template load_piece<KF, TOK>(next, tok0 + i * B::kTok, c, false, code[i], scale[i]);
                }
                fence_async_smem();
                mbar_arrive(&w.k_full[n % kStages]);
                now = next;
                next = pages_of(j + 2);
            }
        }
    }

    // ---- the warp that issues the products.  Step j of tile i goes to pair i, or with one tile to pair j & 1.
    __device__ __forceinline__ void issue(int tiles, uint32_t tmem) {
        constexpr uint32_t kDesc = instr_desc(KF == FMT_BF16, false, kRowTile), kMat16 = S::kMat >> 4;
        const uint64_t q_desc = smem_desc(this->smem + S::kQ, 16), k_desc = smem_desc(this->smem + S::kK, 16);
        for (int i = 0; i < tiles; i++) if (!this->wait_warp(&w.r.q_ready[i], 0)) return;
        const int n = this->end - this->begin;
#pragma unroll 1
        for (int j = 0; j < n; j++) {
            const int st = j % kStages;
            if (!this->wait_warp(&w.k_full[st], turn(j))) return;
#pragma unroll 1
            for (int i = 0; i < tiles; i++) {
                const int pair = ONE ? j & 1 : i, u = ONE ? j >> 1 : j;
                if (!this->wait_warp(&w.s_empty[pair][u & 1], ((u >> 1) & 1) ^ 1)) return;
                tc_after();
                const uint64_t q = q_desc + i * kMat16, k = k_desc + st * (kStage >> 4);
                const uint32_t d = tmem + (2 * pair + (u & 1)) * kRowTile;
                if (elect_lane()) {
#pragma unroll
                    for (int x = 0; x < D / 16; x++) {              // 16 channels: 32 bytes inside a 128-byte row, then the next half
                        const uint32_t o = (x >> 2) * (kRowTile * 8) + (x & 3) * 2;
                        tc_mma_ss(d, COLUMNS ? k + o : q + o, COLUMNS ? q + o : k + o, kDesc, x != 0);
                        if (FINE) tc_mma_ss(d, COLUMNS ? k + o + kMat16 : q + o, COLUMNS ? q + o : k + o + kMat16, kDesc, true);
                    }
                    tc_commit(&w.s_full[pair][u & 1]);
                    if (i == tiles - 1) tc_commit(&w.k_empty[st]);
                }
                __syncwarp();
            }
        }
    }

    // ---- the warpgroups: pair wg >> 1, columns 64 (wg & 1) .. + 63 of a place
    static constexpr int kOnFma = 5;                                // of 16 pairs of exponentials, those that are computed (0 .. 16)
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
    // Queries into shared memory, their factors and positions: a tile by the first warpgroup of a pair.
    __device__ __forceinline__ void queries(int wg, int tiles, int first, int m0, int m_end) {
        const int i = wg >> 1, r = threadIdx.x & 127;
        if (!(wg & 1) && i < tiles) {
            const int m = m0 + 128 * i + r;
            const bool live = m < m_end;
            const int row = live ? first + m / this->p.share : first, hq = live ? this->head * this->p.share + m % this->p.share : 0;
            w.pos[128 * i + r] = live ? max(-1, row_position(this->p.b, this->seq, row)) : -1;
            w.factor[128 * i + r] = this->load_query(i, r, live, row, hq);
            fence_async_smem();
            __syncwarp();
            if ((threadIdx.x & 31) == 0) mbar_arrive(&w.r.q_ready[i]);
        }
        sync_consumers();
    }
    __device__ __forceinline__ void release(int pair, int u) {
        tc_before();
        __syncwarp();
        if ((threadIdx.x & 31) == 0) mbar_arrive(&w.s_empty[pair][u & 1]);
    }
    __device__ __forceinline__ long long vector_index(int first, int m) const {
        return (long long)(first + m / this->p.share) * this->p.Hq + this->head * this->p.share + m % this->p.share;
    }

    // First pass: a thread per query vector.
    __device__ __forceinline__ void rows(int wg, int tiles, int first, int m0, int m_end, uint32_t tmem, const WeighRowsPlan& pl, int split) {
        queries(wg, tiles, first, m0, m_end);
        const int pair = wg >> 1, half = wg & 1;
        if (!ONE && pair >= tiles) return;
        const int r = threadIdx.x & 127, i = ONE ? 0 : pair, m = m0 + 128 * i + r, pos = w.pos[128 * i + r], kv = this->kv;
        float factor = w.factor[128 * i + r];
        const bool broken = factor != factor;
        if (broken) factor = 1.0f;
        if (factor == 0.0f) factor = 1.17549435e-38f;               // a mask is minus infinity over the factor
        const uint32_t at = tmem + ((uint32_t)((threadIdx.x >> 5) & 3) << 21) + 64 * half;
        float ref = kNoMax;
        f32x2 sum2[2] = {pack2(0.0f, 0.0f), pack2(0.0f, 0.0f)};
        const f32x2 factor2 = pack2(factor, factor);
        const int n = this->end - this->begin;
#pragma unroll 1
        for (int u = 0, j = ONE ? pair : 0; j < n; u++, j += ONE ? 2 : 1) {
            const int t0 = this->range.tile(this->begin + j) * kRowTile;
            const uint32_t s_at = at + (2 * pair + (u & 1)) * kRowTile;
            if (!this->wait_warp(&w.s_full[pair][u & 1], (u >> 1) & 1)) return;
            tc_after();
            const uint4 absent = lds128(smem_u32(w.absent[j & 7]));
            const bool gaps = (absent.x | absent.y | absent.z | absent.w) != 0;
            if (gaps || !this->whole(t0)) {                         // what a row does not see becomes minus infinity, in TMEM
                if (IMAGE && gaps && !half) this->latch_absent(t0, absent);
                const int c0 = 64 * half, b = min(pos, kv - 1) - t0, a = this->p.window > 0 ? max(pos - this->p.window + 1, 0) - t0 : -t0, s = this->p.sinks - t0;
                const uint32_t none = factor < 0.0f ? 0x7F800000u : 0xFF800000u;
#pragma unroll 1
                for (int k = 0; k < 4; k++) {
                    const uint32_t gone = (half ? (k < 2 ? absent.z : absent.w) : (k < 2 ? absent.x : absent.y)) >> (16 * (k & 1));
                    const uint32_t in = B::seen(c0 + 16 * k, a, b, s, gone);
                    uint32_t x[16];
                    tc_ld16(x, s_at + 16 * k);
                    tc_wait_ld();
#pragma unroll
                    for (int c = 0; c < 16; c++) x[c] = in >> c & 1u ? x[c] : none;
                    tc_st16(s_at + 16 * k, x);
                }
                tc_wait_st();
            }
            // Against the reference as it stands, a row's largest logit in the first step it had tokens in; where the sum shows that it has become
            // too small (fp32 has room for logits 60 above it) the largest is looked for again and the step done once more.
            f32x2 total[2];
            bool search = u == 0;
            for (;;) {
                if (search) {
                    float y = -INFINITY;
#pragma unroll 1
                    for (int k = 0; k < 4; k++) {
                        uint32_t x[16];
                        tc_ld16(x, s_at + 16 * k);
                        tc_wait_ld();
#pragma unroll
                        for (int c = 0; c < 16; c++) y = fmaxf(y, __uint_as_float(x[c]) * factor);
                    }
                    const float to = fmaxf(y, ref), keep = fast_exp2(ref - to);
                    ref = to;
                    sum2[0] = mul2(sum2[0], pack2(keep, keep));
                    sum2[1] = mul2(sum2[1], pack2(keep, keep));
                }
                const f32x2 ref2 = pack2(-ref, -ref);
                total[0] = sum2[0];
                total[1] = sum2[1];
#pragma unroll
                for (int k = 0; k < 2; k++) {
                    float x[32];
                    tc_ld32(x, s_at + 32 * k);
                    tc_wait_ld();
                    add_row(x, factor2, ref2, total);
                }
                if (search) break;
                float a, b;
                unpack2(add2(total[0], total[1]), a, b);
                search = __any_sync(0xFFFFFFFFu, a + b > 1.0e18f);
                if (!search) break;
            }
            sum2[0] = total[0];
            sum2[1] = total[1];
            release(pair, u);
        }
        if (m >= m_end) return;
        float a, b;
        unpack2(add2(sum2[0], sum2[1]), a, b);
        a += b;
        if (broken && a != 0.0f) a = __uint_as_float(0x7FC00000u);
        const int slot = ONE ? 4 * split + wg : 2 * split + half;
        pl.sums[(long long)slot * this->p.b.n_rows * this->p.Hq + vector_index(first, m)] = make_float2(ref, a);
    }

    // Second pass: a thread per token, the vectors of a tile along its lane; `in`: the vectors that see it, where not all do.
    template <bool MASK>
    __device__ __forceinline__ void add_column(const float (&x)[32], const float4* column, uint32_t in, f32x2 (&total)[2]) const {
#pragma unroll
        for (int c = 0; c < 16; c++) {
            const uint4 v = lds128(smem_u32(column + c));
            float a, b;
            exp2_both(c, fma2(pack2(x[2 * c], x[2 * c + 1]), pack2(__uint_as_float(v.x), __uint_as_float(v.y)), pack2(__uint_as_float(v.z), __uint_as_float(v.w))), a, b);
            if (MASK) {
                a = in >> (2 * c) & 1u ? a : 0.0f;
                b = in >> (2 * c + 1) & 1u ? b : 0.0f;
            }
            total[c & 1] = add2(total[c & 1], pack2(a, b));
        }
    }
    template <bool MASK>
    __device__ __forceinline__ float column_sum(uint32_t s_at, int first, unsigned long long in) const {
        f32x2 total[2] = {pack2(0.0f, 0.0f), pack2(0.0f, 0.0f)};
#pragma unroll
        for (int k = 0; k < 2; k++) {
            float x[32];
            tc_ld32(x, s_at + 32 * k);
            tc_wait_ld();
            add_column<MASK>(x, w.column + first / 2 + 16 * k, (uint32_t)(in >> (32 * k)), total);
        }
        float a, b;
        unpack2(add2(total[0], total[1]), a, b);
        return a + b;
    }
    // Which of 64 vectors from number `first` of the CTA see token t.  A row's vectors lie together.
    __device__ __forceinline__ unsigned long long seeing(int first, int m0, int t) const {
        unsigned long long in = 0;
        const int share = this->p.share;
        int left = share - (m0 + first) % share;                    // of the row's vectors, from this one on
#pragma unroll 1
        for (int c = 0; c < 64; c += left, left = share) {
            const int pos = w.pos[first + c];
            if (t <= pos && sees(this->p, pos, t)) in |= (left < 64 ? (1ull << left) - 1ull : ~0ull) << c;
        }
        return in;
    }
    __device__ __forceinline__ void columns(int wg, int tiles, int first, int m0, int m_end, uint32_t tmem, const WeighRowsPlan& pl, int tile) {
        const int pair = wg >> 1, half = wg & 1, r = threadIdx.x & 127, i = ONE ? 0 : pair, kv = this->kv;
        // -log2 of the rows' sums; minus infinity for a row that sees nothing and for vectors behind the last
        float low = -INFINITY;
        const int m = m0 + 128 * pair + r;
        if (!half && pair < tiles && m < m_end) {
            const long long vec = vector_index(first, m), step = (long long)this->p.b.n_rows * this->p.Hq;
            float top = kNoMax, sum = 0.0f;
            for (int k = 0; k < pl.slots; k++) top = fmaxf(top, pl.sums[k * step + vec].x);
            for (int k = 0; k < pl.slots; k++) {
                const float2 z = pl.sums[k * step + vec];
                sum = fmaf(z.y, fast_exp2(z.x - top), sum);
            }
            if (sum != 0.0f) low = -(top + log2f(sum));
        }
        queries(wg, tiles, first, m0, m_end);
        if (!half && pair < tiles) {
            float factor = w.factor[128 * pair + r];
            if (!(m < m_end)) factor = 0.0f;
            if (factor != factor) factor = 1.0f;
            float* v = reinterpret_cast<float*>(&w.column[64 * pair + (r >> 1)]) + (r & 1);
            v[0] = factor;
            v[2] = low;
        }
        sync_consumers();
        if (!ONE && pair >= tiles) return;
        const uint32_t at = tmem + ((uint32_t)((threadIdx.x >> 5) & 3) << 21) + 64 * half;
        const int n = this->end - this->begin;
        const bool leader = ONE ? half == 0 : wg == 0;              // adds up the other warpgroups' sums of a step, one step later
        float* out = pl.partial + (((long long)this->seq * this->p.c.H + this->head) * pl.chunk_tiles + tile) * pl.tokens + (long long)this->begin * kRowTile + r;
        float sum = 0.0f;
        int u = 0, before = -1;                                     // step whose sum the leader still has
        auto finish = [&]() {
            const int v = u - 1;
            if (!this->wait_warp(&w.part_full[ONE ? pair : 0][v & 3], (v >> 2) & 1)) return false;
            if (ONE) sum += w.part[v & 3][2 * pair][r];
            else for (int k = 0; k < 2 * tiles - 1; k++) sum += w.part[v & 3][k][r];
            out[(long long)before * kRowTile] = sum;
            return true;
        };
#pragma unroll 1
        for (int j = ONE ? pair : 0; j < n; u++, j += ONE ? 2 : 1) {
            const int t0 = this->range.tile(this->begin + j) * kRowTile, t = t0 + r;
            const uint32_t s_at = at + (2 * pair + (u & 1)) * kRowTile;
            if (leader && u && !finish()) return;
            if (!this->wait_warp(&w.s_full[pair][u & 1], (u >> 1) & 1)) return;
            tc_after();
            const uint4 absent = lds128(smem_u32(w.absent[j & 7]));
            const bool gaps = (absent.x | absent.y | absent.z | absent.w) != 0;
            if (gaps || !this->whole(t0)) {
                const uint32_t word = r < 32 ? absent.x : r < 64 ? absent.y : r < 96 ? absent.z : absent.w;
                const bool there = t < kv && !(word >> (r & 31) & 1u);
                sum = column_sum<true>(s_at, 128 * i + 64 * half, there ? seeing(128 * i + 64 * half, m0, t) : 0ull);
            } else {
                sum = column_sum<false>(s_at, 128 * i + 64 * half, 0ull);
            }
            release(pair, u);
            if (leader) {
                before = j;
            } else {
                w.part[u & 3][ONE ? 2 * pair : wg - 1][r] = sum;
                __syncwarp();
                if ((threadIdx.x & 31) == 0) mbar_arrive(&w.part_full[ONE ? pair : 0][u & 3]);
            }
        }
        if (leader && u) finish();
    }
};

template <int KF, int D, bool IMAGE, bool ONE, bool COLUMNS>
__global__ void __launch_bounds__(weigh_threads(IMAGE), 1) weigh_rows_kernel(const __grid_constant__ AttentionParams p, const __grid_constant__ WeighRowsPlan pl) {
    using K = WeighRows<KF, D, IMAGE, ONE, COLUMNS>;
    constexpr int kIssuer = weigh_issuer(IMAGE), kThreads = weigh_threads(IMAGE);
    extern __shared__ uint8_t raw[];
    const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u;
    WeighBars& bars = *reinterpret_cast<WeighBars*>(raw + (base - smem_u32(raw)) + RowsSmem<D>::kBars);
    pdl_trigger();
    const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x >> 5, 0);
    if (threadIdx.x == 0) {
        for (int i = 0; i < 2; i++) {
            mbar_init(&bars.r.q_ready[i], 4);
            for (int k = 0; k < 2; k++) { mbar_init(&bars.s_full[i][k], 1); mbar_init(&bars.s_empty[i][k], 8); }
        }
        for (int i = 0; i < 4; i++) { mbar_init(&bars.k_full[i], IMAGE ? 1 : kWeighProducers); mbar_init(&bars.k_empty[i], 1); }
        mbar_init(&bars.r.drained, 1);
        bars.r.abort = 0; bars.r.lost = 0;
        bars.r.lo = bars.r.least = 0x7FFFFFFF; bars.r.hi = -1;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    pdl_wait();
    // Block order: the last rows (the most tokens) of all heads first.
    int id = blockIdx.x;
    const int split = id % pl.splits; id /= pl.splits;
    const int head = id % p.c.H; id /= p.c.H;
    const int seq = id % p.b.n_seqs, local = pl.chunk_tiles - 1 - id / p.b.n_seqs, tile = pl.chunk + local;
    int first, kv, rows;
    const bool ordered = sequence_rows(p, seq, &first, &kv, &rows);
    if (threadIdx.x == 0 && (!ordered || rows > p.b.max_rows || p.b.kv_len[seq] > kv)) latch(p.status);
    if (!ordered) return;
    rows = min(rows, p.b.max_rows);
    const int m0 = tile * 2 * kRowTile, m_end = min(rows * p.share, m0 + 2 * kRowTile);
    if (m0 >= m_end) return;
    const int tiles = !ONE && m_end - m0 > kRowTile ? 2 : 1;
    if (COLUMNS && threadIdx.x == 0) {          // warps of the warpgroups that are not leaders
        for (int i = 0; i < 2; i++) for (int k = 0; k < 4; k++) mbar_init(&bars.part_full[i][k], ONE ? 4 : 4 * (2 * tiles - 1));
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    {   // positions of the CTA's rows (one below 0 sees nothing: no window need reach back for it)
        uint32_t low = 0x7FFFFFFFu;
        int least = 0x7FFFFFFF, most = -1;
        for (int r = m0 / p.share + threadIdx.x; r <= (m_end - 1) / p.share; r += kThreads) {
            const int x = row_position(p.b, seq, first + r);
            low = min(low, (uint32_t)x);
            least = min(least, x);
            most = max(most, x);
        }
        low = __reduce_min_sync(0xFFFFFFFFu, low);
        least = __reduce_min_sync(0xFFFFFFFFu, least);
        most = __reduce_max_sync(0xFFFFFFFFu, most);
        if (threadIdx.x == 0) { bars.r.first_row = first + m0 / p.share; bars.r.last_row = first + (m_end - 1) / p.share; }
        if ((threadIdx.x & 31) == 0) {
            atomicMin(&bars.r.lo, (int)low);
            atomicMin(&bars.r.least, least);
            atomicMax(&bars.r.hi, most);
        }
    }
    if (warp == kIssuer / 32) tc_alloc(&bars.r.tmem, 512);
    tc_before();
    __syncthreads();
    tc_after();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(&bars.r.tmem);
    K k(p, bars);
    k.smem = base; k.seq = seq; k.head = head; k.kv = kv;
    k.hi = bars.r.hi;
    k.last = min(bars.r.least, kv - 1);
    k.range = step_range(p, kv, bars.r.lo, k.hi);
    k.begin = (int)((long long)k.range.count * split / pl.splits);
    k.end = (int)((long long)k.range.count * (split + 1) / pl.splits);
    if (!COLUMNS && head == 0 && split == 0 && threadIdx.x == 0) pl.ranges[(long long)seq * pl.tiles + tile] = make_int4(k.range.sink_tiles, k.range.first, k.range.count, 0);
    if (warp < kWeighConsumers / 32) {
        if (COLUMNS) k.columns(warp >> 2, tiles, first, m0, m_end, tmem, pl, local);
        else k.rows(warp >> 2, tiles, first, m0, m_end, tmem, pl, split);
    } else if (warp < kIssuer / 32) {
        if constexpr (IMAGE) {
            k.fetch_images(pl);
        } else {
            k.produce(warp - kWeighConsumers / 32);
            cp_wait<0>();
        }
    } else if (k.end > k.begin) {
        k.issue(tiles, tmem);
        if (__any_sync(0xFFFFFFFFu, *reinterpret_cast<volatile int32_t*>(&bars.r.abort))) {    // what was issued must have ended before TMEM goes
            if (elect_lane()) tc_commit(&bars.r.drained);
            __syncwarp();
            for (uint32_t i = 0; i < kWaitLimit && !mbar_try_wait(&bars.r.drained, 0); i++) __nanosleep(40);
        }
    }
    __syncwarp();
    tc_before();
    __syncthreads();
    tc_after();
    if (warp == kIssuer / 32) tc_free(tmem, 512);
    if (threadIdx.x == 0 && bars.r.abort) atomicCAS(p.status, 0, (int)PATCHKV_E_TIMEOUT);
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

// The sum over heads and tiles of vectors (grid: step of 128 tokens, sequence): a thread per token, eight of them share the tiles.  64 bits:
// tens of thousands of numbers are added one by one.
constexpr int kWeighJoin = 1024;
static __global__ void __launch_bounds__(kWeighJoin) weigh_rows_join_kernel(const __grid_constant__ AttentionParams p, const __grid_constant__ WeightParams m,
                                                                            const __grid_constant__ WeighRowsPlan pl) {
    __shared__ double part[kWeighJoin];
    pdl_trigger();
    pdl_wait();
    const int s = blockIdx.y, step = blockIdx.x, r = threadIdx.x & 127, group = threadIdx.x >> 7;
    int first, kv, rows;
    if (!sequence_rows(p, s, &first, &kv, &rows) || step * kRowTile >= kv) return;
    const int tiles = (min(rows, p.b.max_rows) * p.share + 2 * kRowTile - 1) / (2 * kRowTile), end = min(tiles, pl.chunk + pl.chunk_tiles);
    double sum = 0.0;
    for (int tile = pl.chunk + group; tile < end; tile += kWeighJoin / 128) {
        const int4 range = pl.ranges[(long long)s * pl.tiles + tile];
        const int v = step < range.x ? step : step - range.y + range.x;
        if (!(step < range.x || (step >= range.y && v < range.z))) continue;
        const float* from = pl.partial + ((long long)s * p.c.H * pl.chunk_tiles + tile - pl.chunk) * pl.tokens + (long long)v * kRowTile + r;
        float heads = 0.0f;
#pragma unroll 8
        for (int h = 0; h < p.c.H; h++) heads += from[(long long)h * pl.chunk_tiles * pl.tokens];
        sum += heads;
    }
    part[threadIdx.x] = sum;
    __syncthreads();
    const int t = step * kRowTile + r;
    if (group || t >= kv) return;
    for (int i = 1; i < kWeighJoin / 128; i++) sum += part[i * 128 + r];
    double* acc = pl.acc ? pl.acc + (long long)s * p.b.max_kv_len + t : nullptr;
    if (acc && pl.chunk) sum += *acc;
    if (pl.last) store_mass(p, m, s, t, (float)sum);
    else *acc = sum;
}

}  // namespace patchkv
