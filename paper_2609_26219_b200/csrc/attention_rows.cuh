// Attention of many query rows on the 5th-generation tensor cores.
//
// A CTA takes one KV head and up to 256 query vectors of it (128 per tile, 1 or 2 tiles): query head and row are packed one behind
// the other, vector m = row * share + head, so that no row of the tiles is left empty whatever share is.  It walks the
// tokens in tiles of 128:
//   S = Q K^T    tcgen05.mma, 128 x 128 x D, both operands in shared memory, S in TMEM
//   P = 2^(S - ref)   a thread per row; P goes back to TMEM as 16-bit numbers over its S
//   O += P V     tcgen05.mma, 128 x D x 128, P from TMEM, V from shared memory, O in TMEM
// Roles: a warpgroup per tile for the softmax, one thread that issues the products, four warps that bring K and V.  The two tiles
// take turns: while one is in its softmax the tensor cores work for the other.
// K and V are brought by warps and not by TMA because the codes have to become operands on the way: fp16(code * scale), one
// rounding of 2^-12; bf16 pages are copied with cp.async.  Queries over quantised pages are fp16 scaled by a power of two per
// row, so a bf16 query loses nothing.  The weights are fp16 there, bf16 over bf16 pages; sums are fp32 throughout.
// As in the split kernel the softmax reference is only moved (and O rescaled) when a logit exceeds it by more than 8.
#pragma once

#include <stddef.h>

#include "attention_split.cuh"

namespace patchkv {

constexpr int kRowTile = 128;                   // query vectors of a tile, and tokens of a step
constexpr int kRowsThreads = 13 * 32;           // two softmax warpgroups, four producer warps, the issuing warp
constexpr int kProducer0 = 256, kIssuer = 384;  // first threads of the roles

struct RowsPlan {
    float* partial;                             // [split][n_rows * Hq][D], then (m, l) [split][n_rows * Hq]
    int32_t tiles;                              // CTAs along the query vectors of a sequence
    int32_t splits;                             // pieces of the token range (1: no partial results)
};

// ---- tcgen05 --------------------------------------------------------------------------------------------------------
__device__ __forceinline__ void tc_alloc(uint32_t* slot, uint32_t cols) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(slot)), "r"(cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
}
__device__ __forceinline__ void tc_free(uint32_t addr, uint32_t cols) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(cols));
}
__device__ __forceinline__ void tc_commit(uint64_t* bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add) : "memory");
}
__device__ __forceinline__ void tc_mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool add) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"((uint32_t)add) : "memory");
}
__device__ __forceinline__ void tc_ld32(float (&v)[32], uint32_t addr) {
    uint32_t* r = reinterpret_cast<uint32_t*>(v);
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,"
        "%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
          "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
          "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr) : "memory");
}
__device__ __forceinline__ void tc_st32(uint32_t addr, const float (&v)[32]) {
    const uint32_t* r = reinterpret_cast<const uint32_t*>(v);
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,"
        "%27,%28,%29,%30,%31,%32};" ::"r"(addr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
        "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]),
        "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]) : "memory");
}
__device__ __forceinline__ void tc_st16(uint32_t addr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(addr), "r"(r[0]), "r"(r[1]),
        "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]),
        "r"(r[14]), "r"(r[15]) : "memory");
}
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void sts128(uint32_t a, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
    asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(a), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}

// Shared-memory matrices: [64-channel half][row][128 bytes], 16-byte chunks xor-ed with row & 7 (the 128-byte swizzle).
__device__ __forceinline__ uint32_t swizzled(uint32_t row, uint32_t chunk) {        // chunk: 16 bytes, numbered along all channels
    return (chunk >> 3) * (kRowTile * 128) + row * 128 + (((chunk & 7) ^ (row & 7)) << 4);
}
// Matrix descriptor: 128-byte swizzle; stride between groups of 8 rows 1024 bytes; `lead`: stride between 64-channel halves, used
// where the channels are the M or N side (V).
__device__ __forceinline__ uint64_t smem_desc(uint32_t addr, uint32_t lead) {
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | (uint64_t)(lead >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
// Instruction descriptor, kind::f16: fp32 accumulators, both operands bf16 (or fp16), M = 128.
__host__ __device__ constexpr uint32_t instr_desc(bool bf16, bool b_mn_major, int n) {
    return 1u << 4 | (bf16 ? 1u : 0u) << 7 | (bf16 ? 1u : 0u) << 10 | (b_mn_major ? 1u : 0u) << 16 | (uint32_t)(n >> 3) << 17 | (uint32_t)(kRowTile >> 4) << 24;
}

template <int D>
struct RowsSmem {
    static constexpr int kMat = kRowTile * D * 2;               // one 128-row matrix
    static constexpr int kQ = 0, kK = 2 * kMat, kV = 4 * kMat, kBars = 6 * kMat;
    static constexpr int kBytes = kBars + 512 + 1024;           // 1024: the matrices start on a multiple of that
    static constexpr int kLaunch = kBytes > 120 * 1024 ? kBytes : 120 * 1024;   // one CTA per SM: it takes all of TMEM
};
struct RowsBars {
    uint64_t q_ready[2], s_ready[2], p_ready[2], o_ready[2], k_full[2], k_empty[2], v_full[2], v_empty[2], drained;
    alignas(16) uint32_t absent[4][4];                      // per step (mod 4): tokens whose page is out of range
    uint32_t tmem;
    int32_t abort, lo, hi, lost;                // lost: a value that is not finite was taken out of a tile that needs a mask
};
static_assert(sizeof(RowsBars) <= 512 && offsetof(RowsBars, absent) % 16 == 0, "barrier area");

// Steps of 128 tokens that the rows between positions lo and hi see (as tile_range, in other units).
__device__ __forceinline__ TileRange step_range(const AttentionParams& p, int kv, int lo_pos, int hi_pos) {
    TileRange r;
    const int end = min(hi_pos, kv - 1) + 1;
    const int lo = p.window > 0 ? max(0, lo_pos - p.window + 1) : 0;
    r.first = lo / kRowTile;
    const int last = end <= 0 ? 0 : (end - 1) / kRowTile + 1;
    r.sink_tiles = p.window > 0 ? min((min(p.sinks, r.first * kRowTile) + kRowTile - 1) / kRowTile, last) : 0;
    r.count = r.sink_tiles + max(0, last - r.first);
    return r;
}

// Eight fp16 operands of a word of 4-bit codes, in the order 0 4 1 5 2 6 3 7 of its nibbles: 1024 + u (1024 + 16 u) is a bit pattern,
// minus 1032 (times 2^-4, minus 72) the exact code, times the scale the one rounding.
__device__ __forceinline__ uint4 operands4(uint32_t w, uint32_t s, uint32_t m0, uint32_t m1) {
    const uint32_t v = w >> 8;
    uint4 o;
    asm("{\n\t.reg .b32 a;\n\tsub.rn.f16x2 a, %1, %2;\n\tmul.rn.f16x2 %0, a, %3;\n\t}" : "=r"(o.x) : "r"(and_xor<0x000F000Fu>(w, m0)), "r"(0x64086408u), "r"(s));
    asm("{\n\t.reg .b32 a;\n\tfma.rn.f16x2 a, %1, %2, %3;\n\tmul.rn.f16x2 %0, a, %4;\n\t}" : "=r"(o.y) : "r"(and_xor<0x00F000F0u>(w, m1)), "r"(0x2C002C00u), "r"(0xD480D480u), "r"(s));
    asm("{\n\t.reg .b32 a;\n\tsub.rn.f16x2 a, %1, %2;\n\tmul.rn.f16x2 %0, a, %3;\n\t}" : "=r"(o.z) : "r"(and_xor<0x000F000Fu>(v, m0)), "r"(0x64086408u), "r"(s));
    asm("{\n\t.reg .b32 a;\n\tfma.rn.f16x2 a, %1, %2, %3;\n\tmul.rn.f16x2 %0, a, %4;\n\t}" : "=r"(o.w) : "r"(and_xor<0x00F000F0u>(v, m1)), "r"(0x2C002C00u), "r"(0xD480D480u), "r"(s));
    return o;
}
// Four fp16 operands of a word of 8-bit codes, in order: 1024 + u, minus 1152, times the scale.
__device__ __forceinline__ uint2 operands8(uint32_t w, uint32_t s) {
    const uint32_t u = w ^ 0x80808080u;
    uint2 o;
    asm("{\n\t.reg .b32 a;\n\tsub.rn.f16x2 a, %1, %2;\n\tmul.rn.f16x2 %0, a, %3;\n\t}" : "=r"(o.x) : "r"(__byte_perm(u, 0x64646464u, 0x4140)), "r"(0x64806480u), "r"(s));
    asm("{\n\t.reg .b32 a;\n\tsub.rn.f16x2 a, %1, %2;\n\tmul.rn.f16x2 %0, a, %3;\n\t}" : "=r"(o.y) : "r"(__byte_perm(u, 0x64646464u, 0x4342)), "r"(0x64806480u), "r"(s));
    return o;
}

struct StepPlace { TileRange range; int seq, head, kv, lo, hi, begin, end; };
__device__ __forceinline__ bool whole_step(const AttentionParams& p, int kv, int lo, int hi, int t0) {
    return t0 + kRowTile - 1 <= min(lo, kv - 1) && (p.window == 0 || hi - t0 < p.window || t0 + kRowTile <= p.sinks);
}
// Values that are not finite were taken out of the masked steps; a row that sees such a value gets it here.  (Rare: element by
// element, from the pages.)
template <int VF, int D>
__device__ __noinline__ void add_lost(const AttentionParams& p, const StepPlace& at, float (&o)[32], int c0, int pos) {
    for (int j = at.begin; j < at.end; j++) {
        const int t0 = at.range.tile(j) * kRowTile;
        if (whole_step(p, at.kv, at.lo, at.hi, t0)) continue;
        for (int t = t0; t < t0 + kRowTile; t++) {
            if (t > min(pos, at.kv - 1) || !sees(p, pos, t)) continue;
            const int lp = div_page(p.c, t), slot = t - lp * p.c.P;
            const int page = __ldg(p.b.block_table + (long long)at.seq * p.b.table_stride + lp);
            if (page < 0 || page >= p.c.n_pages) continue;
            for (int c = 0; c < 32; c++) {
                float v;
                // column c of the accumulator is channel `ch`
                const int e = c & 7, ch = c0 + (VF == FMT_INT4 ? (c & ~7) + (e & 1 ? 4 + (e >> 1) : e >> 1) : c);
                if (VF == FMT_BF16) {
                    v = bf16_bits_to_float(p.c.v[(long long)page * p.c.stride_page + (long long)slot * p.c.stride_token + (long long)at.head * p.c.stride_head + ch]);
                } else {
                    const uint8_t* pg = p.c.base + (long long)page * p.c.stride_page;
                    const unsigned long long el = ((unsigned long long)slot * p.c.H + at.head) * D + ch;
                    v = (float)code_at(pg + p.c.v_codes, VF, el) * scale_at(pg + p.c.v_scales, el / p.c.G);
                    v = __half2float(__float2half_rn(v));   // as the operand was: beyond 65504 an infinity
                }
                if (!(fabsf(v) <= 3.4e38f)) o[c] += v;
            }
        }
    }
}

// KF / VF: page formats (both FMT_BF16 for the bf16 pool).
template <int KF, int VF, int D>
struct RowsKernel {
    static constexpr bool kPool = KF == FMT_BF16;
    using S = RowsSmem<D>;
    static constexpr int kPer = D / 32;                         // 32-channel pieces (= threads) of a token's row

    const AttentionParams& p;
    RowsBars& bars;
    uint32_t smem;
    int seq, head, kv, lo, hi, begin, end;                      // steps [begin, end) of the range
    TileRange range;

    __device__ __forceinline__ RowsKernel(const AttentionParams& p_, RowsBars& b) : p(p_), bars(b) {}
    __device__ __forceinline__ bool wait(uint64_t* bar, uint32_t parity) { return mbar_wait(bar, parity, &bars.abort); }
    // The same for a whole warp: all of its lanes go on, or none.
    __device__ __forceinline__ bool wait_warp(uint64_t* bar, uint32_t parity) { return __all_sync(0xFFFFFFFFu, wait(bar, parity)); }
    // Seen by some row (or by none): only then does a token's slot take part.
    __device__ __forceinline__ bool any_sees(int t) const { return t <= min(hi, kv - 1) && sees(p, lo, t); }
    __device__ __forceinline__ bool whole(int t0) const { return whole_step(p, kv, lo, hi, t0); }

    // ---- the warps that bring K and V
    __device__ __forceinline__ void produce() {
        const int w = (threadIdx.x - kProducer0) >> 5, lane = threadIdx.x & 31;
        // A warp takes 32 tokens of a step; kPer lanes share a token, 32 / kPer tokens at a time.
        constexpr int kTok = 32 / kPer, kPass = kPer;
        const int c = lane % kPer, tok0 = 32 * w + lane / kPer;
        uint32_t m0, m1;                                        // 1024 + 8 and 1024 + 8 * 16 in every half: magic and offset
        asm volatile("mov.b32 %0, 0x64086408;" : "=r"(m0));
        asm volatile("mov.b32 %0, 0x64806480;" : "=r"(m1));
        int next_page = page_of(begin, 32 * w + (lane & 1) * 16);
        for (int j = begin; j < end; j++) {
            const int n = j - begin, st = n & 1, t0 = range.tile(j) * kRowTile;
            const uint32_t parity = ((n >> 1) & 1) ^ 1;
            const int page_lane = next_page;                    // lane 0: the warp's first 16 tokens, lane 1: the other 16
            if (j + 1 < end) next_page = page_of(j + 1, 32 * w + (lane & 1) * 16);
            const bool masked = !whole(t0);
            uint32_t kw[kPass][8], vw[kPass][8], ks[kPass], vs[kPass];
            bool live[kPass];
            long long at[kPass];
            uint32_t gone = 0;
#pragma unroll
            for (int i = 0; i < kPass; i++) {
                const int tok = tok0 + i * kTok, t = t0 + tok;
                const int page = __shfl_sync(0xFFFFFFFFu, page_lane, (tok - 32 * w) >> 4);
                live[i] = any_sees(t);
                if (live[i] && page < 0) { live[i] = false; gone |= 1u << (tok & 31); latch(p.status); }
                const int slot = t - div_page(p.c, t) * p.c.P;
                at[i] = kPool ? (long long)page * p.c.stride_page + (long long)slot * p.c.stride_token + (long long)head * p.c.stride_head
                              : (long long)page * p.c.stride_page;
                if constexpr (!kPool) {
                    const uint8_t* pg = p.c.base + at[i];
                    const uint32_t row = (uint32_t)slot * p.c.H + head;
                    load_codes<KF>(kw[i], pg + row * (KF == FMT_INT8 ? D : D / 2), c, live[i]);
                    load_codes<VF>(vw[i], pg + p.c.v_codes + row * (VF == FMT_INT8 ? D : D / 2), c, live[i]);
                    const uint32_t s = (row * (D / p.c.G) + c * 32 / p.c.G) * 2;
                    ks[i] = live[i] ? __ldg(reinterpret_cast<const uint16_t*>(pg + p.c.k_scales + s)) : 0u;
                    vs[i] = live[i] ? __ldg(reinterpret_cast<const uint16_t*>(pg + p.c.v_scales + s)) : 0u;
                }
            }
            gone = __reduce_or_sync(0xFFFFFFFFu, gone);
            if (lane == 0) bars.absent[n & 3][w] = gone;
            const uint32_t kb = smem + S::kK + st * S::kMat, vb = smem + S::kV + st * S::kMat;
            if (!wait_warp(&bars.k_empty[st], parity)) return;
            if constexpr (kPool) {
#pragma unroll
                for (int i = 0; i < kPass; i++)
#pragma unroll
                    for (int q = 0; q < 4; q++)                 // chunks kPer apart: a row's lanes read a contiguous run
                        cp16(kb + swizzled(tok0 + i * kTok, q * kPer + c), p.c.k + (live[i] ? at[i] + 8 * (q * kPer + c) : 0), live[i]);
                cp_commit();
                if (!wait_warp(&bars.v_empty[st], parity)) return;
#pragma unroll
                for (int i = 0; i < kPass; i++)
#pragma unroll
                    for (int q = 0; q < 4; q++)
                        cp16(vb + swizzled(tok0 + i * kTok, q * kPer + c), p.c.v + (live[i] ? at[i] + 8 * (q * kPer + c) : 0), live[i]);
                cp_commit();
                cp_wait<1>();
                fence_async_smem();
                mbar_arrive(&bars.k_full[st]);
                cp_wait<0>();
                if (masked) clean<0x7F80u>(vb, tok0, c, 1, kPer);
                fence_async_smem();
                mbar_arrive(&bars.v_full[st]);
            } else {
#pragma unroll
                for (int i = 0; i < kPass; i++) store_operands<KF>(kb, tok0 + i * kTok, c, kw[i], ks[i], m0, m1);
                fence_async_smem();
                mbar_arrive(&bars.k_full[st]);
                if (!wait_warp(&bars.v_empty[st], parity)) return;
#pragma unroll
                for (int i = 0; i < kPass; i++) store_operands<VF>(vb, tok0 + i * kTok, c, vw[i], vs[i], m0, m1);
                if (masked) clean<0x7C00u>(vb, tok0, c, 4, 1);
                fence_async_smem();
                mbar_arrive(&bars.v_full[st]);
            }
        }
    }
    // Page of token `tok` of step j; -1 when it is out of range or lies behind the cache.
    __device__ __forceinline__ int page_of(int j, int tok) const {
        if (j >= end) return -1;
        const int t = range.tile(j) * kRowTile + tok;
        if (t >= kv) return -1;
        const int pg = __ldg(p.b.block_table + (long long)seq * p.b.table_stride + div_page(p.c, t));
        return pg >= 0 && pg < p.c.n_pages ? pg : -1;
    }
    template <int F>
    __device__ __forceinline__ static void load_codes(uint32_t (&w)[8], const uint8_t* row, int c, bool live) {
#pragma unroll
        for (int i = 0; i < 8; i++) w[i] = 0;
        if (!live) return;
        const uint4 a = __ldg(reinterpret_cast<const uint4*>(row + c * (F == FMT_INT8 ? 32 : 16)));
        w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
        if (F == FMT_INT8) {
            const uint4 b = __ldg(reinterpret_cast<const uint4*>(row + c * 32 + 16));
            w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
        }
    }
    // Sets fp16 (EXP 0x7C00) or bf16 (0x7F80) numbers that are not finite to zero; true when there was one.
    template <uint32_t EXP>
    __device__ __forceinline__ static bool finite_only(uint4& x) {
        bool found = false;
        uint32_t* w = &x.x;
#pragma unroll
        for (int i = 0; i < 4; i++) {
            if ((w[i] & EXP) == EXP) { w[i] &= 0xFFFF0000u; found = true; }
            if ((w[i] >> 16 & EXP) == EXP) { w[i] &= 0x0000FFFFu; found = true; }
        }
        return found;
    }
    // In a step that needs a mask a value that is not finite must not meet the weight 0 of a row that does not see it: it is taken out
    // here and given to the rows that see it at the end.  Chunks of the thread: c * lead + q * apart, q = 0 .. 3.
    template <uint32_t EXP>
    __device__ __forceinline__ void clean(uint32_t mat, int tok0, int c, int lead, int apart) {
#pragma unroll 1
        for (int i = 0; i < kPer * 4; i++) {
            const uint32_t a = mat + swizzled(tok0 + (i >> 2) * (32 / kPer), c * lead + (i & 3) * apart);
            uint4 x = lds128(a);
            if (finite_only<EXP>(x)) { sts128(a, x.x, x.y, x.z, x.w); bars.lost = 1; }
        }
    }
    // The 32 channels of a thread into its token's row.
    template <int F>
    __device__ __forceinline__ void store_operands(uint32_t mat, int tok, int c, const uint32_t (&w)[8], uint32_t scale, uint32_t m0, uint32_t m1) {
        const uint32_t s = scale | scale << 16;
        const uint32_t flip = c & 2;                            // the two halves of the channels write different banks
#pragma unroll
        for (int i = 0; i < 4; i++) {
            uint4 o;
            if constexpr (F == FMT_INT4) {
                o = operands4(flip ? w[i ^ 2] : w[i], s, m0, m1);
            } else {
                const uint2 a = operands8(flip ? w[(2 * i) ^ 4] : w[2 * i], s), b = operands8(flip ? w[(2 * i + 1) ^ 4] : w[2 * i + 1], s);
                o = make_uint4(a.x, a.y, b.x, b.y);
            }
            sts128(mat + swizzled(tok, 4 * c + (i ^ flip)), o.x, o.y, o.z, o.w);
        }
    }

    // ---- the thread that issues the products
    __device__ __forceinline__ void issue(int tiles, uint32_t tmem) {
        constexpr uint32_t kQk = instr_desc(kPool, false, kRowTile), kPv = instr_desc(kPool, true, D);
        auto logits = [&](int i, int st) {
            const uint32_t q = smem + S::kQ + i * S::kMat, k = smem + S::kK + st * S::kMat;
#pragma unroll
            for (int x = 0; x < D / 16; x++) {                  // 16 channels: 32 bytes inside a 128-byte row, then the next half
                const uint32_t o = (x >> 2) * (kRowTile * 128) + (x & 3) * 32;
                tc_mma_ss(tmem + i * kRowTile, smem_desc(q + o, 16), smem_desc(k + o, 16), kQk, x != 0);
            }
            tc_commit(&bars.s_ready[i]);
        };
        for (int i = 0; i < tiles; i++) if (!wait(&bars.q_ready[i], 0)) return;
        if (!wait(&bars.k_full[0], 0)) return;
        tc_after();
        for (int i = 0; i < tiles; i++) logits(i, 0);
        tc_commit(&bars.k_empty[0]);
        const int n = end - begin;
        for (int j = 0; j < n; j++) {
            const int st = j & 1;
            for (int i = 0; i < tiles; i++) {
                if (i == 0 && !wait(&bars.v_full[st], (j >> 1) & 1)) return;
                if (!wait(&bars.p_ready[i], j & 1)) return;
                tc_after();
                const uint32_t v = smem + S::kV + st * S::kMat;
#pragma unroll
                for (int x = 0; x < kRowTile / 16; x++)         // 16 tokens: two groups of 8 rows
                    tc_mma_ts(tmem + 2 * kRowTile + i * kRowTile, tmem + i * kRowTile + 8 * x, smem_desc(v + x * 2048, kRowTile * 128), kPv, j != 0 || x != 0);
                if (i == tiles - 1) tc_commit(&bars.v_empty[st]);
                if (j + 1 < n) {
                    if (i == 0) {
                        if (!wait(&bars.k_full[st ^ 1], ((j + 1) >> 1) & 1)) return;
                        tc_after();
                    }
                    logits(i, st ^ 1);
                    if (i == tiles - 1) tc_commit(&bars.k_empty[st ^ 1]);
                } else {
                    tc_commit(&bars.o_ready[i]);
                }
            }
        }
    }

    // Bit c: this row sees column c0 + c.
    __device__ __forceinline__ static uint32_t seen(int c0, int a, int b, int s, const uint4& absent, int k) {
        auto below = [](int n) { return n <= 0 ? 0u : n >= 32 ? 0xFFFFFFFFu : (1u << n) - 1u; };      // bits [0, n)
        const uint32_t gone = k == 0 ? absent.x : k == 1 ? absent.y : k == 2 ? absent.z : absent.w;
        return below(b + 1 - c0) & (~below(a - c0) | below(s - c0)) & ~gone;
    }
    // What a row does not see becomes the value whose weight is zero: times the factor minus infinity.
    __device__ __forceinline__ static void mask_chunk(float (&x)[32], uint32_t seen, float factor) {
        const float none = factor < 0.0f ? INFINITY : -INFINITY;
#pragma unroll
        for (int c = 0; c < 32; c++) x[c] = seen >> c & 1u ? x[c] : none;
    }

    // ---- softmax: one thread per query vector
    __device__ __forceinline__ void softmax(int i, int first, int m, int m_end, uint32_t tmem, const RowsPlan& pl, int split) {
        const int r = threadIdx.x & 127;
        const bool live = m < m_end;
        const int row = live ? first + m / p.share : first, hq = live ? head * p.share + m % p.share : 0;
        const int pos = live ? max(-1, row_position(p.b, seq, row)) : -1;
        // the query into shared memory
        float factor = p.scale_log2;
        {
            const uint16_t* q = p.q + (long long)row * p.q_stride_row + (long long)hq * p.q_stride_head;
            const uint32_t mat = smem + S::kQ + i * S::kMat;
            if constexpr (kPool) {
#pragma unroll 4
                for (int c = 0; c < D / 8; c++) {
                    const uint4 x = live ? __ldg(reinterpret_cast<const uint4*>(q) + c) : make_uint4(0, 0, 0, 0);
                    sts128(mat + swizzled(r, c), x.x, x.y, x.z, x.w);
                }
            } else {
                // scaled so that the largest magnitude lies in [2^13, 2^14); a vector with a NaN or an infinity gives NaN
                float amax = 0.0f, bad = 0.0f;
#pragma unroll 4
                for (int c = 0; c < D / 8; c++) {
                    const uint4 x = live ? __ldg(reinterpret_cast<const uint4*>(q) + c) : make_uint4(0, 0, 0, 0);
                    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                    for (int k = 0; k < 4; k++) {
                        const float a = p.f16 ? low_half(w[k]) : bf16_bits_to_float(w[k] & 0xFFFFu), b = p.f16 ? high_half(w[k]) : __uint_as_float(w[k] & 0xFFFF0000u);
                        amax = fmaxf(amax, fmaxf(fabsf(a), fabsf(b)));
                        bad = fmaf(a, 0.0f, fmaf(b, 0.0f, bad));
                    }
                }
                const int e = (int)(__float_as_uint(amax) >> 23) - 127;
                const int shift = amax > 0.0f ? min(13 - e, 120) : 0;
                const float up = bad == 0.0f ? exp2i(shift) : 0.0f;
                factor = p.scale_log2 * exp2i(-shift) + bad;
#pragma unroll 2
                for (int c = 0; c < D / 8; c++) {
                    const uint4 x = live && bad == 0.0f ? __ldg(reinterpret_cast<const uint4*>(q) + c) : make_uint4(0, 0, 0, 0);
                    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
                    float f[8];
#pragma unroll
                    for (int k = 0; k < 4; k++) {
                        f[2 * k] = (p.f16 ? low_half(w[k]) : bf16_bits_to_float(w[k] & 0xFFFFu)) * up;
                        f[2 * k + 1] = (p.f16 ? high_half(w[k]) : __uint_as_float(w[k] & 0xFFFF0000u)) * up;
                    }
                    if (KF == FMT_INT4)                         // the order operands4 leaves the channels in
                        sts128(mat + swizzled(r, c), half2_bits(f[0], f[4]), half2_bits(f[1], f[5]), half2_bits(f[2], f[6]), half2_bits(f[3], f[7]));
                    else
                        sts128(mat + swizzled(r, c), half2_bits(f[0], f[1]), half2_bits(f[2], f[3]), half2_bits(f[4], f[5]), half2_bits(f[6], f[7]));
                }
            }
        }
        fence_async_smem();
        mbar_arrive(&bars.q_ready[i]);
        // A mask is minus infinity over the factor: a factor of zero is one that leaves no logit, a NaN enters at the end.
        const bool broken = factor != factor;
        if (broken) factor = 1.0f;
        if (factor == 0.0f) factor = 1.17549435e-38f;
        const uint32_t lanes = (uint32_t)((threadIdx.x >> 5) & 3) << 21;              // the warp's quarter of the TMEM lanes
        const uint32_t s_at = tmem + lanes + i * kRowTile, o_at = tmem + lanes + 2 * kRowTile + i * kRowTile;
        float ref = kNoMax;
        f32x2 sum2 = pack2(0.0f, 0.0f);
        const int n = end - begin;
        for (int j = 0; j < n; j++) {
            const int t0 = range.tile(begin + j) * kRowTile;
            if (!wait_warp(&bars.s_ready[i], j & 1)) return;
            tc_after();
            // Columns of the step this row sees: [a, b] and [0, s); what its pages don't hold is in `absent`.
            const uint4 absent = lds128(smem_u32(bars.absent[j & 3]));
            const bool plain = whole(t0) && (absent.x | absent.y | absent.z | absent.w) == 0;
            const int b = min(pos, kv - 1) - t0, a = p.window > 0 ? max(pos - p.window + 1, 0) - t0 : -t0, s = p.sinks - t0;
            // The loops over the step's four chunks stay loops: three roles run different code on an SM, and unrolled it does not
            // stay in the instruction cache (1270 us for 8192 rows of prompt, most of it waiting for instructions).
            float top = -INFINITY;
#pragma unroll 1
            for (int k = 0; k < 4; k++) {
                float x[32];
                tc_ld32(x, s_at + 32 * k);
                tc_wait_ld();
                if (!plain) mask_chunk(x, seen(32 * k, a, b, s, absent, k), factor);
                float y[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                if (factor < 0.0f)
#pragma unroll
                    for (int c = 0; c < 32; c++) x[c] = -x[c];
#pragma unroll
                for (int c = 0; c < 32; c += 2) y[(c >> 1) & 3] = fmaxf(y[(c >> 1) & 3], fmaxf(x[c], x[c + 1]));
                top = fmaxf(top, fmaxf(fmaxf(y[0], y[1]), fmaxf(y[2], y[3])));
            }
            top = top == -INFINITY ? top : top * fabsf(factor);
            const bool move = top > ref + 8.0f;
            if (__any_sync(0xFFFFFFFFu, move)) {
                const float to = move ? top : ref, keep = fast_exp2(ref - to);
                ref = to;
                sum2 = mul2(sum2, pack2(keep, keep));
                if (j > 0)                                      // the products of the steps before are done: s_ready came behind them
#pragma unroll 1
                    for (int k = 0; k < D / 32; k++) {
                        float o[32];
                        tc_ld32(o, o_at + 32 * k);
                        tc_wait_ld();
#pragma unroll
                        for (int c = 0; c < 32; c++) o[c] *= keep;
                        tc_st32(o_at + 32 * k, o);
                    }
            }
            // P lies over the first half of S: a chunk of 32 logits is read before the chunk of 16 columns over it is written
            const f32x2 factor2 = pack2(factor, factor), ref2 = pack2(-ref, -ref);
#pragma unroll 1
            for (int k = 0; k < 4; k++) {
                float x[32];
                tc_ld32(x, s_at + 32 * k);
                tc_wait_ld();
                if (!plain) mask_chunk(x, seen(32 * k, a, b, s, absent, k), factor);
                uint32_t w[16];
#pragma unroll
                for (int c = 0; c < 16; c++) {
                    float u, v;
                    unpack2(fma2(pack2(x[2 * c], x[2 * c + 1]), factor2, ref2), u, v);
                    u = fast_exp2(u);
                    v = fast_exp2(v);
                    sum2 = add2(sum2, pack2(u, v));
                    w[c] = kPool ? bf162_bits(u, v) : half2_bits(u, v);
                }
                tc_st16(s_at + 16 * k, w);
            }
            tc_wait_st();
            tc_before();
            mbar_arrive(&bars.p_ready[i]);
        }
        if (n > 0 && !wait_warp(&bars.o_ready[i], 0)) return;
        tc_after();
        float sum, sum_odd;
        unpack2(sum2, sum, sum_odd);
        sum += sum_odd;
        if (broken && sum != 0.0f) sum = __uint_as_float(0x7FC00000u);
        const bool lost = *reinterpret_cast<volatile int32_t*>(&bars.lost) != 0;
        const float inv = pl.splits > 1 ? 1.0f : (sum != 0.0f ? 1.0f / sum : 0.0f);
        const long long vec = (long long)row * p.Hq + hq;
        float* part = pl.partial + ((long long)split * p.b.n_rows * p.Hq + vec) * D;
        uint16_t* out = p.out + (long long)row * p.out_stride_row + (long long)hq * p.out_stride_head;
#pragma unroll 1
        for (int k = 0; k < D / 32; k++) {
            float o[32];
            if (n > 0) {
                tc_ld32(o, o_at + 32 * k);
                tc_wait_ld();
            } else {
#pragma unroll
                for (int c = 0; c < 32; c++) o[c] = 0.0f;
            }
            if (lost && live) {
                float fixed[32];
#pragma unroll
                for (int c = 0; c < 32; c++) fixed[c] = o[c];
                add_lost<VF, D>(p, {range, seq, head, kv, lo, hi, begin, end}, fixed, 32 * k, pos);
#pragma unroll
                for (int c = 0; c < 32; c++) o[c] = fixed[c];
            }
            if (!live) continue;
#pragma unroll
            for (int c = 0; c < 32; c += 8) {
                float y[8];
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    const int from = VF == FMT_INT4 ? (e < 4 ? 2 * e : 2 * (e - 4) + 1) : e;       // channel e of eight stands there
                    y[e] = o[c + from] * inv;
                }
                if (pl.splits > 1) {
                    float4* d = reinterpret_cast<float4*>(part + 32 * k + c);
                    d[0] = make_float4(y[0], y[1], y[2], y[3]);
                    d[1] = make_float4(y[4], y[5], y[6], y[7]);
                } else {
                    uint4 z;
                    if (p.f16) z = make_uint4(half2_bits(y[0], y[1]), half2_bits(y[2], y[3]), half2_bits(y[4], y[5]), half2_bits(y[6], y[7]));
                    else z = make_uint4(bf162_bits(y[0], y[1]), bf162_bits(y[2], y[3]), bf162_bits(y[4], y[5]), bf162_bits(y[6], y[7]));
                    *reinterpret_cast<uint4*>(out + 32 * k + c) = z;
                }
            }
        }
        if (live && pl.splits > 1) {
            float* ml = pl.partial + (long long)pl.splits * p.b.n_rows * p.Hq * D + ((long long)split * p.b.n_rows * p.Hq + vec) * 2;
            *reinterpret_cast<float2*>(ml) = make_float2(ref, sum);
        }
    }
};

template <int KF, int VF, int D>
__global__ void __launch_bounds__(kRowsThreads, 1) attention_rows_kernel(const __grid_constant__ AttentionParams p, const __grid_constant__ RowsPlan pl) {
    using K = RowsKernel<KF, VF, D>;
    using S = RowsSmem<D>;
    extern __shared__ uint8_t raw[];
    const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u;
    RowsBars& bars = *reinterpret_cast<RowsBars*>(raw + (base - smem_u32(raw)) + S::kBars);
    pdl_trigger();
    const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x >> 5, 0);
    if (threadIdx.x == 0) {
        for (int i = 0; i < 2; i++) {
            mbar_init(&bars.q_ready[i], kRowTile); mbar_init(&bars.p_ready[i], kRowTile);
            mbar_init(&bars.s_ready[i], 1); mbar_init(&bars.o_ready[i], 1);
            mbar_init(&bars.k_full[i], 128); mbar_init(&bars.v_full[i], 128);
            mbar_init(&bars.k_empty[i], 1); mbar_init(&bars.v_empty[i], 1);
        }
        mbar_init(&bars.drained, 1);
        bars.abort = 0; bars.lost = 0;
        bars.lo = 0x7FFFFFFF; bars.hi = -1;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    pdl_wait();
    // Block order: the last rows (the most tokens) of all heads first.
    int id = blockIdx.x;
    const int split = id % pl.splits; id /= pl.splits;
    const int head = id % p.c.H; id /= p.c.H;
    const int seq = id % p.b.n_seqs, tile = pl.tiles - 1 - id / p.b.n_seqs;
    int first, kv, rows;
    const bool ordered = sequence_rows(p, seq, &first, &kv, &rows);
    if (threadIdx.x == 0 && (!ordered || rows > p.b.max_rows || (rows > 0 && __ldg(p.b.kv_len + seq) > kv))) latch(p.status);
    if (!ordered) return;
    rows = min(rows, p.b.max_rows);
    const int m0 = tile * 2 * kRowTile, m_end = min(rows * p.share, m0 + 2 * kRowTile);
    if (m0 >= m_end) return;
    __syncthreads();
    // positions of the CTA's rows
    for (int r = m0 / p.share + threadIdx.x; r <= (m_end - 1) / p.share; r += kRowsThreads) {
        const int x = row_position(p.b, seq, first + r);
        atomicMin(&bars.lo, max(-1, x));
        atomicMax(&bars.hi, x);
    }
    if (warp == kIssuer / 32) tc_alloc(&bars.tmem, 512);
    tc_before();
    __syncthreads();
    tc_after();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(&bars.tmem);
    K k(p, bars);
    k.smem = base; k.seq = seq; k.head = head; k.kv = kv;
    k.lo = bars.lo; k.hi = bars.hi;
    k.range = step_range(p, kv, k.lo, k.hi);
    k.begin = (int)((long long)k.range.count * split / pl.splits);
    k.end = (int)((long long)k.range.count * (split + 1) / pl.splits);
    const int tiles = m_end - m0 > kRowTile ? 2 : 1;
    if (warp < kProducer0 / 32) {
        const int i = warp >> 2;
        if (i < tiles) k.softmax(i, first, m0 + threadIdx.x, m_end, tmem, pl, split);
    } else if (warp < kIssuer / 32) {
        k.produce();
        cp_wait<0>();
    } else if ((threadIdx.x & 31) == 0 && k.end > k.begin) {
        k.issue(tiles, tmem);
        if (bars.abort) {                                       // what was issued must have ended before TMEM goes
            tc_commit(&bars.drained);
            for (uint32_t i = 0; i < kWaitLimit && !mbar_try_wait(&bars.drained, 0); i++) __nanosleep(40);
        }
    }
    __syncwarp();
    tc_before();
    __syncthreads();
    tc_after();
    if (warp == kIssuer / 32) tc_free(tmem, 512);
    if (threadIdx.x == 0 && bars.abort) atomicCAS(p.status, 0, (int)PATCHKV_E_TIMEOUT);
}

// Joins the pieces of split rows: a warp per query vector.
template <int D>
__global__ void __launch_bounds__(128) attention_rows_join_kernel(const AttentionParams p, const RowsPlan pl) {
    pdl_wait();
    const long long n = (long long)p.b.n_rows * p.Hq, vec = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
    const int lane = threadIdx.x & 31;
    if (vec >= n) return;
    const int row = (int)(vec / p.Hq), hq = (int)(vec - (long long)row * p.Hq);
    const int s = find_sequence(p.b, row);
    int first, kv, rows;
    if (s < 0 || !sequence_rows(p, s, &first, &kv, &rows) || row - first >= p.b.max_rows) return;
    const float* ml = pl.partial + pl.splits * n * D;
    float top = kNoMax, sum = 0.0f, y[D / 32];
    for (int i = 0; i < pl.splits; i++) top = fmaxf(top, __ldg(ml + (i * n + vec) * 2));
#pragma unroll
    for (int k = 0; k < D / 32; k++) y[k] = 0.0f;
#pragma unroll 4
    for (int i = 0; i < pl.splits; i++) {
        const float2 x = __ldg(reinterpret_cast<const float2*>(ml + (i * n + vec) * 2));
        const float f = fast_exp2(x.x - top);
        sum = fmaf(f, x.y, sum);
#pragma unroll
        for (int k = 0; k < D / 32; k++) y[k] = fmaf(f, __ldg(pl.partial + (i * n + vec) * D + lane + 32 * k), y[k]);
    }
    uint16_t* o = p.out + (long long)row * p.out_stride_row + (long long)hq * p.out_stride_head;
#pragma unroll
    for (int k = 0; k < D / 32; k++) {
        const float v = sum != 0.0f ? y[k] / sum : 0.0f;
        o[lane + 32 * k] = (uint16_t)(p.f16 ? half2_bits(v, 0.0f) : bf162_bits(v, 0.0f));
    }
}

}  // namespace patchkv
