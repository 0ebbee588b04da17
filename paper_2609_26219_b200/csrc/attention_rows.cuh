// Attention of many query rows on the 5th-generation tensor cores.
//
// A CTA takes one KV head and up to 256 query vectors of it (128 per tile, 1 or 2 tiles): query head and row are packed one behind
// the other, vector m = row * share + head, so that no row of the tiles is left empty whatever share is.  It walks the
// tokens in tiles of 128:
//   S = Q K^T    tcgen05.mma, 128 x 128 x D, both operands in shared memory, S in TMEM
//   P = 2^(S - ref)   a thread per row; P goes back to TMEM as 16-bit numbers over its S
//   O += P V     tcgen05.mma, 128 x D x 128, P from TMEM, V from shared memory, O in TMEM
// Roles: a warpgroup per tile for the softmax, one warp that issues the products, the warps that bring K and V.  The two tiles
// take turns: while one is in its softmax the tensor cores work for the other.  A step's products take 2050 cycles and its
// exponentials as long; what a step takes is the chain of one tile, softmax - P V - Q K^T, and most of the work went into the first.
// The codes have to become operands on the way: fp16(code * scale), one rounding of 2^-12.  Where several CTAs need the same tokens
// (two tiles of CTAs or more) a first kernel does that once per token and leaves images of the two shared-memory matrices of
// each step in the workspace, which a CTA then fetches with one bulk copy each; converting in every CTA kept four warps busy for
// 6000 cycles a step, three times what the products take.  Where one CTA is all there is, its own four warps convert (bf16
// pages: cp.async), and the cache is read once, as it is.  Queries over quantised pages are fp16 scaled by a power of two per
// row, so a bf16 query loses nothing.  The weights are fp16 there, bf16 over bf16 pages; sums are fp32 throughout.
// fp16 queries (FINE) get K as the sum of two fp16 matrices, 22 bits, for one more product per 16 channels: one matrix alone
// rounds code * scale to 11 bits, which in channels far larger than the others was most of an fp16 result's error.
// As in the split kernel the softmax reference is only moved (and O rescaled) when a logit exceeds it by more than 15.
#pragma once

#include <stddef.h>

#include "attention_split.cuh"

namespace patchkv {

constexpr int kRowTile = 128;                   // query vectors of a tile, and tokens of a step
constexpr float kTop = kSplitTop, kPeak = kSplitPeak;
constexpr int kProducer0 = 256;                 // two softmax warpgroups, then the warps that bring K and V (four, or one that copies
__host__ __device__ constexpr int rows_issuer(bool image) { return image ? 288 : 384; }             // images), then the issuing warp
__host__ __device__ constexpr int rows_threads(bool image) { return rows_issuer(image) + 32; }

struct RowsPlan {
    float* partial;                             // [split][n_rows * Hq][D], then (m, l) [split][n_rows * Hq]
    int32_t tiles;                              // CTAs along the query vectors of a sequence
    int32_t splits;                             // pieces of the token range (1: no partial results)
    uint8_t* images;                            // [sequence][step][KV head]: K matrix (FINE: and what it leaves of K), V matrix; null: no images
    uint32_t* meta;                             // of each image: 4 words of absent tokens, 1 word `lost`, 3 unused
    int32_t steps;                              // of a sequence in the two
};
// The image, row and join kernels of a call for head dimension D, 64 or 128 (attention_rows_launch.cuh).
template <int D>
cudaError_t launch_rows(const AttentionParams& p, const RowsPlan& pl, cudaStream_t s);
__device__ __forceinline__ long long image_index(const AttentionParams& p, const RowsPlan& pl, int seq, int step, int head) {
    return ((long long)seq * pl.steps + step) * p.c.H + head;
}

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
__device__ __forceinline__ void tc_ld16(uint32_t (&r)[16], uint32_t addr) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
          "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void tc_st64(uint32_t addr, const uint32_t (&r)[64]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x64.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,"
        "%25,%26,%27,%28,%29,%30,%31,%32,%33,%34,%35,%36,%37,%38,%39,%40,%41,%42,%43,%44,%45,%46,%47,%48,"
        "%49,%50,%51,%52,%53,%54,%55,%56,%57,%58,%59,%60,%61,%62,%63,%64};" ::"r"(addr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]),
        "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]),
        "r"(r[31]), "r"(r[32]), "r"(r[33]), "r"(r[34]), "r"(r[35]), "r"(r[36]), "r"(r[37]), "r"(r[38]), "r"(r[39]), "r"(r[40]),
        "r"(r[41]), "r"(r[42]), "r"(r[43]), "r"(r[44]), "r"(r[45]), "r"(r[46]), "r"(r[47]), "r"(r[48]), "r"(r[49]), "r"(r[50]),
        "r"(r[51]), "r"(r[52]), "r"(r[53]), "r"(r[54]), "r"(r[55]), "r"(r[56]), "r"(r[57]), "r"(r[58]), "r"(r[59]), "r"(r[60]),
        "r"(r[61]), "r"(r[62]), "r"(r[63]) : "memory");
}
// One lane of the warp, always the same one.
__device__ __forceinline__ bool elect_lane() {
    uint32_t yes;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(yes));
    return yes != 0;
}
__device__ __forceinline__ void tc_st16(uint32_t addr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(addr), "r"(r[0]), "r"(r[1]),
        "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]),
        "r"(r[14]), "r"(r[15]) : "memory");
}
__device__ __forceinline__ void bulk_g2s_at(uint32_t dst, const void* src, uint32_t bytes, uint64_t* bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(smem_u32(bar)) : "memory");
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
    alignas(16) uint32_t absent[4][8];          // per step (mod 4): tokens whose page is out of range; word 4: `lost` of an image
    uint32_t tmem;
    int32_t first_row, last_row;                // the CTA's rows
    int32_t abort, lo, hi, least, lost;         // smallest and largest position not below 0; smallest of all; a value that is not finite
                                                // was taken out of a tile that needs a mask
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
// The same and what the rounding took away: code * scale = hi + lo but for bits below 2^-24.  Where 128 * scale may pass fp16's
// range, scales of 512 and more, lo is zero: an infinite hi keeps its sign, and infinity - infinity is never formed.
__device__ __forceinline__ uint32_t rest_mask(uint32_t s) { return (s & 0x7FFFu) < 0x6000u ? 0xFFFFFFFFu : 0u; }
__device__ __forceinline__ uint32_t rest(uint32_t code, uint32_t s, uint32_t hi, uint32_t keep) { return hfma2(code, s, hi ^ 0x80008000u) & keep; }
__device__ __forceinline__ uint32_t hsub2(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __forceinline__ void operands4(uint32_t w, uint32_t s, uint32_t m0, uint32_t m1, uint4& hi, uint4& lo) {
    const uint32_t v = w >> 8;
    const uint32_t a = hsub2(and_xor<0x000F000Fu>(w, m0), 0x64086408u), b = hfma2(and_xor<0x00F000F0u>(w, m1), 0x2C002C00u, 0xD480D480u);
    const uint32_t c = hsub2(and_xor<0x000F000Fu>(v, m0), 0x64086408u), d = hfma2(and_xor<0x00F000F0u>(v, m1), 0x2C002C00u, 0xD480D480u);
    const uint32_t keep = rest_mask(s);
    hi = make_uint4(hmul2(a, s), hmul2(b, s), hmul2(c, s), hmul2(d, s));
    lo = make_uint4(rest(a, s, hi.x, keep), rest(b, s, hi.y, keep), rest(c, s, hi.z, keep), rest(d, s, hi.w, keep));
}
__device__ __forceinline__ void operands8(uint32_t w, uint32_t s, uint2& hi, uint2& lo) {
    const uint32_t u = w ^ 0x80808080u;
    const uint32_t a = hsub2(__byte_perm(u, 0x64646464u, 0x4140), 0x64806480u), b = hsub2(__byte_perm(u, 0x64646464u, 0x4342), 0x64806480u);
    const uint32_t keep = rest_mask(s);
    hi = make_uint2(hmul2(a, s), hmul2(b, s));
    lo = make_uint2(rest(a, s, hi.x, keep), rest(b, s, hi.y, keep));
}
// Four fp16 operands of a word of 8-bit codes, in order: 1024 + u, minus 1152, times the scale.
__device__ __forceinline__ uint2 operands8(uint32_t w, uint32_t s) {
    const uint32_t u = w ^ 0x80808080u;
    uint2 o;
    asm("{\n\t.reg .b32 a;\n\tsub.rn.f16x2 a, %1, %2;\n\tmul.rn.f16x2 %0, a, %3;\n\t}" : "=r"(o.x) : "r"(__byte_perm(u, 0x64646464u, 0x4140)), "r"(0x64806480u), "r"(s));
    asm("{\n\t.reg .b32 a;\n\tsub.rn.f16x2 a, %1, %2;\n\tmul.rn.f16x2 %0, a, %3;\n\t}" : "=r"(o.y) : "r"(__byte_perm(u, 0x64646464u, 0x4342)), "r"(0x64806480u), "r"(s));
    return o;
}

// Sets fp16 (EXP 0x7C00) or bf16 (0x7F80) numbers that are not finite to zero; true when there was one.
template <uint32_t EXP>
__device__ __forceinline__ bool finite_only(uint4& x) {
    bool found = false;
    uint32_t* w = &x.x;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        if ((w[i] & EXP) == EXP) { w[i] &= 0xFFFF0000u; found = true; }
        if ((w[i] >> 16 & EXP) == EXP) { w[i] &= 0x0000FFFFu; found = true; }
    }
    return found;
}
// 32 channels of a token (piece c of its row) as fp16 in channel order.
template <int F>
__device__ __forceinline__ void image_operands(uint4 (&o)[4], const uint8_t* row, int c, uint32_t s, uint32_t m0, uint32_t m1) {
    const uint4 a = *reinterpret_cast<const uint4*>(row + c * (F == FMT_INT8 ? 32 : 16));
    if (F == FMT_INT8) {
        const uint4 b = *reinterpret_cast<const uint4*>(row + c * 32 + 16);
        const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const uint2 x = operands8(w[2 * i], s), y = operands8(w[2 * i + 1], s);
            o[i] = make_uint4(x.x, x.y, y.x, y.y);
        }
    } else {
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int i = 0; i < 4; i++) {                           // 0 4, 1 5, 2 6, 3 7 -> 0 1, 2 3, 4 5, 6 7
            const uint4 x = operands4(w[i], s, m0, m1);
            o[i] = make_uint4(__byte_perm(x.x, x.y, 0x5410), __byte_perm(x.z, x.w, 0x5410), __byte_perm(x.x, x.y, 0x7632), __byte_perm(x.z, x.w, 0x7632));
        }
    }
}
// K of an image: also what the rounding took away.
template <int F>
__device__ __forceinline__ void image_operands(uint4 (&hi)[4], uint4 (&lo)[4], const uint8_t* row, int c, uint32_t s, uint32_t m0, uint32_t m1) {
    const uint4 a = *reinterpret_cast<const uint4*>(row + c * (F == FMT_INT8 ? 32 : 16));
    auto ordered = [](const uint4& x) {                         // 0 4, 1 5, 2 6, 3 7 -> 0 1, 2 3, 4 5, 6 7
        return make_uint4(__byte_perm(x.x, x.y, 0x5410), __byte_perm(x.z, x.w, 0x5410), __byte_perm(x.x, x.y, 0x7632), __byte_perm(x.z, x.w, 0x7632));
    };
    if (F == FMT_INT8) {
        const uint4 b = *reinterpret_cast<const uint4*>(row + c * 32 + 16);
        const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int i = 0; i < 4; i++) {
            uint2 x, y, p, q;
            operands8(w[2 * i], s, x, p);
            operands8(w[2 * i + 1], s, y, q);
            hi[i] = make_uint4(x.x, x.y, y.x, y.y);
            lo[i] = make_uint4(p.x, p.y, q.x, q.y);
        }
    } else {
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int i = 0; i < 4; i++) {
            uint4 x, y;
            operands4(w[i], s, m0, m1, x, y);
            hi[i] = ordered(x);
            lo[i] = ordered(y);
        }
    }
}
// Whether one of the rows at given positions sees token t (they may lie further apart than the window).  Asked only of tokens
// between the rows' positions that have no page.
inline __device__ __noinline__ bool some_row_sees(const AttentionParams& p, int first, int last, int t) {
    for (int r = first; r <= last; r++) {
        const int x = p.b.pos[r];
        if (x >= t && sees(p, x, t)) return true;
    }
    return false;
}
struct StepPlace { TileRange range; int seq, head, kv, last, hi, begin, end; bool order4; };
// A step that every row sees whole: up to token `last`, which is the earliest row's position or the cache's end.
__device__ __forceinline__ bool whole_step(const AttentionParams& p, int last, int hi, int t0) {
    return t0 + kRowTile - 1 <= last && (p.window == 0 || hi - t0 < p.window || t0 + kRowTile <= p.sinks);
}
// Values that are not finite were taken out of the masked steps (of an image: of all); a row that sees such a value gets it here.
// (Rare: element by element, from the pages.)
inline __device__ __noinline__ void add_lost(const AttentionParams& p, const RowsPlan& pl, const StepPlace& at, float (&o)[32], int c0, int pos) {
    const int vf = v_format(p.c.tag), D = p.c.D;
    for (int j = at.begin; j < at.end; j++) {
        const int step = at.range.tile(j), t0 = step * kRowTile;
        if (pl.images ? pl.meta[image_index(p, pl, at.seq, step, at.head) * 8 + 4] == 0 : whole_step(p, at.last, at.hi, t0)) continue;
        for (int t = t0; t < t0 + kRowTile; t++) {
            if (t > min(pos, at.kv - 1) || !sees(p, pos, t)) continue;
            const int lp = div_page(p.c, t), slot = t - lp * p.c.P;
            const int page = p.b.block_table[(long long)at.seq * p.b.table_stride + lp];
            if (page < 0 || page >= p.c.n_pages) continue;
            for (int c = 0; c < 32; c++) {
                float v;
                // column c of the accumulator is channel `ch`
                const int e = c & 7, ch = c0 + (at.order4 ? (c & ~7) + (e & 1 ? 4 + (e >> 1) : e >> 1) : c);
                if (vf == FMT_BF16) {
                    v = bf16_bits_to_float(p.c.v[(long long)page * p.c.stride_page + (long long)slot * p.c.stride_token + (long long)at.head * p.c.stride_head + ch]);
                } else {
                    const uint8_t* pg = p.c.base + (long long)page * p.c.stride_page;
                    const unsigned long long el = ((unsigned long long)slot * p.c.H + at.head) * D + ch;
                    v = (float)code_at(pg + p.c.v_codes, vf, el) * scale_at(pg + p.c.v_scales, el / p.c.G);
                    v = __half2float(__float2half_rn(v));   // as the operand was: beyond 65504 an infinity
                }
                if (!(fabsf(v) <= 3.4e38f)) o[c] += v;
            }
        }
    }
}

// KF / VF: page formats (both FMT_BF16 for the bf16 pool).  IMAGE: operands come as images, in channel order (KF = VF = FMT_INT8
// stands for fp16 images, FMT_BF16 for bf16).
template <int KF, int VF, int D, bool IMAGE, bool FINE>
struct RowsKernel {
    static constexpr bool kPool = KF == FMT_BF16;
    using S = RowsSmem<D>;
    static constexpr int kPer = D / 32;                         // 32-channel pieces (= threads) of a token's row
    // K's ring: two stages, or one of two matrices (the next K has the whole softmax of a step to arrive).
    __device__ __forceinline__ static int k_stage(int n) { return FINE ? 0 : n & 1; }
    __device__ __forceinline__ static uint32_t k_turn(int n) { return (FINE ? n : n >> 1) & 1; }

    const AttentionParams& p;
    RowsBars& bars;
    uint32_t smem;
    int seq, head, kv, last, hi, begin, end;                    // steps [begin, end) of the range
    TileRange range;

    __device__ __forceinline__ RowsKernel(const AttentionParams& p_, RowsBars& b) : p(p_), bars(b) {}
    __device__ __forceinline__ bool wait(uint64_t* bar, uint32_t parity) { return mbar_wait(bar, parity, &bars.abort); }
    // The same for a whole warp: all of its lanes go on, or none.
    __device__ __forceinline__ bool wait_warp(uint64_t* bar, uint32_t parity) { return __all_sync(0xFFFFFFFFu, wait(bar, parity)); }
    // Seen by some row (or by none): only then does a token's slot take part.
    __device__ __forceinline__ bool any_sees(int t) const { return t <= min(hi, kv - 1) && sees(p, bars.lo, t); }
    // The same exactly, for what counts as an error.
    __device__ __forceinline__ bool really_seen(int t) const {
        return any_sees(t) && (!p.b.pos || p.window == 0 || some_row_sees(p, bars.first_row, bars.last_row, t));
    }
    __device__ __forceinline__ bool whole(int t0) const { return whole_step(p, last, hi, t0); }

    // ---- the warps that bring K and V
    // A warp takes TOK = 32 tokens of a step, or 16 where a call has one tile only and the second tile's softmax warps bring too; kPer lanes share a
    // token, 32 / kPer tokens at a time (a pass).
    static constexpr int kTok = 32 / kPer;
    struct Pages { int page, t0; };                             // lane 0: page of the warp's first 16 tokens, lane 1: of the other 16

    // Address of the thread's token of pass i (quantised: its page, and its row in *row); live: some row sees it and it has a page.
    template <int TOK>
    __device__ __forceinline__ long long token_at(const Pages& g, int tok, uint32_t* row, bool* live) const {
        const int t = g.t0 + tok;
        const int page = __shfl_sync(0xFFFFFFFFu, g.page, TOK == 16 ? 0 : tok >> 4 & 1);
        const int slot = t - div_page(p.c, t) * p.c.P;
        *live = page >= 0 && any_sees(t);
        *row = (uint32_t)slot * p.c.H + head;
        if (!*live) return 0;
        return (long long)page * p.c.stride_page + (kPool ? (long long)slot * p.c.stride_token + (long long)head * p.c.stride_head : 0ll);
    }
    // Tokens of the warp that some row sees but whose page is out of range.
    template <int TOK>
    __device__ __forceinline__ uint32_t missing(const Pages& g, int w) const {
        const int lane = threadIdx.x & 31, page = __shfl_sync(0xFFFFFFFFu, g.page, lane >> 4);
        const uint32_t gone = __ballot_sync(0xFFFFFFFFu, lane < TOK && page < 0 && any_sees(g.t0 + TOK * w + lane));
        if (gone >> lane & 1u && really_seen(g.t0 + TOK * w + lane)) latch(p.status);
        return gone;
    }
    // The thread's 32 channels of pass i, K or V: codes and their scale.
    template <int F, int TOK>
    __device__ __forceinline__ void load_piece(const Pages& g, int tok, int c, bool is_v, uint32_t (&w)[8], uint32_t& scale) const {
        uint32_t row;
        bool live;
        const uint8_t* pg = p.c.base + token_at<TOK>(g, tok, &row, &live);
#pragma unroll
        for (int i = 0; i < 8; i++) w[i] = 0;
        scale = 0;
        if (!live) return;
        const uint8_t* codes = pg + (is_v ? p.c.v_codes : 0u) + row * (F == FMT_INT8 ? D : D / 2) + c * (F == FMT_INT8 ? 32 : 16);
        const uint4 a = *reinterpret_cast<const uint4*>(codes);
        w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
        if (F == FMT_INT8) {
            const uint4 b = *reinterpret_cast<const uint4*>(codes + 16);
            w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
        }
        const uint32_t s = (row * (D / p.c.G) + c * 32 / p.c.G) * 2 + (is_v ? p.c.v_scales : p.c.k_scales);
        scale = *reinterpret_cast<const uint16_t*>(pg + s);
    }

    // Images: one lane copies.  Returns with the copies in flight counted in `sent` (bit 2 st + (0 for K, 1 for V): a copy into stage st
    // has been issued), so that after an abort they can be waited for.
    __device__ __forceinline__ void fetch_images(const RowsPlan& pl) {
        int j = begin;
        uint32_t k_uses = 0, v_uses = 0;                        // copies issued
        for (; j < end; j++) {
            const int n = j - begin, st = n & 1;
            const uint32_t parity = ((n >> 1) & 1) ^ 1;
            constexpr uint32_t kBytes = (FINE ? 2 : 1) * S::kMat;
            const long long at = image_index(p, pl, seq, range.tile(j), head);
            const uint8_t* image = pl.images + at * (kBytes + S::kMat);
            uint64_t* full = &bars.k_full[k_stage(n)];
            if (!wait_warp(&bars.k_empty[k_stage(n)], k_turn(n) ^ 1)) break;
            if (elect_lane()) {
                mbar_arrive_expect_tx(full, kBytes + 32);
                bulk_g2s_at(smem + S::kK + k_stage(n) * S::kMat, image, kBytes, full);
                bulk_g2s_at(smem_u32(bars.absent[n & 3]), pl.meta + at * 8, 32, full);
            }
            __syncwarp();
            k_uses++;
            if (!wait_warp(&bars.v_empty[st], parity)) break;
            if (elect_lane()) {
                mbar_arrive_expect_tx(&bars.v_full[st], S::kMat);
                bulk_g2s_at(smem + S::kV + st * S::kMat, image + kBytes, S::kMat, &bars.v_full[st]);
            }
            __syncwarp();
            v_uses++;
        }
        // The last copies (after an abort they may have no reader) must have landed before the CTA goes.
        for (int back = 1; back <= 2; back++) {
            const uint32_t k = k_uses - back, v = v_uses - back;
            for (uint32_t i = 0; k_uses >= (uint32_t)back && (!FINE || back == 1) && i < kWaitLimit && !mbar_try_wait(&bars.k_full[k_stage((int)k)], k_turn((int)k)); i++) __nanosleep(40);
            for (uint32_t i = 0; v_uses >= (uint32_t)back && i < kWaitLimit && !mbar_try_wait(&bars.v_full[v & 1], (v >> 1) & 1); i++) __nanosleep(40);
        }
    }

    template <int TOK>
    __device__ __forceinline__ void produce(int w) {
        constexpr int kPass = TOK / kTok;
        const int lane = threadIdx.x & 31;
        const int c = lane % kPer, tok0 = TOK * w + lane / kPer;
        uint32_t m0, m1;                                        // 1024 + 8 and 1024 + 8 * 16 in every half: magic and offset
        asm volatile("mov.b32 %0, 0x64086408;" : "=r"(m0));
        asm volatile("mov.b32 %0, 0x64806480;" : "=r"(m1));
        if (begin >= end) return;
        auto pages_of = [&](int j) { return Pages{page_of(j, TOK * w + (TOK == 32 ? (lane & 1) * 16 : 0)), j < end ? range.tile(j) * kRowTile : 0}; };
        Pages now = pages_of(begin), next = pages_of(begin + 1);
        // One set of registers for the codes in flight: as soon as K's have become operands V's are asked for, then the next K's.
        uint32_t code[kPass][8], scale[kPass];
        if constexpr (!kPool)
#pragma unroll
            for (int i = 0; i < kPass; i++) load_piece<KF, TOK>(now, tok0 + i * kTok, c, false, code[i], scale[i]);
#pragma unroll 1
        for (int j = begin; j < end; j++) {
            const int n = j - begin, st = n & 1;
            const uint32_t parity = ((n >> 1) & 1) ^ 1;
            const bool masked = !whole(now.t0);
            const uint32_t gone = missing<TOK>(now, w);
            if (lane == 0) {
                if (TOK == 32) bars.absent[n & 3][w] = gone;
                else reinterpret_cast<uint16_t*>(bars.absent[n & 3])[w] = (uint16_t)gone;
            }
            const uint32_t kb = smem + S::kK + k_stage(n) * S::kMat, vb = smem + S::kV + st * S::kMat;
            uint64_t* k_full = &bars.k_full[k_stage(n)];
            if (!wait_warp(&bars.k_empty[k_stage(n)], k_turn(n) ^ 1)) return;
            if constexpr (kPool) {
                // chunks kPer apart: a row's lanes read a contiguous run
                auto copy = [&](const uint16_t* from, uint32_t mat) {
#pragma unroll
                    for (int i = 0; i < kPass; i++) {
                        uint32_t row;
                        bool live;
                        const uint16_t* x = from + token_at<TOK>(now, tok0 + i * kTok, &row, &live) + 8 * c;
#pragma unroll
                        for (int q = 0; q < 4; q++) cp16(mat + swizzled(tok0 + i * kTok, q * kPer + c), live ? x + 8 * q * kPer : from, live);
                    }
                    cp_commit();
                };
                copy(p.c.k, kb);
                if (!wait_warp(&bars.v_empty[st], parity)) return;
                copy(p.c.v, vb);
                cp_wait<1>();
                fence_async_smem();
                mbar_arrive(k_full);
                cp_wait<0>();
                if (masked) clean<0x7F80u, kPass>(vb, tok0, c, 1, kPer);
            } else {
#pragma unroll
                for (int i = 0; i < kPass; i++) {
                    store_operands<KF, FINE>(kb, tok0 + i * kTok, c, code[i], scale[i], m0, m1);
                    load_piece<VF, TOK>(now, tok0 + i * kTok, c, true, code[i], scale[i]);
                }
                fence_async_smem();
                mbar_arrive(k_full);
                if (!wait_warp(&bars.v_empty[st], parity)) return;
#pragma unroll
                for (int i = 0; i < kPass; i++) {
                    store_operands<VF, false>(vb, tok0 + i * kTok, c, code[i], scale[i], m0, m1);
                    load_piece<KF, TOK>(next, tok0 + i * kTok, c, false, code[i], scale[i]);
                }
                if (masked) clean<0x7C00u, kPass>(vb, tok0, c, 4, 1);
            }
            fence_async_smem();
            mbar_arrive(&bars.v_full[st]);
            now = next;
            next = pages_of(j + 2);
        }
    }
    // Page of token `tok` of step j; -1 when it is out of range or lies behind the cache.
    __device__ __forceinline__ int page_of(int j, int tok) const {
        if (j >= end) return -1;
        const int t = range.tile(j) * kRowTile + tok;
        if (t >= kv) return -1;
        const int pg = p.b.block_table[(long long)seq * p.b.table_stride + div_page(p.c, t)];
        return pg >= 0 && pg < p.c.n_pages ? pg : -1;
    }
    // In a step that needs a mask a value that is not finite must not meet the weight 0 of a row that does not see it: it is taken out
    // here and given to the rows that see it at the end.  Chunks of the thread: c * lead + q * apart, q = 0 .. 3.
    template <uint32_t EXP, int PASSES>
    __device__ __forceinline__ void clean(uint32_t mat, int tok0, int c, int lead, int apart) {
#pragma unroll 1
        for (int i = 0; i < PASSES * 4; i++) {
            const uint32_t a = mat + swizzled(tok0 + (i >> 2) * (32 / kPer), c * lead + (i & 3) * apart);
            uint4 x = lds128(a);
            if (finite_only<EXP>(x)) { sts128(a, x.x, x.y, x.z, x.w); bars.lost = 1; }
        }
    }
    // The 32 channels of a thread into its token's row.
    template <int F, bool REST>
    __device__ __forceinline__ void store_operands(uint32_t mat, int tok, int c, const uint32_t (&w)[8], uint32_t scale, uint32_t m0, uint32_t m1) {
        const uint32_t s = scale | scale << 16;
        const uint32_t flip = c & 2;                            // the two halves of the channels write different banks
#pragma unroll
        for (int i = 0; i < 4; i++) {
            uint4 o, lo;
            if constexpr (F == FMT_INT4) {
                const uint32_t x = flip ? w[i ^ 2] : w[i];
                if (REST) operands4(x, s, m0, m1, o, lo); else o = operands4(x, s, m0, m1);
            } else {
                const uint32_t x = flip ? w[(2 * i) ^ 4] : w[2 * i], y = flip ? w[(2 * i + 1) ^ 4] : w[2 * i + 1];
                uint2 a, b, c2, d2;
                if (REST) { operands8(x, s, a, c2); operands8(y, s, b, d2); lo = make_uint4(c2.x, c2.y, d2.x, d2.y); }
                else { a = operands8(x, s); b = operands8(y, s); }
                o = make_uint4(a.x, a.y, b.x, b.y);
            }
            const uint32_t at = mat + swizzled(tok, 4 * c + (i ^ flip));
            sts128(at, o.x, o.y, o.z, o.w);
            if (REST) sts128(at + S::kMat, lo.x, lo.y, lo.z, lo.w);
        }
    }

    // ---- the warp that issues the products (one lane of it; the whole warp waits, so that all else is known to be uniform)
    __device__ __forceinline__ void issue(int tiles, uint32_t tmem) {
        constexpr uint32_t kQk = instr_desc(kPool, false, kRowTile), kPv = instr_desc(kPool, true, D);
        const uint64_t q_desc = smem_desc(smem + S::kQ, 16), k_desc = smem_desc(smem + S::kK, 16), v_desc = smem_desc(smem + S::kV, kRowTile * 128);
        constexpr uint32_t kMat16 = S::kMat >> 4;
        auto logits = [&](int i, int st, uint64_t* k_free) {
            const uint64_t q = q_desc + i * kMat16, k = k_desc + st * kMat16;
            if (elect_lane()) {
#pragma unroll
                for (int x = 0; x < D / 16; x++) {              // 16 channels: 32 bytes inside a 128-byte row, then the next half
                    const uint32_t o = (x >> 2) * (kRowTile * 8) + (x & 3) * 2;
                    tc_mma_ss(tmem + i * kRowTile, q + o, k + o, kQk, x != 0);
                    if (FINE) tc_mma_ss(tmem + i * kRowTile, q + o, k + o + kMat16, kQk, true);
                }
                tc_commit(&bars.s_ready[i]);
                if (k_free) tc_commit(k_free);
            }
            __syncwarp();
        };
        for (int i = 0; i < tiles; i++) if (!wait_warp(&bars.q_ready[i], 0)) return;
        if (!wait_warp(&bars.k_full[0], 0)) return;
        tc_after();
        for (int i = 0; i < tiles; i++) logits(i, 0, i == tiles - 1 ? &bars.k_empty[0] : nullptr);
        const int n = end - begin;
#pragma unroll 1
        for (int j = 0; j < n; j++) {
            const int st = j & 1;
            if (!wait_warp(&bars.v_full[st], (j >> 1) & 1)) return;
            if (j + 1 < n && !wait_warp(&bars.k_full[k_stage(j + 1)], k_turn(j + 1))) return;
#pragma unroll 1
            for (int i = 0; i < tiles; i++) {
                if (!wait_warp(&bars.p_ready[i], j & 1)) return;
                tc_after();
                const uint64_t v = v_desc + st * kMat16;
                const uint32_t o = tmem + (2 + i) * kRowTile, a = tmem + i * kRowTile;
                if (elect_lane()) {
                    tc_mma_ts(o, a, v, kPv, j != 0);
#pragma unroll
                    for (int x = 1; x < kRowTile / 16; x++)       // 16 tokens: 8 columns of P, two groups of 8 rows of V
                        tc_mma_ts(o, a + 8 * x, v + x * 128, kPv, true);
                    if (i == tiles - 1) tc_commit(&bars.v_empty[st]);
                    if (j + 1 == n) tc_commit(&bars.o_ready[i]);
                }
                __syncwarp();
                if (j + 1 < n) logits(i, k_stage(j + 1), i == tiles - 1 ? &bars.k_empty[k_stage(j + 1)] : nullptr);
            }
        }
    }

    // Tokens on pages out of range count when some row sees them (with images nobody has looked at that yet).
    __device__ __forceinline__ void latch_absent(int t0, const uint4& absent) const {
        const int lane = threadIdx.x & 31;
        const uint32_t gone[4] = {absent.x, absent.y, absent.z, absent.w};
#pragma unroll
        for (int k = 0; k < 4; k++)
            if (gone[k] >> lane & 1u && really_seen(t0 + 32 * k + lane)) latch(p.status);
    }

    // Bit c: this row sees column c0 + c.
    __device__ __forceinline__ static uint32_t seen(int c0, int a, int b, int s, uint32_t gone) {
        auto below = [](int n) { return n <= 0 ? 0u : n >= 32 ? 0xFFFFFFFFu : (1u << n) - 1u; };      // bits [0, n)
        return below(b + 1 - c0) & (~below(a - c0) | below(s - c0)) & ~gone;
    }
    // ---- softmax: a thread per query vector
    // The query into shared memory: cp.async, then (bf16 over quantised pages) in place to fp16, scaled so that the largest magnitude
    // lies in [2^13, 2^14).  A vector with a NaN or an infinity gives NaN.  Returns the factor of its logits.
    __device__ __forceinline__ float load_query(int i, int r, bool live, int row, int hq) {
        const long long mine = (long long)row * p.q_stride_row + (long long)hq * p.q_stride_head;
        const uint32_t mat = smem + S::kQ + i * S::kMat;
        // The warp's 32 rows, a run of D / 8 lanes each: row by row of a thread is 32 cache lines an instruction.
        constexpr int kRun = D / 8;
        const int lane = threadIdx.x & 31;
#pragma unroll 4
        for (int k = 0; k < kRun; k++) {
            const int from = k * (32 / kRun) + lane / kRun;
            const long long at = __shfl_sync(0xFFFFFFFFu, mine, from);
            const bool there = __shfl_sync(0xFFFFFFFFu, (int)live, from) != 0;
            cp16(mat + swizzled((r & ~31) + from, lane % kRun), p.q + at + 8 * (lane % kRun), there);
        }
        cp_commit();
        cp_wait<0>();
        __syncwarp();
        if (kPool) return p.scale_log2;
        // Magnitudes are ordered as their bit patterns.
        uint32_t most = 0;
#pragma unroll 4
        for (int c = 0; c < D / 8; c++) {
            const uint4 v = lds128(mat + swizzled(r, c));
            most = __vmaxu2(__vmaxu2(most, v.x & 0x7FFF7FFFu), __vmaxu2(v.y & 0x7FFF7FFFu, __vmaxu2(v.z & 0x7FFF7FFFu, v.w & 0x7FFF7FFFu)));
        }
        most = max(most & 0xFFFFu, most >> 16);
        const bool bad = most >= (p.f16 ? 0x7C00u : 0x7F80u);
        // fp16 stays as it is
        const int shift = p.f16 || most == 0 ? 0 : min(13 - ((int)(most >> 7) - 127), 120);
        const float up = exp2i(shift);
        if (!p.f16 || KF == FMT_INT4 || __any_sync(0xFFFFFFFFu, bad))
#pragma unroll 2
            for (int c = 0; c < D / 8; c++) {
                uint4 v = lds128(mat + swizzled(r, c));
                if (bad) v = make_uint4(0, 0, 0, 0);
                uint32_t w[4] = {v.x, v.y, v.z, v.w};
                if (!p.f16)
#pragma unroll
                    for (int k = 0; k < 4; k++) w[k] = half2_bits(__uint_as_float(w[k] << 16) * up, __uint_as_float(w[k] & 0xFFFF0000u) * up);
                if (KF == FMT_INT4)                             // the order operands4 leaves the channels in: 0 4, 1 5, 2 6, 3 7
                    sts128(mat + swizzled(r, c), __byte_perm(w[0], w[2], 0x5410), __byte_perm(w[0], w[2], 0x7632), __byte_perm(w[1], w[3], 0x5410), __byte_perm(w[1], w[3], 0x7632));
                else
                    sts128(mat + swizzled(r, c), w[0], w[1], w[2], w[3]);
            }
        return bad ? __uint_as_float(0x7FC00000u) : p.scale_log2 * exp2i(-shift);
    }

    // 2^y for two y on the fma pipe: y = n + f with n whole and |f| <= 1/2, 2^f by a polynomial (fitted for the least relative
    // error on that interval: 2.6e-6), times 2^n put together as bits.  At -127, where all below is put, those bits are +0: a masked
    // logit has the weight 0, as from ex2.  (2^-126 instead is a normal bf16 number, and times a finite 3e38 in a slot that the row
    // does not see it shows.)  Above 126 (a row that has had no token yet: its reference is far below all logits) the result is
    // 2^126, which the check behind finds; NaN stays NaN.
    __device__ __forceinline__ static void exp2_pair(f32x2 y2, float& a, float& b) {
        float u, v;
        unpack2(y2, u, v);
        asm("max.NaN.f32 %0, %0, %1;" : "+f"(u) : "f"(-127.0f));
        asm("max.NaN.f32 %0, %0, %1;" : "+f"(v) : "f"(-127.0f));
        asm("min.NaN.f32 %0, %0, %1;" : "+f"(u) : "f"(126.0f));
        asm("min.NaN.f32 %0, %0, %1;" : "+f"(v) : "f"(126.0f));
        const f32x2 y = pack2(u, v), magic = pack2(12582912.0f, 12582912.0f);       // 1.5 * 2^23
        const f32x2 t = add2(y, magic), f = sub2(y, sub2(t, magic));
        f32x2 e = fma2(f, pack2(0.009570097550749779f, 0.009570097550749779f), pack2(0.05591786280274391f, 0.05591786280274391f));
        e = fma2(e, f, pack2(0.240247443318367f, 0.240247443318367f));
        e = fma2(e, f, pack2(0.6931217908859253f, 0.6931217908859253f));
        e = fma2(e, f, pack2(0.9999992847442627f, 0.9999992847442627f));
        float n0, n1;
        unpack2(t, n0, n1);
        unpack2(mul2(e, pack2(__uint_as_float((__float_as_uint(n0) << 23) + 0x3F800000u), __uint_as_float((__float_as_uint(n1) << 23) + 0x3F800000u))), a, b);
    }

    // 32 logits -> 16 words of weights against the reference; their sum onto `total`.  The exponential unit does 16 a cycle and SM, a
    // step's 32768 would keep it as busy as the products keep the tensor cores: kOnFma of 16 pairs are computed instead.
    static constexpr int kOnFma = 4;
    __device__ __forceinline__ static void weigh(const float (&x)[32], uint32_t* w, f32x2 factor2, f32x2 ref2, f32x2& total) {
#pragma unroll
        for (int c = 0; c < 16; c++) {
            float e, f;
            unpack2(fma2(pack2(x[2 * c], x[2 * c + 1]), factor2, ref2), e, f);
            if (c % 4 < kOnFma / 4) {
                exp2_pair(pack2(e, f), e, f);
            } else {
                e = fast_exp2(e);
                f = fast_exp2(f);
            }
            total = add2(total, pack2(e, f));
            w[c] = kPool ? bf162_bits(e, f) : half2_bits(e, f);
        }
    }

    __device__ __forceinline__ void softmax(int i, int first, int m, int m_end, uint32_t tmem, const RowsPlan& pl, int split) {
        const int r = threadIdx.x & 127;
        const bool live = m < m_end;
        const int row = live ? first + m / p.share : first, hq = live ? head * p.share + m % p.share : 0;
        const int pos = live ? max(-1, row_position(p.b, seq, row)) : -1;
        float factor = load_query(i, r, live, row, hq);
        fence_async_smem();
        __syncwarp();
        if ((threadIdx.x & 31) == 0) mbar_arrive(&bars.q_ready[i]);
        // A mask is minus infinity over the factor: a factor of zero is one that leaves no logit, a NaN enters at the end.
        const bool broken = factor != factor;
        if (broken) factor = 1.0f;
        if (factor == 0.0f) factor = 1.17549435e-38f;
        const uint32_t lanes = (uint32_t)((threadIdx.x >> 5) & 3) << 21;              // the warp's quarter of the TMEM lanes
        const uint32_t s_at = tmem + lanes + i * kRowTile, o_at = tmem + lanes + (2 + i) * kRowTile;
        float ref = kNoMax;
        uint32_t lost_seen = 0;
        f32x2 sum2 = pack2(0.0f, 0.0f);
        const f32x2 factor2 = pack2(factor, factor);
        const int n = end - begin;
#pragma unroll 1
        for (int j = 0; j < n; j++) {
            const int t0 = range.tile(begin + j) * kRowTile;
            if (!wait_warp(&bars.s_ready[i], j & 1)) return;
            tc_after();
            const uint4 absent = lds128(smem_u32(bars.absent[j & 3]));
            if (IMAGE) lost_seen |= bars.absent[j & 3][4];
            const bool gaps = (absent.x | absent.y | absent.z | absent.w) != 0;
            if (gaps || !whole(t0)) {
                // What a row does not see becomes the logit whose product with the factor is minus infinity, in TMEM: steps that
                // need a mask are few, and the code below stays free of it.
                if (IMAGE && gaps) latch_absent(t0, absent);
                const int b = min(pos, kv - 1) - t0, a = p.window > 0 ? max(pos - p.window + 1, 0) - t0 : -t0, s = p.sinks - t0;
                const uint32_t none = factor < 0.0f ? 0x7F800000u : 0xFF800000u;
#pragma unroll 1
                for (int k = 0; k < 8; k++) {
                    const uint32_t gone = (k < 2 ? absent.x : k < 4 ? absent.y : k < 6 ? absent.z : absent.w) >> (16 * (k & 1));
                    const uint32_t in = seen(16 * k, a, b, s, gone);
                    uint32_t x[16];
                    tc_ld16(x, s_at + 16 * k);
                    tc_wait_ld();
#pragma unroll
                    for (int c = 0; c < 16; c++) x[c] = in >> c & 1u ? x[c] : none;
                    tc_st16(s_at + 16 * k, x);
                }
                tc_wait_st();
            }
            // Weights are made against the reference as it stands, and checked: nothing is stored before it is known that none exceeds
            // 2^15.  Else (a row's first step, and rarely) the largest logits are found, the references of the warp's rows moved to
            // 3 below them, and the weights made again.  fp16 then holds weights down to 2^-17 of the largest to all its bits (the many
            // small weights of a long context matter: with a largest weight of 2^-4 fp16 results were 7.7e-4 off, 7.0e-4
            // so, with K as one fp16 matrix), and a logit may still grow by 12: a step made twice costs 4500 cycles, and at 8
            // below 8192 rows over 8192 tokens (32 query heads) take 610 us instead of 562.
            uint32_t w[64];
            f32x2 total;
            bool search = j == 0;
            for (;;) {
                if (search) {
                    float y = -INFINITY;
#pragma unroll 1
                    for (int k = 0; k < 8; k++) {
                        uint32_t x[16];
                        tc_ld16(x, s_at + 16 * k);
                        tc_wait_ld();
#pragma unroll
                        for (int c = 0; c < 16; c++) y = fmaxf(y, __uint_as_float(x[c]) * factor);
                    }
                    const float to = y > ref + kTop ? y - kPeak : ref, keep = fast_exp2(ref - to);
                    ref = to;
                    sum2 = mul2(sum2, pack2(keep, keep));
                    if (j > 0)                                  // the products of the steps before are done: s_ready came behind them
#pragma unroll 1
                        for (int k = 0; k < D / 16; k++) {
                            uint32_t o[16];
                            tc_ld16(o, o_at + 16 * k);
                            tc_wait_ld();
#pragma unroll
                            for (int c = 0; c < 16; c++) o[c] = __float_as_uint(__uint_as_float(o[c]) * keep);
                            tc_st16(o_at + 16 * k, o);
                        }
                }
                const f32x2 ref2 = pack2(-ref, -ref);
                total = sum2;
                float x[32];
                if constexpr (IMAGE) {                          // registers for two chunks: one on its way while the other is weighed
                    float z[32];
                    tc_ld32(x, s_at);
                    tc_wait_ld();
                    tc_ld32(z, s_at + 32);
                    weigh(x, w, factor2, ref2, total);
                    tc_wait_ld();
                    tc_ld32(x, s_at + 64);
                    weigh(z, w + 16, factor2, ref2, total);
                    tc_wait_ld();
                    tc_ld32(z, s_at + 96);
                    weigh(x, w + 32, factor2, ref2, total);
                    tc_wait_ld();
                    weigh(z, w + 48, factor2, ref2, total);
                } else {
#pragma unroll
                    for (int k = 0; k < 4; k++) {
                        tc_ld32(x, s_at + 32 * k);
                        tc_wait_ld();
                        weigh(x, w + 16 * k, factor2, ref2, total);
                    }
                }
                if (search) break;
                uint32_t most[4] = {0, 0, 0, 0};                // weights are not negative: their bit patterns order them
#pragma unroll
                for (int c = 0; c < 64; c++) most[c & 3] = __vmaxu2(most[c & 3], w[c]);
                const uint32_t top = __vmaxu2(__vmaxu2(most[0], most[1]), __vmaxu2(most[2], most[3]));
                constexpr uint32_t kLimit = kPool ? 0x4700u : 0x7800u;                  // 2^15
                search = __any_sync(0xFFFFFFFFu, max(top & 0xFFFFu, top >> 16) > kLimit);
                if (!search) break;
            }
            sum2 = total;
            tc_st64(s_at, w);                                   // over the first half of S
            tc_wait_st();
            tc_before();
            __syncwarp();
            if ((threadIdx.x & 31) == 0) mbar_arrive(&bars.p_ready[i]);
        }
        if (n > 0 && !wait_warp(&bars.o_ready[i], 0)) return;
        tc_after();
        float sum, sum_odd;
        unpack2(sum2, sum, sum_odd);
        sum += sum_odd;
        if (broken && sum != 0.0f) sum = __uint_as_float(0x7FC00000u);
        const bool lost = IMAGE ? lost_seen != 0 : *reinterpret_cast<volatile int32_t*>(&bars.lost) != 0;
        const float inv = pl.splits > 1 ? 1.0f : (sum != 0.0f ? 1.0f / sum : 0.0f);
        const long long vec = (long long)row * p.Hq + hq;
        float* part = pl.partial + ((long long)split * p.b.n_rows * p.Hq + vec) * D;
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
                add_lost(p, pl, {range, seq, head, kv, last, hi, begin, end, VF == FMT_INT4}, fixed, 32 * k, pos);
#pragma unroll
                for (int c = 0; c < 32; c++) o[c] = fixed[c];
            }
#pragma unroll
            for (int c = 0; c < 32; c += 8) {
                float y[8];
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    const int from = VF == FMT_INT4 ? (e < 4 ? 2 * e : 2 * (e - 4) + 1) : e;       // channel e of eight stands there
                    y[e] = o[c + from] * inv;
                }
                if (pl.splits > 1) {
                    if (!live) continue;
                    float4* d = reinterpret_cast<float4*>(part + 32 * k + c);
                    d[0] = make_float4(y[0], y[1], y[2], y[3]);
                    d[1] = make_float4(y[4], y[5], y[6], y[7]);
                } else {                                        // by way of the query's place in shared memory
                    const uint32_t at = smem + S::kQ + i * S::kMat + swizzled(r, 4 * k + c / 8);
                    if (p.f16) sts128(at, half2_bits(y[0], y[1]), half2_bits(y[2], y[3]), half2_bits(y[4], y[5]), half2_bits(y[6], y[7]));
                    else sts128(at, bf162_bits(y[0], y[1]), bf162_bits(y[2], y[3]), bf162_bits(y[4], y[5]), bf162_bits(y[6], y[7]));
                }
            }
        }
        if (pl.splits == 1) {
            __syncwarp();
            const long long mine = (long long)row * p.out_stride_row + (long long)hq * p.out_stride_head;
            constexpr int kRun = D / 8;
            const int lane = threadIdx.x & 31;
#pragma unroll 4
            for (int k = 0; k < kRun; k++) {
                const int from = k * (32 / kRun) + lane / kRun;
                const long long at = __shfl_sync(0xFFFFFFFFu, mine, from);
                const bool there = __shfl_sync(0xFFFFFFFFu, (int)live, from) != 0;
                const uint4 z = lds128(smem + S::kQ + i * S::kMat + swizzled((r & ~31) + from, lane % kRun));
                if (there) *reinterpret_cast<uint4*>(p.out + at + 8 * (lane % kRun)) = z;
            }
        }
        if (live && pl.splits > 1) {
            float* ml = pl.partial + (long long)pl.splits * p.b.n_rows * p.Hq * D + ((long long)split * p.b.n_rows * p.Hq + vec) * 2;
            *reinterpret_cast<float2*>(ml) = make_float2(ref, sum);
        }
    }
};

// ONE: no sequence has more than one tile of vectors; the second tile's warps then help to bring K and V.
template <int KF, int VF, int D, bool IMAGE, bool ONE, bool FINE>
__global__ void __launch_bounds__(rows_threads(IMAGE), 1) attention_rows_kernel(const __grid_constant__ AttentionParams p, const __grid_constant__ RowsPlan pl) {
    using K = RowsKernel<KF, VF, D, IMAGE, FINE>;
    using S = RowsSmem<D>;
    constexpr int kIssuer = rows_issuer(IMAGE), kThreads = rows_threads(IMAGE);
    extern __shared__ uint8_t raw[];
    const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u;
    RowsBars& bars = *reinterpret_cast<RowsBars*>(raw + (base - smem_u32(raw)) + S::kBars);
    pdl_trigger();
    const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x >> 5, 0);
    if (threadIdx.x == 0) {
        for (int i = 0; i < 2; i++) {
            mbar_init(&bars.q_ready[i], 4); mbar_init(&bars.p_ready[i], 4);          // the four warps of a tile
            mbar_init(&bars.s_ready[i], 1); mbar_init(&bars.o_ready[i], 1);
            mbar_init(&bars.k_full[i], IMAGE ? 1 : ONE ? 256 : 128); mbar_init(&bars.v_full[i], IMAGE ? 1 : ONE ? 256 : 128);
            mbar_init(&bars.k_empty[i], 1); mbar_init(&bars.v_empty[i], 1);
        }
        mbar_init(&bars.drained, 1);
        bars.abort = 0; bars.lost = 0;
        bars.lo = bars.least = 0x7FFFFFFF; bars.hi = -1;
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
    if (threadIdx.x == 0 && (!ordered || rows > p.b.max_rows || (rows > 0 && p.b.kv_len[seq] > kv))) latch(p.status);
    if (!ordered) return;
    rows = min(rows, p.b.max_rows);
    const int m0 = tile * 2 * kRowTile, m_end = min(rows * p.share, m0 + 2 * kRowTile);
    if (m0 >= m_end) return;
    const int tiles = !ONE && m_end - m0 > kRowTile ? 2 : 1;
    __syncthreads();
    // positions of the CTA's rows (one below 0 sees nothing: no window need reach back for it)
    {
        uint32_t low = 0x7FFFFFFFu;                             // below 0 is above that
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
        if (threadIdx.x == 0) { bars.first_row = first + m0 / p.share; bars.last_row = first + (m_end - 1) / p.share; }
        if ((threadIdx.x & 31) == 0) {
            atomicMin(&bars.lo, (int)low);
            atomicMin(&bars.least, least);
            atomicMax(&bars.hi, most);
        }
    }
    if (warp == kIssuer / 32) tc_alloc(&bars.tmem, 512);
    tc_before();
    __syncthreads();
    tc_after();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(&bars.tmem);
    K k(p, bars);
    k.smem = base; k.seq = seq; k.head = head; k.kv = kv;
    k.hi = bars.hi;
    k.last = min(bars.least, kv - 1);
    k.range = step_range(p, kv, bars.lo, k.hi);
    k.begin = (int)((long long)k.range.count * split / pl.splits);
    k.end = (int)((long long)k.range.count * (split + 1) / pl.splits);
    if (warp < (ONE ? 4 : kProducer0 / 32)) {
        if (warp < 4 * tiles) k.softmax(warp >> 2, first, m0 + (int)threadIdx.x, m_end, tmem, pl, split);
    } else if (warp < kIssuer / 32) {
        if constexpr (IMAGE) {
            k.fetch_images(pl);
        } else {
            k.template produce<ONE ? 16 : 32>(warp - (ONE ? 4 : 8));
            cp_wait<0>();
        }
    } else if (k.end > k.begin) {
        k.issue(tiles, tmem);
        if (__any_sync(0xFFFFFFFFu, *reinterpret_cast<volatile int32_t*>(&bars.abort))) {      // what was issued must have ended before TMEM goes
            if (elect_lane()) tc_commit(&bars.drained);
            __syncwarp();
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

// Images of the two matrices of a step (grid: step, KV head, sequence): the operands of 128 tokens in channel order, laid out and
// swizzled as in shared memory, tokens behind the cache or on a page out of range zero.  Values that are not finite are set to
// zero in V and noted.  Bound by memory: reads the cache once, writes 4 bytes per element pair.
constexpr int kImageThreads = 256;
template <int KF, int VF, int D, bool FINE>
__global__ void __launch_bounds__(kImageThreads) attention_image_kernel(const AttentionParams p, const RowsPlan pl) {
    using S = RowsSmem<D>;
    constexpr bool kPool = KF == FMT_BF16;
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
    uint32_t m0 = 0x64086408u, m1 = 0x64806480u;
    uint8_t* k_image = pl.images + image_index(p, pl, seq, step, head) * ((FINE ? 3 : 2) * S::kMat);
    uint8_t* v_image = k_image + (FINE ? 2 : 1) * S::kMat;
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
        uint4 ko[4], kr[4], vo[4];
        if (page < 0) {
#pragma unroll
            for (int q = 0; q < 4; q++) ko[q] = kr[q] = vo[q] = make_uint4(0, 0, 0, 0);
        } else if constexpr (kPool) {
            const long long o = (long long)page * p.c.stride_page + (long long)slot * p.c.stride_token + (long long)head * p.c.stride_head + 32 * c;
#pragma unroll
            for (int q = 0; q < 4; q++) {
                ko[q] = *(reinterpret_cast<const uint4*>(p.c.k + o) + q);
                vo[q] = *(reinterpret_cast<const uint4*>(p.c.v + o) + q);
            }
        } else {
            const uint8_t* pg = p.c.base + (long long)page * p.c.stride_page;
            const uint32_t row = (uint32_t)slot * p.c.H + head, sc = (row * (D / p.c.G) + c * 32 / p.c.G) * 2;
            uint32_t ks = *reinterpret_cast<const uint16_t*>(pg + p.c.k_scales + sc), vs = *reinterpret_cast<const uint16_t*>(pg + p.c.v_scales + sc);
            ks |= ks << 16; vs |= vs << 16;
            if (FINE) image_operands<KF>(ko, kr, pg + row * (KF == FMT_INT8 ? D : D / 2), c, ks, m0, m1);
            else image_operands<KF>(ko, pg + row * (KF == FMT_INT8 ? D : D / 2), c, ks, m0, m1);
            image_operands<VF>(vo, pg + p.c.v_codes + row * (VF == FMT_INT8 ? D : D / 2), c, vs, m0, m1);
        }
        bool lost = false;
#pragma unroll
        for (int q = 0; q < 4; q++) {
            lost = finite_only<kPool ? 0x7F80u : 0x7C00u>(vo[q]) || lost;
            *reinterpret_cast<uint4*>(k_image + swizzled(tok, 4 * c + q)) = ko[q];
            if (FINE) *reinterpret_cast<uint4*>(k_image + S::kMat + swizzled(tok, 4 * c + q)) = kr[q];
            *reinterpret_cast<uint4*>(v_image + swizzled(tok, 4 * c + q)) = vo[q];
        }
        if (lost) meta[4] = 1;
    }
    __syncthreads();
    if (threadIdx.x < 8) pl.meta[image_index(p, pl, seq, step, head) * 8 + threadIdx.x] = meta[threadIdx.x];
}

// Joins the pieces of split rows: a warp per query vector, sequence by sequence as they were made (a search for a row's sequence would
// lose those in front of row_start entries that descend).
template <int D>
__global__ void __launch_bounds__(128) attention_rows_join_kernel(const AttentionParams p, const RowsPlan pl) {
    pdl_wait();
    const int lane = threadIdx.x & 31;
    int first, kv, rows;
    if (!sequence_rows(p, blockIdx.y, &first, &kv, &rows)) return;
    const long long n = (long long)p.b.n_rows * p.Hq, at = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
    if (at >= (long long)min(rows, p.b.max_rows) * p.Hq) return;
    const int row = first + (int)(at / p.Hq), hq = (int)(at % p.Hq);
    const long long vec = (long long)row * p.Hq + hq;
    const float* ml = pl.partial + pl.splits * n * D;
    float top = kNoMax, sum = 0.0f, y[D / 32];
    for (int i = 0; i < pl.splits; i++) top = fmaxf(top, ml[(i * n + vec) * 2]);
#pragma unroll
    for (int k = 0; k < D / 32; k++) y[k] = 0.0f;
#pragma unroll 4
    for (int i = 0; i < pl.splits; i++) {
        const float2 x = *reinterpret_cast<const float2*>(ml + (i * n + vec) * 2);
        const float f = fast_exp2(x.x - top);
        sum = fmaf(f, x.y, sum);
#pragma unroll
        for (int k = 0; k < D / 32; k++) y[k] = fmaf(f, pl.partial[(i * n + vec) * D + lane + 32 * k], y[k]);
    }
    uint16_t* o = p.out + (long long)row * p.out_stride_row + (long long)hq * p.out_stride_head;
#pragma unroll
    for (int k = 0; k < D / 32; k++) {
        const float v = sum != 0.0f ? y[k] / sum : 0.0f;
        o[lane + 32 * k] = (uint16_t)(p.f16 ? half2_bits(v, 0.0f) : bf162_bits(v, 0.0f));
    }
}

}  // namespace patchkv
