// Attention of few query columns: the cache is split over the grid along the tokens and read once.
//
// A column is a (row, query head of one KV head) pair; up to 8 * NT of them (NT 1 or 2) ride on one pass over a KV head.
// Both products run on mma.m16n8k16 with the cache as the M side, so a cached number becomes a matrix operand once
// and 8 columns use it: logits^T[16 tokens][8 columns] = K * q^T, out^T[channels][8 columns] += V^T * p^T.  The matrix
// pipe is far from its limit here (tcgen05 would want 128 rows); what bounds the kernel is the bytes of the cache
// and, for 4-bit pages, the instructions that turn codes into operands, which is where the work below went.
//
// Codes as operands.  A code plus its offset (u = q + 8 or q + 128) put into the low bits of a half is the subnormal u * 2^-24,
// exactly, so an operand register costs one logic instruction, and the products and fp32 sums take it from there.
//   K: each 32-channel chunk is summed on its own in fp32 from a start value that takes the offset out again
//      (-8 * sum of the chunk's q), then enters the logit with the token's fp32 scale: no rounding of K at all.
//      q is fp16 scaled by a power of two per column (bf16 has fewer bits, so nothing is lost but far below 2^-24 of
//      the column's largest).
//   V: v = (u * 2^-24) * S - offset * S in one half fma, S the token's scale times a power of two that follows the
//      largest V scale seen: one rounding of 2^-12, as p's own to fp16.
// Softmax on powers of two against a reference that is only moved when a logit exceeds it by more than 8 (p <= 256): one
// vote per tile instead of a maximum across lanes.
#pragma once

#include "attention.cuh"

namespace patchkv {

constexpr int kTile = 16;                       // tokens a warp takes at a time: one mma K (M) step
constexpr float kNoMax = -3.0e38f;

// What the combine kernel needs of a split launch, and where partial results lie.
struct SplitPlan {
    float* partial;                             // [item][head][regs][32 lanes], then m and l [cols] each
    int32_t* items;                             // per sequence: first item, number of items
    int32_t regs, cols_max;                     // floats a lane holds, columns (8 * NT)
    int32_t item_stride;                        // floats per (item, head)
    int32_t max_items;                          // grid bound
    int32_t target;                             // pieces the whole batch is cut into (0: one piece per sequence, no combine)
    int32_t heads, head_groups, warps_per_head; // heads of a CTA, CTAs across the heads
};

__device__ __forceinline__ void cp16(uint32_t dst, const void* src, bool live) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(live ? 16 : 0) : "memory");
}
template <int BYTES>
__device__ __forceinline__ void cp_small(uint32_t dst, const void* src, bool live) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(dst), "l"(src), "n"(BYTES), "r"(live ? BYTES : 0) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t hfma2(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t d;
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}
__device__ __forceinline__ uint32_t hmul2(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __forceinline__ float fast_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t half2_bits(float lo, float hi) {
    uint32_t d;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}
__device__ __forceinline__ uint32_t bf162_bits(float lo, float hi) {
    uint32_t d;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}
__device__ __forceinline__ uint32_t both(float x) { return half2_bits(x, x); }
__device__ __forceinline__ float exp2i(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }   // -126 <= e <= 127
__device__ __forceinline__ float low_half(uint32_t x) { return half_bits_to_float(x & 0xFFFFu); }
__device__ __forceinline__ float high_half(uint32_t x) { return half_bits_to_float(x >> 16); }

// The tokens a sequence's rows see: tiles [0, sink_tiles) and [first, end_tile), numbered through as `count` virtual tiles.
struct TileRange {
    int sink_tiles, first, count;
    __device__ __forceinline__ int tile(int i) const { return i < sink_tiles ? i : first + (i - sink_tiles); }
};
__device__ __forceinline__ TileRange tile_range(const AttentionParams& p, int kv, int lo_pos, int hi_pos) {
    TileRange r;
    const int end = min(hi_pos, kv - 1) + 1;                 // hi_pos < 0: nothing
    const int lo = p.window > 0 ? max(0, lo_pos - p.window + 1) : 0;
    r.first = lo / kTile;
    r.sink_tiles = p.window > 0 ? (min(p.sinks, r.first * kTile) + kTile - 1) / kTile : 0;
    const int last = end <= 0 ? 0 : (end - 1) / kTile + 1;
    r.sink_tiles = min(r.sink_tiles, last);
    r.count = r.sink_tiles + max(0, last - r.first);
    return r;
}
// Smallest (but -1 for any below) and largest position of the first max_rows of a sequence's rows.
__device__ __forceinline__ void position_range(const AttentionParams& p, int s, int first, int rows, int* lo, int* hi) {
    const int n = min(rows, p.b.max_rows);
    if (!p.b.pos) {
        const int a = __ldg(p.b.kv_len + s) - rows;
        *lo = max(-1, a);
        *hi = a + n - 1;
        return;
    }
    *lo = 0x7FFFFFFF;
    *hi = -1;
    for (int i = 0; i < n; i++) {
        const int x = __ldg(p.b.pos + first + i);
        *lo = min(*lo, x);
        *hi = max(*hi, x);
    }
    *lo = max(-1, *lo);
}

// ---------------------------------------------------------------------------------------------------------------------
// KF / VF: page formats (both FMT_BF16 for the bf16 pool); G32: one scale per 32 channels (else G is 64 or 128).
template <int KF, int VF, int D, int NT, int STAGES, int WARPS, bool G32>
struct SplitKernel {
    static constexpr bool kPool = KF == FMT_BF16;
    static constexpr int kKRow = KF == FMT_BF16 ? 2 * D : (KF == FMT_INT8 ? D : D / 2);     // bytes of a head's row
    static constexpr int kVRow = VF == FMT_BF16 ? 2 * D : (VF == FMT_INT8 ? D : D / 2);
    static constexpr int kKStride = kKRow + 16, kVStride = kVRow + 16;                      // bank-conflict-free for every access below
    static constexpr int kV = kTile * kKStride, kScales = kV + kTile * kVStride;
    static constexpr int kStage = kScales + (kPool ? 0 : 2 * kTile * 8);                    // 8 bytes of scales per token, K then V
    static constexpr int kChunks = D / 32, kMT = D / 16, kRegs = 4 * kMT * NT;
    static constexpr int kSmem = WARPS * STAGES * kStage;
    static constexpr int kMerge = WARPS * (kRegs * 32 + 2 * 8 * NT) * 4;                    // the warps' results, in the same memory

    const AttentionParams& p;
    uint32_t ring;
    int lane, g, t;
    uint32_t qf[NT][kPool ? kMT : 2 * kChunks][2];
    float bias[NT][kPool ? 1 : kChunks][2];
    float factor[NT][2], ref[NT][2], sum[NT][2];
    int pos[NT][2];
    float acc[NT][kMT][4];
    int v_exp;                                  // V scales are multiplied by 2^v_exp
    int kv, lo_pos, hi_pos;

    __device__ SplitKernel(const AttentionParams& p_) : p(p_) {}

    __device__ __forceinline__ bool visible(int ps, int tok) const {
        return tok <= ps && tok < kv && sees(p, ps, tok);
    }

    // Queries of column n = 8 * nt + (lane / 4) as B operands, and the per-column numbers of the lane's two logit columns.
    __device__ __forceinline__ void load_queries(int first, int cols, int head) {
#pragma unroll
        for (int nt = 0; nt < NT; nt++) {
            const int n = 8 * nt + g, row = n / p.share, hq = head * p.share + n % p.share;
            const uint16_t* q = p.q + (long long)(first + row) * p.q_stride_row + (long long)hq * p.q_stride_head;
            const bool live = n < cols;
            if constexpr (kPool) {
#pragma unroll
                for (int k = 0; k < kMT; k++)
#pragma unroll
                    for (int e = 0; e < 2; e++)
                        qf[nt][k][e] = live ? __ldg(reinterpret_cast<const uint32_t*>(q + 16 * k + 8 * e + 2 * t)) : 0u;
#pragma unroll
                for (int e = 0; e < 2; e++) factor[nt][e] = p.scale_log2;
            } else {
                // the lane's channels: 8 of each chunk, in the order the codes of a 32-bit word come out
                float x[kChunks][8];
                float amax = 0.0f;
#pragma unroll
                for (int j = 0; j < kChunks; j++) {
                    uint32_t w[4] = {0, 0, 0, 0};
                    if (live) {
                        if (KF == FMT_INT4) {
                            const uint4 v = __ldg(reinterpret_cast<const uint4*>(q + 32 * j + 8 * t));
                            w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
                        } else {
                            const uint2 a = __ldg(reinterpret_cast<const uint2*>(q + 32 * j + 4 * t));
                            const uint2 b = __ldg(reinterpret_cast<const uint2*>(q + 32 * j + 16 + 4 * t));
                            w[0] = a.x; w[1] = a.y; w[2] = b.x; w[3] = b.y;
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 8; i++) {
                        const uint32_t h = i & 1 ? w[i >> 1] >> 16 : w[i >> 1] & 0xFFFFu;
                        x[j][i] = p.f16 ? half_bits_to_float(h) : bf16_bits_to_float(h);
                        amax = fmaxf(amax, fabsf(x[j][i]));
                    }
                }
                amax = fmaxf(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, 1));
                amax = fmaxf(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, 2));
                // largest magnitude into [2^13, 2^14); zeros, NaN and infinities as they are
                const int e = (int)(__float_as_uint(amax) >> 23) - 127;
                const int shift = amax > 0.0f && e < 128 ? min(13 - e, 120) : 0;
                const float up = exp2i(shift);
                const float down = p.scale_log2 * exp2i(-shift) * 16777216.0f;
                float off[kChunks];
#pragma unroll
                for (int j = 0; j < kChunks; j++) {
#pragma unroll
                    for (int m = 0; m < 2; m++) {
                        if (KF == FMT_INT4) {                // word's nibbles: (0,4) (1,5) / (2,6) (3,7), odd ones 16 times up
                            qf[nt][2 * j + m][0] = half2_bits(x[j][2 * m] * up, x[j][2 * m + 4] * up);
                            qf[nt][2 * j + m][1] = half2_bits(x[j][2 * m + 1] * up * 0.0625f, x[j][2 * m + 5] * up * 0.0625f);
                        } else {
                            qf[nt][2 * j + m][0] = half2_bits(x[j][4 * m] * up, x[j][4 * m + 1] * up);
                            qf[nt][2 * j + m][1] = half2_bits(x[j][4 * m + 2] * up, x[j][4 * m + 3] * up);
                        }
                    }
                    float a = 0.0f;
#pragma unroll
                    for (int m = 0; m < 2; m++) {
                        a += low_half(qf[nt][2 * j + m][0]) + high_half(qf[nt][2 * j + m][0]);
                        const float b = low_half(qf[nt][2 * j + m][1]) + high_half(qf[nt][2 * j + m][1]);
                        a += KF == FMT_INT4 ? 16.0f * b : b;
                    }
                    a += __shfl_xor_sync(0xFFFFFFFFu, a, 1);
                    a += __shfl_xor_sync(0xFFFFFFFFu, a, 2);
                    off[j] = a * (KF == FMT_INT4 ? -4.76837158203125e-07f : -7.62939453125e-06f);    // -8 * 2^-24, -128 * 2^-24
                }
#pragma unroll
                for (int e2 = 0; e2 < 2; e2++) {
                    const int src = (2 * t + e2) * 4;
                    factor[nt][e2] = __shfl_sync(0xFFFFFFFFu, down, src);
#pragma unroll
                    for (int j = 0; j < kChunks; j++) bias[nt][j][e2] = __shfl_sync(0xFFFFFFFFu, off[j], src);
                }
            }
        }
    }

    // Enqueues tile `tile` of the head into stage `st`; page < 0: zeros.
    __device__ __forceinline__ void fetch(int st, int tile, int page, int head) {
        const uint32_t base = ring + st * kStage;
        const int t0 = tile * kTile, slot0 = t0 - div_page(p.c, t0) * p.c.P;
        // a token that no row sees is filled with zeros: nothing of its slot takes part
        const int end = min(hi_pos, kv - 1);
        if constexpr (kPool) {
            const long long o = page < 0 ? 0 : (long long)page * p.c.stride_page + (long long)slot0 * p.c.stride_token + (long long)head * p.c.stride_head;
#pragma unroll
            for (int i = lane; i < kTile * kKRow / 16; i += 32) {
                const int tok = i / (kKRow / 16), c = i % (kKRow / 16);
                const bool live = page >= 0 && t0 + tok <= end && sees(p, lo_pos, t0 + tok);
                const long long a = o + (live ? tok * p.c.stride_token + 8 * c : 0);
                cp16(base + tok * kKStride + 16 * c, p.c.k + a, live);
                cp16(base + kV + tok * kVStride + 16 * c, p.c.v + a, live);
            }
        } else {
            const uint8_t* pg = p.c.base + (page < 0 ? 0ll : (long long)page * p.c.stride_page);
            const uint32_t row0 = (uint32_t)slot0 * p.c.H + head;          // (token, head) rows of a page, H apart per token
#pragma unroll
            for (int i = lane; i < kTile * kKRow / 16; i += 32) {
                const int tok = i / (kKRow / 16), c = i % (kKRow / 16);
                cp16(base + tok * kKStride + 16 * c, pg + (row0 + tok * p.c.H) * kKRow + 16 * c, page >= 0);
            }
#pragma unroll
            for (int i = lane; i < kTile * kVRow / 16; i += 32) {
                const int tok = i / (kVRow / 16), c = i % (kVRow / 16);
                cp16(base + kV + tok * kVStride + 16 * c, pg + p.c.v_codes + (row0 + tok * p.c.H) * kVRow + 16 * c, page >= 0);
            }
            const int tok = lane & 15;
            const bool live = page >= 0 && t0 + tok <= end && sees(p, lo_pos, t0 + tok);
            const uint8_t* sc = pg + (lane < 16 ? p.c.k_scales : p.c.v_scales);
            const uint32_t e = (row0 + tok * p.c.H) * (D / (G32 ? 32 : p.c.G)) * 2;
            const uint32_t dst = base + kScales + lane * 8;
            if (D == 128 && G32) cp_small<8>(dst, sc + e, live);
            else cp_small<4>(dst, sc + (e & ~3u), live);                   // a lone fp16: its word, picked apart below
        }
    }

    // Scale of 32-channel chunk j from a token's 8 bytes.
    __device__ __forceinline__ float chunk_scale(const uint2& s, int j, uint32_t odd) const {
        if (G32) return half_bits_to_float(j & 1 ? (j < 2 ? s.x : s.y) >> 16 : (j < 2 ? s.x : s.y) & 0xFFFFu);
        const int i = p.c.G == D ? (int)odd : j * 32 / p.c.G;
        return half_bits_to_float(i ? s.x >> 16 : s.x & 0xFFFFu);
    }

    __device__ __forceinline__ void rescale(int nt, int e, float to) {
        const float keep = fast_exp2(ref[nt][e] - to);
        ref[nt][e] = to;
        sum[nt][e] *= keep;
#pragma unroll
        for (int i = 0; i < kMT; i++) { acc[nt][i][e] *= keep; acc[nt][i][2 + e] *= keep; }
    }

    // One tile: logits, weights, and the weighted values.
    __device__ __forceinline__ void tile(int st, int tl, int page, int head) {
        const uint32_t base = ring + st * kStage;
        const int t0 = tl * kTile;
        // (row of logits: token g and g + 8; column 2t and 2t + 1 of each eight)
        float x[NT][4];
        const int slot0 = t0 - div_page(p.c, t0) * p.c.P;
        uint32_t odd_a = 0, odd_b = 0;
        if constexpr (kPool) {
#pragma unroll
            for (int nt = 0; nt < NT; nt++)
#pragma unroll
                for (int i = 0; i < 4; i++) x[nt][i] = 0.0f;
            const uint32_t a = base + ((lane & 7) + (lane & 8)) * kKStride + (lane >> 4) * 16;
#pragma unroll
            for (int k = 0; k < kMT; k++) {
                uint32_t r[4];
                ldmatrix4(r, a + 32 * k);
#pragma unroll
                for (int nt = 0; nt < NT; nt++) mma_bf16(x[nt], r[0], r[1], r[2], r[3], qf[nt][k][0], qf[nt][k][1]);
            }
        } else {
            if (!G32 && p.c.G == D) {                                      // which half of the word a lone scale is
                odd_a = ((slot0 + g) * p.c.H + head) & 1;
                odd_b = ((slot0 + g + 8) * p.c.H + head) & 1;
            }
            const uint2 sa = lds64(base + kScales + 8 * g), sb = lds64(base + kScales + 8 * (g + 8));
#pragma unroll
            for (int nt = 0; nt < NT; nt++)
#pragma unroll
                for (int i = 0; i < 4; i++) x[nt][i] = 0.0f;
            const uint32_t ra = base + g * kKStride + 4 * t, rb = ra + 8 * kKStride;
#pragma unroll
            for (int j = 0; j < kChunks; j++) {
                float y[NT][4];
#pragma unroll
                for (int nt = 0; nt < NT; nt++) {
                    y[nt][0] = y[nt][2] = bias[nt][j][0];
                    y[nt][1] = y[nt][3] = bias[nt][j][1];
                }
                if constexpr (KF == FMT_INT4) {
                    uint32_t wa = lds32(ra + 16 * j), wb = lds32(rb + 16 * j);
#pragma unroll
                    for (int m = 0; m < 2; m++) {
                        const uint32_t a0 = (wa & 0x000F000Fu) ^ 0x00080008u, a1 = (wb & 0x000F000Fu) ^ 0x00080008u;
                        const uint32_t a2 = (wa & 0x00F000F0u) ^ 0x00800080u, a3 = (wb & 0x00F000F0u) ^ 0x00800080u;
#pragma unroll
                        for (int nt = 0; nt < NT; nt++) mma_f16(y[nt], a0, a1, a2, a3, qf[nt][2 * j + m][0], qf[nt][2 * j + m][1]);
                        wa >>= 8; wb >>= 8;
                    }
                } else {
#pragma unroll
                    for (int m = 0; m < 2; m++) {
                        const uint32_t wa = lds32(ra + 32 * j + 16 * m) ^ 0x80808080u, wb = lds32(rb + 32 * j + 16 * m) ^ 0x80808080u;
                        const uint32_t a0 = __byte_perm(wa, 0, 0x4140), a1 = __byte_perm(wb, 0, 0x4140);
                        const uint32_t a2 = __byte_perm(wa, 0, 0x4342), a3 = __byte_perm(wb, 0, 0x4342);
#pragma unroll
                        for (int nt = 0; nt < NT; nt++) mma_f16(y[nt], a0, a1, a2, a3, qf[nt][2 * j + m][0], qf[nt][2 * j + m][1]);
                    }
                }
                const float fa = chunk_scale(sa, j, odd_a), fb = chunk_scale(sb, j, odd_b);
#pragma unroll
                for (int nt = 0; nt < NT; nt++) {
                    x[nt][0] = fmaf(y[nt][0], fa, x[nt][0]); x[nt][1] = fmaf(y[nt][1], fa, x[nt][1]);
                    x[nt][2] = fmaf(y[nt][2], fb, x[nt][2]); x[nt][3] = fmaf(y[nt][3], fb, x[nt][3]);
                }
            }
        }
        // Whole tiles need no mask: seen by the earliest row and inside the latest row's window, or among the sinks.
        const bool whole = page >= 0 && t0 + kTile - 1 <= min(lo_pos, kv - 1) &&
                           (p.window == 0 || hi_pos - t0 < p.window || t0 + kTile <= p.sinks);
        bool move = false;
#pragma unroll
        for (int nt = 0; nt < NT; nt++)
#pragma unroll
            for (int i = 0; i < 4; i++) {
                x[nt][i] *= factor[nt][i & 1];
                if (!whole && !(page >= 0 && visible(pos[nt][i & 1], t0 + g + 8 * (i >> 1)))) x[nt][i] = -INFINITY;
                move = move || x[nt][i] > ref[nt][i & 1] + 8.0f;
            }
        if (__any_sync(0xFFFFFFFFu, move)) {
#pragma unroll
            for (int nt = 0; nt < NT; nt++)
#pragma unroll
                for (int e = 0; e < 2; e++) {
                    float m = fmaxf(x[nt][e], x[nt][2 + e]);
                    m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 4));
                    m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 8));
                    m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 16));
                    if (m > ref[nt][e]) rescale(nt, e, m);
                }
        }
        uint32_t pf[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; nt++) {
#pragma unroll
            for (int i = 0; i < 4; i++) x[nt][i] = fast_exp2(x[nt][i] - ref[nt][i & 1]);
            sum[nt][0] += x[nt][0] + x[nt][2];
            sum[nt][1] += x[nt][1] + x[nt][3];
#pragma unroll
            for (int k = 0; k < 2; k++)
                pf[nt][k] = transpose8x8(kPool ? bf162_bits(x[nt][2 * k], x[nt][2 * k + 1]) : half2_bits(x[nt][2 * k], x[nt][2 * k + 1]));
        }
        if constexpr (kPool) {
            const uint32_t a = base + kV + ((lane & 7) + ((lane >> 4) << 3)) * kVStride + (lane & 8) * 2;
            if (!whole) {
                // A value that is not finite must not meet the weight 0 of a row that does not see it.
                uint32_t bad = 0;
#pragma unroll
                for (int i = 0; i < kMT; i++) {
                    uint32_t r[4];
                    ldmatrix4_trans(r, a + 32 * i);
#pragma unroll
                    for (int k = 0; k < 4; k++) bad |= ((r[k] & 0x7F807F80u) + 0x00800080u) & 0x80008000u;
                }
                if (__any_sync(0xFFFFFFFFu, bad != 0)) { values_one_by_one(base, x, 0u); return; }
            }
#pragma unroll
            for (int i = 0; i < kMT; i++) {
                uint32_t r[4];
                ldmatrix4_trans(r, a + 32 * i);
#pragma unroll
                for (int nt = 0; nt < NT; nt++) mma_bf16(acc[nt][i], r[0], r[1], r[2], r[3], pf[nt][0], pf[nt][1]);
            }
        } else {
            // scales of the lane's channels (one group: channels [g * D / 8, (g + 1) * D / 8)) for tokens 2t, 2t+1, 2t+8, 2t+9
            const int group = g * (D / 8) / (G32 ? 32 : p.c.G);
            uint32_t s[4];
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const int tok = 2 * t + (i & 1) + 8 * (i >> 1);
                uint32_t at = base + kScales + 128 + 8 * tok + 2 * group;
                if (!G32 && p.c.G == D) at += 2 * (((slot0 + tok) * p.c.H + head) & 1);
                s[i] = lds16(at);
            }
            uint32_t sp[2] = {s[0] | s[1] << 16, s[2] | s[3] << 16};
            const uint32_t mag = __vmaxu2(sp[0] & 0x7FFF7FFFu, sp[1] & 0x7FFF7FFFu), top = max(mag & 0xFFFFu, mag >> 16);
            // exponent field e: s < 2^(e - 14); the power of two keeps s * 2^v_exp below 2^15
            if (__any_sync(0xFFFFFFFFu, (int)(top >> 10) - 14 + v_exp > 15 || top >= 0x7C00u)) {
                uint32_t m = top >= 0x7C00u ? 0u : top;
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, d));
                const int to = min(v_exp, 29 - (int)(m >> 10));
                if (to < v_exp) {
                    const float keep = exp2i(to - v_exp);
                    v_exp = to;
#pragma unroll
                    for (int nt = 0; nt < NT; nt++)
#pragma unroll
                        for (int i = 0; i < kMT; i++)
#pragma unroll
                            for (int k = 0; k < 4; k++) acc[nt][i][k] *= keep;
                }
                if (!whole && __any_sync(0xFFFFFFFFu, top >= 0x7C00u)) { values_one_by_one(base, x, (uint32_t)(slot0 * p.c.H + head)); return; }
            }
            // 2^v_exp as a product of two halves (v_exp is between -1 and 29): exact, a scale only grows
            const uint32_t up0 = both(exp2i(min(v_exp, 15))), up1 = both(exp2i(max(v_exp - 15, 0)));
            uint32_t S[2], S16[2], off[2];
#pragma unroll
            for (int k = 0; k < 2; k++) {
                S[k] = hmul2(hmul2(sp[k], up0), up1);
                S16[k] = hmul2(S[k], 0x2C002C00u);                          // 2^-4
                off[k] = hmul2(S[k], VF == FMT_INT4 ? 0x80088008u : 0x80808080u);   // -8 * 2^-24, -128 * 2^-24
            }
            const uint32_t rv = base + kV + 2 * t * kVStride + g * (kVRow / 8);
            constexpr int kWords = kVRow / 32;                              // words of a lane's channels in one token
            uint32_t w[4][kWords];
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const uint32_t a = rv + ((i & 1) + 8 * (i >> 1)) * kVStride;
                if constexpr (kWords == 4) {
                    const uint4 v = lds128(a);
                    w[i][0] = v.x; w[i][1] = v.y; w[i][2] = v.z; w[i][3] = v.w;
                } else if constexpr (kWords == 2) {
                    const uint2 v = lds64(a);
                    w[i][0] = v.x; w[i][1] = v.y;
                } else {
                    w[i][0] = lds32(a);
                }
            }
#pragma unroll
            for (int k = 0; k < kWords; k++) {
#pragma unroll
                for (int h = 0; h < 2; h++) {                               // low and high halves of the words
                    uint32_t a = __byte_perm(w[0][k], w[1][k], h ? 0x7632 : 0x5410);
                    uint32_t b = __byte_perm(w[2][k], w[3][k], h ? 0x7632 : 0x5410);
                    if constexpr (VF == FMT_INT4) {
#pragma unroll
                        for (int m = 0; m < 2; m++) {
                            const uint32_t a0 = hfma2((a & 0x000F000Fu) ^ 0x00080008u, S[0], off[0]);
                            const uint32_t a1 = hfma2((a & 0x00F000F0u) ^ 0x00800080u, S16[0], off[0]);
                            const uint32_t a2 = hfma2((b & 0x000F000Fu) ^ 0x00080008u, S[1], off[1]);
                            const uint32_t a3 = hfma2((b & 0x00F000F0u) ^ 0x00800080u, S16[1], off[1]);
#pragma unroll
                            for (int nt = 0; nt < NT; nt++) mma_f16(acc[nt][4 * k + 2 * h + m], a0, a1, a2, a3, pf[nt][0], pf[nt][1]);
                            a >>= 8; b >>= 8;
                        }
                    } else {
                        const uint32_t a0 = hfma2((a & 0x00FF00FFu) ^ 0x00800080u, S[0], off[0]);
                        const uint32_t a1 = hfma2(((a >> 8) & 0x00FF00FFu) ^ 0x00800080u, S[0], off[0]);
                        const uint32_t a2 = hfma2((b & 0x00FF00FFu) ^ 0x00800080u, S[1], off[1]);
                        const uint32_t a3 = hfma2(((b >> 8) & 0x00FF00FFu) ^ 0x00800080u, S[1], off[1]);
#pragma unroll
                        for (int nt = 0; nt < NT; nt++) mma_f16(acc[nt][2 * k + h], a0, a1, a2, a3, pf[nt][0], pf[nt][1]);
                    }
                }
            }
        }
    }

    // Channel of accumulator (i, e) of this lane.
    __device__ __forceinline__ int channel(int i, int e) const { return kPool ? 16 * i + 8 * e + g : g * (D / 8) + 2 * i + e; }

    // The rare tile with values that are not finite, some of them unseen by some rows: every weight that is not zero times its value.
    __device__ __forceinline__ void values_one_by_one(uint32_t base, float (&x)[NT][4], uint32_t row0) {
        for (int tok = 0; tok < kTile; tok++) {
#pragma unroll
            for (int nt = 0; nt < NT; nt++) {
                float w[2];
#pragma unroll
                for (int e = 0; e < 2; e++) {
                    const float a = __shfl_sync(0xFFFFFFFFu, x[nt][e], (tok & 7) * 4 + t);
                    const float b = __shfl_sync(0xFFFFFFFFu, x[nt][2 + e], (tok & 7) * 4 + t);
                    w[e] = tok < 8 ? a : b;
                }
#pragma unroll
                for (int i = 0; i < kMT; i++)
#pragma unroll
                    for (int e = 0; e < 2; e++) {
                        const int c = channel(i, e);
                        float v;
                        if (kPool) {
                            v = bf16_bits_to_float(lds16(base + kV + tok * kVStride + 2 * c));
                        } else {
                            uint32_t at = base + kScales + 128 + 8 * tok + 2 * (c / (G32 ? 32 : p.c.G));
                            if (!G32 && p.c.G == D) at += 2 * ((row0 + tok * p.c.H) & 1);
                            const uint32_t byte = base + kV + tok * kVStride + (VF == FMT_INT8 ? c : c >> 1);
                            uint32_t u = lds32(byte & ~3u) >> ((byte & 3u) * 8);
                            if (VF == FMT_INT4) u = ((u >> ((c & 1) * 4)) & 15u) ^ 8u; else u = (u & 255u) ^ 128u;
                            v = ((float)u - (VF == FMT_INT4 ? 8.0f : 128.0f)) * half_bits_to_float(lds16(at)) * 5.9604644775390625e-08f * exp2i(v_exp);
                        }
                        if (w[0] != 0.0f) acc[nt][i][2 * e] = fmaf(w[0], v, acc[nt][i][2 * e]);
                        if (w[1] != 0.0f) acc[nt][i][2 * e + 1] = fmaf(w[1], v, acc[nt][i][2 * e + 1]);
                    }
            }
        }
    }
};

// Result of one column: value of accumulator r of a lane as (channel, column).
template <bool POOL, int D>
__device__ __forceinline__ void place(int r, int lane, int* channel, int* col) {
    const int per = 4 * (D / 16), nt = r / per, i = (r % per) >> 2, e = (r >> 1) & 1, f = r & 1;
    const int g = lane >> 2, t = lane & 3;
    *channel = POOL ? 16 * i + 8 * e + g : g * (D / 8) + 2 * i + e;
    *col = 8 * nt + 2 * t + f;
}

template <bool POOL, int D>
__device__ __forceinline__ void store_out(const AttentionParams& p, int first, int head, int r, int lane, int cols, float y) {
    int c, n;
    place<POOL, D>(r, lane, &c, &n);
    if (n >= cols) return;
    uint16_t* o = p.out + (long long)(first + n / p.share) * p.out_stride_row + (long long)(head * p.share + n % p.share) * p.out_stride_head + c;
    *o = (uint16_t)(p.f16 ? half2_bits(y, 0.0f) : bf162_bits(y, 0.0f));
}

// The piece of the batch that item `item` stands for: sequence and virtual tiles [begin, end).  All lanes of a warp agree.
// With a target, the batch's tiles are cut into about that many pieces of equal length, none across two sequences.
struct Item { int seq, split, splits, first_item, begin, end, first, rows, kv, lo, hi; bool ok; };
__device__ __forceinline__ Item find_item(const AttentionParams& p, const SplitPlan& pl, int item) {
    const int lane = threadIdx.x & 31;
    Item it;
    it.ok = false;
    it.splits = 1; it.split = 0; it.first_item = item;
    if (pl.target == 0) {
        it.seq = item;
    } else {
        int total = 0;
        for (int s0 = 0; s0 < p.b.n_seqs; s0 += 32) {
            int n = 0;
            if (s0 + lane < p.b.n_seqs) {
                int first, kv, rows, lo, hi;
                const bool ordered = sequence_rows(p, s0 + lane, &first, &kv, &rows);
                if (!ordered && item == 0) latch(p.status);
                if (ordered && rows > 0) {
                    position_range(p, s0 + lane, first, rows, &lo, &hi);
                    n = tile_range(p, kv, lo, hi).count;
                }
            }
            total += __reduce_add_sync(0xFFFFFFFFu, n);
        }
        const int least = pl.warps_per_head;                 // a piece gives every warp a tile
        const int piece = max((total + pl.target - 1) / pl.target, least);
        int at = 0;
        it.seq = -1;
        for (int s0 = 0; s0 < p.b.n_seqs && it.seq < 0; s0 += 32) {
            int n = 0;
            if (s0 + lane < p.b.n_seqs) {
                int first, kv, rows, lo, hi;
                if (sequence_rows(p, s0 + lane, &first, &kv, &rows) && rows > 0) {
                    position_range(p, s0 + lane, first, rows, &lo, &hi);
                    n = max(1, (tile_range(p, kv, lo, hi).count + piece - 1) / piece);
                }
            }
            int inc = n;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int o = __shfl_up_sync(0xFFFFFFFFu, inc, d);
                if (lane >= d) inc += o;
            }
            const unsigned hit = __ballot_sync(0xFFFFFFFFu, item < at + inc);
            if (hit) {
                const int src = __ffs(hit) - 1;
                it.seq = s0 + src;
                it.splits = __shfl_sync(0xFFFFFFFFu, n, src);
                it.first_item = at + __shfl_sync(0xFFFFFFFFu, inc - n, src);
                it.split = item - it.first_item;
                it.begin = it.split * piece;
                it.end = it.begin + piece;
            }
            at += __shfl_sync(0xFFFFFFFFu, inc, 31);
        }
        if (it.seq < 0) return it;
    }
    const bool ordered = sequence_rows(p, it.seq, &it.first, &it.kv, &it.rows);
    if (lane == 0 && (!ordered || it.rows > p.b.max_rows || __ldg(p.b.kv_len + it.seq) > it.kv)) latch(p.status);
    if (!ordered || it.rows == 0) return it;
    position_range(p, it.seq, it.first, it.rows, &it.lo, &it.hi);
    it.rows = min(it.rows, p.b.max_rows);
    const int count = tile_range(p, it.kv, it.lo, it.hi).count;
    if (pl.target == 0) { it.begin = 0; it.end = count; }
    it.end = min(it.end, count);
    it.ok = true;
    return it;
}

template <int KF, int VF, int D, int NT, int STAGES, int WARPS, bool G32>
__global__ void __launch_bounds__(WARPS * 32) attention_split_kernel(const AttentionParams p, const SplitPlan pl) {
    using K = SplitKernel<KF, VF, D, NT, STAGES, WARPS, G32>;
    extern __shared__ __align__(16) uint8_t smem[];
    pdl_trigger();
    pdl_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const Item it = find_item(p, pl, blockIdx.x);
    if (!it.ok) return;                                      // the same in every warp
    const int head = blockIdx.y * pl.heads + warp % pl.heads, sub = warp / pl.heads;
    const bool live = head < p.c.H;
    const int cols = min(it.rows * p.share, 8 * NT);
    K k(p);
    k.ring = smem_u32(smem) + warp * STAGES * K::kStage;
    k.lane = lane; k.g = lane >> 2; k.t = lane & 3;
    k.kv = it.kv; k.lo_pos = it.lo; k.hi_pos = it.hi;
    k.v_exp = 29;
    const TileRange range = tile_range(p, it.kv, it.lo, it.hi);
#pragma unroll
    for (int nt = 0; nt < NT; nt++) {
#pragma unroll
        for (int e = 0; e < 2; e++) {
            const int n = 8 * nt + 2 * k.t + e;
            k.pos[nt][e] = n < cols ? row_position(p.b, it.seq, it.first + n / p.share) : -1;
            k.ref[nt][e] = kNoMax;
            k.sum[nt][e] = 0.0f;
        }
#pragma unroll
        for (int i = 0; i < K::kMT; i++)
#pragma unroll
            for (int j = 0; j < 4; j++) k.acc[nt][i][j] = 0.0f;
    }
    if (live) {
        const int step = pl.warps_per_head, n = it.begin + sub < it.end ? (it.end - it.begin - sub + step - 1) / step : 0;
        // pages of the warp's next 64 tiles: a lane each of the current 32 and the 32 behind them
        auto page_of = [&](int i) {
            if (i >= n) return -1;
            const int lp = div_page(p.c, range.tile(it.begin + sub + i * step) * kTile);
            int pg = __ldg(p.b.block_table + (long long)it.seq * p.b.table_stride + lp);
            if (pg < 0 || pg >= p.c.n_pages) { latch(p.status); pg = -1; }
            return pg;
        };
        int pages = page_of(lane), pages_next = page_of(lane + 32);
        k.load_queries(it.first, cols, head);
        int fetched = 0;
        auto fetch = [&](int i) {
            // i runs through 0, 1, 2 ...; the pages in registers are those of the 32-block of i
            const int pg = __shfl_sync(0xFFFFFFFFu, pages, i & 31);
            if (i < n) k.fetch(i % STAGES, range.tile(it.begin + sub + i * step), pg, head);
            cp_commit();
            if ((i & 31) == 31) { pages = pages_next; pages_next = page_of(i + 33 + lane); }
            return pg;
        };
        int pg_ring[STAGES];
#pragma unroll
        for (int i = 0; i < STAGES - 1; i++) pg_ring[i] = fetch(fetched++);
        for (int i0 = 0; i0 < n; i0 += STAGES) {
#pragma unroll
            for (int u = 0; u < STAGES; u++) {
                const int i = i0 + u;
                if (i < n) {
                    pg_ring[(u + STAGES - 1) % STAGES] = fetch(fetched++);
                    cp_wait<STAGES - 1>();
                    __syncwarp();
                    k.tile(u, range.tile(it.begin + sub + i * step), pg_ring[u], head);
                    __syncwarp();                            // the stage may be filled again
                }
            }
        }
        cp_wait<0>();
    }
    __syncthreads();
    // results of the warps into shared memory, [warp][register][lane], with m and l per column; V's power of two taken out
    float* res = reinterpret_cast<float*>(smem);
    float* ml = res + WARPS * K::kRegs * 32;
    if (live) {
        const float down = K::kPool ? 1.0f : 16777216.0f * exp2i(-k.v_exp);
#pragma unroll
        for (int nt = 0; nt < NT; nt++) {
#pragma unroll
            for (int i = 0; i < K::kMT; i++)
#pragma unroll
                for (int j = 0; j < 4; j++) res[(warp * K::kRegs + (nt * K::kMT + i) * 4 + j) * 32 + lane] = k.acc[nt][i][j] * down;
#pragma unroll
            for (int e = 0; e < 2; e++) {
                float s = k.sum[nt][e];
                s += __shfl_xor_sync(0xFFFFFFFFu, s, 4);
                s += __shfl_xor_sync(0xFFFFFFFFu, s, 8);
                s += __shfl_xor_sync(0xFFFFFFFFu, s, 16);
                if (lane < 4) {
                    ml[(warp * 8 * NT + 8 * nt + 2 * lane + e) * 2] = k.ref[nt][e];
                    ml[(warp * 8 * NT + 8 * nt + 2 * lane + e) * 2 + 1] = s;
                }
            }
        }
    }
    __syncthreads();
    if (pl.target && it.split == 0 && blockIdx.y == 0 && threadIdx.x == 0) {
        pl.items[2 * it.seq] = it.first_item;
        pl.items[2 * it.seq + 1] = it.splits;
    }
    for (int i = threadIdx.x; i < pl.heads * K::kRegs * 32; i += WARPS * 32) {
        const int hl = i / (K::kRegs * 32), r = (i / 32) % K::kRegs, ln = i & 31, h = blockIdx.y * pl.heads + hl;
        if (h >= p.c.H) continue;
        int c, n;
        place<K::kPool, D>(r, ln, &c, &n);
        if (n >= cols) continue;
        float m = kNoMax;
        for (int w = 0; w < pl.warps_per_head; w++) m = fmaxf(m, ml[((hl + w * pl.heads) * 8 * NT + n) * 2]);
        float l = 0.0f, y = 0.0f;
        for (int w = 0; w < pl.warps_per_head; w++) {
            const int wi = hl + w * pl.heads;
            const float f = fast_exp2(ml[(wi * 8 * NT + n) * 2] - m);
            l = fmaf(f, ml[(wi * 8 * NT + n) * 2 + 1], l);
            y = fmaf(f, res[(wi * K::kRegs + r) * 32 + ln], y);
        }
        if (pl.target == 0) {
            store_out<K::kPool, D>(p, it.first, h, r, ln, cols, l != 0.0f ? y / l : 0.0f);
        } else {
            float* out = pl.partial + ((long long)blockIdx.x * p.c.H + h) * pl.item_stride;
            out[r * 32 + ln] = y;
            if (c == 0) { out[pl.regs * 32 + 2 * n] = m; out[pl.regs * 32 + 2 * n + 1] = l; }
        }
    }
}

// Joins the pieces of a sequence: grid (sequence, KV head, quarter of the registers), the CTA's warps share the pieces.
constexpr int kJoinThreads = 256;
template <bool POOL, int D, int NT>
__global__ void __launch_bounds__(kJoinThreads) attention_join_kernel(const AttentionParams p, const SplitPlan pl) {
    constexpr int kRegs = 4 * (D / 16) * NT, kPart = kRegs / 4;         // registers of this CTA: a warp takes one of them at a time
    __shared__ float acc[kJoinThreads / 32][kPart][32];
    __shared__ float top[kJoinThreads / 32][8 * NT], norm[kJoinThreads / 32][8 * NT];
    pdl_wait();
    const int s = blockIdx.x, h = blockIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int first, kv, rows;
    if (!sequence_rows(p, s, &first, &kv, &rows) || rows == 0) return;
    const int cols = min(min(rows, p.b.max_rows) * p.share, 8 * NT);
    const int first_item = pl.items[2 * s], n = pl.items[2 * s + 1];
    const float* part = pl.partial + ((long long)first_item * p.c.H + h) * pl.item_stride;
    const long long step = (long long)p.c.H * pl.item_stride;
    // largest reference of each of the lane's two columns (2t, 2t + 1 of each eight), over the warp's pieces, then over all
    const int t = lane & 3;
    float m[NT][2], l[NT][2], y[kPart];
#pragma unroll
    for (int nt = 0; nt < NT; nt++)
#pragma unroll
        for (int e = 0; e < 2; e++) { m[nt][e] = kNoMax; l[nt][e] = 0.0f; }
    for (int i = warp; i < n; i += kJoinThreads / 32)
#pragma unroll
        for (int nt = 0; nt < NT; nt++)
#pragma unroll
            for (int e = 0; e < 2; e++) {
                const int c = 8 * nt + 2 * t + e;
                if (c < cols) m[nt][e] = fmaxf(m[nt][e], __ldg(part + i * step + kRegs * 32 + 2 * c));
            }
#pragma unroll
    for (int k = 0; k < kPart; k++) y[k] = 0.0f;
#pragma unroll 4
    for (int i = warp; i < n; i += kJoinThreads / 32) {
        const float* q = part + i * step;
        float f[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; nt++)
#pragma unroll
            for (int e = 0; e < 2; e++) {
                const int c = 8 * nt + 2 * t + e;
                f[nt][e] = 0.0f;
                if (c < cols) {
                    f[nt][e] = fast_exp2(__ldg(q + kRegs * 32 + 2 * c) - m[nt][e]);
                    l[nt][e] = fmaf(f[nt][e], __ldg(q + kRegs * 32 + 2 * c + 1), l[nt][e]);
                }
            }
#pragma unroll
        for (int k = 0; k < kPart; k++) {
            const int r = blockIdx.z * kPart + k;
            const float w = f[NT == 1 ? 0 : r / (kRegs / NT)][k & 1];
            if (8 * (r / (kRegs / NT)) + 2 * t + (k & 1) < cols) y[k] = fmaf(w, __ldg(q + r * 32 + lane), y[k]);
        }
    }
#pragma unroll
    for (int k = 0; k < kPart; k++) acc[warp][k][lane] = y[k];
    if (lane < 4)
#pragma unroll
        for (int nt = 0; nt < NT; nt++)
#pragma unroll
            for (int e = 0; e < 2; e++) { top[warp][8 * nt + 2 * t + e] = m[nt][e]; norm[warp][8 * nt + 2 * t + e] = l[nt][e]; }
    __syncthreads();
    for (int i = threadIdx.x; i < kPart * 32; i += kJoinThreads) {
        const int k = i / 32, ln = i & 31, r = blockIdx.z * kPart + k;
        int c, col;
        place<POOL, D>(r, ln, &c, &col);
        if (col >= cols) continue;
        float mx = kNoMax, sum = 0.0f, v = 0.0f;
        for (int w = 0; w < kJoinThreads / 32; w++) mx = fmaxf(mx, top[w][col]);
        for (int w = 0; w < kJoinThreads / 32; w++) {
            const float f = fast_exp2(top[w][col] - mx);
            sum = fmaf(f, norm[w][col], sum);
            v = fmaf(f, acc[w][k][ln], v);
        }
        store_out<POOL, D>(p, first, h, r, ln, cols, sum != 0.0f ? v / sum : 0.0f);
    }
}

}  // namespace patchkv
