// Attention of few query columns: the cache is split over the grid along the tokens and read once.
//
// A column is a (row, query head of one KV head) pair; up to 16 of them ride on one pass over a KV head.
// Both products run on warp-level mma with the cache as the M side, so a cached number becomes a matrix operand once and
// all columns use it: logits^T[16 tokens][columns] = K * q^T, out^T[channels][columns] += V^T * p^T.  The matrix pipe is
// far from its limit here (31 % with 8 columns); what bounds the kernel is the bytes of the cache and, for 4-bit pages, the instructions
// that turn codes into operands, which is where the work below went.  (tcgen05 with 128 tokens as its M side and 8 or 16
// columns as N would take the same operands from shared memory; it has not been tried.)
//
// Codes as operands.  The bit pattern u < 2048 is the half u * 2^-24, so a code plus its offset (u = q + 8 or q + 128) is an exact
// operand once it stands in the low bits of its half: one logic instruction per register.  (e4m3 operands would take half
// of those, two per 8 codes, with q as a sum of two or three e4m3 numbers; but an e4m3 mma here turns its operands into halves
// with instructions of its own: 580 instructions a tile instead of 480, measured.)
//   K: q is fp16 (bf16 has fewer bits), scaled by a power of two per column, so what is lost lies 2^-24 below the column's
//      largest; each 32-channel chunk is summed on its own in fp32 from a start value that takes the offset out again (-8 * sum of
//      the chunk's q), then enters the logit with the token's fp32 scale: no rounding of K at all.
//   V: v = (u * 2^-24) * S - offset * S in one half fma, S the token's scale times a power of two that follows the
//      V scales: one rounding, of 2^-12, as p's own to fp16, or of 2^-25 where v is subnormal.  For the latter to stay below
//      2^-12 of a group's largest value S has to be 2^8 at least (8-bit codes: 2^4), and it is 2^15 at most: the power of two
//      moves both ways, and a tile whose scales have a wider range goes through again for the smaller ones.
//   p: where its rounding would be as large as the result's own, for fp16 results and over bf16 pages, it is the sum of two such
//      numbers, for one more product per operand (bf16 pages, 8 x 16k tokens: 2.0e-3 -> 1.7e-3 off, which is the result's rounding, 99.1 ->
//      99.3 us; the matrix pipe has room).
// Softmax on powers of two against a reference that is only moved when a logit exceeds it by more than 15 (p <= 2^15), to 3 below
// the largest (fp16 then holds weights down to 2^-17 of it to all its bits): one vote per tile instead of a maximum across lanes.
#pragma once

#include "attention.cuh"

namespace patchkv {

constexpr int kTile = 16;                       // tokens a warp takes at a time: one mma K (M) step
constexpr float kNoMax = -3.0e38f;
constexpr float kSplitTop = 15.0f, kSplitPeak = 3.0f;   // logits reach that far above the reference at most; it is put that far below the largest

// What the combine kernel needs of a split launch, and where partial results lie.
struct SplitPlan {
    float* partial;                             // [item][head]: [registers][32 lanes], then (m, l) per column
    int32_t* items;                             // per sequence: first item, number of items
    int32_t item_stride;                        // floats per (item, head)
    int32_t max_items;                          // grid bound
    int32_t target;                             // pieces the whole batch is cut into (0: one piece per sequence, no combine)
    int32_t heads_log2, per_head_log2;          // heads of a CTA, warps that share a head's tiles: powers of two
    uint32_t share_magic;                       // row of a column n < 16: n * share_magic >> 16
};
// The split kernels for head dimension D (64, 128) and 4 * nc columns, and the join where there is one (attention_split_launch.cuh).
template <int D>
cudaError_t launch_split(const AttentionParams& p, const SplitPlan& pl, int nc, int groups, cudaStream_t s);

// Warps and ring depth of the kernels: sixteen warps hide the latency of the page look-ups and of the operand
// work best where 128 registers a thread are enough (8 columns), the ring takes what shared memory is left.
constexpr int split_warps(bool pool, int nc) { return !pool && nc <= 2 ? 16 : 8; }

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
// d = a * b + {c0, c1, c0, c1}: the start values of the two columns.
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1, float c0, float c1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%10,%11};"
                 : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(c0), "f"(c1));
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
// (w & MASK) ^ flip in one instruction (the compiler makes two of it when both are constants).
template <uint32_t MASK>
__device__ __forceinline__ uint32_t and_xor(uint32_t w, uint32_t flip) {
    uint32_t d;
    asm("lop3.b32 %0, %1, %2, %3, 0x6A;" : "=r"(d) : "r"(w), "n"(MASK), "r"(flip));
    return d;
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
__device__ __forceinline__ uint32_t add_u16x2(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("add.u16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __forceinline__ uint32_t both(float x) { return half2_bits(x, x); }
__device__ __forceinline__ float exp2i(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }   // -126 <= e <= 127
__device__ __forceinline__ float low_half(uint32_t x) {
    float y;
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tcvt.f32.f16 %0, l;\n\t}" : "=f"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ float high_half(uint32_t x) {
    float y;
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tcvt.f32.f16 %0, h;\n\t}" : "=f"(y) : "r"(x));
    return y;
}

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
// Smallest and largest position of the first max_rows of a sequence's rows, those below 0 left out: they see nothing, and a window
// need not reach back for them.  `least`: the smallest of all, but -1 for any below (a tile needs its mask then).
__device__ __forceinline__ void position_range(const AttentionParams& p, int s, int first, int rows, int* lo, int* hi, int* least) {
    const int n = min(rows, p.b.max_rows);
    if (!p.b.pos) {
        const int a = p.b.kv_len[s] - rows;
        *least = max(-1, a);
        *lo = max(0, a);
        *hi = a + n - 1;
        return;
    }
    uint32_t low = 0x7FFFFFFF;                               // below 0 is above that
    *least = 0x7FFFFFFF;
    *hi = -1;
#pragma unroll 1
    for (int i = 0; i < n; i++) {
        const int x = p.b.pos[first + i];
        low = min(low, (uint32_t)x);
        *least = min(*least, x);
        *hi = max(*hi, x);
    }
    *lo = (int)low;
    *least = max(-1, *least);
}

// ---------------------------------------------------------------------------------------------------------------------
// Column n of a KV head is number e = (n / 4) & 1 of lane column t = n % 4 in the n / 8-th eight: an accumulator's columns 2t and
// 2t + 1 are n = 4e + t.  (Four query heads per KV head then fill every lane once.)  NC: columns of a lane, 1, 2 or 4.
__device__ __forceinline__ int column_of(int nc, int t) { return 8 * (nc >> 1) + 4 * (nc & 1) + t; }

// KF / VF: page formats (both FMT_BF16 for the bf16 pool); G32: one scale per 32 channels (else G is 64 or 128).
template <int KF, int VF, int D, int NC, int STAGES, int WARPS, bool G32>
struct SplitKernel {
    static constexpr bool kPool = KF == FMT_BF16, kK4 = KF == FMT_INT4;
    static constexpr int NT = (NC + 1) / 2;                                                 // column tiles of the mma
    static constexpr int kKRow = KF == FMT_BF16 ? 2 * D : (KF == FMT_INT8 ? D : D / 2);     // bytes of a head's row
    static constexpr int kVRow = VF == FMT_BF16 ? 2 * D : (VF == FMT_INT8 ? D : D / 2);
    static constexpr int kKStride = kKRow + 16, kVStride = kVRow + 16;                      // bank-conflict-free for every access below
    static constexpr int kV = kTile * kKStride, kScales = kV + kTile * kVStride;
    static constexpr int kStage = kScales + (kPool ? 0 : 2 * kTile * 8);                    // 8 bytes of scales per token, K then V
    static constexpr int kChunks = D / 32, kMT = D / 16;
    static constexpr int kRegs = (NC == 1 ? 2 : 4 * NT) * kMT;                              // accumulators of a lane that hold a column
    static constexpr int kCold = 4 * (12 + 4 * NC);                                         // a warp's numbers that only masks need
    static constexpr int kSmem = WARPS * (STAGES * kStage + kCold);
    static constexpr int kMerge = WARPS * (kRegs * 32 + 2 * 4 * NC) * 4;                    // the warps' results, in the same memory

    const AttentionParams& p;
    uint32_t ring;
    int lane, g, t;
    uint32_t qf[NT][kMT][2];
    float bias[kPool ? 1 : NT][kPool ? 1 : kChunks][2];
    float factor[NC], ref[NC], sum[NC];
    float acc[NT][kMT][4];
    uint32_t v_up0, v_up1, v_most;              // V scales are multiplied by a power of two: two halves, and the bits of the first scale too large for it
    uint32_t cold;                              // shared memory: kv, smallest and largest position (not below 0), and the positions of the columns
    uint32_t k_off, v_off, s_off;               // the lane's places in a tile's rows, relative to its first
    uint32_t flip0, flip1;                      // 8 in every half's low nibble, 8 in the next one (constants the compiler must keep in registers)

    __device__ __forceinline__ SplitKernel(const AttentionParams& p_) : p(p_) {}

    // 128 registers a thread are what sixteen warps leave: what only tiles with a mask need lives in shared memory.
    __device__ __forceinline__ int kv() const { return (int)lds32(cold); }
    __device__ __forceinline__ int lo_pos() const { return (int)lds32(cold + 4); }
    __device__ __forceinline__ int lo_whole() const { return (int)lds32(cold + 28); }       // lo_pos, or -1 with a row below 0
    __device__ __forceinline__ int hi_pos() const { return (int)lds32(cold + 8); }
    __device__ __forceinline__ int pos(int c) const { return (int)lds32(cold + 48 + 4 * column_of(c, t)); }
    // First token of the warp's tile i.
    __device__ __forceinline__ int first_token(int i) const {
        const int v = (int)lds32(cold + 12) + (i << lds32(cold + 16)), sinks = (int)lds32(cold + 20);
        return (v < sinks ? v : (int)lds32(cold + 24) + v - sinks) * kTile;
    }
    // Whether one of the rows sees a token of the tile: rows at given positions may lie further apart than the window, or behind the
    // cache's end.
    __device__ __forceinline__ bool some_row_sees(int t0) const {
        if (!p.b.pos || p.window == 0 || t0 < p.sinks) return true;
        const int last = min(t0 + kTile, kv()) - 1;
        bool seen = false;
#pragma unroll 1
        for (int c = 0; c < 4 * NC; c++) {
            const int x = (int)lds32(cold + 48 + 4 * c);
            seen = seen || (x >= t0 && x - last < p.window);
        }
        return seen;
    }
    __device__ __forceinline__ const int32_t* table() const {
        const uint2 x = lds64(cold + 32);
        return reinterpret_cast<const int32_t*>((uint64_t)x.y << 32 | x.x);
    }
    __device__ __forceinline__ int v_exp() const { return 30 - (int)(v_most >> 10); }
    __device__ __forceinline__ int scales_per_row() const { return G32 ? kChunks : D / p.c.G; }

    __device__ __forceinline__ void start(int lane_, uint32_t ring_, uint32_t cold_) {
        lane = lane_; g = lane >> 2; t = lane & 3; ring = ring_; cold = cold_;
        constexpr int kc = kKRow / 16, vc = kVRow / 16;       // 16-byte chunks of a row, a power of two
        k_off = (lane / kc) * p.c.H * kKRow + (lane % kc) * 16;
        v_off = (lane / vc) * p.c.H * kVRow + (lane % vc) * 16;
        if (!kPool) {
            s_off = (lane & 15) * p.c.H * scales_per_row() * 2 + (lane < 16 ? p.c.k_scales : p.c.v_scales);
            v_off += p.c.v_codes;
        }
        set_v_exp(29);
        asm volatile("mov.b32 %0, 0x00080008;" : "=r"(flip0));
        asm volatile("mov.b32 %0, 0x00800080;" : "=r"(flip1));
#pragma unroll
        for (int c = 0; c < NC; c++) { ref[c] = kNoMax; sum[c] = 0.0f; }
#pragma unroll
        for (int nt = 0; nt < NT; nt++)
#pragma unroll
            for (int i = 0; i < kMT; i++)
#pragma unroll
                for (int j = 0; j < 4; j++) acc[nt][i][j] = 0.0f;
    }
    __device__ __forceinline__ void set_v_exp(int e) {       // -1 <= e <= 29: exact
        v_up0 = both(exp2i(min(e, 15)));
        v_up1 = both(exp2i(max(e - 15, 0)));
        v_most = (uint32_t)(30 - e) << 10;                   // exponent field x: s < 2^(x - 14), so s * 2^e stays at 2^15 at most
    }

    // Asks for the queries: 32-bit words of column n = column_of(2 nt + (g & 1), g / 2), into the operands' own registers.
    __device__ __forceinline__ void ask_queries(int first, int cols, int head, uint32_t share_magic) {
#pragma unroll
        for (int nt = 0; nt < NT; nt++) {
            const int n = column_of(2 * nt + (g & 1), g >> 1), row = (int)(n * share_magic >> 16);
            const bool live = n < cols && (g & 1) < NC;
            const uint16_t* q = p.q + (long long)(first + row) * p.q_stride_row + (long long)(head * p.share + n - row * p.share) * p.q_stride_head;
            if constexpr (kPool) {
#pragma unroll
                for (int k = 0; k < kMT; k++)
#pragma unroll
                    for (int e = 0; e < 2; e++) qf[nt][k][e] = live ? *reinterpret_cast<const uint32_t*>(q + 16 * k + 8 * e + 2 * t) : 0u;
            } else {
#pragma unroll
                for (int j = 0; j < kChunks; j++) {           // 8 channels of each chunk, in the order the codes of a word come out
                    uint4 v = make_uint4(0, 0, 0, 0);
                    if (live) {
                        if (kK4) {
                            v = *reinterpret_cast<const uint4*>(q + 32 * j + 8 * t);
                        } else {
                            const uint2 a = *reinterpret_cast<const uint2*>(q + 32 * j + 4 * t);
                            const uint2 b = *reinterpret_cast<const uint2*>(q + 32 * j + 16 + 4 * t);
                            v = make_uint4(a.x, a.y, b.x, b.y);
                        }
                    }
                    qf[nt][2 * j][0] = v.x; qf[nt][2 * j][1] = v.y; qf[nt][2 * j + 1][0] = v.z; qf[nt][2 * j + 1][1] = v.w;
                }
            }
        }
    }
    // Queries as B operands, and the per-column numbers of the lane's logit columns.
    __device__ __forceinline__ void load_queries() {
#pragma unroll
        for (int nt = 0; nt < NT; nt++) {
            if constexpr (kPool) {
                factor[2 * nt] = p.scale_log2;
                if (NC > 1) factor[2 * nt + (NC > 1)] = p.scale_log2;
            } else {
                uint32_t w[kChunks][4];
#pragma unroll
                for (int j = 0; j < kChunks; j++) {
                    w[j][0] = qf[nt][2 * j][0]; w[j][1] = qf[nt][2 * j][1]; w[j][2] = qf[nt][2 * j + 1][0]; w[j][3] = qf[nt][2 * j + 1][1];
                }
                // Largest magnitude (ordered as the bit patterns are) into [2^13, 2^14); zeros as they are.  A column with a NaN or an
                // infinity has no result but NaN: its factor is NaN.
                uint32_t most = 0;
#pragma unroll
                for (int j = 0; j < kChunks; j++)
#pragma unroll
                    for (int i = 0; i < 4; i++) most = __vmaxu2(most, w[j][i] & 0x7FFF7FFFu);
                most = max(most & 0xFFFFu, most >> 16);
                most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, 1));
                most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, 2));
                const bool bad = most >= (p.f16 ? 0x7C00u : 0x7F80u);
                const float amax = p.f16 ? half_bits_to_float(most) : bf16_bits_to_float(most);
                const int shift = most == 0 ? 0 : min(13 - ((int)(__float_as_uint(amax) >> 23) - 127), 120);
                const float up = bad ? 0.0f : exp2i(shift);
                const float down = bad ? __uint_as_float(0x7FC00000u) : p.scale_log2 * exp2i(-shift) * 16777216.0f;
#pragma unroll
                for (int j = 0; j < kChunks; j++) {
                    float x[8], a = 0.0f;
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        x[2 * i] = p.f16 ? low_half(w[j][i]) : __uint_as_float(w[j][i] << 16);
                        x[2 * i + 1] = p.f16 ? high_half(w[j][i]) : __uint_as_float(w[j][i] & 0xFFFF0000u);
                    }
                    if (bad)
#pragma unroll
                        for (int i = 0; i < 8; i++) x[i] = 0.0f;
#pragma unroll
                    for (int i = 0; i < 8; i++) { x[i] *= up; a += x[i]; }
#pragma unroll
                    for (int m = 0; m < 2; m++) {
                        uint32_t* f = qf[nt][2 * j + m];
                        if (kK4) {                            // nibbles of a word: (0, 4) (1, 5) / (2, 6) (3, 7), odd ones 16 times up
                            f[0] = half2_bits(x[2 * m], x[2 * m + 4]);
                            f[1] = half2_bits(x[2 * m + 1] * 0.0625f, x[2 * m + 5] * 0.0625f);
                        } else {
                            f[0] = half2_bits(x[4 * m], x[4 * m + 1]);
                            f[1] = half2_bits(x[4 * m + 2], x[4 * m + 3]);
                        }
                    }
                    // the chunk's sum (what rounding to half took away lies 2^-25 below the largest)
                    a += __shfl_xor_sync(0xFFFFFFFFu, a, 1);
                    a += __shfl_xor_sync(0xFFFFFFFFu, a, 2);
                    a *= kK4 ? -4.76837158203125e-07f : -7.62939453125e-06f;        // -8 * 2^-24, -128 * 2^-24
                    bias[nt][j][0] = __shfl_sync(0xFFFFFFFFu, a, 8 * t);
                    bias[nt][j][1] = __shfl_sync(0xFFFFFFFFu, a, 8 * t + 4);
                }
                factor[2 * nt] = __shfl_sync(0xFFFFFFFFu, down, 8 * t);
                if (NC > 1) factor[2 * nt + (NC > 1)] = __shfl_sync(0xFFFFFFFFu, down, 8 * t + 4);
            }
        }
    }

    // Enqueues a tile into the stage at `base`: `at` is the place of its page (of a pool: of its first token), in bytes; row0 its first
    // (token, head) row there, H apart per token.  A token that no row sees is filled with zeros (of quantised pages: its
    // scales), and so is a tile without a page: nothing of its slot takes part.
    __device__ __forceinline__ void fetch(uint32_t base, long long at, uint32_t row0, bool whole, bool present, int t0) {
        if constexpr (kPool) {
            constexpr int kc = kKRow / 16;
            const uint8_t* k = reinterpret_cast<const uint8_t*>(p.c.k) + at + (lane % kc) * 16;
            const uint8_t* v = reinterpret_cast<const uint8_t*>(p.c.v) + at + (lane % kc) * 16;
            const uint32_t dst = base + (lane / kc) * kKStride + (lane % kc) * 16;
#pragma unroll
            for (int i = 0; i < kTile * kc / 32; i++) {
                const int tok = lane / kc + i * (32 / kc);
                const bool live = whole || (present && t0 + tok <= min(hi_pos(), kv() - 1) && sees(p, lo_pos(), t0 + tok));
                const long long o = live ? 2 * tok * p.c.stride_token : 0;
                cp16(dst + i * (32 / kc) * kKStride, k + o, live);
                cp16(dst + kV + i * (32 / kc) * kVStride, v + o, live);
            }
        } else {
            const uint8_t* pg = p.c.base + at;
            constexpr int kc = kKRow / 16, vc = kVRow / 16;
            const uint8_t* ks = pg + (row0 * kKRow + k_off);
            const uint8_t* vs = pg + (row0 * kVRow + v_off);
            const uint8_t* sc = pg + (row0 * (uint32_t)scales_per_row() * 2 + s_off);
            const uint32_t kd = base + (lane / kc) * kKStride + (lane % kc) * 16, vd = base + kV + (lane / vc) * kVStride + (lane % vc) * 16;
            const uint32_t sd = base + kScales + lane * 8;
            bool live = true, all = true;
            if (!whole) {
                const int tok = t0 + (lane & 15);
                live = present && tok <= min(hi_pos(), kv() - 1) && sees(p, lo_pos(), tok);
                all = present;
            }
#pragma unroll
            for (int i = 0; i < kTile * kc / 32; i++) cp16(kd + i * (32 / kc) * kKStride, ks + i * (32 / kc) * kKRow * p.c.H, all);
#pragma unroll
            for (int i = 0; i < kTile * vc / 32; i++) cp16(vd + i * (32 / vc) * kVStride, vs + i * (32 / vc) * kVRow * p.c.H, all);
            if (D == 128 && G32) cp_small<8>(sd, sc, live);
            else cp_small<4>(sd, reinterpret_cast<const uint8_t*>(reinterpret_cast<uintptr_t>(sc) & ~(uintptr_t)3), live);   // a lone fp16: its word, picked apart below
        }
    }

    // Scale of 32-channel chunk j from a token's 8 bytes.
    __device__ __forceinline__ float chunk_scale(const uint2& s, int j, uint32_t odd) const {
        if (G32) return j & 1 ? high_half(j < 2 ? s.x : s.y) : low_half(j < 2 ? s.x : s.y);
        const int i = p.c.G == D ? (int)odd : j * 32 / p.c.G;
        return i ? high_half(s.x) : low_half(s.x);
    }

    __device__ __forceinline__ void rescale(int c, float to) {
        const float keep = fast_exp2(ref[c] - to);
        ref[c] = to;
        sum[c] *= keep;
#pragma unroll
        for (int i = 0; i < kMT; i++) { acc[c >> 1][i][c & 1] *= keep; acc[c >> 1][i][2 + (c & 1)] *= keep; }
    }

    // V scales of one pass have bit patterns in [v_most - kSpread, v_most): S in [2^8, 2^15), or [2^4, 2^15) (file header).
    static constexpr int kSpread = (VF == FMT_INT8 ? 11 : 7) << 10;
    // Largest magnitude of four halves, and the smallest that is not zero, minus 1.
    __device__ __forceinline__ static void magnitudes(const uint32_t (&s)[2], uint32_t* top, int* low) {
        const uint32_t a = s[0] & 0x7FFF7FFFu, b = s[1] & 0x7FFF7FFFu, most = __vmaxu2(a, b);
        const uint32_t least = __vminu2(add_u16x2(a, 0xFFFFFFFFu), add_u16x2(b, 0xFFFFFFFFu));
        *top = max(most & 0xFFFFu, most >> 16);
        *low = (int)min(least & 0xFFFFu, least >> 16);
    }

    // One tile: logits, weights, and the weighted values.  `below`: 0, or the tile once more for its V scales below that bit pattern;
    // returns the next such, 0 when all are done.
    __device__ __forceinline__ uint32_t tile(uint32_t base, bool whole, bool present, int t0, uint32_t row0, uint32_t below) {
        float x[NC][2];                                                    // tokens g and g + 8
        if constexpr (kPool) {
            float y[NT][4];
#pragma unroll
            for (int nt = 0; nt < NT; nt++)
#pragma unroll
                for (int i = 0; i < 4; i++) y[nt][i] = 0.0f;
            const uint32_t a = base + ((lane & 7) + (lane & 8)) * kKStride + (lane >> 4) * 16;
#pragma unroll
            for (int k = 0; k < kMT; k++) {
                uint32_t r[4];
                ldmatrix4(r, a + 32 * k);
#pragma unroll
                for (int nt = 0; nt < NT; nt++) mma_bf16(y[nt], r[0], r[1], r[2], r[3], qf[nt][k][0], qf[nt][k][1]);
            }
#pragma unroll
            for (int c = 0; c < NC; c++) { x[c][0] = y[c >> 1][c & 1]; x[c][1] = y[c >> 1][2 + (c & 1)]; }
        } else {
            uint32_t odd_a = 0, odd_b = 0;
            if (!G32 && p.c.G == D) {                                      // which half of the word a lone scale is
                odd_a = (row0 + g * p.c.H) & 1;
                odd_b = (row0 + (g + 8) * p.c.H) & 1;
            }
            const uint2 sa = lds64(base + kScales + 8 * g), sb = lds64(base + kScales + 8 * (g + 8));
            const uint32_t ra = base + g * kKStride + 4 * t, rb = ra + 8 * kKStride;
#pragma unroll
            for (int j = 0; j < kChunks; j++) {
                float y[NT][4];
                if constexpr (kK4) {
                    uint32_t wa = lds32(ra + 16 * j), wb = lds32(rb + 16 * j);
#pragma unroll
                    for (int m = 0; m < 2; m++) {
                        const uint32_t a0 = and_xor<0x000F000Fu>(wa, flip0), a1 = and_xor<0x000F000Fu>(wb, flip0);
                        const uint32_t a2 = and_xor<0x00F000F0u>(wa, flip1), a3 = and_xor<0x00F000F0u>(wb, flip1);
#pragma unroll
                        for (int q = 0; q < NT; q++) {
                            if (m == 0) mma_f16(y[q], a0, a1, a2, a3, qf[q][2 * j][0], qf[q][2 * j][1], bias[q][j][0], bias[q][j][1]);
                            else mma_f16(y[q], a0, a1, a2, a3, qf[q][2 * j + 1][0], qf[q][2 * j + 1][1]);
                        }
                        if (m == 0) { wa >>= 8; wb >>= 8; }
                    }
                } else {
#pragma unroll
                    for (int m = 0; m < 2; m++) {
                        const uint32_t wa = lds32(ra + 32 * j + 16 * m) ^ 0x80808080u, wb = lds32(rb + 32 * j + 16 * m) ^ 0x80808080u;
                        const uint32_t a0 = __byte_perm(wa, 0, 0x4140), a1 = __byte_perm(wb, 0, 0x4140);
                        const uint32_t a2 = __byte_perm(wa, 0, 0x4342), a3 = __byte_perm(wb, 0, 0x4342);
#pragma unroll
                        for (int q = 0; q < NT; q++) {
                            if (m == 0) mma_f16(y[q], a0, a1, a2, a3, qf[q][2 * j][0], qf[q][2 * j][1], bias[q][j][0], bias[q][j][1]);
                            else mma_f16(y[q], a0, a1, a2, a3, qf[q][2 * j + 1][0], qf[q][2 * j + 1][1]);
                        }
                    }
                }
                const float fa = chunk_scale(sa, j, odd_a), fb = chunk_scale(sb, j, odd_b);
#pragma unroll
                for (int c = 0; c < NC; c++) {
                    const float ya = y[c >> 1][c & 1], yb = y[c >> 1][2 + (c & 1)];
                    x[c][0] = j ? fmaf(ya, fa, x[c][0]) : ya * fa;
                    x[c][1] = j ? fmaf(yb, fb, x[c][1]) : yb * fb;
                }
            }
        }
#pragma unroll
        for (int c = 0; c < NC; c++) { x[c][0] *= factor[c]; x[c][1] *= factor[c]; }
        if (!whole)
#pragma unroll
            for (int c = 0; c < NC; c++)
#pragma unroll
                for (int i = 0; i < 2; i++) {
                    const int tok = t0 + g + 8 * i, ps = pos(c);
                    if (!(present && tok <= ps && tok < kv() && sees(p, ps, tok))) x[c][i] = -INFINITY;
                }
        float most = kNoMax;
#pragma unroll
        for (int c = 0; c < NC; c++) most = fmaxf(most, fmaxf(x[c][0], x[c][1]) - ref[c]);
        // V scales of the lane's channels (one group: channels [g * D / 8, (g + 1) * D / 8)) for tokens 2t, 2t+1, 2t+8, 2t+9
        uint32_t sp[2] = {0, 0}, top = 0, next = 0;
        int low = 0;
        if constexpr (!kPool) {
            uint32_t s[4];
            const int group = g * (D / 8) / (G32 ? 32 : p.c.G);
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const int tok = 2 * t + (i & 1) + 8 * (i >> 1);
                uint32_t at = base + kScales + 128 + 8 * tok + 2 * group;
                if (!G32 && p.c.G == D) at += 2 * ((row0 + tok * p.c.H) & 1);
                s[i] = lds16(at);
            }
            sp[0] = s[0] | s[1] << 16;
            sp[1] = s[2] | s[3] << 16;
            magnitudes(sp, &top, &low);
        }
        // One vote for the two references that may have to move.
        if (__any_sync(0xFFFFFFFFu, most > kSplitTop || (!kPool && (top >= v_most || low < (int)v_most - kSpread || below)))) {
#pragma unroll
            for (int c = 0; c < NC; c++) {
                float m = fmaxf(x[c][0], x[c][1]);
                m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 4));
                m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 8));
                m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 16));
                if (m > ref[c] + kSplitTop) rescale(c, m - kSplitPeak);
            }
            if constexpr (!kPool) {
                if (below) {                                        // the weights are in the sums already
#pragma unroll
                    for (int c = 0; c < NC; c++) sum[c] -= fast_exp2(x[c][0] - ref[c]) + fast_exp2(x[c][1] - ref[c]);
#pragma unroll
                    for (int k = 0; k < 2; k++) sp[k] &= __vcmpltu2(sp[k] & 0x7FFF7FFFu, below * 0x00010001u);
                    magnitudes(sp, &top, &low);
                }
                const uint32_t m = __reduce_max_sync(0xFFFFFFFFu, top >= 0x7C00u ? 0u : top);   // a scale that is not finite always gets here
                if (m >= v_most || (m && __any_sync(0xFFFFFFFFu, low < (int)v_most - kSpread))) {
                    const int from = v_exp(), to = 29 - (int)(m >> 10);
                    const float keep = exp2i(to - from);
                    set_v_exp(to);
#pragma unroll
                    for (int nt = 0; nt < NT; nt++)
#pragma unroll
                        for (int i = 0; i < kMT; i++)
#pragma unroll
                            for (int k = 0; k < 4; k++) acc[nt][i][k] *= keep;
                }
                if (__any_sync(0xFFFFFFFFu, low < (int)v_most - kSpread)) {
                    next = v_most - kSpread;
#pragma unroll
                    for (int k = 0; k < 2; k++) sp[k] &= __vcmpgeu2(sp[k] & 0x7FFF7FFFu, next * 0x00010001u);
                }
            }
        }
        uint32_t pf[NT][2], pr[NT][2];                              // weights, and where that shows what their rounding took
        const bool fine = kPool || p.f16;
#pragma unroll
        for (int c = 0; c < NC; c++) {
#pragma unroll
            for (int i = 0; i < 2; i++) x[c][i] = fast_exp2(x[c][i] - ref[c]);
            sum[c] += x[c][0] + x[c][1];
        }
#pragma unroll
        for (int nt = 0; nt < NT; nt++)
#pragma unroll
            for (int i = 0; i < 2; i++) {
                const float lo = x[2 * nt][i], hi = NC > 1 ? x[(2 * nt + 1) % NC][i] : 0.0f;
                const uint32_t w = kPool ? bf162_bits(lo, hi) : half2_bits(lo, hi);
                pf[nt][i] = transpose8x8(w);
                pr[nt][i] = 0;
                if constexpr (kPool) pr[nt][i] = transpose8x8(bf162_bits(lo - __uint_as_float(w << 16), hi - __uint_as_float(w & 0xFFFF0000u)));
                else if (fine) pr[nt][i] = transpose8x8(half2_bits(lo - low_half(w), hi - high_half(w)));
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
                if (__any_sync(0xFFFFFFFFu, bad != 0)) { values_one_by_one(base, x, 0u); return 0; }
            }
#pragma unroll
            for (int i = 0; i < kMT; i++) {
                uint32_t r[4];
                ldmatrix4_trans(r, a + 32 * i);
#pragma unroll
                for (int nt = 0; nt < NT; nt++) {
                    mma_bf16(acc[nt][i], r[0], r[1], r[2], r[3], pf[nt][0], pf[nt][1]);
                    mma_bf16(acc[nt][i], r[0], r[1], r[2], r[3], pr[nt][0], pr[nt][1]);
                }
            }
        } else {
            if (!whole && __any_sync(0xFFFFFFFFu, top >= 0x7C00u)) { values_one_by_one(base, x, row0); return 0; }
            uint32_t S[2], S16[2], off[2];
#pragma unroll
            for (int k = 0; k < 2; k++) {
                S[k] = hmul2(hmul2(sp[k], v_up0), v_up1);
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
                            const uint32_t a0 = hfma2(and_xor<0x000F000Fu>(a, flip0), S[0], off[0]);
                            const uint32_t a1 = hfma2(and_xor<0x00F000F0u>(a, flip1), S16[0], off[0]);
                            const uint32_t a2 = hfma2(and_xor<0x000F000Fu>(b, flip0), S[1], off[1]);
                            const uint32_t a3 = hfma2(and_xor<0x00F000F0u>(b, flip1), S16[1], off[1]);
#pragma unroll
                            for (int nt = 0; nt < NT; nt++) {
                                mma_f16(acc[nt][4 * k + 2 * h + m], a0, a1, a2, a3, pf[nt][0], pf[nt][1]);
                                if (fine) mma_f16(acc[nt][4 * k + 2 * h + m], a0, a1, a2, a3, pr[nt][0], pr[nt][1]);
                            }
                            a >>= 8; b >>= 8;
                        }
                    } else {
                        const uint32_t a0 = hfma2(and_xor<0x00FF00FFu>(a, flip1), S[0], off[0]);
                        const uint32_t a1 = hfma2(and_xor<0x00FF00FFu>(a >> 8, flip1), S[0], off[0]);
                        const uint32_t a2 = hfma2(and_xor<0x00FF00FFu>(b, flip1), S[1], off[1]);
                        const uint32_t a3 = hfma2(and_xor<0x00FF00FFu>(b >> 8, flip1), S[1], off[1]);
#pragma unroll
                        for (int nt = 0; nt < NT; nt++) {
                            mma_f16(acc[nt][2 * k + h], a0, a1, a2, a3, pf[nt][0], pf[nt][1]);
                            if (fine) mma_f16(acc[nt][2 * k + h], a0, a1, a2, a3, pr[nt][0], pr[nt][1]);
                        }
                    }
                }
            }
        }
        return next;
    }

    // Channel of accumulator (i, e) of this lane.
    __device__ __forceinline__ int channel(int i, int e) const { return kPool ? 16 * i + 8 * e + g : g * (D / 8) + 2 * i + e; }

    // The rare tile with values that are not finite, some of them unseen by some rows: every weight that is not zero times its value.
    __device__ __forceinline__ void values_one_by_one(uint32_t base, float (&x)[NC][2], uint32_t row0) {
#pragma unroll 1
        for (int tok = 0; tok < kTile; tok++) {
            float w[NC];
#pragma unroll
            for (int c = 0; c < NC; c++) {
                const float a = __shfl_sync(0xFFFFFFFFu, x[c][0], (tok & 7) * 4 + t);
                const float b = __shfl_sync(0xFFFFFFFFu, x[c][1], (tok & 7) * 4 + t);
                w[c] = tok < 8 ? a : b;
            }
#pragma unroll
            for (int i = 0; i < kMT; i++)
#pragma unroll
                for (int e = 0; e < 2; e++) {
                    const int ch = channel(i, e);
                    float v;
                    if (kPool) {
                        v = bf16_bits_to_float(lds16(base + kV + tok * kVStride + 2 * ch));
                    } else {
                        uint32_t at = base + kScales + 128 + 8 * tok + 2 * (ch / (G32 ? 32 : p.c.G));
                        if (!G32 && p.c.G == D) at += 2 * ((row0 + tok * p.c.H) & 1);
                        const uint32_t byte = base + kV + tok * kVStride + (VF == FMT_INT8 ? ch : ch >> 1);
                        uint32_t u = lds32(byte & ~3u) >> ((byte & 3u) * 8);
                        if (VF == FMT_INT4) u = ((u >> ((ch & 1) * 4)) & 15u) ^ 8u; else u = (u & 255u) ^ 128u;
                        v = ((float)u - (VF == FMT_INT4 ? 8.0f : 128.0f)) * half_bits_to_float(lds16(at)) * 5.9604644775390625e-08f * exp2i(v_exp());
                    }
#pragma unroll
                    for (int c = 0; c < NC; c++)
                        if (w[c] != 0.0f) acc[c >> 1][i][2 * e + (c & 1)] = fmaf(w[c], v, acc[c >> 1][i][2 * e + (c & 1)]);
                }
        }
    }
};

// Register r of the stored results (accumulators that hold a column, in order) of a lane: channel and column.
template <bool POOL, int D, int NC>
__device__ __forceinline__ void place(int r, int lane, int* channel, int* col) {
    const int g = lane >> 2, t = lane & 3, pairs = NC == 1 ? 1 : 2;
    const int f = NC == 1 ? 0 : r & 1, q = r / pairs, nt = q / (2 * (D / 16)), i = (q / 2) % (D / 16), e = q & 1;
    *channel = POOL ? 16 * i + 8 * e + g : g * (D / 8) + 2 * i + e;
    *col = 8 * nt + 4 * f + t;
}

__device__ __forceinline__ void store_out(const AttentionParams& p, uint32_t share_magic, int first, int head, int c, int n, float y) {
    const int row = (int)(n * share_magic >> 16);
    uint16_t* o = p.out + (long long)(first + row) * p.out_stride_row + (long long)(head * p.share + n - row * p.share) * p.out_stride_head + c;
    *o = (uint16_t)(p.f16 ? half2_bits(y, 0.0f) : bf162_bits(y, 0.0f));
}

// The piece of the batch that item `item` stands for: sequence and virtual tiles [begin, end).  All lanes of a warp agree.
// With a target, the batch's tiles are cut into about that many pieces of equal length, none across two sequences.
struct Item { int seq, split, splits, first_item, begin, end, first, rows, kv, lo, hi, least; bool ok; };
__device__ __forceinline__ Item find_item(const AttentionParams& p, const SplitPlan& pl, int item) {
    const int lane = threadIdx.x & 31;
    Item it;
    it.ok = false;
    it.splits = 1; it.split = 0; it.first_item = item;
    it.seq = p.b.n_seqs == 1 ? 0 : item;
    if (pl.target && p.b.n_seqs > 1) {
        // tiles of sequence s0 + lane; -1 for one without rows
        auto tiles_of = [&](int s0) {
            int first, kv, rows, lo, hi, least;
            if (s0 + lane >= p.b.n_seqs) return -1;
            if (!sequence_rows(p, s0 + lane, &first, &kv, &rows)) { if (item == 0) latch(p.status); return -1; }
            if (rows == 0) return -1;
            position_range(p, s0 + lane, first, rows, &lo, &hi, &least);
            return tile_range(p, kv, lo, hi).count;
        };
        int tiles = tiles_of(0), total = __reduce_add_sync(0xFFFFFFFFu, max(tiles, 0));
#pragma unroll 1
        for (int s0 = 32; s0 < p.b.n_seqs; s0 += 32) total += __reduce_add_sync(0xFFFFFFFFu, max(tiles_of(s0), 0));
        const int least = 1 << pl.per_head_log2;             // a piece gives every warp a tile
        const int piece = max((int)((uint32_t)(total + pl.target - 1) / (uint32_t)pl.target), least);
        int at = 0;
        it.seq = -1;
#pragma unroll 1
        for (int s0 = 0; s0 < p.b.n_seqs && it.seq < 0; s0 += 32) {
            if (s0) tiles = tiles_of(s0);
            const int n = tiles < 0 ? 0 : max(1, (int)((uint32_t)(tiles + piece - 1) / (uint32_t)piece));
            const int even = n ? (int)((uint32_t)(tiles + n - 1) / (uint32_t)n) : 0;      // the sequence's pieces of equal length
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
                const int length = __shfl_sync(0xFFFFFFFFu, even, src);
                it.begin = it.split * length;
                it.end = it.begin + length;
            }
            at += __shfl_sync(0xFFFFFFFFu, inc, 31);
        }
        if (it.seq < 0) return it;
    }
    const bool ordered = sequence_rows(p, it.seq, &it.first, &it.kv, &it.rows);
    if (lane == 0 && (!ordered || it.rows > p.b.max_rows || p.b.kv_len[it.seq] > it.kv)) latch(p.status);
    if (!ordered || it.rows == 0) return it;
    position_range(p, it.seq, it.first, it.rows, &it.lo, &it.hi, &it.least);
    it.rows = min(it.rows, p.b.max_rows);
    const int count = tile_range(p, it.kv, it.lo, it.hi).count;
    if (pl.target == 0) {
        it.begin = 0; it.end = count;
    } else if (p.b.n_seqs == 1) {                            // no search
        const int piece = max((int)((uint32_t)(count + pl.target - 1) / (uint32_t)pl.target), 1 << pl.per_head_log2);
        it.splits = max(1, (int)((uint32_t)(count + piece - 1) / (uint32_t)piece));
        if (item >= it.splits) return it;
        it.split = item;
        it.first_item = 0;
        it.begin = item * piece;
        it.end = it.begin + piece;
    }
    it.end = min(it.end, count);
    it.ok = true;
    return it;
}

template <int KF, int VF, int D, int NC, int STAGES, int WARPS, bool G32>
__global__ void __launch_bounds__(WARPS * 32) attention_split_kernel(const __grid_constant__ AttentionParams p, const __grid_constant__ SplitPlan pl) {
    using K = SplitKernel<KF, VF, D, NC, STAGES, WARPS, G32>;
    extern __shared__ __align__(16) uint8_t smem[];
    pdl_trigger();
    pdl_wait();
    // the warp's number through a shuffle: the compiler then knows that it is the same in all lanes
    const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    // One warp looks the piece up (sixteen at once would share its schedulers for three microseconds), the others read it.
    __shared__ Item found;
    if (warp == 0) {
        const Item x = find_item(p, pl, blockIdx.x);
        if (lane == 0) found = x;
    }
    __syncthreads();
    const Item it = found;
    if (!it.ok) return;
    const int heads = 1 << pl.heads_log2, local = warp & (heads - 1), sub = warp >> pl.heads_log2, head = blockIdx.y * heads + local;
    const bool live = head < p.c.H;
    const int cols = min(it.rows * p.share, 4 * NC);
    K k(p);
    k.start(lane, smem_u32(smem) + warp * STAGES * K::kStage, smem_u32(smem) + WARPS * STAGES * K::kStage + warp * K::kCold);
    if (live) {
        k.ask_queries(it.first, cols, head, pl.share_magic);
        const int step = 1 << pl.per_head_log2, n = it.begin + sub < it.end ? (it.end - it.begin - sub + step - 1) >> pl.per_head_log2 : 0;
        uint32_t* cold = reinterpret_cast<uint32_t*>(smem + WARPS * STAGES * K::kStage + warp * K::kCold);
        if (lane == 0) {
            const TileRange range = tile_range(p, it.kv, it.lo, it.hi);
            const uint64_t table = reinterpret_cast<uint64_t>(p.b.block_table + (long long)it.seq * p.b.table_stride);
            cold[0] = it.kv; cold[1] = it.lo; cold[2] = it.hi;
            cold[3] = it.begin + sub; cold[4] = pl.per_head_log2; cold[5] = range.sink_tiles; cold[6] = range.first;
            cold[7] = it.least;
            cold[8] = (uint32_t)table; cold[9] = (uint32_t)(table >> 32);
        }
        if (lane < 4 * NC) cold[12 + lane] = lane < cols ? row_position(p.b, it.seq, it.first + (int)(lane * pl.share_magic >> 16)) : -1;
        __syncwarp();
        // The warp's next 32 tiles, a lane each: place, first row and flags.  Whole tiles need no mask: seen by the earliest row and
        // inside the latest row's window, or among the sinks.
        struct Place { long long at; uint32_t row0, flags; };        // flags: bit 0 whole, bit 1 has a page
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
        // One copy of the tile's code, stage and all else in registers: the instruction cache is cold at every launch, and a
        // short context runs each instruction a few times only.
        uint32_t whole = 0, present = 0, odd = 0;            // bit j: flags (and row0 & 1) of the tile fetched j ago
        uint32_t fetch_base = k.ring, base = k.ring;
        auto fetch = [&](int i) {
            // i runs through 0, 1, 2 ...; `here` is the 32-block of i
            const uint32_t flags = __shfl_sync(0xFFFFFFFFu, here.flags, i & 31), row0 = __shfl_sync(0xFFFFFFFFu, here.row0, i & 31);
            const long long at = __shfl_sync(0xFFFFFFFFu, here.at, i & 31);
            if (i < n) k.fetch(fetch_base, at, row0, flags & 1, flags >> 1, flags & 1 ? 0 : k.first_token(i));
            cp_commit();
            if ((i & 31) == 31) here = place_of(i + 1 + lane);
            whole = whole << 1 | (flags & 1);
            present = present << 1 | flags >> 1;
            if (!G32) odd = odd << 1 | (row0 & 1);
            fetch_base = fetch_base == k.ring + (STAGES - 1) * K::kStage ? k.ring : fetch_base + K::kStage;
        };
#pragma unroll 1
        for (int i = 0; i < STAGES - 1; i++) fetch(i);
        k.load_queries();
#pragma unroll 1
        for (int i = 0; i < n; i++) {
            fetch(i + STAGES - 1);
            cp_wait<STAGES - 1>();
            __syncwarp();
            const bool w = whole >> (STAGES - 1) & 1;
            uint32_t below = 0;
            do below = k.tile(base, w, present >> (STAGES - 1) & 1, w ? 0 : k.first_token(i), odd >> (STAGES - 1) & 1, below);
            while (!K::kPool && below);
            __syncwarp();                                    // the stage may be filled again
            base = base == k.ring + (STAGES - 1) * K::kStage ? k.ring : base + K::kStage;
        }
        cp_wait<0>();
    }
    if (pl.target && it.split == 0 && blockIdx.y == 0 && threadIdx.x == 0) {
        pl.items[2 * it.seq] = it.first_item;
        pl.items[2 * it.seq + 1] = it.splits;
    }
    // V's power of two out of the result; l over the lanes.
    const float down = K::kPool ? 1.0f : 16777216.0f * exp2i(-k.v_exp());
#pragma unroll
    for (int c = 0; c < NC; c++) {
        k.sum[c] += __shfl_xor_sync(0xFFFFFFFFu, k.sum[c], 4);
        k.sum[c] += __shfl_xor_sync(0xFFFFFFFFu, k.sum[c], 8);
        k.sum[c] += __shfl_xor_sync(0xFFFFFFFFu, k.sum[c], 16);
    }
    // The warps of a head agree on a reference (m and l per column through shared memory), bring their results to it, and each
    // sums up its share of the registers, which lie as [warp][register][lane].
    float weight[NC];
    __syncthreads();                                         // the rings are done with
    float* res = reinterpret_cast<float*>(smem);
    float* ml = res + WARPS * K::kRegs * 32;
    if (lane < 4)
#pragma unroll
        for (int c = 0; c < NC; c++) *reinterpret_cast<float2*>(ml + (warp * 4 * NC + column_of(c, lane)) * 2) = make_float2(k.ref[c], k.sum[c]);
    __syncthreads();
    float m[NC], l[NC];
#pragma unroll
    for (int c = 0; c < NC; c++) {
        m[c] = k.ref[c];
        l[c] = 0.0f;
        const float* o = ml + (local * 4 * NC + column_of(c, k.t)) * 2;
        for (int w = 0; w < WARPS >> pl.heads_log2; w++) m[c] = fmaxf(m[c], o[(w << pl.heads_log2) * 8 * NC]);
        for (int w = 0; w < WARPS >> pl.heads_log2; w++)
            l[c] = fmaf(fast_exp2(o[(w << pl.heads_log2) * 8 * NC] - m[c]), o[(w << pl.heads_log2) * 8 * NC + 1], l[c]);
        weight[c] = fast_exp2(k.ref[c] - m[c]) * down;
    }
    {
        int r = 0;
#pragma unroll
        for (int nt = 0; nt < K::NT; nt++)
#pragma unroll
            for (int i = 0; i < K::kMT; i++)
#pragma unroll
                for (int j = 0; j < 4; j += NC == 1 ? 2 : 1) res[(warp * K::kRegs + r++) * 32 + lane] = k.acc[nt][i][j] * weight[(2 * nt + (j & 1)) % NC];
    }
    __syncthreads();
    if (!live) return;
    float* out = pl.partial + ((long long)blockIdx.x * p.c.H + head) * pl.item_stride;
    const float* mine = res + local * K::kRegs * 32 + lane;
#pragma unroll 4
    for (int r = sub; r < K::kRegs; r += 1 << pl.per_head_log2) {
        float y = 0.0f;
#pragma unroll 1                                          // code that runs once from a cold instruction cache: 16.9 -> 16.2 us, 16k 4-bit tokens
        for (int w = 0; w < WARPS >> pl.heads_log2; w++) y += mine[((w << pl.heads_log2) * K::kRegs + r) * 32];
        if (pl.target) {
            out[r * 32 + lane] = y;
        } else {
            int ch, col;
            place<K::kPool, D, NC>(r, lane, &ch, &col);
            float lc = l[0];
#pragma unroll
            for (int j = 1; j < NC; j++) if (2 * (col >> 3) + ((col >> 2) & 1) == j) lc = l[j];
            if (col < cols) store_out(p, pl.share_magic, it.first, head, ch, col, lc != 0.0f ? y / lc : 0.0f);
        }
    }
    if (pl.target && sub == 0 && lane < 4)
#pragma unroll
        for (int c = 0; c < NC; c++) *reinterpret_cast<float2*>(out + K::kRegs * 32 + 2 * column_of(c, lane)) = make_float2(m[c], l[c]);
}

// Joins the pieces of a sequence.  Grid (sequence, KV head, slice of 128 numbers): a warp takes every WARPS-th piece, a lane four
// neighbouring numbers of it (one register, four lanes of the split kernel: four columns).  The weights of all pieces are found
// first, a column per warp, while the warp's first pieces are on their way.  Sixteen warps where one sequence has many
// pieces, four where many sequences share them (18 us against 11 for 32 sequences of 4 pieces).
constexpr int kMaxPieces = 160;
template <bool POOL, int D, int NC, int WARPS>
__global__ void __launch_bounds__(32 * WARPS) attention_join_kernel(const AttentionParams p, const SplitPlan pl) {
    constexpr int kRegs = (NC == 1 ? 2 : 2 * NC) * (D / 16), kCols = 4 * NC;
    constexpr int kFirst = WARPS == 16 ? kMaxPieces / WARPS : 4;        // pieces of a warp that are asked for at once
    __shared__ float4 acc[WARPS][32];
    __shared__ float weight[kMaxPieces][kCols];
    __shared__ float norm[kCols];
    pdl_wait();
    const int s = blockIdx.x, h = blockIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int first, kv, rows;
    const bool ordered = sequence_rows(p, s, &first, &kv, &rows);
    const int first_item = pl.items[2 * s], n = pl.items[2 * s + 1];
    if (!ordered || rows == 0) return;                       // then the two numbers above mean nothing
    const int cols = min(min(rows, p.b.max_rows) * p.share, kCols);
    const float* part = pl.partial + ((long long)first_item * p.c.H + h) * pl.item_stride;
    const long long step = (long long)p.c.H * pl.item_stride;
    const int at = blockIdx.z * 32 + lane;                   // numbers 4 at .. 4 at + 3: one register of four lanes, four columns
    int ch0, col0;
    place<POOL, D, NC>(at >> 3, 0, &ch0, &col0);
    auto piece = [&](int i) { return *(reinterpret_cast<const float4*>(part + i * step) + at); };
    float4 x[kFirst];
#pragma unroll
    for (int i = 0; i < kFirst; i++)
        x[i] = col0 < cols && warp + i * WARPS < n ? piece(warp + i * WARPS) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int c = warp; c < cols; c += WARPS) {
        float m[kMaxPieces / 32], l[kMaxPieces / 32], top = kNoMax, sum = 0.0f;
#pragma unroll
        for (int i = 0; i < kMaxPieces / 32; i++) {
            m[i] = kNoMax; l[i] = 0.0f;
            if (32 * i + lane < n) {
                const float2 z = *reinterpret_cast<const float2*>(part + (32 * i + lane) * step + kRegs * 32 + 2 * c);
                m[i] = z.x; l[i] = z.y;
            }
            top = fmaxf(top, m[i]);
        }
#pragma unroll
        for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
#pragma unroll
        for (int i = 0; i < kMaxPieces / 32; i++) {
            if (WARPS < 16 && 32 * i >= n) break;
            const float f = fast_exp2(m[i] - top);
            sum = fmaf(f, l[i], sum);
            if (32 * i + lane < n) weight[32 * i + lane][c] = f;
        }
#pragma unroll
        for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
        if (lane == 0) norm[c] = sum;
    }
    __syncthreads();
    float4 y = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (col0 < cols) {
        auto add = [&](int k, const float4& v) {
            y.x = fmaf(weight[k][col0], v.x, y.x);
            if (col0 + 1 < cols) y.y = fmaf(weight[k][col0 + 1], v.y, y.y);
            if (col0 + 2 < cols) y.z = fmaf(weight[k][col0 + 2], v.z, y.z);
            if (col0 + 3 < cols) y.w = fmaf(weight[k][col0 + 3], v.w, y.w);
        };
#pragma unroll
        for (int i = 0; i < kFirst; i++) {
            if (warp + i * WARPS >= n) break;
            add(warp + i * WARPS, x[i]);
        }
#pragma unroll 4
        for (int i = warp + kFirst * WARPS; i < n; i += WARPS) add(i, piece(i));
    }
    acc[warp][lane] = y;
    __syncthreads();
    if (threadIdx.x >= 128) return;
    const int e = blockIdx.z * 128 + threadIdx.x;
    int c, col;
    place<POOL, D, NC>(e >> 5, e & 31, &c, &col);
    if (col >= cols) return;
    float v = 0.0f;
#pragma unroll
    for (int w = 0; w < WARPS; w++) v += reinterpret_cast<const float*>(acc[w])[threadIdx.x];
    store_out(p, pl.share_magic, first, h, c, col, norm[col] != 0.0f ? v / norm[col] : 0.0f);
}

}  // namespace patchkv
