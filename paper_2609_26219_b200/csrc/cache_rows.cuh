// Rows on their way into the cache: where a row's slot is, and the quantiser (cache.cu, rotary.cu).
#pragma once

#include "live.cuh"

namespace patchkv {

__device__ __forceinline__ void latch_bounds(int32_t* status) { atomicCAS(status, 0, (int)PATCHKV_E_BOUNDS); }

// Page (its number) and slot of row r; -1 (latched once per row by the caller's `first` thread) when the row is skipped.
template <bool WRITE, class PARAMS>
__device__ __forceinline__ int find_page(const PARAMS& p, int r, bool first, int* slot, int* position = nullptr) {
    const int s = find_sequence(p.b, r);
    if (s < 0) return -1;                                   // a row of no sequence: not an error
    const int pos = row_position(p.b, s, r), a = p.b.row_start[s];
    if (position) *position = pos;
    // (A sequence that starts below row 0 has no row in front of row 0 to look at.)
    bool ok = a >= 0 && p.b.row_start[s + 1] <= p.b.n_rows;
    if (WRITE && ok && p.b.pos && r > a) ok = p.b.pos[r - 1] < pos;
    const int pg = ok ? locate(p.b, p.c, s, pos, slot) : -1;
    if (pg < 0 && first) latch_bounds(p.status);
    return pg;
}
// The same with the place of a quantised page.
template <bool WRITE, class PARAMS>
__device__ __forceinline__ bool find_slot(const PARAMS& p, int r, bool first, uint8_t** page, int* slot) {
    const int pg = find_page<WRITE>(p, r, first, slot);
    if (pg < 0) return false;
    *page = p.c.base + (long long)pg * p.c.stride_page;
    return true;
}

// Entries of row_start that descend or lie outside [0, n_rows] are an error, although the rows of such a sequence may be found in
// none.  The launch's threads share the sequences; at a kernel's end, so that nothing waits for these loads.
__device__ __forceinline__ void check_entries(const BatchDev& b, int32_t* status, uint32_t thread, uint32_t threads) {
    for (uint32_t s = thread; s < (uint32_t)b.n_seqs; s += threads) {
        const int a = b.row_start[s], e = b.row_start[s + 1];
        if (a < 0 || e < a || e > b.n_rows) latch_bounds(status);
    }
}

template <int TYPE>
__device__ __forceinline__ float to_float(uint32_t h) {
    return TYPE == PATCHKV_ROWS_F16 ? half_bits_to_float(h) : bf16_bits_to_float(h);
}
template <int TYPE>
__device__ __forceinline__ uint32_t pack_pair(float lo, float hi) {
    if (TYPE == PATCHKV_ROWS_F16) {
        const __half2 h = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}

// CH = 8, 16 or 32 channels (w) -> codes and, from the group's first lane, its scale.  `seg` lanes share a group (a power of two).
//   Group maximum: magnitudes are ordered as their 16-bit patterns, two at a time.
//   s = fp16(amax / qmax): q0 = amax * y, q = q0 + (amax - q0 * qmax) * y with y = fp32(1 / qmax), fused, is the correctly rounded fp32
//   quotient for every bf16 and fp16 amax and qmax 7 or 127 (gone through in exact arithmetic).
//   code = rint(x / s): t = x * r with r = 1 / s to an ulp or two, corrected to t' = t + (x - t * s) * r, the remainder exact.  x and s have 11
//   bits at most, so x / s is a half-integer or 2^-12 away from one: t' is within 2^-15 of it, and where x / s is a half-integer h
//   the correction differs from h - t by 2^-22 of itself, which rounds away: t' = h.  Adding 1.5 * 2^23 rounds to the integer,
//   ties to even.  |x / s| <= qmax (1 + 2^-11) unless s is subnormal; then the quotients are clamped.
template <int TYPE, int FMT, int CH>
__device__ __forceinline__ void encode(const uint4 (&w)[CH / 8], uint8_t* codes, uint8_t* scale, int seg, bool live) {
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < CH / 8; i++)
        most = __vmaxu2(most, __vmaxu2(__vmaxu2(w[i].x & 0x7FFF7FFFu, w[i].y & 0x7FFF7FFFu), __vmaxu2(w[i].z & 0x7FFF7FFFu, w[i].w & 0x7FFF7FFFu)));
    for (int d = 1; d < seg; d <<= 1) most = __vmaxu2(most, __shfl_xor_sync(0xFFFFFFFFu, most, d));
    if (!live) return;
    constexpr float qmax = FMT == FMT_INT8 ? 127.0f : 7.0f, y = 1.0f / qmax;
    const float amax = to_float<TYPE>(max(most & 0xFFFFu, most >> 16));
    const float q0 = __fmul_rn(amax, y), q = __fmaf_rn(__fmaf_rn(-q0, qmax, amax), y, q0);
    const uint32_t s16 = pack_pair<PATCHKV_ROWS_F16>(amax > 3.0e38f ? INFINITY : q, 0.0f) & 0xFFFFu;
    const bool usable = s16 != 0 && s16 < 0x7C00u;          // a zero or infinite scale: all codes zero
    const float s = half_bits_to_float(usable ? s16 : 0x3C00u);
    float r;
    asm("rcp.approx.f32 %0, %1;" : "=f"(r) : "f"(s));
    const f32x2 r2 = pack2(r, r), s2 = pack2(-s, -s), magic = pack2(12582912.0f, 12582912.0f);
    uint32_t out[CH / 8][2];
#pragma unroll
    for (int k = 0; k < CH / 8; k++) {
        const uint32_t ws[4] = {w[k].x, w[k].y, w[k].z, w[k].w};
        uint32_t kb[8];
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const f32x2 x = pack2(to_float<TYPE>(ws[i] & 0xFFFFu), to_float<TYPE>(ws[i] >> 16));
            f32x2 t = mul2(x, r2);
            t = fma2(fma2(t, s2, x), r2, t);
            float a, b;
            if (s16 < 0x0400u) {                            // subnormal
                unpack2(t, a, b);
                t = pack2(fminf(fmaxf(a, -qmax), qmax), fminf(fmaxf(b, -qmax), qmax));
            }
            unpack2(add2(t, magic), a, b);
            kb[2 * i] = __float_as_uint(a);
            kb[2 * i + 1] = __float_as_uint(b);
        }
        const uint32_t w0 = __byte_perm(__byte_perm(kb[0], kb[1], 0x0040), __byte_perm(kb[2], kb[3], 0x0040), 0x5410);
        const uint32_t w1 = __byte_perm(__byte_perm(kb[4], kb[5], 0x0040), __byte_perm(kb[6], kb[7], 0x0040), 0x5410);
        if (FMT == FMT_INT8) {
            out[k][0] = w0; out[k][1] = w1;
        } else {
            uint32_t a = w0 & 0x0F0F0F0Fu, b = w1 & 0x0F0F0F0Fu;
            a = (a | (a >> 4)) & 0x00FF00FFu; b = (b | (b >> 4)) & 0x00FF00FFu;
            out[k][0] = __byte_perm(a, b, 0x6420);
        }
        if (!usable) out[k][0] = out[k][1] = 0;
    }
    if constexpr (CH == 8) {
        if (FMT == FMT_INT8) *reinterpret_cast<uint2*>(codes) = make_uint2(out[0][0], out[0][1]);
        else *reinterpret_cast<uint32_t*>(codes) = out[0][0];
    } else if constexpr (CH == 16) {
        if (FMT == FMT_INT8) *reinterpret_cast<uint4*>(codes) = make_uint4(out[0][0], out[0][1], out[1][0], out[1][1]);
        else *reinterpret_cast<uint2*>(codes) = make_uint2(out[0][0], out[1][0]);
    } else if constexpr (FMT == FMT_INT8) {
        reinterpret_cast<uint4*>(codes)[0] = make_uint4(out[0][0], out[0][1], out[1][0], out[1][1]);
        reinterpret_cast<uint4*>(codes)[1] = make_uint4(out[2][0], out[2][1], out[3][0], out[3][1]);
    } else {
        *reinterpret_cast<uint4*>(codes) = make_uint4(out[0][0], out[1][0], out[2][0], out[3][0]);
    }
    if (scale) *reinterpret_cast<uint16_t*>(scale) = (uint16_t)s16;
}

}  // namespace patchkv
