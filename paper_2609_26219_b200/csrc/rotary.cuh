// Cosines and sines of rotary positions (rotary.cu, evict.cu).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>

#include "common.cuh"

namespace patchkv {

// Frequencies of the rotary pairs in 64 bits, as the restore path defines them: inv_freq[i], or rope_base^(-2i/Dr).
struct Frequencies { double theta[PATCHKV_MAX_ROTARY_DIM / 2]; };

// Checks the rotary fields of a geometry and fills the frequencies.
int fill_frequencies(patchkv_ctx* ctx, const char* who, const patchkv_geom* g, Frequencies* f);

// cos and sin of an angle in radians, |angle| < 2^48, to 2^-52 or so.  The angle comes to [-pi/4, pi/4] by multiples of pi/2 taken off in
// two parts (the first product and difference are exact in the fused operation: both are multiples of 2^-52 below 1), then the two
// Taylor series, cut where the next term is below 2^-53.  64 bits because a position of 10^5 leaves an fp32 angle 2^-7 off, and so that a
// key next to the border of two codes falls on the side that the formula says; some 25 operations of the fp64 pipe for both.
__device__ __forceinline__ void cos_sin(double angle, double* c, double* s) {
    constexpr double kRound = 6755399441055744.0;           // 1.5 * 2^52: adding it rounds to an integer, in the low word
    const double t = fma(angle, 0.63661977236758134308, kRound);      // 2 / pi
    const int quarter = __double2loint(t);
    const double k = t - kRound;
    double r = fma(k, -1.57079632679489655800, angle);      // pi / 2 in 53 bits, and what that leaves of it
    r = fma(k, -6.12323399573676603587e-17, r);
    const double z = r * r;
    double p = -1.0 / 1307674368000.0, q = 1.0 / 20922789888000.0;    // 1 / 15!, 1 / 16!
    p = fma(p, z, 1.0 / 6227020800.0);
    q = fma(q, z, -1.0 / 87178291200.0);
    p = fma(p, z, -1.0 / 39916800.0);
    q = fma(q, z, 1.0 / 479001600.0);
    p = fma(p, z, 1.0 / 362880.0);
    q = fma(q, z, -1.0 / 3628800.0);
    p = fma(p, z, -1.0 / 5040.0);
    q = fma(q, z, 1.0 / 40320.0);
    p = fma(p, z, 1.0 / 120.0);
    q = fma(q, z, -1.0 / 720.0);
    p = fma(p, z, -1.0 / 6.0);
    q = fma(q, z, 1.0 / 24.0);
    q = fma(q, z, -0.5);
    const double sn = fma(p * z, r, r), cs = fma(q, z, 1.0);
    const double a = quarter & 1 ? sn : cs, b = quarter & 1 ? cs : sn;
    *c = (quarter + 1) & 2 ? -a : a;
    *s = quarter & 2 ? -b : b;
}

// A lane of the fast kernels has 16 channels of a head, two runs of eight, such that it has both channels of its eight rotary pairs: in the
// half layout the runs lie Dr / 2 apart, in the interleaved one, and behind the rotary channels, side by side.  Angle 8 u + i belongs to pair i
// of lane u of the head.
__device__ __forceinline__ int first_run(bool half, int Dr, int u) { return half && 16 * u < Dr ? 8 * u : 16 * u; }
__device__ __forceinline__ int second_run(bool half, int Dr, int u) { return half && 16 * u < Dr ? Dr / 2 + 8 * u : 16 * u + 8; }

// The runs' eight words in bf16 or fp16 (TYPE), turned by c[i], s[i] in fp32.
template <int TYPE>
__device__ __forceinline__ float low_float(uint32_t w) {
    if (TYPE == PATCHKV_ROWS_F16) return __half2float(__ushort_as_half((unsigned short)(w & 0xFFFFu)));
    return __uint_as_float(w << 16);
}
template <int TYPE>
__device__ __forceinline__ float high_float(uint32_t w) {
    if (TYPE == PATCHKV_ROWS_F16) return __half2float(__ushort_as_half((unsigned short)(w >> 16)));
    return __uint_as_float(w & 0xFFFF0000u);
}
template <int TYPE>
__device__ __forceinline__ uint32_t pack_floats(float lo, float hi) {
    uint32_t d;
    if (TYPE == PATCHKV_ROWS_F16) asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}
template <int TYPE, bool HALF>
__device__ __forceinline__ void turn_words(uint32_t (&w)[8], const float (&c)[8], const float (&s)[8]) {
    if (HALF) {
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const f32x2 a = pack2(low_float<TYPE>(w[i]), high_float<TYPE>(w[i])), b = pack2(low_float<TYPE>(w[4 + i]), high_float<TYPE>(w[4 + i]));
            const f32x2 cc = pack2(c[2 * i], c[2 * i + 1]), ss = pack2(s[2 * i], s[2 * i + 1]);
            float lo, hi;
            unpack2(sub2(mul2(a, cc), mul2(b, ss)), lo, hi);
            w[i] = pack_floats<TYPE>(lo, hi);
            unpack2(fma2(a, ss, mul2(b, cc)), lo, hi);
            w[4 + i] = pack_floats<TYPE>(lo, hi);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const float a = low_float<TYPE>(w[i]), b = high_float<TYPE>(w[i]);
            w[i] = pack_floats<TYPE>(fmaf(-b, s[i], a * c[i]), fmaf(b, c[i], a * s[i]));
        }
    }
}

}  // namespace patchkv
