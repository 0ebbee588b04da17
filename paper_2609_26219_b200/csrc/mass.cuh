// Parameters and the last step shared by the kernels of patchkv_attention_mass (mass.cu).
#pragma once

#include "attention.cuh"

namespace patchkv {

// What is added to an AttentionParams (its q, masks and cache).
struct WeightParams {
    const void* in;
    void* out;
    long long stride;
    float decay;
    int32_t u64;
};

// Whether the row at position pos sees a token at all.
__device__ __forceinline__ bool sees_some(const AttentionParams& p, int pos, int kv) {
    const int end = min(pos, kv - 1);
    return end >= 0 && (p.window == 0 || pos - end < p.window || p.sinks > 0);
}

// The call's sum for token t of sequence s, onto what was there.
__device__ __forceinline__ void store_mass(const AttentionParams& p, const WeightParams& m, int s, int t, float sum) {
    const long long at = (long long)s * m.stride + t;
    const bool add = m.in && m.decay != 0.0f;
    if (m.u64) {
        unsigned long long units = 0;
        if (fabsf(sum) <= 3.0e38f) units = (unsigned long long)__double2ll_rn((double)sum * 16777216.0);
        else atomicCAS(p.status, 0, (int)PATCHKV_E_BADINPUT);
        static_cast<unsigned long long*>(m.out)[at] = (add ? static_cast<const unsigned long long*>(m.in)[at] : 0ull) + units;
    } else {
        static_cast<float*>(m.out)[at] = add ? fmaf(m.decay, static_cast<const float*>(m.in)[at], sum) : sum;
    }
}

}  // namespace patchkv
