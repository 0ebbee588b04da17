// Parameters and masks shared by the attention kernels (attention.cu).
#pragma once

#include "live.cuh"

namespace patchkv {

struct AttentionParams {
    CacheDev c;
    BatchDev b;
    const uint16_t* q;
    uint16_t* out;
    long long q_stride_row, q_stride_head, out_stride_row, out_stride_head;
    int32_t Hq, share;              // query heads, and query heads per KV head
    int32_t window, sinks;
    int32_t f16;                    // type of q and out: fp16 (1) or bf16 (0)
    float scale_log2;               // scale * log2(e): the softmax runs on powers of two
    int32_t* status;
};

__device__ __forceinline__ void latch(int32_t* status) { atomicCAS(status, 0, (int)PATCHKV_E_BOUNDS); }

// Whether the row at position pos sees token t < kv (t <= pos is the caller's).
__device__ __forceinline__ bool sees(const AttentionParams& p, int pos, int t) {
    return p.window == 0 || pos - t < p.window || t < p.sinks;
}

// First row of a sequence and the tokens it may use; false when its row_start entries are out of order or out of range.
__device__ __forceinline__ bool sequence_rows(const AttentionParams& p, int s, int* first, int* kv, int* rows = nullptr) {
    const int a = p.b.row_start[s], e = p.b.row_start[s + 1];
    *first = a;
    const long long cap = (long long)p.b.table_stride * p.c.P;
    long long n = min(p.b.kv_len[s], p.b.max_kv_len);
    if (n > cap) n = cap;
    *kv = n < 0 ? 0 : (int)n;
    if (rows) *rows = e - a;
    return a >= 0 && e >= a && e <= p.b.n_rows;
}

}  // namespace patchkv
