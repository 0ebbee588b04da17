// What the live-cache calls (cache.cu, attention.cu) share: the batch and the page pool as a kernel sees them.
// All their kernels read global memory with plain loads: launched as dependents, they are resident while the kernel in front of
// them writes what they will read, which the read-only path rules out (and the compiler may move such loads across the wait).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "common.cuh"

namespace patchkv {

struct BatchDev {
    const int32_t* row_start;
    const int32_t* kv_len;
    const int32_t* pos;
    const int32_t* block_table;
    int32_t n_seqs, n_rows, max_rows, max_kv_len, table_stride;
};

// One layer of a pool: quantised pages (base, stride_page in bytes; sections of a page by their byte offsets), or the two
// tensors of a bf16 pool (k, v; strides in elements).
struct CacheDev {
    uint8_t* base;
    long long stride_page;              // bytes (quantised) or elements (bf16)
    const uint16_t* k;
    const uint16_t* v;
    long long stride_token, stride_head;
    uint32_t k_scales, v_codes, v_scales;   // section offsets inside a page; the K codes are at 0
    int32_t n_pages, H, D, P, G;
    int32_t P_shift;                    // log2 of P when it is a power of two, else -1
    int32_t tag;
};

__device__ __forceinline__ int div_page(const CacheDev& c, int t) { return c.P_shift >= 0 ? t >> c.P_shift : t / c.P; }

// The sequence of a packed row: the first b with row_start[b + 1] > r; -1 for a row of no sequence.
__device__ __forceinline__ int find_sequence(const BatchDev& b, int r) {
    int lo = 0, hi = b.n_seqs;          // answer in [lo, hi]
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (b.row_start[mid + 1] > r) hi = mid; else lo = mid + 1;
    }
    return lo < b.n_seqs && b.row_start[lo] <= r ? lo : -1;
}

// Position of row r of sequence s (which ends at row `end`).
__device__ __forceinline__ int row_position(const BatchDev& b, int s, int r) {
    return b.pos ? b.pos[r] : b.kv_len[s] - (b.row_start[s + 1] - r);
}

// Page and slot of a position inside [0, kv_len); page -1 when it is out of range.
__device__ __forceinline__ int locate(const BatchDev& b, const CacheDev& c, int s, int pos, int* slot) {
    if (pos < 0 || pos >= b.kv_len[s]) return -1;
    const int lp = div_page(c, pos);
    *slot = pos - lp * c.P;
    if (lp >= b.table_stride) return -1;
    const int page = b.block_table[(long long)s * b.table_stride + lp];
    return page >= 0 && page < c.n_pages ? page : -1;
}

__device__ __forceinline__ float half_bits_to_float(uint32_t h) { return __half2float(__ushort_as_half((unsigned short)h)); }
__device__ __forceinline__ float bf16_bits_to_float(uint32_t h) { return __uint_as_float(h << 16); }

// Code `e` (element index of a section) as a signed integer, byte accesses only.
__device__ __forceinline__ int code_at(const uint8_t* codes, int fmt, unsigned long long e) {
    if (fmt == FMT_INT8) return (int)(int8_t)codes[e];
    const int n = (codes[e >> 1] >> ((e & 1) * 4)) & 15;
    return n >= 8 ? n - 16 : n;
}
__device__ __forceinline__ float scale_at(const uint8_t* scales, unsigned long long i) {
    return half_bits_to_float((uint32_t)scales[2 * i] | (uint32_t)scales[2 * i + 1] << 8);
}

// Host side: validation, and the device form of the structs.  Without a context (a size is asked for) arrays may be null.
int fill_batch(patchkv_ctx* ctx, const char* who, const patchkv_batch* b, BatchDev* out);
int fill_cache(patchkv_ctx* ctx, const char* who, const patchkv_geom* g, const patchkv_qpool* q, int layer, CacheDev* out);
int check_live_geometry(patchkv_ctx* ctx, const char* who, const patchkv_geom* g, int layer);
// Whether two of the n * H vectors of D elements at these strides share an element (rows within heads or heads within rows).
bool rows_overlap(long long n, long long H, long long D, long long stride_row, long long stride_head);
inline int log2_exact(int x) {
    for (int i = 0; i < 31; i++) if (x == 1 << i) return i;
    return -1;
}

}  // namespace patchkv
