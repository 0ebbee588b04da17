// Rows into and out of a cache of quantised pages: patchkv_cache_append, patchkv_cache_read, and the checks that the
// live-cache calls share.
#include <math.h>

#include "live.cuh"

namespace patchkv {

constexpr int kRowThreads = 128;

struct RowsDev {
    uint16_t* k;
    uint16_t* v;
    long long stride_row, stride_head;
};

struct RowParams {
    CacheDev c;
    BatchDev b;
    RowsDev rows;
    int32_t* status;
    int32_t vecs;               // vectors of a row: H * D / 8, or / 32
    int32_t seg;                // lanes per scale group: G / 8, or / 32
    int32_t parts;              // warps that share a row (32 vectors each at a time)
    int32_t G_shift, D_shift;   // log2 of G; of D when it is a power of two, else -1
};

__device__ __forceinline__ void latch_bounds(int32_t* status) { atomicCAS(status, 0, (int)PATCHKV_E_BOUNDS); }

// Page and slot of row r; false (latched once per row by the caller's `first` thread) when the row is skipped.
template <bool WRITE>
__device__ __forceinline__ bool find_slot(const RowParams& p, int r, bool first, uint8_t** page, int* slot) {
    const int s = find_sequence(p.b, r);
    if (s < 0) return false;                                // a row of no sequence: not an error
    const int pos = row_position(p.b, s, r), a = p.b.row_start[s];
    // (A sequence that starts below row 0 has no row in front of row 0 to look at.)
    bool ok = a >= 0 && p.b.row_start[s + 1] <= p.b.n_rows;
    if (WRITE && ok && p.b.pos && r > a) ok = p.b.pos[r - 1] < pos;
    const int pg = ok ? locate(p.b, p.c, s, pos, slot) : -1;
    if (pg < 0) {
        if (first) latch_bounds(p.status);
        return false;
    }
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

// CH = 8 or 32 channels (w) -> codes and, from the group's first lane, its scale.  `seg` lanes share a group (a power of two).
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
    } else if constexpr (FMT == FMT_INT8) {
        reinterpret_cast<uint4*>(codes)[0] = make_uint4(out[0][0], out[0][1], out[1][0], out[1][1]);
        reinterpret_cast<uint4*>(codes)[1] = make_uint4(out[2][0], out[2][1], out[3][0], out[3][1]);
    } else {
        *reinterpret_cast<uint4*>(codes) = make_uint4(out[0][0], out[1][0], out[2][0], out[3][0]);
    }
    if (scale) *reinterpret_cast<uint16_t*>(scale) = (uint16_t)s16;
}

// A warp takes a row (or a share of one), a lane a vector of K and of V, several times 32 of them at once: the row's slot is looked up
// once, loads and stores of a warp are contiguous, the groups' maxima go through shuffles.  (With a thread per vector of a row
// the look-up was most of the instructions: 170 us to read 2 x 64k tokens, 116 so.)  Bound by memory, the append of few bits by
// its instructions too: a vector there is 32 channels of one group, so that its scale is found once, or 8 where groups are smaller.
// Row and first vector of a warp.
__device__ __forceinline__ bool warp_place(const RowParams& p, int* r, int* v_first) {
    const uint32_t w = (blockIdx.x * kRowThreads + threadIdx.x) >> 5, q = p.parts == 1 ? w : w / (uint32_t)p.parts;
    *r = (int)q;
    *v_first = (int)(w - q * p.parts) * 32;
    return *r < p.b.n_rows;
}
// Element offset of channel e of a row (counted over its heads) inside a row of the caller's tensors.
__device__ __forceinline__ long long row_element(const RowParams& p, int e) {
    if (p.rows.stride_head == p.c.D) return e;
    const int h = p.D_shift >= 0 ? e >> p.D_shift : e / p.c.D;
    return (long long)h * p.rows.stride_head + (e - h * p.c.D);
}

template <int TYPE, int KF, int VF, int CH>
__global__ void __launch_bounds__(kRowThreads) cache_append_kernel(const __grid_constant__ RowParams p) {
    constexpr int kBatch = CH == 8 ? 4 : 1;
    pdl_trigger();
    int r, v_first;
    if (!warp_place(p, &r, &v_first)) return;
    pdl_wait();
    uint8_t* page = nullptr;
    int slot = 0;
    bool found = false;
    const int lane = threadIdx.x & 31, stride = 32 * p.parts;
    for (int v0 = v_first; v0 < p.vecs; v0 += stride * kBatch) {
        uint4 kw[kBatch][CH / 8], vw[kBatch][CH / 8];
#pragma unroll
        for (int i = 0; i < kBatch; i++) {
            const int vec = v0 + stride * i + lane;
#pragma unroll
            for (int q = 0; q < CH / 8; q++) kw[i][q] = vw[i][q] = make_uint4(0, 0, 0, 0);
            if (vec < p.vecs) {
                const long long src = (long long)r * p.rows.stride_row + row_element(p, vec * CH);
#pragma unroll
                for (int q = 0; q < CH / 8; q++) {
                    kw[i][q] = *(reinterpret_cast<const uint4*>(p.rows.k + src) + q);
                    vw[i][q] = *(reinterpret_cast<const uint4*>(p.rows.v + src) + q);
                }
            }
        }
        if (v0 == v_first) found = find_slot<true>(p, r, lane == 0 && v_first == 0, &page, &slot);      // while the row is on its way
        if (!found) break;                                   // the same for all lanes
#pragma unroll
        for (int i = 0; i < kBatch; i++) {
            if (v0 + stride * i >= p.vecs) break;
            const int vec = v0 + stride * i + lane;
            const uint32_t at = ((uint32_t)slot * p.vecs + vec) * CH;
            const bool first = (vec & (p.seg - 1)) == 0;
            const uint32_t group = at >> p.G_shift;
            encode<TYPE, KF, CH>(kw[i], page + (KF == FMT_INT8 ? at : at >> 1), first ? page + p.c.k_scales + 2 * group : nullptr, p.seg, vec < p.vecs);
            encode<TYPE, VF, CH>(vw[i], page + p.c.v_codes + (VF == FMT_INT8 ? at : at >> 1), first ? page + p.c.v_scales + 2 * group : nullptr,
                                 p.seg, vec < p.vecs);
        }
    }
    check_entries(p.b, p.status, blockIdx.x * kRowThreads + threadIdx.x, (uint32_t)p.b.n_rows * p.parts * 32);
}

// Eight codes and their scale -> eight channels.  An integer u < 2^23 in the low bits of 2^23's pattern is the float
// 2^23 + u, so the codes need no conversion instruction; code * scale is exact in fp32 and rounded once.
template <int TYPE, int FMT>
__device__ __forceinline__ uint4 decode8(const uint2& w, float s) {
    float x[8];
    if (FMT == FMT_INT8) {
        const uint32_t a = w.x ^ 0x80808080u, b = w.y ^ 0x80808080u;
#pragma unroll
        for (int i = 0; i < 4; i++) {
            x[i] = __uint_as_float(__byte_perm(a, 0x4B000000u, 0x7540 + i)) - 8388736.0f;
            x[4 + i] = __uint_as_float(__byte_perm(b, 0x4B000000u, 0x7540 + i)) - 8388736.0f;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++)
            x[i] = __uint_as_float((((w.x >> (4 * i)) & 15u) ^ 8u) | 0x4B000000u) - 8388616.0f;
    }
    uint4 o;
    o.x = pack_pair<TYPE>(x[0] * s, x[1] * s);
    o.y = pack_pair<TYPE>(x[2] * s, x[3] * s);
    o.z = pack_pair<TYPE>(x[4] * s, x[5] * s);
    o.w = pack_pair<TYPE>(x[6] * s, x[7] * s);
    return o;
}
template <int FMT>
__device__ __forceinline__ uint2 load_codes8(const uint8_t* codes, uint32_t at) {
    if (FMT == FMT_INT8) return *reinterpret_cast<const uint2*>(codes + at);
    return make_uint2(*reinterpret_cast<const uint32_t*>(codes + (at >> 1)), 0u);
}

template <int TYPE, int KF, int VF>
__global__ void __launch_bounds__(kRowThreads) cache_read_kernel(const __grid_constant__ RowParams p) {
    pdl_trigger();
    int r, v_first;
    if (!warp_place(p, &r, &v_first)) return;
    const int lane = threadIdx.x & 31, stride = 32 * p.parts;
    uint8_t* page = nullptr;
    int slot = 0;
    pdl_wait();
    const bool found = find_slot<false>(p, r, lane == 0 && v_first == 0, &page, &slot);
    constexpr int kBatch = 4;
    for (int v0 = found ? v_first : p.vecs; v0 < p.vecs; v0 += stride * kBatch) {
        uint2 kc[kBatch], vc[kBatch];
        uint16_t ks[kBatch], vs[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; i++) {
            const int vec = min(v0 + stride * i + lane, p.vecs - 1);
            const uint32_t at = ((uint32_t)slot * p.vecs + vec) * 8, group = at >> p.G_shift;
            kc[i] = load_codes8<KF>(page, at);
            vc[i] = load_codes8<VF>(page + p.c.v_codes, at);
            ks[i] = *reinterpret_cast<const uint16_t*>(page + p.c.k_scales + 2 * group);
            vs[i] = *reinterpret_cast<const uint16_t*>(page + p.c.v_scales + 2 * group);
        }
#pragma unroll
        for (int i = 0; i < kBatch; i++) {
            const int vec = v0 + stride * i + lane;
            if (vec < p.vecs) {
                const long long dst = (long long)r * p.rows.stride_row + row_element(p, vec * 8);
                *reinterpret_cast<uint4*>(p.rows.k + dst) = decode8<TYPE, KF>(kc[i], half_bits_to_float(ks[i]));
                *reinterpret_cast<uint4*>(p.rows.v + dst) = decode8<TYPE, VF>(vc[i], half_bits_to_float(vs[i]));
            }
        }
    }
    check_entries(p.b, p.status, blockIdx.x * kRowThreads + threadIdx.x, (uint32_t)p.b.n_rows * p.parts * 32);
}

// Any geometry, any strides: one thread per (row, section, head) walks the head's groups with byte accesses to the page.
// (A byte may hold codes of two groups, so the head is the smallest piece that one thread can own.)
template <int TYPE, bool WRITE>
__global__ void __launch_bounds__(kRowThreads) cache_rows_any_kernel(const RowParams p) {
    const uint32_t i = blockIdx.x * kRowThreads + threadIdx.x, per_row = 2u * p.c.H;
    const int r = (int)(i / per_row), q = (int)(i - (uint32_t)r * per_row), h = q >> 1;
    if (r >= p.b.n_rows) return;
    check_entries(p.b, p.status, i, (uint32_t)p.b.n_rows * per_row);
    uint8_t* page = nullptr;
    int slot = 0;
    if (!find_slot<WRITE>(p, r, q == 0, &page, &slot)) return;
    const bool is_v = q & 1;
    const int fmt = is_v ? v_format(p.c.tag) : k_format(p.c.tag);
    uint8_t* codes = page + (is_v ? p.c.v_codes : 0u);
    uint8_t* scales = page + (is_v ? p.c.v_scales : p.c.k_scales);
    uint16_t* x = (is_v ? p.rows.v : p.rows.k) + (long long)r * p.rows.stride_row + (long long)h * p.rows.stride_head;
    const unsigned long long e0 = ((unsigned long long)slot * p.c.H + h) * p.c.D;
    const float qmax = fmt == FMT_INT8 ? 127.0f : 7.0f;
    int low = 0;
    for (int c0 = 0; c0 < p.c.D; c0 += p.c.G) {
        const unsigned long long group = (e0 + c0) / p.c.G;
        if (WRITE) {
            float amax = 0.0f;
            for (int c = c0; c < c0 + p.c.G; c++) amax = fmaxf(amax, fabsf(to_float<TYPE>(x[c])));
            const uint32_t sb = pack_pair<PATCHKV_ROWS_F16>(__fdiv_rn(amax, qmax), 0.0f);
            const float s = half_bits_to_float(sb & 0xFFFFu);
            scales[2 * group] = (uint8_t)sb;
            scales[2 * group + 1] = (uint8_t)(sb >> 8);
            const bool usable = s > 0.0f && s <= 65504.0f;
            for (int c = c0; c < c0 + p.c.G; c++) {
                float t = usable ? rintf(__fdiv_rn(to_float<TYPE>(x[c]), s)) : 0.0f;
                const int code = (int)fminf(fmaxf(t, -qmax), qmax);
                if (fmt == FMT_INT8) codes[e0 + c] = (uint8_t)code;
                else if ((c & 1) == 0) low = code & 15;                   // D is even: the pair is this thread's
                else codes[(e0 + c) >> 1] = (uint8_t)(low | (code & 15) << 4);
            }
        } else {
            const float s = scale_at(scales, group);
            for (int c = c0; c < c0 + p.c.G; c++)
                x[c] = (uint16_t)pack_pair<TYPE>((float)code_at(codes, fmt, e0 + c) * s, 0.0f);
        }
    }
}

bool rows_overlap(long long n, long long H, long long D, long long stride_row, long long stride_head) {
    const bool by_row = (H == 1 || stride_head >= D) && (n == 1 || stride_row >= (H - 1) * stride_head + D);
    const bool by_head = (n == 1 || stride_row >= D) && (H == 1 || stride_head >= (n - 1) * stride_row + D);
    return !by_row && !by_head;
}

int check_live_geometry(patchkv_ctx* ctx, const char* who, const patchkv_geom* g, int layer) {
    const std::string w(who);
    if (!g || g->struct_size != sizeof(patchkv_geom)) return fail(ctx, PATCHKV_E_INVALID, w + ": null geom or wrong struct_size");
    if (g->n_layers <= 0 || g->n_kv_heads <= 0 || g->head_dim <= 0 || (g->head_dim & 1) || g->page_tokens <= 0 || g->group <= 0 ||
        g->head_dim % g->group)
        return fail(ctx, PATCHKV_E_INVALID, w + ": geometry needs L, H, P > 0, D even, G dividing D");
    if (layer < 0 || layer >= g->n_layers) return fail(ctx, PATCHKV_E_INVALID, w + ": layer out of range");
    // element indexes inside a page, and its byte offsets, are 32-bit
    if ((unsigned long long)g->page_tokens * g->n_kv_heads > (1ull << 29) / g->head_dim)
        return fail(ctx, PATCHKV_E_UNSUPPORTED, w + ": a page holds more than 2^29 elements");
    return PATCHKV_OK;
}

int fill_cache(patchkv_ctx* ctx, const char* who, const patchkv_geom* g, const patchkv_qpool* q, int layer, CacheDev* c) {
    const std::string w(who);
    if (!q || q->struct_size != sizeof(patchkv_qpool)) return fail(ctx, PATCHKV_E_INVALID, w + ": null cache or wrong struct_size");
    if (q->tag < PATCHKV_TAG_INT8 || q->tag > PATCHKV_TAG_K4V4) return fail(ctx, PATCHKV_E_INVALID, w + ": tag of a quantised cache must be INT8, INT4 or K4V4");
    if (!q->base || (reinterpret_cast<uintptr_t>(q->base) & 15u) || q->n_pages <= 0)
        return fail(ctx, PATCHKV_E_INVALID, w + ": cache base null or not 16-byte aligned, or no pages");
    const uint64_t elems = (uint64_t)g->page_tokens * g->n_kv_heads * g->head_dim;
    if (q->stride_layer < 0 || (q->stride_layer & 15) || (q->stride_page & 15) || q->stride_page < 0 ||
        (uint64_t)q->stride_page < record_bytes(q->tag, elems, g->group))
        return fail(ctx, PATCHKV_E_INVALID, w + ": cache strides must be multiples of 16, a page at least one record");
    memset(c, 0, sizeof(*c));
    c->base = static_cast<uint8_t*>(q->base) + (long long)layer * q->stride_layer;
    c->stride_page = q->stride_page;
    const int kf = k_format(q->tag), vf = v_format(q->tag);
    c->k_scales = (uint32_t)code_bytes(kf, elems);
    c->v_codes = c->k_scales + (uint32_t)scale_bytes(kf, elems, g->group);
    c->v_scales = c->v_codes + (uint32_t)code_bytes(vf, elems);
    c->n_pages = q->n_pages; c->H = g->n_kv_heads; c->D = g->head_dim; c->P = g->page_tokens; c->G = g->group;
    c->P_shift = log2_exact(g->page_tokens);
    c->tag = q->tag;
    return PATCHKV_OK;
}

int fill_batch(patchkv_ctx* ctx, const char* who, const patchkv_batch* b, BatchDev* o) {
    const std::string w(who);
    if (!b || b->struct_size != sizeof(patchkv_batch)) return fail(ctx, PATCHKV_E_INVALID, w + ": null batch or wrong struct_size");
    if (b->n_seqs < 0 || b->n_rows < 0 || b->max_rows < 0 || b->max_kv_len < 0 || b->table_stride < 0)
        return fail(ctx, PATCHKV_E_INVALID, w + ": negative count in the batch");
    if (ctx && b->n_seqs > 0 && b->n_rows > 0 && (!b->row_start || !b->kv_len || (!b->block_table && b->table_stride > 0)))
        return fail(ctx, PATCHKV_E_INVALID, w + ": null row_start, kv_len or block_table");
    o->row_start = b->row_start; o->kv_len = b->kv_len; o->pos = b->pos; o->block_table = b->block_table;
    o->n_seqs = b->n_seqs; o->n_rows = b->n_rows; o->max_rows = b->max_rows; o->max_kv_len = b->max_kv_len;
    o->table_stride = b->table_stride;
    return PATCHKV_OK;
}

namespace {

template <int TYPE, int KF, int VF>
cudaError_t launch_rows_fast(const RowParams& p, bool write, unsigned grid, cudaStream_t stream) {
    if (write && p.seg << 5 == p.c.G) return launch_pdl(cache_append_kernel<TYPE, KF, VF, 32>, dim3(grid), dim3(kRowThreads), 0, stream, p);
    return write ? launch_pdl(cache_append_kernel<TYPE, KF, VF, 8>, dim3(grid), dim3(kRowThreads), 0, stream, p)
                 : launch_pdl(cache_read_kernel<TYPE, KF, VF>, dim3(grid), dim3(kRowThreads), 0, stream, p);
}
template <int TYPE>
cudaError_t launch_rows_tag(const RowParams& p, bool write, unsigned grid, cudaStream_t stream) {
    if (p.c.tag == PATCHKV_TAG_INT8) return launch_rows_fast<TYPE, FMT_INT8, FMT_INT8>(p, write, grid, stream);
    if (p.c.tag == PATCHKV_TAG_INT4) return launch_rows_fast<TYPE, FMT_INT8, FMT_INT4>(p, write, grid, stream);
    return launch_rows_fast<TYPE, FMT_INT4, FMT_INT4>(p, write, grid, stream);
}

int cache_rows(patchkv_ctx* ctx, const char* who, const patchkv_geom* g, const patchkv_qpool* cache, int layer,
               const patchkv_batch* batch, const patchkv_rows* rows, bool write, cudaStream_t stream) {
    const std::string w(who);
    RowParams p;
    int rc = check_live_geometry(ctx, who, g, layer);
    if (rc == PATCHKV_OK) rc = fill_cache(ctx, who, g, cache, layer, &p.c);
    if (rc == PATCHKV_OK) rc = fill_batch(ctx, who, batch, &p.b);
    if (rc != PATCHKV_OK) return rc;
    if (!rows || rows->struct_size != sizeof(patchkv_rows)) return fail(ctx, PATCHKV_E_INVALID, w + ": null rows or wrong struct_size");
    if (rows->type != PATCHKV_ROWS_BF16 && rows->type != PATCHKV_ROWS_F16) return fail(ctx, PATCHKV_E_INVALID, w + ": unknown row type");
    if (rows->stride_row < 0 || rows->stride_head < 0) return fail(ctx, PATCHKV_E_INVALID, w + ": negative row stride");
    if (p.b.n_rows == 0 || p.b.n_seqs == 0) return PATCHKV_OK;
    const uintptr_t ka = reinterpret_cast<uintptr_t>(rows->k), va = reinterpret_cast<uintptr_t>(rows->v);
    if (!ka || !va || (ka & 1) || (va & 1)) return fail(ctx, PATCHKV_E_INVALID, w + ": null or misaligned rows");
    if (!write && rows_overlap(p.b.n_rows, p.c.H, p.c.D, rows->stride_row, rows->stride_head))
        return fail(ctx, PATCHKV_E_INVALID, w + ": rows or heads of the output overlap");
    p.rows = {static_cast<uint16_t*>(rows->k), static_cast<uint16_t*>(rows->v), rows->stride_row, rows->stride_head};
    p.status = ctx->d_status;
    const long long elems = (long long)g->page_tokens * g->n_kv_heads * g->head_dim;
    const int gs = log2_exact(g->group);
    const bool fast = g->head_dim % 8 == 0 && gs >= 3 && gs <= 8 && elems % 32 == 0 && (elems / g->group) % 8 == 0 &&
                      ((ka | va) & 15) == 0 && rows->stride_row % 8 == 0 && rows->stride_head % 8 == 0;
    const int channels = write && g->group % 32 == 0 ? 32 : 8;         // of a vector
    p.vecs = (int)((long long)g->n_kv_heads * g->head_dim / channels);
    p.seg = g->group / channels;
    p.G_shift = gs; p.D_shift = log2_exact(g->head_dim);
    // Few rows: a warp for every 32 vectors of a row (8 rows of 128 vectors, append and read: 7.2 us in one warp each, 4.7 in four).
    const int groups = (p.vecs + 31) / 32;
    p.parts = (long long)p.b.n_rows * groups <= 16 * 148 ? groups : 1;
    const long long threads = (long long)p.b.n_rows * (fast ? 32 * p.parts : 2 * g->n_kv_heads);
    const long long grid = (threads + kRowThreads - 1) / kRowThreads;
    if (grid * kRowThreads > (1ll << 32) - 1) return fail(ctx, PATCHKV_E_UNSUPPORTED, w + ": too many rows for one call");
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return fail(ctx, PATCHKV_E_CUDA, "cudaSetDevice failed");
    const bool f16 = rows->type == PATCHKV_ROWS_F16;
    if (fast) {
        PKV_CUDA(ctx, f16 ? launch_rows_tag<PATCHKV_ROWS_F16>(p, write, (unsigned)grid, stream)
                          : launch_rows_tag<PATCHKV_ROWS_BF16>(p, write, (unsigned)grid, stream));
        return PATCHKV_OK;
    }
    auto kernel = f16 ? (write ? cache_rows_any_kernel<PATCHKV_ROWS_F16, true> : cache_rows_any_kernel<PATCHKV_ROWS_F16, false>)
                      : (write ? cache_rows_any_kernel<PATCHKV_ROWS_BF16, true> : cache_rows_any_kernel<PATCHKV_ROWS_BF16, false>);
    kernel<<<(unsigned)grid, kRowThreads, 0, stream>>>(p);
    PKV_CUDA(ctx, cudaGetLastError());
    return PATCHKV_OK;
}

}  // namespace
}  // namespace patchkv

using namespace patchkv;

extern "C" int patchkv_cache_append(patchkv_ctx* ctx, const patchkv_geom* geom, const patchkv_qpool* cache, int layer,
                                    const patchkv_batch* batch, const patchkv_rows* rows, void* stream) {
    if (!ctx) return PATCHKV_E_INVALID;
    std::lock_guard<std::mutex> lock(ctx->mu);
    return cache_rows(ctx, "cache_append", geom, cache, layer, batch, rows, true, static_cast<cudaStream_t>(stream));
}

extern "C" int patchkv_cache_read(patchkv_ctx* ctx, const patchkv_geom* geom, const patchkv_qpool* cache, int layer,
                                  const patchkv_batch* batch, const patchkv_rows* rows, void* stream) {
    if (!ctx) return PATCHKV_E_INVALID;
    std::lock_guard<std::mutex> lock(ctx->mu);
    return cache_rows(ctx, "cache_read", geom, cache, layer, batch, rows, false, static_cast<cudaStream_t>(stream));
}
