// Rows that get their rotary positions on their way into the cache: patchkv_rotary_append.
#include "cache_rows.cuh"
#include "rotary.cuh"

namespace patchkv {

constexpr int kRotaryThreads = 128;

struct RotaryParams {
    CacheDev c;
    BatchDev b;
    const uint16_t* q;
    uint16_t* q_out;
    const uint16_t* k;
    const uint16_t* v;
    uint16_t* k_pool;           // of a bf16 pool
    uint16_t* v_pool;
    long long q_stride_row, q_stride_head, out_stride_row, out_stride_head, k_stride_row, k_stride_head, v_stride_row, v_stride_head;
    const int32_t* rope_pos;
    int32_t* status;
    double factor;
    int32_t Hq, Dr, half;
    int32_t parts;              // warps that share a row
    int32_t q_passes, kv_passes;    // passes of a warp over the queries, and over the keys and values
    int32_t U_shift;            // log2 of the 16-channel units of a head
    int32_t G_shift;            // log2 of G
    Frequencies f;
};

// The larger of two numbers that are not negative: their bit patterns order them.
__device__ __forceinline__ unsigned long long magnitude(double x) { return __double_as_longlong(x) & 0x7FFFFFFFFFFFFFFFull; }

// Eight channels of keys -> codes and, from the group's first lane, its scale: the quantiser's definition in 64 bits, as a rotated key is not a
// 16-bit number.  (In fp32 a key within 2^-24 of the border of two codes would fall on either side, and a code is a step of up to a seventh
// of the group's largest value.)  code = rint(x / s): t = x * r with r = 1 / s to 2^-46, corrected once by its remainder; where x / s is a
// half-integer the remainder is exact and the correction gives it.  Adding 1.5 * 2^52 rounds, ties to even.
template <int FMT>
__device__ __forceinline__ uint32_t scale64(double amax) {
    return __half_as_ushort(__double2half(amax * (1.0 / (FMT == FMT_INT8 ? 127.0 : 7.0))));
}
template <int FMT>
__device__ __forceinline__ void codes64(const double* x, uint32_t s16, uint8_t* codes) {
    constexpr double qmax = FMT == FMT_INT8 ? 127.0 : 7.0;
    const bool usable = s16 != 0 && s16 < 0x7C00u;          // a zero or infinite scale: all codes zero
    const float sf = half_bits_to_float(usable ? s16 : 0x3C00u);
    float rf;
    asm("rcp.approx.f32 %0, %1;" : "=f"(rf) : "f"(sf));
    const double s = sf;
    double r = rf;
    r = fma(fma(-s, r, 1.0), r, r);
    uint32_t code[8];
#pragma unroll
    for (int i = 0; i < 8; i++) {
        double t = x[i] * r;
        t = fma(fma(-t, s, x[i]), r, t);
        code[i] = (uint32_t)__double2loint(t + 6755399441055744.0);
    }
    if (s16 < 0x0400u)                                      // a subnormal scale; else |t| <= qmax (1 + 2^-11), which rounds to qmax
#pragma unroll
        for (int i = 0; i < 8; i++) code[i] = (uint32_t)min(max((int)code[i], -(int)qmax), (int)qmax);
    uint32_t w[2];
#pragma unroll
    for (int i = 0; i < 2; i++)
        w[i] = usable ? __byte_perm(__byte_perm(code[4 * i], code[4 * i + 1], 0x0040), __byte_perm(code[4 * i + 2], code[4 * i + 3], 0x0040), 0x5410) : 0u;
    if (FMT == FMT_INT8) {
        *reinterpret_cast<uint2*>(codes) = make_uint2(w[0], w[1]);
    } else {
#pragma unroll
        for (int i = 0; i < 2; i++) {
            w[i] &= 0x0F0F0F0Fu;
            w[i] = (w[i] | w[i] >> 4) & 0x00FF00FFu;
        }
        *reinterpret_cast<uint32_t*>(codes) = __byte_perm(w[0], w[1], 0x6420);
    }
}

// A warp takes a row, or every `parts`-th pass of one; a pass is 32 units of 16 channels of the queries, or of the keys and the values.  A lane has
// the same channels of a head in every pass, both of each rotary pair among them (rotary.cuh), so it keeps their cosines and sines in registers
// and exchanges nothing but the maxima of the keys' groups (with the pairs' other halves brought by shuffles 166 us where this takes 116, 16384
// rows of 32 query heads and 8 KV heads into 4-bit pages).  Two units of a lane are on their way at a time (95 us for 116).  Bound by
// memory into a bf16 pool (403 MB in 68 us, 5.9 TB/s); for quantised pages (354 MB in 76 us) by latency beside the 64-bit work on the keys: fp64
// pipe 12 %, issue slots 49 %, a third of the warps active, most of them waiting on loads.
template <int TYPE, int KF, int VF, bool HALF>
__global__ void __launch_bounds__(kRotaryThreads, KF == FMT_BF16 ? 8 : 6) rotary_append_kernel(const __grid_constant__ RotaryParams p) {
    constexpr bool kPool = KF == FMT_BF16;
    constexpr int kPairs = PATCHKV_MAX_ROTARY_DIM / 2, kWarps = kRotaryThreads / 32;
    __shared__ double2 exact[kPool ? 1 : kWarps][kPool ? 1 : kPairs];       // of angle 8 u + i at i * Dr / 16 + u
    __shared__ __align__(16) float cosine[kWarps][kPairs], sine[kWarps][kPairs];
    pdl_trigger();
    const uint32_t wid = (blockIdx.x * kRotaryThreads + threadIdx.x) >> 5;
    const int r = (int)(wid / (uint32_t)p.parts), part = (int)(wid - (uint32_t)r * p.parts), lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (r >= p.b.n_rows) return;
    pdl_wait();
    const int u = lane & ((1 << p.U_shift) - 1), sub = lane >> p.U_shift, per_pass = 32 >> p.U_shift;       // unit, head of a pass, heads of a pass
    const int ch0 = first_run(HALF, p.Dr, u), ch1 = second_run(HALF, p.Dr, u);
    struct Unit { uint4 a, b; };
    auto load = [&](const uint16_t* from, int c0, int c1, bool live) {
        Unit x = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
        if (live) {
            x.a = *reinterpret_cast<const uint4*>(from + c0);
            x.b = *reinterpret_cast<const uint4*>(from + c1);
        }
        return x;
    };
    auto store = [&](uint16_t* to, int c0, int c1, const uint32_t (&w)[8]) {
        *reinterpret_cast<uint4*>(to + c0) = make_uint4(w[0], w[1], w[2], w[3]);
        *reinterpret_cast<uint4*>(to + c1) = make_uint4(w[4], w[5], w[6], w[7]);
    };
    int slot = 0, pos = 0;
    const int pg = find_page<true>(p, r, lane == 0 && part == 0, &slot, &pos);
    if (pg >= 0) {
        if (p.rope_pos) pos = p.rope_pos[r];
        for (int i = lane; i < p.Dr >> 1; i += 32) {
            double c, s;
            cos_sin((double)pos * p.f.theta[i], &c, &s);
            c *= p.factor;
            s *= p.factor;
            if (!kPool) exact[warp][(i & 7) * (p.Dr >> 4) + (i >> 3)] = make_double2(c, s);
            cosine[warp][i] = (float)c;
            sine[warp][i] = (float)s;
        }
        __syncwarp();
        const bool turns = 16 * u < p.Dr;
        float c[8], s[8];
        {
            const float4* a = reinterpret_cast<const float4*>(&cosine[warp][turns ? 8 * u : 0]);
            const float4* b = reinterpret_cast<const float4*>(&sine[warp][turns ? 8 * u : 0]);
            const float4 c0 = a[0], c1 = a[1], s0 = b[0], s1 = b[1];
            c[0] = c0.x; c[1] = c0.y; c[2] = c0.z; c[3] = c0.w; c[4] = c1.x; c[5] = c1.y; c[6] = c1.z; c[7] = c1.w;
            s[0] = s0.x; s[1] = s0.y; s[2] = s0.z; s[3] = s0.w; s[4] = s1.x; s[5] = s1.y; s[6] = s1.z; s[7] = s1.w;
        }
        int pass = part;
        {
            const uint16_t* q = p.q + (long long)r * p.q_stride_row + (long long)(pass * per_pass + sub) * p.q_stride_head;
            uint16_t* out = p.q_out + (long long)r * p.out_stride_row + (long long)(pass * per_pass + sub) * p.out_stride_head;
            const long long q_step = (long long)p.parts * per_pass * p.q_stride_head, out_step = (long long)p.parts * per_pass * p.out_stride_head;
            const int h_step = p.parts * per_pass;
            int h = pass * per_pass + sub;
#pragma unroll 1
            for (; pass < p.q_passes; pass += 2 * p.parts, h += 2 * h_step) {
                const bool live0 = h < p.Hq, live1 = h + h_step < p.Hq;
                const Unit x = load(q, ch0, ch1, live0), y = load(q + q_step, ch0, ch1, live1);
                uint32_t w[8] = {x.a.x, x.a.y, x.a.z, x.a.w, x.b.x, x.b.y, x.b.z, x.b.w};
                if (turns) turn_words<TYPE, HALF>(w, c, s);
                if (live0) store(out, ch0, ch1, w);
                uint32_t v[8] = {y.a.x, y.a.y, y.a.z, y.a.w, y.b.x, y.b.y, y.b.z, y.b.w};
                if (turns) turn_words<TYPE, HALF>(v, c, s);
                if (live1) store(out + out_step, ch0, ch1, v);
                q += 2 * q_step;
                out += 2 * out_step;
            }
            // (a warp whose second unit would have been the first pass behind the queries has not done that one)
            if (pass - p.parts >= p.q_passes) pass -= p.parts;
        }
        const long long row = kPool ? (long long)pg * p.c.stride_page + (long long)slot * p.c.stride_token : (long long)pg * p.c.stride_page;
#pragma unroll 1
        for (; pass < p.q_passes + p.kv_passes; pass += p.parts) {
            const int h = (pass - p.q_passes) * per_pass + sub;
            const bool live = h < p.c.H;
            const Unit x = load(p.k + (long long)r * p.k_stride_row + (long long)h * p.k_stride_head, ch0, ch1, live);
            const Unit y = load(p.v + (long long)r * p.v_stride_row + (long long)h * p.v_stride_head, 16 * u, 16 * u + 8, live);
            uint32_t w[8] = {x.a.x, x.a.y, x.a.z, x.a.w, x.b.x, x.b.y, x.b.z, x.b.w};
            if constexpr (kPool) {
                if (turns) turn_words<TYPE, HALF>(w, c, s);
                const uint32_t v[8] = {y.a.x, y.a.y, y.a.z, y.a.w, y.b.x, y.b.y, y.b.z, y.b.w};
                if (live) {
                    store(p.k_pool + row + (long long)h * p.c.stride_head, ch0, ch1, w);
                    store(p.v_pool + row + (long long)h * p.c.stride_head, 16 * u, 16 * u + 8, v);
                }
            } else {
                uint8_t* page = p.c.base + row;
                const uint32_t head = ((uint32_t)slot * p.c.H + h) * p.c.D;
                {
                    const uint4 v[2] = {y.a, y.b};
                    const uint32_t at = head + 16 * u, seg = 1u << (p.G_shift - 4);
                    encode<TYPE, VF, 16>(v, page + p.c.v_codes + (VF == FMT_INT8 ? at : at >> 1),
                                         (u & (seg - 1)) == 0 ? page + p.c.v_scales + 2 * (at >> p.G_shift) : nullptr, (int)seg, live);
                }
                double z[16];                               // the runs: 0 .. 7 and 8 .. 15
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    z[2 * i] = low_float<TYPE>(w[i]);
                    z[2 * i + 1] = high_float<TYPE>(w[i]);
                }
                if (turns)
#pragma unroll
                    for (int i = 0; i < 8; i++) {
                        const double2 t = exact[warp][i * (p.Dr >> 4) + u];
                        double& a = z[HALF ? i : 2 * i];
                        double& b = z[HALF ? 8 + i : 2 * i + 1];
                        const double e = fma(-b, t.y, a * t.x);
                        b = fma(b, t.x, a * t.y);
                        a = e;
                    }
                // A group lies in 8 channels of each of G / 8 lanes, or (joint) in all 16 of G / 16: behind the rotary channels, where it has
                // them all, and in the interleaved layout.
                const bool joint = !HALF || !turns || p.Dr <= 1 << p.G_shift;
                unsigned long long m0 = 0, m1 = 0;
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    m0 = max(m0, magnitude(z[i]));
                    m1 = max(m1, magnitude(z[8 + i]));
                }
                if (joint) m0 = m1 = max(m0, m1);
                const int lanes = 1 << (p.G_shift - (joint ? 4 : 3));
                for (int d = 1; d < 1 << (p.G_shift - 3) && d < 1 << p.U_shift; d <<= 1) {
                    const unsigned long long a = __shfl_xor_sync(0xFFFFFFFFu, m0, d), b = __shfl_xor_sync(0xFFFFFFFFu, m1, d);
                    if (d < lanes) { m0 = max(m0, a); m1 = max(m1, b); }
                }
                if (live) {
                    const uint32_t s0 = scale64<KF>(__longlong_as_double((long long)m0)), s1 = joint ? s0 : scale64<KF>(__longlong_as_double((long long)m1));
                    const uint32_t at0 = head + ch0, at1 = head + ch1;
                    codes64<KF>(z, s0, page + (KF == FMT_INT8 ? at0 : at0 >> 1));
                    codes64<KF>(z + 8, s1, page + (KF == FMT_INT8 ? at1 : at1 >> 1));
                    if ((u & (lanes - 1)) == 0) {
                        *reinterpret_cast<uint16_t*>(page + p.c.k_scales + 2 * (at0 >> p.G_shift)) = (uint16_t)s0;
                        if (!joint) *reinterpret_cast<uint16_t*>(page + p.c.k_scales + 2 * (at1 >> p.G_shift)) = (uint16_t)s1;
                    }
                }
            }
        }
    }
    check_entries(p.b, p.status, blockIdx.x * kRotaryThreads + threadIdx.x, (uint32_t)p.b.n_rows * p.parts * 32);
}

// Any geometry, any strides: one thread per (row, head) of the queries, keys and values.
template <int TYPE>
__global__ void __launch_bounds__(kRotaryThreads) rotary_any_kernel(const __grid_constant__ RotaryParams p) {
    const uint32_t i = blockIdx.x * kRotaryThreads + threadIdx.x, per_row = (uint32_t)p.Hq + 2u * p.c.H;
    const int r = (int)(i / per_row), q = (int)(i - (uint32_t)r * per_row);
    if (r >= p.b.n_rows) return;
    check_entries(p.b, p.status, i, (uint32_t)p.b.n_rows * per_row);
    int slot = 0, pos = 0;
    const int pg = find_page<true>(p, r, q == 0, &slot, &pos);
    if (pg < 0) return;
    if (p.rope_pos) pos = p.rope_pos[r];
    const int kind = q < p.Hq ? 0 : q < p.Hq + p.c.H ? 1 : 2, h = q - (kind == 0 ? 0 : kind == 1 ? p.Hq : p.Hq + p.c.H), D = p.c.D;
    const uint16_t* x = kind == 0 ? p.q + (long long)r * p.q_stride_row + (long long)h * p.q_stride_head
                      : kind == 1 ? p.k + (long long)r * p.k_stride_row + (long long)h * p.k_stride_head
                                  : p.v + (long long)r * p.v_stride_row + (long long)h * p.v_stride_head;
    const int Dr = kind == 2 ? 0 : p.Dr;
    const bool half = p.half, pool = p.c.tag == PATCHKV_TAG_BF16;
    if (kind == 0 || pool) {
        const long long row = (long long)pg * p.c.stride_page + (long long)slot * p.c.stride_token + (long long)h * p.c.stride_head;
        uint16_t* y = kind == 0 ? p.q_out + (long long)r * p.out_stride_row + (long long)h * p.out_stride_head : (kind == 1 ? p.k_pool : p.v_pool) + row;
        for (int j = 0; j < Dr >> 1; j++) {
            const int c0 = half ? j : 2 * j, c1 = half ? j + (Dr >> 1) : 2 * j + 1;
            double c, s;
            cos_sin((double)pos * p.f.theta[j], &c, &s);
            const float cf = (float)(p.factor * c), sf = (float)(p.factor * s), a = to_float<TYPE>(x[c0]), b = to_float<TYPE>(x[c1]);
            y[c0] = (uint16_t)pack_pair<TYPE>(fmaf(-b, sf, a * cf), 0.0f);
            y[c1] = (uint16_t)pack_pair<TYPE>(fmaf(b, cf, a * sf), 0.0f);
        }
        for (int c = Dr; c < D; c++) y[c] = x[c];
        return;
    }
    const int fmt = kind == 2 ? v_format(p.c.tag) : k_format(p.c.tag);
    uint8_t* page = p.c.base + (long long)pg * p.c.stride_page;
    uint8_t* codes = page + (kind == 2 ? p.c.v_codes : 0u);
    uint8_t* scales = page + (kind == 2 ? p.c.v_scales : p.c.k_scales);
    const unsigned long long e0 = ((unsigned long long)slot * p.c.H + h) * D;
    auto value = [&](int ch) {                              // the rotated key, or the value
        if (ch >= Dr) return (double)to_float<TYPE>(x[ch]);
        const int n = Dr >> 1, j = half ? ch % n : ch >> 1, second = half ? ch >= n : ch & 1;
        double c, s;
        cos_sin((double)pos * p.f.theta[j], &c, &s);
        const double a = to_float<TYPE>(x[half ? j : 2 * j]), b = to_float<TYPE>(x[half ? j + n : 2 * j + 1]);
        c *= p.factor;
        s *= p.factor;
        return second ? fma(b, c, a * s) : fma(-b, s, a * c);
    };
    const double qmax = fmt == FMT_INT8 ? 127.0 : 7.0;
    int low = 0;
    for (int c0 = 0; c0 < D; c0 += p.c.G) {
        const unsigned long long group = (e0 + c0) / p.c.G;
        double amax = 0.0;
        for (int c = c0; c < c0 + p.c.G; c++) amax = fmax(amax, fabs(value(c)));
        const float sf = __half2float(__double2half(amax / qmax));
        const uint32_t sb = pack_pair<PATCHKV_ROWS_F16>(sf, 0.0f);      // its bits: exact (stored byte by byte from
                                                                        // the 64-bit conversion itself the low byte came out wrong)
        const double s = sf;
        scales[2 * group] = (uint8_t)sb;
        scales[2 * group + 1] = (uint8_t)(sb >> 8);
        const bool usable = s > 0.0 && s <= 65504.0;
        for (int c = c0; c < c0 + p.c.G; c++) {
            const int code = usable ? (int)fmin(fmax(rint(value(c) / s), -qmax), qmax) : 0;
            if (fmt == FMT_INT8) codes[e0 + c] = (uint8_t)code;
            else if ((c & 1) == 0) low = code & 15;         // D is even: the pair is this thread's
            else codes[(e0 + c) >> 1] = (uint8_t)(low | (code & 15) << 4);
        }
    }
}

int fill_frequencies(patchkv_ctx* ctx, const char* who, const patchkv_geom* g, Frequencies* f) {
    const std::string w(who);
    if (g->rotary_dim < 0 || g->rotary_dim > g->head_dim || (g->rotary_dim & 1)) return fail(ctx, PATCHKV_E_INVALID, w + ": rotary_dim must be even and at most head_dim");
    if (g->rope_style != PATCHKV_ROPE_HALF && g->rope_style != PATCHKV_ROPE_INTERLEAVED) return fail(ctx, PATCHKV_E_INVALID, w + ": unknown rope_style");
    if (g->rotary_dim > PATCHKV_MAX_ROTARY_DIM) return fail(ctx, PATCHKV_E_UNSUPPORTED, w + ": rotary_dim above 256");
    if (!g->inv_freq && g->rotary_dim > 0 && !(g->rope_base > 0.0 && g->rope_base <= 1e300)) return fail(ctx, PATCHKV_E_INVALID, w + ": rope_base must be positive and finite");
    const int n = g->rotary_dim / 2;
    for (int i = 0; i < n; i++) {
        f->theta[i] = g->inv_freq ? (double)g->inv_freq[i] : pow(g->rope_base, -2.0 * (double)i / (double)g->rotary_dim);
        if (!(fabs(f->theta[i]) <= 65536.0)) return fail(ctx, PATCHKV_E_INVALID, w + ": a frequency is above 65536 or not a number");
    }
    return PATCHKV_OK;
}

namespace {

template <int TYPE, int KF, int VF>
cudaError_t launch_rotary_style(const RotaryParams& p, bool half, unsigned grid, cudaStream_t stream) {
    return half ? launch_pdl(rotary_append_kernel<TYPE, KF, VF, true>, dim3(grid), dim3(kRotaryThreads), 0, stream, p)
                : launch_pdl(rotary_append_kernel<TYPE, KF, VF, false>, dim3(grid), dim3(kRotaryThreads), 0, stream, p);
}
template <int TYPE>
cudaError_t launch_rotary_tag(const RotaryParams& p, bool half, unsigned grid, cudaStream_t stream) {
    if (p.c.tag == PATCHKV_TAG_INT8) return launch_rotary_style<TYPE, FMT_INT8, FMT_INT8>(p, half, grid, stream);
    if (p.c.tag == PATCHKV_TAG_INT4) return launch_rotary_style<TYPE, FMT_INT8, FMT_INT4>(p, half, grid, stream);
    return launch_rotary_style<TYPE, FMT_INT4, FMT_INT4>(p, half, grid, stream);
}

bool vectors(const void* x, int64_t stride_row, int64_t stride_head) {
    return (reinterpret_cast<uintptr_t>(x) & 15) == 0 && stride_row % 8 == 0 && stride_head % 8 == 0;
}

}  // namespace
}  // namespace patchkv

using namespace patchkv;

extern "C" int patchkv_rotary_append(patchkv_ctx* ctx, const patchkv_geom* g, const patchkv_pool* pool, const patchkv_qpool* cache,
                                     int layer, const patchkv_batch* batch, const patchkv_rotary_args* a, void* stream_) {
    if (!ctx) return PATCHKV_E_INVALID;
    std::lock_guard<std::mutex> lock(ctx->mu);
    RotaryParams p;
    if ((pool != nullptr) == (cache != nullptr)) return fail(ctx, PATCHKV_E_INVALID, "rotary_append: give a pool or a cache, one of the two");
    int rc = check_live_geometry(ctx, "rotary_append", g, layer);
    if (rc == PATCHKV_OK) rc = fill_frequencies(ctx, "rotary_append", g, &p.f);
    if (rc == PATCHKV_OK) rc = fill_batch(ctx, "rotary_append", batch, &p.b);
    if (rc == PATCHKV_OK) rc = pool ? fill_pool(ctx, "rotary_append", g, pool, layer, &p.c) : fill_cache(ctx, "rotary_append", g, cache, layer, &p.c);
    if (rc == PATCHKV_OK && pool) rc = check_written_pool(ctx, "rotary_append", g, pool);
    if (rc != PATCHKV_OK) return rc;
    if (!a || a->struct_size != sizeof(patchkv_rotary_args)) return fail(ctx, PATCHKV_E_INVALID, "rotary_append: null args or wrong struct_size");
    if (a->type != PATCHKV_ROWS_BF16 && a->type != PATCHKV_ROWS_F16) return fail(ctx, PATCHKV_E_INVALID, "rotary_append: unknown row type");
    if (pool && a->type != PATCHKV_ROWS_BF16) return fail(ctx, PATCHKV_E_INVALID, "rotary_append: rows into a bf16 pool must be bf16");
    if (!(fabsf(a->factor) <= 3.0e38f)) return fail(ctx, PATCHKV_E_INVALID, "rotary_append: factor must be finite");
    if (a->n_q_heads < 0 || a->n_q_heads > 65535) return fail(ctx, PATCHKV_E_INVALID, "rotary_append: n_q_heads must lie in [0, 65535]");
    if (a->q_stride_row < 0 || a->q_stride_head < 0 || a->q_out_stride_row < 0 || a->q_out_stride_head < 0 || a->k_stride_row < 0 ||
        a->k_stride_head < 0 || a->v_stride_row < 0 || a->v_stride_head < 0)
        return fail(ctx, PATCHKV_E_INVALID, "rotary_append: negative stride");
    if (p.b.n_rows == 0 || p.b.n_seqs == 0) return PATCHKV_OK;
    const uintptr_t ka = reinterpret_cast<uintptr_t>(a->k), va = reinterpret_cast<uintptr_t>(a->v), qa = reinterpret_cast<uintptr_t>(a->q),
                    oa = reinterpret_cast<uintptr_t>(a->q_out);
    if (!ka || !va || ((ka | va) & 1)) return fail(ctx, PATCHKV_E_INVALID, "rotary_append: null or misaligned k or v");
    if (a->n_q_heads > 0) {
        if (!qa || !oa || ((qa | oa) & 1)) return fail(ctx, PATCHKV_E_INVALID, "rotary_append: null or misaligned q or q_out");
        if (rows_overlap(p.b.n_rows, a->n_q_heads, p.c.D, a->q_out_stride_row, a->q_out_stride_head))
            return fail(ctx, PATCHKV_E_INVALID, "rotary_append: rows or heads of q_out overlap");
        if (qa == oa && (a->q_stride_row != a->q_out_stride_row || a->q_stride_head != a->q_out_stride_head))
            return fail(ctx, PATCHKV_E_INVALID, "rotary_append: q in place needs the same strides");
    }
    p.q = static_cast<const uint16_t*>(a->q); p.q_out = static_cast<uint16_t*>(a->q_out);
    p.k = static_cast<const uint16_t*>(a->k); p.v = static_cast<const uint16_t*>(a->v);
    p.k_pool = const_cast<uint16_t*>(p.c.k); p.v_pool = const_cast<uint16_t*>(p.c.v);
    p.q_stride_row = a->q_stride_row; p.q_stride_head = a->q_stride_head;
    p.out_stride_row = a->q_out_stride_row; p.out_stride_head = a->q_out_stride_head;
    p.k_stride_row = a->k_stride_row; p.k_stride_head = a->k_stride_head;
    p.v_stride_row = a->v_stride_row; p.v_stride_head = a->v_stride_head;
    p.rope_pos = a->rope_pos;
    p.status = ctx->d_status;
    p.factor = a->factor;
    p.Hq = a->n_q_heads; p.Dr = g->rotary_dim;
    const bool half = g->rope_style == PATCHKV_ROPE_HALF, f16 = a->type == PATCHKV_ROWS_F16;
    const int D = g->head_dim, ds = log2_exact(D), gs = log2_exact(g->group);
    bool fast = ds >= 4 && ds <= 8 && g->rotary_dim % 16 == 0 && vectors(a->k, a->k_stride_row, a->k_stride_head) &&
                vectors(a->v, a->v_stride_row, a->v_stride_head);
    if (p.Hq) fast = fast && vectors(a->q, a->q_stride_row, a->q_stride_head) && vectors(a->q_out, a->q_out_stride_row, a->q_out_stride_head);
    const long long elems = (long long)g->page_tokens * g->n_kv_heads * D;
    if (pool) fast = fast && p.c.stride_page % 8 == 0 && p.c.stride_token % 8 == 0 && p.c.stride_head % 8 == 0 && pool->stride_layer % 8 == 0;
    // (a group's channels have to lie in one run of each of its lanes, or in both)
    else fast = fast && gs >= 4 && elems % 32 == 0 && (elems / g->group) % 8 == 0 && (!half || p.Dr <= g->group || (p.Dr / 2) % g->group == 0);
    p.G_shift = gs < 0 ? 0 : gs;
    p.U_shift = fast ? ds - 4 : 0;
    p.half = half;
    p.parts = 1;
    if (fast) {
        const int per_pass = 32 >> p.U_shift;               // heads
        p.q_passes = (p.Hq + per_pass - 1) / per_pass;
        p.kv_passes = (g->n_kv_heads + per_pass - 1) / per_pass;
        // Few rows: a warp for each pass of a row (32 query heads and 8 KV heads of 128 channels, replayed: 8, 64, 256 and 512 rows 3.4, 4.8, 6.6
        // and 9.8 us; with a warp for a row 5.6, 6.2, 6.8 and 8.7).
        const int passes = p.q_passes + p.kv_passes;
        if ((long long)p.b.n_rows * passes <= 32 * 148) p.parts = passes;
    }
    const long long threads = (long long)p.b.n_rows * (fast ? 32 * p.parts : p.Hq + 2 * g->n_kv_heads);
    const long long grid = (threads + kRotaryThreads - 1) / kRotaryThreads;
    if (grid * kRotaryThreads > (1ll << 32) - 1) return fail(ctx, PATCHKV_E_UNSUPPORTED, "rotary_append: too many rows for one call");
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return fail(ctx, PATCHKV_E_CUDA, "cudaSetDevice failed");
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    if (fast) {
        const cudaError_t e = pool ? launch_rotary_style<PATCHKV_ROWS_BF16, FMT_BF16, FMT_BF16>(p, half, (unsigned)grid, stream)
                            : f16 ? launch_rotary_tag<PATCHKV_ROWS_F16>(p, half, (unsigned)grid, stream)
                                  : launch_rotary_tag<PATCHKV_ROWS_BF16>(p, half, (unsigned)grid, stream);
        PKV_CUDA(ctx, e);
        return PATCHKV_OK;
    }
    if (f16) rotary_any_kernel<PATCHKV_ROWS_F16><<<(unsigned)grid, kRotaryThreads, 0, stream>>>(p);
    else rotary_any_kernel<PATCHKV_ROWS_BF16><<<(unsigned)grid, kRotaryThreads, 0, stream>>>(p);
    PKV_CUDA(ctx, cudaGetLastError());
    return PATCHKV_OK;
}
