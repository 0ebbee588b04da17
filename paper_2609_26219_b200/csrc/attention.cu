// Attention over a cache of quantised pages or over the bf16 pool (patchkv_attention).
#include <math.h>

#include <algorithm>

#include "attention.cuh"
#include "attention_rows.cuh"
#include "attention_split.cuh"

namespace patchkv {

// ---------------------------------------------------------------- any geometry, any strides
// One CTA per (row, query head): tiles of 128 tokens, a token per thread for the logits, channels across threads for the
// second product.  Every token a row does not see is passed over, so nothing of its slot reaches the row.
constexpr int kAnyThreads = 128;

template <int TYPE>
__global__ void __launch_bounds__(kAnyThreads) attention_any_kernel(const AttentionParams p) {
    __shared__ float q[PATCHKV_MAX_ATTENTION_DIM];
    __shared__ float w[kAnyThreads];
    __shared__ long long off_k[kAnyThreads], off_v[kAnyThreads];
    __shared__ float red[kAnyThreads / 32];
    const int s = blockIdx.z, hq = blockIdx.y, h = hq / p.share;
    int first, kv, rows;
    const bool ordered = sequence_rows(p, s, &first, &kv, &rows);
    if (threadIdx.x == 0 && (!ordered || rows > p.b.max_rows)) latch(p.status);
    if (!ordered || (int)blockIdx.x >= rows) return;
    const int r = first + blockIdx.x;
    if (p.b.kv_len[s] > kv && threadIdx.x == 0) latch(p.status);
    const int pos = row_position(p.b, s, r);
    const uint16_t* qs = p.q + (long long)r * p.q_stride_row + (long long)hq * p.q_stride_head;
    for (int c = threadIdx.x; c < p.c.D; c += kAnyThreads)
        q[c] = TYPE == PATCHKV_ROWS_F16 ? half_bits_to_float(qs[c]) : bf16_bits_to_float(qs[c]);
    __syncthreads();
    const int end = min(pos, kv - 1) + 1;                       // tokens [0, end), those outside the window by `sees`
    float m = -INFINITY, l = 0.0f, acc[2] = {0.0f, 0.0f};
    const int kf = k_format(p.c.tag), vf = v_format(p.c.tag);
    int t0 = 0;
    while (t0 < end) {
        const int t = t0 + threadIdx.x;
        float x = -INFINITY;
        off_v[threadIdx.x] = -1;
        if (t < end && sees(p, pos, t)) {
            const int lp = div_page(p.c, t), slot = t - lp * p.c.P;
            const int page = p.b.block_table[(long long)s * p.b.table_stride + lp];
            if (page < 0 || page >= p.c.n_pages) {
                latch(p.status);
            } else if (p.c.tag == PATCHKV_TAG_BF16) {
                const long long o = (long long)page * p.c.stride_page + (long long)slot * p.c.stride_token + (long long)h * p.c.stride_head;
                off_v[threadIdx.x] = o;
                x = 0.0f;
                for (int c = 0; c < p.c.D; c++) x = fmaf(q[c], bf16_bits_to_float(p.c.k[o + c]), x);
            } else {
                const uint8_t* pg = p.c.base + (long long)page * p.c.stride_page;
                const unsigned long long e = ((unsigned long long)slot * p.c.H + h) * p.c.D;
                off_v[threadIdx.x] = (long long)page;
                off_k[threadIdx.x] = (long long)e;
                x = 0.0f;
                for (int c0 = 0; c0 < p.c.D; c0 += p.c.G) {
                    float y = 0.0f;
                    for (int c = c0; c < c0 + p.c.G; c++) y = fmaf(q[c], (float)code_at(pg, kf, e + c), y);
                    x = fmaf(y, scale_at(pg + p.c.k_scales, (e + c0) / p.c.G), x);
                }
            }
            x *= p.scale_log2;
        }
        float mt = x;
        for (int d = 16; d; d >>= 1) mt = fmaxf(mt, __shfl_xor_sync(0xFFFFFFFFu, mt, d));
        if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = mt;
        __syncthreads();
        mt = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
        const float mn = fmaxf(m, mt), ref = mn == -INFINITY ? 0.0f : mn;
        const float e = off_v[threadIdx.x] >= 0 ? exp2f(x - ref) : 0.0f;
        w[threadIdx.x] = e;
        const float keep = exp2f(m - ref);
        m = mn;
        __syncthreads();
        l *= keep;
        acc[0] *= keep; acc[1] *= keep;
        for (int j = 0; j < min(kAnyThreads, end - t0); j++) {
            const long long o = off_v[j];
            if (o < 0) continue;
            l += w[j];
#pragma unroll
            for (int k = 0; k < 2; k++) {
                const int c = threadIdx.x + k * kAnyThreads;
                if (c >= p.c.D) continue;
                if (p.c.tag == PATCHKV_TAG_BF16) {
                    acc[k] = fmaf(w[j], bf16_bits_to_float(p.c.v[o + c]), acc[k]);
                } else {
                    const uint8_t* pg = p.c.base + o * p.c.stride_page;
                    const unsigned long long ec = (unsigned long long)off_k[j] + c;
                    acc[k] = fmaf(w[j], (float)code_at(pg + p.c.v_codes, vf, ec) * scale_at(pg + p.c.v_scales, ec / p.c.G), acc[k]);
                }
            }
        }
        __syncthreads();
        t0 += kAnyThreads;
        if (p.window > 0 && t0 >= p.sinks && t0 <= pos - p.window)       // skip what lies between the sinks and the window
            t0 = pos - p.window + 1;
    }
    uint16_t* o = p.out + (long long)r * p.out_stride_row + (long long)hq * p.out_stride_head;
    const float inv = l != 0.0f ? 1.0f / l : 0.0f;              // a row that sees nothing: zeros
#pragma unroll
    for (int k = 0; k < 2; k++) {
        const int c = threadIdx.x + k * kAnyThreads;
        if (c < p.c.D) {
            const float y = acc[k] * inv;
            o[c] = TYPE == PATCHKV_ROWS_F16 ? __half_as_ushort(__float2half_rn(y)) : __bfloat16_as_ushort(__float2bfloat16_rn(y));
        }
    }
}

namespace {

// Checks everything but the workspace; with `ctx` null only what the workspace's size depends on.
int check_attention(patchkv_ctx* ctx, const patchkv_geom* g, int tag, const patchkv_batch* b, int Hq, int window, int sinks) {
    if (g->head_dim > PATCHKV_MAX_ATTENTION_DIM) return fail(ctx, PATCHKV_E_UNSUPPORTED, "attention: head_dim above 256");
    if (Hq <= 0 || Hq % g->n_kv_heads) return fail(ctx, PATCHKV_E_INVALID, "attention: n_q_heads must be a positive multiple of n_kv_heads");
    if (window < 0 || sinks < 0) return fail(ctx, PATCHKV_E_INVALID, "attention: negative window or sinks");
    if (Hq > 65535 || b->n_seqs > 65535) return fail(ctx, PATCHKV_E_UNSUPPORTED, "attention: more than 65535 query heads or sequences");
    if (tag < PATCHKV_TAG_BF16 || tag > PATCHKV_TAG_K4V4) return fail(ctx, PATCHKV_E_INVALID, "attention: unknown tag");
    return PATCHKV_OK;
}

int fill_pool(patchkv_ctx* ctx, const patchkv_geom* g, const patchkv_pool* q, int layer, CacheDev* c) {
    if (q->struct_size != sizeof(patchkv_pool)) return fail(ctx, PATCHKV_E_INVALID, "attention: wrong struct_size of the pool");
    const uintptr_t k = reinterpret_cast<uintptr_t>(q->k_base), v = reinterpret_cast<uintptr_t>(q->v_base);
    if (!k || !v || ((k | v) & 15u) || q->n_pages <= 0) return fail(ctx, PATCHKV_E_INVALID, "attention: pool base null or not 16-byte aligned, or no pages");
    if (q->stride_layer < 0 || q->stride_page < 0 || q->stride_token < 0 || q->stride_head < 0)
        return fail(ctx, PATCHKV_E_INVALID, "attention: negative pool stride");
    memset(c, 0, sizeof(*c));
    c->k = static_cast<const uint16_t*>(q->k_base) + (long long)layer * q->stride_layer;
    c->v = static_cast<const uint16_t*>(q->v_base) + (long long)layer * q->stride_layer;
    c->stride_page = q->stride_page; c->stride_token = q->stride_token; c->stride_head = q->stride_head;
    c->n_pages = q->n_pages; c->H = g->n_kv_heads; c->D = g->head_dim; c->P = g->page_tokens; c->G = g->group;
    c->P_shift = log2_exact(g->page_tokens);
    c->tag = PATCHKV_TAG_BF16;
    return PATCHKV_OK;
}

constexpr int kSms = 148;                        // B200; only sizes launches, so that results don't depend on the context

// How a call is served.
struct AttentionPlan {
    int nc;                     // columns of a lane of the split kernel; 0: another kernel
    int row_tiles, row_splits;  // CTAs along the query vectors of a sequence, and along the tokens, of the row kernel; 0: another
    int heads, groups, warps_per_head;
    int target, max_items;
    long long item_stride;      // floats
    uint64_t partial_bytes, items_bytes;
    int image_steps;            // steps of a sequence whose operands are laid out in the workspace first; 0: none
    uint64_t image_bytes, meta_bytes;
};

constexpr uint64_t kMaxImageBytes = 3ull << 29;

AttentionPlan plan_attention(const patchkv_geom* g, int tag, const patchkv_batch* b, int Hq, int window, int sinks) {
    AttentionPlan a;
    memset(&a, 0, sizeof(a));
    const int D = g->head_dim, H = g->n_kv_heads;
    const bool pool = tag == PATCHKV_TAG_BF16;
    const bool shape = (D == 64 || D == 128) && g->page_tokens % kTile == 0 && (pool || g->group % 32 == 0);
    const long long cols = (long long)std::min(b->max_rows, b->n_rows) * (Hq / H);
    if (!shape || cols == 0) return a;
    if (cols > 16) {
        // Whole CTAs along the query vectors; where they leave SMs idle the tokens are split, two steps a piece at least.
        const long long tiles = (cols + 2 * kRowTile - 1) / (2 * kRowTile), ctas = tiles * H * b->n_seqs;
        if (ctas > 1 << 24 || cols > 1 << 30) return a;
        long long steps = ((long long)b->max_kv_len + kRowTile - 1) / kRowTile;
        if (window > 0) steps = std::min(steps, ((long long)window + sinks + b->max_rows) / kRowTile + 3);
        a.row_tiles = (int)tiles;
        a.row_splits = (int)std::max(1ll, std::min((long long)kSms / ctas, steps / 2));
        // Images pay where a token is needed by several CTAs of vectors: by two where they save converting codes, by eight over bf16 pages, which
        // they only copy.  With and without, 8 KV heads, 32 query heads, D 128, 64k tokens: 4-bit pages and 2, 4, 8 CTAs
        // 232 and 241, 362 and 479, 602 and 942 us; bf16 pages 245 and 172, 374 and 353, 633 and 674, and with 32 of them
        // 2091 and 2626 us.  Up to 1.5 GiB of workspace.
        const uint64_t all_steps = ((uint64_t)b->max_kv_len + kRowTile - 1) / kRowTile, images = all_steps * H * b->n_seqs;
        const uint64_t image = (pool ? 4ull : 6ull) * kRowTile * D;         // room for fp16 queries' two matrices of K
        if (tiles >= (pool ? 8 : 2) && images > 0 && images <= kMaxImageBytes / image) {
            a.image_steps = (int)all_steps;
            a.image_bytes = images * image;
            a.meta_bytes = images * 32;
        }
        if (a.row_splits > 1) a.partial_bytes = (uint64_t)a.row_splits * b->n_rows * Hq * (D + 2) * 4;
        return a;
    }
    a.nc = cols <= 4 ? 1 : cols <= 8 ? 2 : 4;
    const int warps = split_warps(pool, a.nc);
    a.heads = 1;
    for (int h = 2; h <= warps; h *= 2)         // the most heads a CTA can take without more idle warps
        if ((H + h - 1) / h * h <= (H + a.heads - 1) / a.heads * a.heads || h <= H) a.heads = h;
    a.groups = (H + a.heads - 1) / a.heads;
    a.warps_per_head = warps / a.heads;
    // Pieces: as many CTAs as there are SMs, one per SM; a sequence leaves one piece partly filled.
    const int slots = std::max(1, kSms / a.groups);
    a.target = b->n_seqs >= 2 * slots ? 0 : std::max(slots - b->n_seqs, (slots + 1) / 2);
    a.max_items = b->n_seqs + a.target;
    if (a.target) {
        a.item_stride = (a.nc == 1 ? 2 : 2 * a.nc) * (D / 16) * 32 + 2 * 4 * a.nc;
        a.items_bytes = ((uint64_t)b->n_seqs * 8 + 15) / 16 * 16;
        a.partial_bytes = (uint64_t)a.max_items * H * a.item_stride * 4;
    }
    return a;
}

bool aligned_rows(const void* x, int64_t stride_row, int64_t stride_head) {
    return (reinterpret_cast<uintptr_t>(x) & 15) == 0 && stride_row % 8 == 0 && stride_head % 8 == 0;
}

}  // namespace
}  // namespace patchkv

using namespace patchkv;

extern "C" uint64_t patchkv_attention_workspace_bytes(const patchkv_geom* g, int tag, const patchkv_batch* b, int n_q_heads,
                                                      int window, int sinks) {
    BatchDev bd;
    if (check_live_geometry(nullptr, "attention", g, 0) != PATCHKV_OK || fill_batch(nullptr, "attention", b, &bd) != PATCHKV_OK ||
        check_attention(nullptr, g, tag, b, n_q_heads, window, sinks) != PATCHKV_OK)
        return 0;
    const AttentionPlan a = plan_attention(g, tag, b, n_q_heads, window, sinks);
    return a.partial_bytes + a.items_bytes + a.image_bytes + a.meta_bytes;
}

extern "C" int patchkv_attention(patchkv_ctx* ctx, const patchkv_geom* g, const patchkv_pool* pool, const patchkv_qpool* cache,
                                 int layer, const patchkv_batch* batch, const patchkv_attention_args* a, void* stream_) {
    if (!ctx) return PATCHKV_E_INVALID;
    std::lock_guard<std::mutex> lock(ctx->mu);
    AttentionParams p;
    if ((pool != nullptr) == (cache != nullptr)) return fail(ctx, PATCHKV_E_INVALID, "attention: give a pool or a cache, one of the two");
    int rc = check_live_geometry(ctx, "attention", g, layer);
    if (rc == PATCHKV_OK) rc = fill_batch(ctx, "attention", batch, &p.b);
    if (rc == PATCHKV_OK) rc = pool ? fill_pool(ctx, g, pool, layer, &p.c) : fill_cache(ctx, "attention", g, cache, layer, &p.c);
    if (rc != PATCHKV_OK) return rc;
    if (!a || a->struct_size != sizeof(patchkv_attention_args)) return fail(ctx, PATCHKV_E_INVALID, "attention: null args or wrong struct_size");
    rc = check_attention(ctx, g, p.c.tag, batch, a->n_q_heads, a->window, a->sinks);
    if (rc != PATCHKV_OK) return rc;
    if (a->type != PATCHKV_ROWS_BF16 && a->type != PATCHKV_ROWS_F16) return fail(ctx, PATCHKV_E_INVALID, "attention: unknown row type");
    if (pool && a->type != PATCHKV_ROWS_BF16) return fail(ctx, PATCHKV_E_INVALID, "attention: over a bf16 pool q and out must be bf16");
    if (!(fabsf(a->scale) <= 3.0e38f)) return fail(ctx, PATCHKV_E_INVALID, "attention: scale must be finite");
    if (a->q_stride_row < 0 || a->q_stride_head < 0 || a->out_stride_row < 0 || a->out_stride_head < 0)
        return fail(ctx, PATCHKV_E_INVALID, "attention: negative stride");
    if (p.b.n_rows == 0 || p.b.n_seqs == 0 || p.b.max_rows == 0) return PATCHKV_OK;
    const uintptr_t qa = reinterpret_cast<uintptr_t>(a->q), oa = reinterpret_cast<uintptr_t>(a->out);
    if (!qa || !oa || (qa & 1) || (oa & 1)) return fail(ctx, PATCHKV_E_INVALID, "attention: null or misaligned q or out");
    if (rows_overlap(p.b.n_rows, a->n_q_heads, p.c.D, a->out_stride_row, a->out_stride_head))
        return fail(ctx, PATCHKV_E_INVALID, "attention: rows or heads of out overlap");
    const uint64_t need = patchkv_attention_workspace_bytes(g, p.c.tag, batch, a->n_q_heads, a->window, a->sinks);
    if (need && (!a->workspace || (reinterpret_cast<uintptr_t>(a->workspace) & 15) || a->workspace_bytes < need))
        return fail(ctx, PATCHKV_E_INVALID, "attention: workspace null, misaligned or too small");
    p.q = static_cast<const uint16_t*>(a->q); p.out = static_cast<uint16_t*>(a->out);
    p.q_stride_row = a->q_stride_row; p.q_stride_head = a->q_stride_head;
    p.out_stride_row = a->out_stride_row; p.out_stride_head = a->out_stride_head;
    p.Hq = a->n_q_heads; p.share = a->n_q_heads / g->n_kv_heads;
    p.window = a->window; p.sinks = a->sinks;
    p.scale_log2 = (float)((double)a->scale * 1.4426950408889634);
    p.status = ctx->d_status;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return fail(ctx, PATCHKV_E_CUDA, "cudaSetDevice failed");
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    p.f16 = a->type == PATCHKV_ROWS_F16;
    const AttentionPlan plan = plan_attention(g, p.c.tag, batch, a->n_q_heads, a->window, a->sinks);
    const bool aligned = aligned_rows(a->q, a->q_stride_row, a->q_stride_head) &&
                         (!pool || (pool->stride_page % 8 == 0 && pool->stride_token % 8 == 0 && pool->stride_head % 8 == 0 && pool->stride_layer % 8 == 0));
    if (plan.nc && aligned) {
        SplitPlan pl;
        memset(&pl, 0, sizeof(pl));
        pl.items = static_cast<int32_t*>(a->workspace);
        pl.partial = reinterpret_cast<float*>(static_cast<uint8_t*>(a->workspace) + plan.items_bytes);
        pl.item_stride = (int32_t)plan.item_stride;
        pl.max_items = plan.max_items; pl.target = plan.target;
        pl.heads_log2 = log2_exact(plan.heads); pl.per_head_log2 = log2_exact(plan.warps_per_head);
        pl.share_magic = (65536u + p.share - 1) / p.share;
        PKV_CUDA(ctx, p.c.D == 128 ? launch_split<128>(p, pl, plan.nc, plan.groups, stream)
                                   : launch_split<64>(p, pl, plan.nc, plan.groups, stream));
        return PATCHKV_OK;
    }
    if (plan.row_tiles && aligned && aligned_rows(a->out, a->out_stride_row, a->out_stride_head)) {
        uint8_t* ws = static_cast<uint8_t*>(a->workspace);
        const RowsPlan pl = {reinterpret_cast<float*>(ws + plan.image_bytes + plan.meta_bytes), plan.row_tiles, plan.row_splits,
                             plan.image_steps ? ws : nullptr, reinterpret_cast<uint32_t*>(ws + plan.image_bytes), plan.image_steps};
        PKV_CUDA(ctx, p.c.D == 128 ? launch_rows<128>(p, pl, stream) : launch_rows<64>(p, pl, stream));
        return PATCHKV_OK;
    }
    auto kernel = a->type == PATCHKV_ROWS_F16 ? attention_any_kernel<PATCHKV_ROWS_F16> : attention_any_kernel<PATCHKV_ROWS_BF16>;
    kernel<<<dim3(std::min(p.b.max_rows, p.b.n_rows), p.Hq, p.b.n_seqs), kAnyThreads, 0, stream>>>(p);
    PKV_CUDA(ctx, cudaGetLastError());
    return PATCHKV_OK;
}
