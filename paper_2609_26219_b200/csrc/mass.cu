// The attention weight that cached tokens receive (patchkv_attention_mass).
#include <math.h>

#include <algorithm>

#include "mass_rows.cuh"
#include "mass_split.cuh"

namespace patchkv {

// ---------------------------------------------------------------- any geometry, any strides
constexpr int kMassThreads = 128;

// scale * log2(e) * q . k of a token at a place of the cache (pools: element offset; quantised pages: page and element index).
struct KeyPlace { long long at; unsigned long long e; };
__device__ __forceinline__ bool find_key(const AttentionParams& p, int s, int t, int h, KeyPlace* k) {
    const int lp = div_page(p.c, t), slot = t - lp * p.c.P;
    const int page = p.b.block_table[(long long)s * p.b.table_stride + lp];
    if (page < 0 || page >= p.c.n_pages) return false;
    if (p.c.tag == PATCHKV_TAG_BF16) {
        k->at = (long long)page * p.c.stride_page + (long long)slot * p.c.stride_token + (long long)h * p.c.stride_head;
    } else {
        k->at = (long long)page * p.c.stride_page;
        k->e = ((unsigned long long)slot * p.c.H + h) * p.c.D;
    }
    return true;
}
__device__ __forceinline__ float logit(const AttentionParams& p, const KeyPlace& k, const float* q) {
    float x = 0.0f;
    if (p.c.tag == PATCHKV_TAG_BF16) {
        for (int c = 0; c < p.c.D; c++) x = fmaf(q[c], bf16_bits_to_float(p.c.k[k.at + c]), x);
    } else {
        const uint8_t* pg = p.c.base + k.at;
        const int fmt = k_format(p.c.tag);
        for (int c0 = 0; c0 < p.c.D; c0 += p.c.G) {
            float y = 0.0f;
            for (int c = c0; c < c0 + p.c.G; c++) y = fmaf(q[c], (float)code_at(pg, fmt, k.e + c), y);
            x = fmaf(y, scale_at(pg + p.c.k_scales, (k.e + c0) / p.c.G), x);
        }
    }
    return x * p.scale_log2;
}
__device__ __forceinline__ void load_query(const AttentionParams& p, int r, int hq, float* q) {
    const uint16_t* qs = p.q + (long long)r * p.q_stride_row + (long long)hq * p.q_stride_head;
    for (int c = threadIdx.x; c < p.c.D; c += kMassThreads) q[c] = p.f16 ? half_bits_to_float(qs[c]) : bf16_bits_to_float(qs[c]);
}

// One CTA per (row, query head): log2 of the sum of 2^logit over the tokens that the row sees; NaN for a row whose logits are all minus
// infinity, infinity for one that sees none.
__global__ void __launch_bounds__(kMassThreads) mass_sums_any_kernel(const AttentionParams p, float* sums) {
    __shared__ float q[PATCHKV_MAX_ATTENTION_DIM];
    __shared__ float2 red[kMassThreads];
    const int s = blockIdx.z, hq = blockIdx.y, h = hq / p.share;
    int first, kv, rows;
    const bool ordered = sequence_rows(p, s, &first, &kv, &rows);
    if (threadIdx.x == 0 && (!ordered || rows > p.b.max_rows || (rows > 0 && p.b.kv_len[s] > kv))) latch(p.status);
    if (!ordered || (int)blockIdx.x >= min(rows, p.b.max_rows)) return;
    const int r = first + blockIdx.x, pos = row_position(p.b, s, r);
    load_query(p, r, hq, q);
    __syncthreads();
    float m = -INFINITY, l = 0.0f;
    bool saw = false;
    const int end = min(pos, kv - 1) + 1;
    for (uint32_t at = threadIdx.x; end > 0 && at < (uint32_t)end; at += kMassThreads) {       // (of 2^31 - 1 tokens the step behind the last is above 2^31)
        const int t = (int)at;
        if (!sees(p, pos, t)) continue;
        KeyPlace k;
        if (!find_key(p, s, t, h, &k)) { latch(p.status); continue; }
        const float x = logit(p, k, q), to = fmaxf(m, x);      // (a NaN leaves the maximum as it is, and stays in the sum)
        saw = true;
        if (x == -INFINITY) continue;
        l = x != x ? x : l * exp2f(m - to) + exp2f(x - to);
        m = to;
    }
    red[threadIdx.x] = make_float2(m, l);
    saw = __syncthreads_or(saw);
    if (threadIdx.x != 0) return;
    for (int i = 0; i < kMassThreads; i++) m = fmaxf(m, red[i].x);
    l = 0.0f;
    for (int i = 0; i < kMassThreads; i++) l += red[i].x == m ? red[i].y : red[i].y * exp2f(red[i].x - m);      // (m may be -infinity)
    sums[(long long)r * p.Hq + hq] = l != 0.0f ? m + log2f(l) : saw ? NAN : INFINITY;
}

// A thread per token: the weights of all rows and heads, in order.
__global__ void __launch_bounds__(kMassThreads) mass_columns_any_kernel(const AttentionParams p, const WeightParams m, const float* sums) {
    __shared__ float q[PATCHKV_MAX_ATTENTION_DIM];
    const int s = blockIdx.y, t = blockIdx.x * kMassThreads + threadIdx.x;
    int first, kv, rows;
    if (!sequence_rows(p, s, &first, &kv, &rows)) {
        if (threadIdx.x == 0) latch(p.status);                  // (of a call without rows nobody has looked)
        return;
    }
    rows = min(rows, p.b.max_rows);
    float total = 0.0f;
    for (int hq = 0; hq < p.Hq; hq++) {
        KeyPlace k;
        const bool there = t < kv && find_key(p, s, t, hq / p.share, &k);
        float sum = 0.0f;
        for (int i = 0; i < rows; i++) {
            const int r = first + i, pos = row_position(p.b, s, r);
            __syncthreads();
            load_query(p, r, hq, q);
            __syncthreads();
            if (there && t <= pos && sees(p, pos, t)) sum += exp2f(logit(p, k, q) - sums[(long long)r * p.Hq + hq]);
        }
        total += sum;
    }
    if (t < kv) store_mass(p, m, s, t, total);
}

namespace {

int check_mass(patchkv_ctx* ctx, const patchkv_geom* g, int tag, const patchkv_batch* b, int Hq, int window, int sinks) {
    if (g->head_dim > PATCHKV_MAX_ATTENTION_DIM) return fail(ctx, PATCHKV_E_UNSUPPORTED, "attention_mass: head_dim above 256");
    if (Hq <= 0 || Hq % g->n_kv_heads) return fail(ctx, PATCHKV_E_INVALID, "attention_mass: n_q_heads must be a positive multiple of n_kv_heads");
    if (window < 0 || sinks < 0) return fail(ctx, PATCHKV_E_INVALID, "attention_mass: negative window or sinks");
    if (Hq > 65535 || b->n_seqs > 65535) return fail(ctx, PATCHKV_E_UNSUPPORTED, "attention_mass: more than 65535 query heads or sequences");
    if (tag < PATCHKV_TAG_BF16 || tag > PATCHKV_TAG_K4V4) return fail(ctx, PATCHKV_E_INVALID, "attention_mass: unknown tag");
    return PATCHKV_OK;
}

constexpr int kSms = 148;                        // B200; only sizes launches, so that results don't depend on the context

// How a call is served, and its workspace.
struct MassPlan {
    int nc;                     // columns of a lane of the split kernel; 0: another kernel
    int heads, groups, warps_per_head, target, max_items, cols, tokens;
    uint64_t items_bytes, sums_bytes, bytes;
    int row_tiles, row_splits, one, chunk, steps;       // the row kernels (0 tiles: another): CTAs along the vectors and the tokens, whether there is one tile
                                // of vectors, CTAs along the vectors of a launch of the second pass, steps of a sequence that have images
    uint64_t ranges_bytes, acc_bytes, partial_bytes, image_bytes, meta_bytes;
};

// Steps of an item of the row kernels: some of their waits take as long as an item (a million tokens, 30 ms), well below the limit of a wait.
constexpr long long kMaxItemSteps = 8192;
constexpr uint64_t kMaxMassImages = 3ull << 29, kMaxMassPartial = 1ull << 28;
uint64_t round16(uint64_t x) { return (x + 15) / 16 * 16; }

// Tokens that a sequence can have: max_kv_len, or what its block table has room for.
long long longest_sequence(const patchkv_geom* g, const patchkv_batch* b) {
    return std::min((long long)b->max_kv_len, (long long)b->table_stride * g->page_tokens);
}

MassPlan plan_mass(const patchkv_geom* g, int tag, const patchkv_batch* b, int Hq, int window, int sinks) {
    MassPlan a;
    memset(&a, 0, sizeof(a));
    const int D = g->head_dim, H = g->n_kv_heads;
    const bool pool = tag == PATCHKV_TAG_BF16;
    const bool shape = (D == 64 || D == 128) && g->page_tokens % kTile == 0 && (pool || g->group % 32 == 0);
    const long long cols = (long long)std::min(b->max_rows, b->n_rows) * (Hq / H);
    const uint64_t any_bytes = round16((uint64_t)b->n_rows * Hq * 4);       // of the element-wise kernel, which unaligned queries go to
    a.bytes = any_bytes;
    const long long longest = longest_sequence(g, b);
    if (!shape || cols == 0 || longest > 1 << 30) return a;
    // The longest run of rows decides for the whole batch: a prompt chunk beside decode steps (2048 rows over 8192 tokens and 7 rows over 65536 each, bf16
    // pool) takes 1694 us in one call, and 567 in two.
    // Up to 16 columns the split kernel: 32 query heads over 8 KV heads, 32k tokens, 1, 2 and 4 rows take 27, 34 and 49 us of it on a bf16 pool
    // and 22, 28 and 43 us on 4-bit pages; the row kernels take 60 and 68 us for any of them.
    if (cols > 16) {
        // Whole CTAs along the query vectors; where they leave SMs idle the tokens are split, two steps a piece at least.  (32 rows of 32 query
        // heads over 8 KV heads, 32k tokens of a bf16 pool: 58 us split, 490 us on eight SMs.)
        const long long tiles = (cols + 2 * kRowTile - 1) / (2 * kRowTile), ctas = tiles * H * b->n_seqs;
        if (ctas == 0 || ctas > 1 << 24 || cols > 1 << 30) return a;
        const long long all = (longest + kRowTile - 1) / kRowTile;
        long long steps = all;                  // that the rows of a CTA see at most
        const long long cta_rows = std::min((long long)b->max_rows, 2ll * kRowTile / (Hq / H) + 2);
        if (window > 0 && !b->pos) steps = std::min(all, ((long long)window + sinks + cta_rows) / kRowTile + 3);
        a.row_tiles = (int)tiles;
        a.row_splits = (int)std::max({1ll, std::min((long long)kSms / ctas, steps / 2), (steps + kMaxItemSteps - 1) / kMaxItemSteps});
        a.one = cols <= kRowTile;
        a.tokens = (int)(steps * kRowTile);
        const uint64_t tile_bytes = (uint64_t)b->n_seqs * H * a.tokens * 4;
        a.chunk = (int)std::min<uint64_t>(tiles, std::max<uint64_t>(1, kMaxMassPartial / std::max<uint64_t>(tile_bytes, 1)));
        a.sums_bytes = (uint64_t)a.row_splits * b->n_rows * Hq * 8;
        a.ranges_bytes = (uint64_t)b->n_seqs * tiles * 16;
        a.acc_bytes = a.chunk < tiles ? round16((uint64_t)b->n_seqs * longest * 8) : 0;
        a.partial_bytes = a.chunk * tile_bytes;
        // Images pay where many CTAs would make the same operands from codes (8-bit keys, 8192 tokens, 32 query heads over 8 KV heads, with images and
        // without: 74 and 58 us for 2 tiles, 154 and 150 for 8, 260 and 275 for 16, 430 and 465 for 32).
        const uint64_t images = (uint64_t)all * H * b->n_seqs, image = 4ull * kRowTile * D;
        if (!pool && tiles > 8 && images > 0 && images <= kMaxMassImages / image) {
            a.steps = (int)all;
            a.image_bytes = images * image;
            a.meta_bytes = images * 32;
        }
        a.bytes = std::max(any_bytes, round16(a.sums_bytes) + a.ranges_bytes + a.acc_bytes + a.partial_bytes + a.image_bytes + a.meta_bytes);
        return a;
    }
    a.nc = cols <= 4 ? 1 : cols <= 8 ? 2 : 4;
    a.cols = (int)cols;
    const int warps = split_warps(pool, a.nc);
    a.heads = 1;                                // heads of a CTA, and pieces of the batch, as the attention has them
    for (int h = 2; h <= warps; h *= 2)
        if ((H + h - 1) / h * h <= (H + a.heads - 1) / a.heads * a.heads || h <= H) a.heads = h;
    a.groups = (H + a.heads - 1) / a.heads;
    a.warps_per_head = warps / a.heads;
    const int slots = std::max(1, kSms / a.groups);
    a.target = b->n_seqs >= 2 * slots ? 0 : std::max(slots - b->n_seqs, (slots + 1) / 2);
    a.max_items = b->n_seqs + a.target;
    // Tiles that a sequence's rows can see: with a window, and rows one behind the other, not all of them.
    long long tiles = (longest + kTile - 1) / kTile;
    if (window > 0 && !b->pos) tiles = std::min(tiles, ((long long)window + b->max_rows + kTile - 1) / kTile + 1 + ((long long)sinks + kTile - 1) / kTile);
    a.tokens = (int)(tiles * kTile);
    a.items_bytes = ((uint64_t)b->n_seqs * 8 + 15) / 16 * 16;
    a.sums_bytes = (uint64_t)a.max_items * H * 4 * a.nc * 8;
    a.bytes = std::max(any_bytes, a.items_bytes + a.sums_bytes + (uint64_t)b->n_seqs * H * a.cols * a.tokens * 4);
    return a;
}

}  // namespace
}  // namespace patchkv

using namespace patchkv;

extern "C" uint64_t patchkv_attention_mass_workspace_bytes(const patchkv_geom* g, int tag, const patchkv_batch* b, int n_q_heads,
                                                           int window, int sinks) {
    BatchDev bd;
    if (check_live_geometry(nullptr, "attention_mass", g, 0) != PATCHKV_OK || fill_batch(nullptr, "attention_mass", b, &bd) != PATCHKV_OK ||
        check_mass(nullptr, g, tag, b, n_q_heads, window, sinks) != PATCHKV_OK)
        return 0;
    return plan_mass(g, tag, b, n_q_heads, window, sinks).bytes;
}

extern "C" int patchkv_attention_mass(patchkv_ctx* ctx, const patchkv_geom* g, const patchkv_pool* pool, const patchkv_qpool* cache,
                                      int layer, const patchkv_batch* batch, const patchkv_mass_args* a, void* stream_) {
    if (!ctx) return PATCHKV_E_INVALID;
    std::lock_guard<std::mutex> lock(ctx->mu);
    AttentionParams p;
    if ((pool != nullptr) == (cache != nullptr)) return fail(ctx, PATCHKV_E_INVALID, "attention_mass: give a pool or a cache, one of the two");
    int rc = check_live_geometry(ctx, "attention_mass", g, layer);
    if (rc == PATCHKV_OK) rc = fill_batch(ctx, "attention_mass", batch, &p.b);
    if (rc == PATCHKV_OK) rc = pool ? fill_pool(ctx, "attention_mass", g, pool, layer, &p.c) : fill_cache(ctx, "attention_mass", g, cache, layer, &p.c);
    if (rc != PATCHKV_OK) return rc;
    if (!a || a->struct_size != sizeof(patchkv_mass_args)) return fail(ctx, PATCHKV_E_INVALID, "attention_mass: null args or wrong struct_size");
    rc = check_mass(ctx, g, p.c.tag, batch, a->n_q_heads, a->window, a->sinks);
    if (rc != PATCHKV_OK) return rc;
    if (a->type != PATCHKV_ROWS_BF16 && a->type != PATCHKV_ROWS_F16) return fail(ctx, PATCHKV_E_INVALID, "attention_mass: unknown row type");
    if (pool && a->type != PATCHKV_ROWS_BF16) return fail(ctx, PATCHKV_E_INVALID, "attention_mass: over a bf16 pool q must be bf16");
    if (!(fabsf(a->scale) <= 3.0e38f)) return fail(ctx, PATCHKV_E_INVALID, "attention_mass: scale must be finite");
    if (!(fabsf(a->decay) <= 3.0e38f)) return fail(ctx, PATCHKV_E_INVALID, "attention_mass: decay must be finite");
    if (a->mass_type != PATCHKV_MASS_F32 && a->mass_type != PATCHKV_MASS_U64) return fail(ctx, PATCHKV_E_INVALID, "attention_mass: unknown mass type");
    if (a->mass_type == PATCHKV_MASS_U64 && a->decay != 0.0f && a->decay != 1.0f)
        return fail(ctx, PATCHKV_E_INVALID, "attention_mass: decay of whole masses must be 0 or 1");
    if (a->q_stride_row < 0 || a->q_stride_head < 0) return fail(ctx, PATCHKV_E_INVALID, "attention_mass: negative stride");
    if (a->mass_stride < longest_sequence(g, batch)) return fail(ctx, PATCHKV_E_INVALID, "attention_mass: mass_stride is smaller than the longest sequence");
    if (p.b.n_seqs == 0 || p.b.max_kv_len == 0) return PATCHKV_OK;
    const uintptr_t unit = a->mass_type == PATCHKV_MASS_U64 ? 7 : 3;
    if (!a->mass || (reinterpret_cast<uintptr_t>(a->mass) & unit) || (reinterpret_cast<uintptr_t>(a->mass_in) & unit))
        return fail(ctx, PATCHKV_E_INVALID, "attention_mass: null or misaligned mass");
    if (!p.b.row_start || !p.b.kv_len) return fail(ctx, PATCHKV_E_INVALID, "attention_mass: null row_start or kv_len");
    const uintptr_t qa = reinterpret_cast<uintptr_t>(a->q);
    const bool any_rows = p.b.n_rows > 0 && p.b.max_rows > 0;
    if (any_rows && (!qa || (qa & 1))) return fail(ctx, PATCHKV_E_INVALID, "attention_mass: null or misaligned q");
    const uint64_t need = patchkv_attention_mass_workspace_bytes(g, p.c.tag, batch, a->n_q_heads, a->window, a->sinks);
    if (need && (!a->workspace || (reinterpret_cast<uintptr_t>(a->workspace) & 15) || a->workspace_bytes < need))
        return fail(ctx, PATCHKV_E_INVALID, "attention_mass: workspace null, misaligned or too small");
    p.b.max_kv_len = (int)longest_sequence(g, batch);           // sizes the launches
    if (p.b.max_kv_len == 0) return PATCHKV_OK;
    p.q = static_cast<const uint16_t*>(a->q); p.out = nullptr;
    p.q_stride_row = a->q_stride_row; p.q_stride_head = a->q_stride_head;
    p.out_stride_row = p.out_stride_head = 0;
    p.Hq = a->n_q_heads; p.share = a->n_q_heads / g->n_kv_heads;
    p.window = a->window; p.sinks = a->sinks;
    p.scale_log2 = (float)((double)a->scale * 1.4426950408889634);
    p.status = ctx->d_status;
    p.f16 = a->type == PATCHKV_ROWS_F16;
    const WeightParams m = {a->mass_in, a->mass, a->mass_stride, a->decay, a->mass_type == PATCHKV_MASS_U64};
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return fail(ctx, PATCHKV_E_CUDA, "cudaSetDevice failed");
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    const MassPlan plan = plan_mass(g, p.c.tag, batch, a->n_q_heads, a->window, a->sinks);
    const bool aligned = (qa & 15) == 0 && a->q_stride_row % 8 == 0 && a->q_stride_head % 8 == 0 &&
                         (!pool || (pool->stride_page % 8 == 0 && pool->stride_token % 8 == 0 && pool->stride_head % 8 == 0 && pool->stride_layer % 8 == 0));
    if (plan.nc && aligned) {
        uint8_t* ws = static_cast<uint8_t*>(a->workspace);
        WeighPlan pl;
        memset(&pl, 0, sizeof(pl));
        pl.s.items = reinterpret_cast<int32_t*>(ws);
        pl.s.max_items = plan.max_items; pl.s.target = plan.target;
        pl.s.heads_log2 = log2_exact(plan.heads); pl.s.per_head_log2 = log2_exact(plan.warps_per_head);
        pl.s.share_magic = (65536u + p.share - 1) / p.share;
        pl.sums = reinterpret_cast<float2*>(ws + plan.items_bytes);
        pl.logits = reinterpret_cast<float*>(ws + plan.items_bytes + plan.sums_bytes);
        pl.tokens = plan.tokens; pl.cols = plan.cols;
        PKV_CUDA(ctx, p.c.D == 128 ? launch_weigh<128>(p, m, pl, plan.nc, plan.groups, stream) : launch_weigh<64>(p, m, pl, plan.nc, plan.groups, stream));
        return PATCHKV_OK;
    }
    if (plan.row_tiles && aligned) {
        uint8_t* ws = static_cast<uint8_t*>(a->workspace);
        WeighRowsPlan pl;
        memset(&pl, 0, sizeof(pl));
        auto take = [&](uint64_t bytes) { uint8_t* at = bytes ? ws : nullptr; ws += round16(bytes); return at; };
        pl.images = take(plan.image_bytes);
        pl.meta = reinterpret_cast<uint32_t*>(take(plan.meta_bytes));
        pl.sums = reinterpret_cast<float2*>(take(plan.sums_bytes));
        pl.ranges = reinterpret_cast<int4*>(take(plan.ranges_bytes));
        pl.acc = reinterpret_cast<double*>(take(plan.acc_bytes));
        pl.partial = reinterpret_cast<float*>(take(plan.partial_bytes));
        pl.tiles = plan.row_tiles; pl.splits = plan.row_splits; pl.one = plan.one;
        pl.chunk_tiles = plan.chunk; pl.tokens = plan.tokens; pl.steps = plan.steps;
        PKV_CUDA(ctx, p.c.D == 128 ? launch_weigh_rows<128>(p, m, pl, stream) : launch_weigh_rows<64>(p, m, pl, stream));
        return PATCHKV_OK;
    }
    float* sums = static_cast<float*>(a->workspace);
    if (any_rows) {
        mass_sums_any_kernel<<<dim3(std::min(p.b.max_rows, p.b.n_rows), p.Hq, p.b.n_seqs), kMassThreads, 0, stream>>>(p, sums);
        PKV_CUDA(ctx, cudaGetLastError());
    }
    mass_columns_any_kernel<<<dim3((unsigned)((p.b.max_kv_len + (long long)kMassThreads - 1) / kMassThreads), p.b.n_seqs), kMassThreads, 0, stream>>>(p, m, sums);
    PKV_CUDA(ctx, cudaGetLastError());
    return PATCHKV_OK;
}
