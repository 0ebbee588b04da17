// Cutting a cache down: which tokens stay (patchkv_evict_select), and their rows' way into other pages (patchkv_cache_gather).
#include <cooperative_groups.h>

#include "attention_launch.cuh"
#include "rotary.cuh"

namespace patchkv {

namespace cg = cooperative_groups;

// ---------------------------------------------------------------- which tokens stay
constexpr int kSelectThreads = 1024, kSelectWarps = kSelectThreads / 32, kSelectBins = 2048, kSelectHeld = 16384, kSelectList = 4096, kMaxCluster = 8;
constexpr int kStays = 0x7FFFFFFF, kAbsent = (int)0x80000000;      // keys of tokens that stay in any case, and of those behind the last

struct EvictParams {
    const float* mass;
    const int32_t* kv_len;
    const int32_t* budget;
    int32_t* keep;
    int32_t* kept;
    float* mass_out;
    long long mass_stride, keep_stride, out_stride;
    int32_t max_len, max_keep, recent, sinks;
    int32_t* status;
};

// A cluster takes a sequence, each of its CTAs a run of the tokens, each lane some that lie together.  Masses are keys, bit patterns, which order
// numbers that are not negative, with the tokens that stay in any case above all.  The key of the last token that stays is found digit by digit
// (11, 11 and 10 bits): a CTA counts its keys by digit in shared memory, and every CTA adds up the counts of all (distributed shared memory) and
// finds the digit by itself.  After the first digit few keys are left as a rule; every CTA then gets the list of them and finds the other
// two digits without the cluster (where they are many, ties above all, the cluster counts on).  Each lane counts what of its tokens
// stays, a prefix over lanes, warps and CTAs gives every kept token its place, and the indices leave by way of shared memory, so that they
// are written side by side.  All counts are whole numbers: the order of the atomics does not matter.  Bound by latencies: a
// barrier of the cluster takes 2000 cycles, counts read from eight CTAs 4000, from sixteen 12000, which is 5 to 6 of the 21 us that eight sequences
// of 128k tokens take; the rest, the walks over the keys and the atomics on bins that keys of one scale share, has not been taken apart.
// 32 sequences of 4096 tokens 7.1 us.
// HELD: keys and indices of a run fit shared memory, else keys are made again each time and indices written one by one.  The bound on the lengths
// decides (131072: 21.6 us for eight sequences of that length; 131073: 42.0).
struct SelectSmem {
    alignas(16) int bins[3][kSelectBins];
    int list[kSelectList];                      // keys that are left after the first digit
    int sums[kSelectWarps];
    int found[3];                               // digit, how many keys lie above it, and how many have it
    int2 warp_count[kSelectWarps];              // tokens above the border, and those at it
    int2 cta_count[kMaxCluster];                // of every CTA of the cluster
    int listed[kMaxCluster];                    // keys that every CTA has put on its list
    int n_list;
};
// The bin, from the top, in which the need-th key lies: found = {bin, keys above it, keys in it}.  c: counts of bins 2046 - 2i and 2047 - 2i.
__device__ __forceinline__ void find_bin(SelectSmem& m, int2 c, int need) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, own = c.x + c.y;
    int inc = own;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int o = __shfl_up_sync(0xFFFFFFFFu, inc, d);
        if (lane >= d) inc += o;
    }
    if (lane == 31) m.sums[warp] = inc;
    __syncthreads();
    const int before = __reduce_add_sync(0xFFFFFFFFu, lane < warp ? m.sums[lane] : 0) + inc - own;
    if (before < need && need <= before + own) {
        const bool second = need > before + c.y;
        m.found[0] = kSelectBins - 1 - 2 * (int)threadIdx.x - second;
        m.found[1] = before + (second ? c.y : 0);
        m.found[2] = second ? c.x : c.y;
    }
    __syncthreads();
}
template <bool HELD>
__global__ void __launch_bounds__(kSelectThreads) evict_select_kernel(const EvictParams p) {
    extern __shared__ int held[];               // keys [lane's token][33] of each warp, then the indices of the kept
    __shared__ SelectSmem m;
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = (int)cluster.block_rank(), ctas = (int)cluster.num_blocks();
    const int s = blockIdx.x / ctas, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    pdl_trigger();
    for (int i = tid; i < 3 * kSelectBins / 4; i += kSelectThreads) reinterpret_cast<int4*>(m.bins[0])[i] = make_int4(0, 0, 0, 0);
    if (tid == 0) m.n_list = 0;
    auto all_there = cluster.barrier_arrive();
    pdl_wait();
    int n = p.kv_len[s], B = p.budget ? p.budget[s] : p.max_keep;
    if (rank == 0 && tid == 0 && (n > p.max_len || B > p.max_keep)) atomicCAS(p.status, 0, (int)PATCHKV_E_BOUNDS);
    n = max(0, min(n, p.max_len));
    B = max(0, min(B, p.max_keep));
    const int kept = min(n, B), last = n <= B ? n : min(p.recent, B), first = n <= B ? 0 : min(p.sinks, B - last);
    // `steps` tokens a lane
    const int steps = (n + ctas * kSelectThreads - 1) / (ctas * kSelectThreads), run = steps * kSelectThreads;
    const int base = rank * run + warp * 32 * steps, begin = base + lane * steps;
    int* const mine = held + warp * 33 * steps;
    int* const indices = held + kSelectWarps * 33 * steps;
    const float* mass = p.mass + (long long)s * p.mass_stride;
    auto mass_of = [&](int t) {
        const uint32_t bits = __float_as_uint(mass[t]);
        return bits < 0x7F800000u ? (int)bits : 0;
    };
    auto key_of = [&](int t) {
        if (t >= n) return kAbsent;
        const uint32_t bits = __float_as_uint(mass[t]);
        if (bits >= 0x7F800000u && bits != 0x80000000u) atomicCAS(p.status, 0, (int)PATCHKV_E_BADINPUT);
        return t < first || t >= n - last ? kStays : bits < 0x7F800000u ? (int)bits : 0;
    };
    auto key = [&](int i) { return HELD ? mine[33 * i + lane] : key_of(begin + i); };
    if (HELD)
#pragma unroll 4
        for (int i = lane; i < 32 * steps; i += 32) {
            const int owner = i / steps;
            mine[33 * (i - owner * steps) + owner] = key_of(base + i);
        }
    cluster.barrier_wait(std::move(all_there)); // all bins are empty, and every CTA is there to be read
    auto barrier = [&]() { if (ctas > 1) cluster.sync(); else __syncthreads(); };
    int border = kept > 0 && first + last < kept ? 0 : kStays;     // key of the last token that stays, so far as it is known
    int need = kept;                            // how many of those keys that agree with it so far stay
    auto shift_of = [](int digit) { return digit == 0 ? 21 : digit == 1 ? 10 : 0; };
    auto mask_of = [](int digit) { return digit == 2 ? 1023u : 2047u; };
    auto known_of = [](int digit) { return digit == 0 ? 0x80000000u : digit == 1 ? 0xFFE00000u : 0xFFFFFC00u; };
    auto found = [&](int digit) {
        border |= m.found[0] << shift_of(digit);
        need -= m.found[1];
    };
    // A digit by the whole cluster.
    auto count_all = [&](int digit) {
        const int shift = shift_of(digit);
        const uint32_t known = known_of(digit), mask = mask_of(digit);
        int* count = m.bins[digit];
#pragma unroll 4
        for (int i = 0; i < steps; i++) {
            const uint32_t k = (uint32_t)key(i);
            if (((k ^ (uint32_t)border) & known) == 0) atomicAdd(&count[k >> shift & mask], 1);
        }
        barrier();
        int2 c = make_int2(0, 0);
        if (digit != 0 || tid >= kSelectThreads / 2)        // the first digit's upper half stands for a sign
#pragma unroll 8
            for (int i = 0; i < ctas; i++) {
                const int2 x = *reinterpret_cast<const int2*>(cluster.map_shared_rank(count, i) + kSelectBins - 2 - 2 * tid);
                c.x += x.x;
                c.y += x.y;
            }
        find_bin(m, c, need);
        found(digit);
    };
    if (border == 0) {
        count_all(0);
        const int left = m.found[2];
        if (left > kSelectList) {
            count_all(1);
            count_all(2);
        } else {
#pragma unroll 4
            for (int i = 0; i < steps; i++) {
                const int k = key(i);
                if (((uint32_t)(k ^ border) & known_of(1)) == 0) m.list[atomicAdd(&m.n_list, 1)] = k;
            }
            __syncthreads();
            if (tid < ctas) cluster.map_shared_rank(m.listed, tid)[rank] = m.n_list;
            barrier();
            // The lists of all CTAs, a key to a thread and round: the i-th key is on the list of the CTA whose share of the numbers has i.
            for (int digit = 1; digit < 3; digit++) {
                const int shift = shift_of(digit);
                const uint32_t known = known_of(digit), mask = mask_of(digit);
                int* count = m.bins[digit];
                for (int i = tid; i < left; i += kSelectThreads) {
                    int from = 0, at = i;
                    while (at >= m.listed[from]) at -= m.listed[from++];
                    const uint32_t k = (uint32_t)cluster.map_shared_rank(m.list, from)[at];
                    if (((k ^ (uint32_t)border) & known) == 0) atomicAdd(&count[k >> shift & mask], 1);
                }
                __syncthreads();
                find_bin(m, *reinterpret_cast<const int2*>(count + kSelectBins - 2 - 2 * tid), need);
                found(digit);
            }
        }
    }
    int2 count = make_int2(0, 0);
#pragma unroll 4
    for (int i = 0; i < steps; i++) {
        const int k = key(i);
        count.x += k > border;
        count.y += k == border;
    }
    int2 sum = count;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int a = __shfl_up_sync(0xFFFFFFFFu, sum.x, d), b = __shfl_up_sync(0xFFFFFFFFu, sum.y, d);
        if (lane >= d) { sum.x += a; sum.y += b; }
    }
    if (lane == 31) m.warp_count[warp] = sum;
    __syncthreads();
    int2 at;                                    // of this CTA, in front of the lane's tokens
    {
        const int2 c = m.warp_count[lane];
        at.x = __reduce_add_sync(0xFFFFFFFFu, lane < warp ? c.x : 0) + sum.x - count.x;
        at.y = __reduce_add_sync(0xFFFFFFFFu, lane < warp ? c.y : 0) + sum.y - count.y;
        const int2 all = make_int2(__reduce_add_sync(0xFFFFFFFFu, c.x), __reduce_add_sync(0xFFFFFFFFu, c.y));
        if (warp == 0 && lane < ctas) cluster.map_shared_rank(m.cta_count, lane)[rank] = all;
    }
    barrier();                                  // (and behind it nobody reads another CTA's shared memory)
    int2 front = make_int2(0, 0);               // of the CTAs in front
    for (int i = 0; i < rank; i++) { front.x += m.cta_count[i].x; front.y += m.cta_count[i].y; }
    const int2 own = m.cta_count[rank];
    const int start = front.x + min(front.y, need), end = front.x + own.x + min(front.y + own.y, need);
    int32_t* keep = p.keep + (long long)s * p.keep_stride;
    float* out = p.mass_out ? p.mass_out + (long long)s * p.out_stride : nullptr;
    int place = front.x + at.x + min(front.y + at.y, need), ties = front.y + at.y;
#pragma unroll 4
    for (int i = 0; i < steps; i++) {
        const int k = key(i);
        const bool stays = k > border || (k == border && ties < need);
        ties += k == border;
        if (stays) {
            if (HELD) {
                indices[place - start] = begin + i;
            } else {
                keep[place] = begin + i;
                if (out) out[place] = __int_as_float(mass_of(begin + i));
            }
        }
        place += stays;
    }
    if (HELD) {
        __syncthreads();
#pragma unroll 4
        for (int i = start + tid; i < end; i += kSelectThreads) {
            const int t = indices[i - start];
            keep[i] = t;
            if (out) out[i] = __int_as_float(mass_of(t));
        }
    }
    for (int i = kept + rank * kSelectThreads + tid; i < p.max_keep; i += ctas * kSelectThreads) keep[i] = -1;
    if (rank == 0 && tid == 0) p.kept[s] = kept;
}

// ---------------------------------------------------------------- their rows
constexpr int kGatherThreads = 128;

struct MoveParams {
    CacheDev c;
    uint16_t* k_pool;
    uint16_t* v_pool;
    const int32_t* keep;
    const int32_t* kept;
    const int32_t* kv_len;
    const int32_t* src_table;
    const int32_t* dst_table;
    long long keep_stride;
    int32_t* status;
    int32_t n_seqs, max_keep, src_stride, dst_stride, rotate, Dr, half;
    int32_t parts, passes, U_shift;             // pools: warps that share a row; passes over K or V; 16-channel units of a head
    uint32_t k_row, s_row, v_row;               // quantised pages: bytes of a row's K codes, scales (of K or V) and V codes
    Frequencies f;
};

struct Move { int from, to, slot, to_slot, turn; };         // pages and slots; positions moved
// Where row i of sequence s comes from and goes to; false when it is skipped (latched by the caller's `report` thread).
__device__ __forceinline__ bool find_move(const MoveParams& p, int s, int i, bool report, Move* m) {
    const int old = p.keep[(long long)s * p.keep_stride + i];
    bool ok = old >= 0 && old < p.kv_len[s];
    if (ok) {
        const int lp = div_page(p.c, old), tp = div_page(p.c, i);
        ok = lp < p.src_stride && tp < p.dst_stride;
        if (ok) {
            m->from = p.src_table[(long long)s * p.src_stride + lp];
            m->to = p.dst_table[(long long)s * p.dst_stride + tp];
            m->slot = old - lp * p.c.P;
            m->to_slot = i - tp * p.c.P;
            m->turn = i - old;
            ok = m->from >= 0 && m->from < p.c.n_pages && m->to >= 0 && m->to < p.c.n_pages;
        }
    }
    if (!ok && report) atomicCAS(p.status, 0, (int)PATCHKV_E_BOUNDS);
    return ok;
}
__device__ __forceinline__ int rows_of(const MoveParams& p, int s) {
    const int n = p.kept[s];
    if (n > p.max_keep && blockIdx.x == 0 && threadIdx.x == 0) atomicCAS(p.status, 0, (int)PATCHKV_E_BOUNDS);
    return min(n, p.max_keep);
}

// Rows of a bf16 pool (grid: warps, sequence): a warp takes a row, or every `parts`-th pass of one; a pass is 32 units of 16 channels, keys and
// then values, laid out over the lanes as in rotary_append_kernel.  Bound by memory: 32768 rows of 8 heads of 128 channels, keys turned, 268 MB in
// 47 us replayed (5.7 TB/s); without the lines asked for ahead 53.
template <bool HALF>
__global__ void __launch_bounds__(kGatherThreads) gather_pool_kernel(const __grid_constant__ MoveParams p) {
    __shared__ __align__(16) float cosine[kGatherThreads / 32][PATCHKV_MAX_ROTARY_DIM / 2], sine[kGatherThreads / 32][PATCHKV_MAX_ROTARY_DIM / 2];
    pdl_trigger();
    pdl_wait();
    const int s = blockIdx.y, lane = threadIdx.x & 31;
    const uint32_t wid = (blockIdx.x * kGatherThreads + threadIdx.x) >> 5;
    const int i = (int)(wid / (uint32_t)p.parts), part = (int)(wid - (uint32_t)i * p.parts);
    if (i >= rows_of(p, s)) return;
    Move m;
    if (!find_move(p, s, i, lane == 0 && part == 0, &m)) return;
    const int u = lane & ((1 << p.U_shift) - 1), sub = lane >> p.U_shift, total = 2 * p.passes;
    const long long from = (long long)m.from * p.c.stride_page + (long long)m.slot * p.c.stride_token;
    const long long to = (long long)m.to * p.c.stride_page + (long long)m.to_slot * p.c.stride_token;
    const bool rotate = p.rotate && m.turn != 0, turns = rotate && 16 * u < p.Dr;
    const int ch0 = first_run(HALF && rotate, p.Dr, u), ch1 = second_run(HALF && rotate, p.Dr, u);
    struct Unit { uint4 a, b; };
    auto head_of = [&](int pass) { return ((pass < p.passes ? pass : pass - p.passes) << (5 - p.U_shift)) + sub; };
    auto load = [&](int pass) {
        Unit x = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
        const int h = head_of(pass);
        if (pass >= total || h >= p.c.H) return x;
        const uint16_t* a = (pass < p.passes ? p.c.k : p.c.v) + from + (long long)h * p.c.stride_head;
        x.a = *reinterpret_cast<const uint4*>(a + ch0);
        x.b = *reinterpret_cast<const uint4*>(a + ch1);
        return x;
    };
    if (p.parts == 1)
        for (int c = 0; c < p.c.D; c += 64)                 // 128 bytes
            for (int h = lane; h < p.c.H; h += 32) {
                prefetch_l2(p.c.k + from + (long long)h * p.c.stride_head + c);
                prefetch_l2(p.c.v + from + (long long)h * p.c.stride_head + c);
            }
    Unit next = load(part);
    const int warp = threadIdx.x >> 5;
    if (rotate && part < p.passes)
        for (int j = lane; j < p.Dr >> 1; j += 32) {
            double c, sn;
            cos_sin((double)m.turn * p.f.theta[j], &c, &sn);
            cosine[warp][j] = (float)c;
            sine[warp][j] = (float)sn;
        }
    __syncwarp();
    float c[8], sn[8];
    {
        const float4* a = reinterpret_cast<const float4*>(&cosine[warp][turns ? 8 * u : 0]);
        const float4* b = reinterpret_cast<const float4*>(&sine[warp][turns ? 8 * u : 0]);
        const float4 c0 = a[0], c1 = a[1], s0 = b[0], s1 = b[1];
        c[0] = c0.x; c[1] = c0.y; c[2] = c0.z; c[3] = c0.w; c[4] = c1.x; c[5] = c1.y; c[6] = c1.z; c[7] = c1.w;
        sn[0] = s0.x; sn[1] = s0.y; sn[2] = s0.z; sn[3] = s0.w; sn[4] = s1.x; sn[5] = s1.y; sn[6] = s1.z; sn[7] = s1.w;
    }
#pragma unroll 1
    for (int pass = part; pass < total; pass += p.parts) {
        const Unit x = next;
        next = load(pass + p.parts);
        const int h = head_of(pass);
        uint32_t w[8] = {x.a.x, x.a.y, x.a.z, x.a.w, x.b.x, x.b.y, x.b.z, x.b.w};
        if (turns && pass < p.passes) turn_words<PATCHKV_ROWS_BF16, HALF>(w, c, sn);
        if (h < p.c.H) {
            uint16_t* a = (pass < p.passes ? p.k_pool : p.v_pool) + to + (long long)h * p.c.stride_head;
            *reinterpret_cast<uint4*>(a + ch0) = make_uint4(w[0], w[1], w[2], w[3]);
            *reinterpret_cast<uint4*>(a + ch1) = make_uint4(w[4], w[5], w[6], w[7]);
        }
    }
}

// Rows of quantised pages (grid: warps, sequence): a row's codes and scales are a run of bytes in each of the page's four sections.
// A warp takes a row, codes by 16 bytes and scales by 4.  8192 rows of 1152 bytes: 4.5 us replayed (4.2 TB/s), where the call takes 6.5 on the host.
__global__ void __launch_bounds__(kGatherThreads) gather_codes_kernel(const __grid_constant__ MoveParams p) {
    pdl_trigger();
    pdl_wait();
    const int s = blockIdx.y, lane = threadIdx.x & 31, i = (int)((blockIdx.x * kGatherThreads + threadIdx.x) >> 5);
    if (i >= rows_of(p, s)) return;
    Move m;
    if (!find_move(p, s, i, lane == 0, &m)) return;
    const uint8_t* from = p.c.base + (long long)m.from * p.c.stride_page;
    uint8_t* to = p.c.base + (long long)m.to * p.c.stride_page;
    const uint32_t ks = p.c.k_scales + m.slot * p.s_row, kd = p.c.k_scales + m.to_slot * p.s_row;
    const uint32_t vs = p.c.v_scales + m.slot * p.s_row, vd = p.c.v_scales + m.to_slot * p.s_row;
    const uint32_t k16 = p.k_row / 16, v16 = p.v_row / 16, s4 = p.s_row / 4, steps = max(max(k16, v16), s4);
#pragma unroll 1
    for (uint32_t j = lane; j < steps; j += 32) {
        uint4 k = make_uint4(0, 0, 0, 0), v = k;
        uint32_t a = 0, b = 0;
        if (j < k16) k = *(reinterpret_cast<const uint4*>(from + m.slot * p.k_row) + j);
        if (j < v16) v = *(reinterpret_cast<const uint4*>(from + p.c.v_codes + m.slot * p.v_row) + j);
        if (j < s4) { a = *(reinterpret_cast<const uint32_t*>(from + ks) + j); b = *(reinterpret_cast<const uint32_t*>(from + vs) + j); }
        if (j < k16) *(reinterpret_cast<uint4*>(to + m.to_slot * p.k_row) + j) = k;
        if (j < v16) *(reinterpret_cast<uint4*>(to + p.c.v_codes + m.to_slot * p.v_row) + j) = v;
        if (j < s4) { *(reinterpret_cast<uint32_t*>(to + kd) + j) = a; *(reinterpret_cast<uint32_t*>(to + vd) + j) = b; }
    }
}

// Any geometry, any strides: a thread per row and head (grid: threads, sequence), byte by byte and pair by pair.
__global__ void __launch_bounds__(kGatherThreads) gather_any_kernel(const __grid_constant__ MoveParams p) {
    const int s = blockIdx.y;
    const uint32_t id = blockIdx.x * kGatherThreads + threadIdx.x;
    const int i = (int)(id / (uint32_t)p.c.H), h = (int)(id - (uint32_t)i * p.c.H), D = p.c.D;
    if (i >= rows_of(p, s)) return;
    Move m;
    if (!find_move(p, s, i, h == 0, &m)) return;
    if (p.c.tag == PATCHKV_TAG_BF16) {
        const long long from = (long long)m.from * p.c.stride_page + (long long)m.slot * p.c.stride_token + (long long)h * p.c.stride_head;
        const long long to = (long long)m.to * p.c.stride_page + (long long)m.to_slot * p.c.stride_token + (long long)h * p.c.stride_head;
        const int Dr = p.rotate && m.turn != 0 ? p.Dr : 0;
        for (int j = 0; j < Dr >> 1; j++) {
            const int c0 = p.half ? j : 2 * j, c1 = p.half ? j + (Dr >> 1) : 2 * j + 1;
            double c, sn;
            cos_sin((double)m.turn * p.f.theta[j], &c, &sn);
            const float cf = (float)c, sf = (float)sn, a = bf16_bits_to_float(p.c.k[from + c0]), b = bf16_bits_to_float(p.c.k[from + c1]);
            p.k_pool[to + c0] = __bfloat16_as_ushort(__float2bfloat16_rn(fmaf(-b, sf, a * cf)));
            p.k_pool[to + c1] = __bfloat16_as_ushort(__float2bfloat16_rn(fmaf(b, cf, a * sf)));
        }
        for (int c = Dr; c < D; c++) p.k_pool[to + c] = p.c.k[from + c];
        for (int c = 0; c < D; c++) p.v_pool[to + c] = p.c.v[from + c];
        return;
    }
    const uint8_t* from = p.c.base + (long long)m.from * p.c.stride_page;
    uint8_t* to = p.c.base + (long long)m.to * p.c.stride_page;
    const uint32_t section[4] = {0, p.c.k_scales, p.c.v_codes, p.c.v_scales}, row[4] = {p.k_row, p.s_row, p.v_row, p.s_row};
    for (int q = 0; q < 4; q++)
        for (uint32_t j = row[q] / p.c.H * h; j < row[q] / p.c.H * (h + 1); j++)        // a head's bytes: whole ones, D is even
            to[section[q] + m.to_slot * row[q] + j] = from[section[q] + m.slot * row[q] + j];
}

namespace {

int evict_select(patchkv_ctx* ctx, const patchkv_evict_args* a, cudaStream_t stream) {
    if (!a || a->struct_size != sizeof(patchkv_evict_args)) return fail(ctx, PATCHKV_E_INVALID, "evict_select: null args or wrong struct_size");
    if (a->n_seqs < 0 || a->max_len < 0 || a->max_keep < 0 || a->recent < 0 || a->sinks < 0)
        return fail(ctx, PATCHKV_E_INVALID, "evict_select: negative count");
    if (a->max_len > 1 << 24) return fail(ctx, PATCHKV_E_UNSUPPORTED, "evict_select: max_len above 2^24");
    if (a->n_seqs > 65535) return fail(ctx, PATCHKV_E_UNSUPPORTED, "evict_select: more than 65535 sequences");
    if (a->mass_stride < a->max_len || a->keep_stride < a->max_keep || (a->mass_out && a->mass_out_stride < a->max_keep))
        return fail(ctx, PATCHKV_E_INVALID, "evict_select: a stride is smaller than its row");
    if (a->n_seqs == 0) return PATCHKV_OK;
    if (!a->kv_len || !a->kept || (a->max_keep > 0 && !a->keep) || (a->max_len > 0 && !a->mass))
        return fail(ctx, PATCHKV_E_INVALID, "evict_select: null mass, kv_len, keep or kept");
    if (((reinterpret_cast<uintptr_t>(a->mass) | reinterpret_cast<uintptr_t>(a->kv_len) | reinterpret_cast<uintptr_t>(a->budget) |
          reinterpret_cast<uintptr_t>(a->keep) | reinterpret_cast<uintptr_t>(a->kept) | reinterpret_cast<uintptr_t>(a->mass_out)) & 3) != 0)
        return fail(ctx, PATCHKV_E_INVALID, "evict_select: misaligned array");
    if (a->kept == a->kv_len || a->kept == a->budget || a->mass_out == a->mass)
        return fail(ctx, PATCHKV_E_INVALID, "evict_select: an output is an input");
    const EvictParams p = {a->mass, a->kv_len, a->budget, a->keep, a->kept, a->mass_out, a->mass_stride, a->keep_stride, a->mass_out_stride,
                           a->max_len, a->max_keep, a->recent, a->sinks, ctx->d_status};
    // CTAs of a cluster: one for every 4096 tokens, up to eight.  (32 sequences of 16000 tokens: 16.1, 12.7, 14.3 and 14.9 us with one for every
    // 2048, 4096, 8192 and 16384; eight of 128k: 22 us with eight CTAs, 336 with one.)
    int ctas = 1;
    while (ctas < kMaxCluster && (long long)ctas * 4096 < a->max_len) ctas *= 2;
    const int run = (a->max_len + ctas * kSelectThreads - 1) / (ctas * kSelectThreads) * kSelectThreads;
    const bool held = run <= kSelectHeld;
    auto bytes = [](int tokens) { return tokens / 32 * 33 * 4 + tokens * 4; };
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return fail(ctx, PATCHKV_E_CUDA, "cudaSetDevice failed");
    static std::atomic<uint64_t> allowed{0};
    if (held) PKV_CUDA(ctx, allow_smem((const void*)evict_select_kernel<true>, bytes(kSelectHeld), &allowed));
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof(cfg));
    cfg.gridDim = dim3(a->n_seqs * ctas); cfg.blockDim = dim3(kSelectThreads); cfg.dynamicSmemBytes = held ? bytes(run) : 0; cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = ctas; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr; cfg.numAttrs = 2;
    PKV_CUDA(ctx, held ? cudaLaunchKernelEx(&cfg, evict_select_kernel<true>, p) : cudaLaunchKernelEx(&cfg, evict_select_kernel<false>, p));
    return PATCHKV_OK;
}

int cache_gather(patchkv_ctx* ctx, const patchkv_geom* g, const patchkv_pool* pool, const patchkv_qpool* cache, int layer,
                 const patchkv_gather_args* a, cudaStream_t stream) {
    MoveParams p;
    if ((pool != nullptr) == (cache != nullptr)) return fail(ctx, PATCHKV_E_INVALID, "cache_gather: give a pool or a cache, one of the two");
    int rc = check_live_geometry(ctx, "cache_gather", g, layer);
    if (rc == PATCHKV_OK) rc = pool ? fill_pool(ctx, "cache_gather", g, pool, layer, &p.c) : fill_cache(ctx, "cache_gather", g, cache, layer, &p.c);
    if (rc == PATCHKV_OK && pool) rc = check_written_pool(ctx, "cache_gather", g, pool);
    if (rc != PATCHKV_OK) return rc;
    if (!a || a->struct_size != sizeof(patchkv_gather_args)) return fail(ctx, PATCHKV_E_INVALID, "cache_gather: null args or wrong struct_size");
    if (a->n_seqs < 0 || a->max_keep < 0 || a->src_stride < 0 || a->dst_stride < 0) return fail(ctx, PATCHKV_E_INVALID, "cache_gather: negative count");
    if (a->n_seqs > 65535) return fail(ctx, PATCHKV_E_UNSUPPORTED, "cache_gather: more than 65535 sequences");
    if (a->rotate != 0 && a->rotate != 1) return fail(ctx, PATCHKV_E_INVALID, "cache_gather: rotate must be 0 or 1");
    if (a->rotate && !pool) return fail(ctx, PATCHKV_E_UNSUPPORTED, "cache_gather: keys of quantised pages are moved as they are; rotate needs a bf16 pool");
    if (a->keep_stride < a->max_keep) return fail(ctx, PATCHKV_E_INVALID, "cache_gather: keep_stride is smaller than max_keep");
    if (a->n_seqs == 0 || a->max_keep == 0) return PATCHKV_OK;
    if (!a->keep || !a->kept || !a->kv_len || (a->src_stride > 0 && !a->src_table) || (a->dst_stride > 0 && !a->dst_table))
        return fail(ctx, PATCHKV_E_INVALID, "cache_gather: null keep, kept, kv_len or table");
    p.Dr = 0;
    if (a->rotate) {
        rc = fill_frequencies(ctx, "cache_gather", g, &p.f);
        if (rc != PATCHKV_OK) return rc;
        p.Dr = g->rotary_dim;
    }
    const bool half = a->rotate && g->rope_style == PATCHKV_ROPE_HALF;
    p.k_pool = const_cast<uint16_t*>(p.c.k); p.v_pool = const_cast<uint16_t*>(p.c.v);
    p.keep = a->keep; p.kept = a->kept; p.kv_len = a->kv_len; p.src_table = a->src_table; p.dst_table = a->dst_table;
    p.keep_stride = a->keep_stride;
    p.status = ctx->d_status;
    p.n_seqs = a->n_seqs; p.max_keep = a->max_keep; p.src_stride = a->src_stride; p.dst_stride = a->dst_stride;
    p.rotate = a->rotate; p.half = half;
    const int H = g->n_kv_heads, D = g->head_dim, ds = log2_exact(D);
    p.k_row = (uint32_t)code_bytes(k_format(p.c.tag), (uint64_t)H * D);
    p.v_row = (uint32_t)code_bytes(v_format(p.c.tag), (uint64_t)H * D);
    p.s_row = 2u * (uint32_t)(H * (D / g->group));
    p.parts = 1; p.passes = 0; p.U_shift = 0;
    bool fast;
    long long threads;                                      // of a sequence
    if (pool) {
        fast = ds >= 4 && ds <= 8 && p.Dr % 16 == 0 && p.c.stride_page % 8 == 0 && p.c.stride_token % 8 == 0 &&
               p.c.stride_head % 8 == 0 && pool->stride_layer % 8 == 0;
        if (fast) {
            p.U_shift = ds - 4;
            const int per_pass = 32 >> p.U_shift;           // heads
            p.passes = (H + per_pass - 1) / per_pass;
            // Few rows: a warp for each pass of a row (8 heads of 128 channels, replayed: 64, 512 and 4096 rows 3.1, 4.0 and 12.6 us; with a warp
            // for a row 4.3, 5.1 and 9.3).
            if ((long long)a->n_seqs * a->max_keep * 2 * p.passes <= 32 * 148) p.parts = 2 * p.passes;
        }
        threads = (long long)a->max_keep * (fast ? 32 * p.parts : H);
    } else {
        fast = p.k_row % 16 == 0 && p.v_row % 16 == 0 && p.s_row % 4 == 0 && p.c.k_scales % 16 == 0 && p.c.v_codes % 16 == 0 && p.c.v_scales % 16 == 0;
        threads = (long long)a->max_keep * (fast ? 32 : H);
    }
    const long long grid = (threads + kGatherThreads - 1) / kGatherThreads;
    if (grid * kGatherThreads > (1ll << 32) - 1) return fail(ctx, PATCHKV_E_UNSUPPORTED, "cache_gather: too many rows for one call");
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return fail(ctx, PATCHKV_E_CUDA, "cudaSetDevice failed");
    const dim3 blocks((unsigned)grid, a->n_seqs), block(kGatherThreads);
    if (!fast) {
        gather_any_kernel<<<blocks, block, 0, stream>>>(p);
        PKV_CUDA(ctx, cudaGetLastError());
    } else if (!pool) {
        PKV_CUDA(ctx, launch_pdl(gather_codes_kernel, blocks, block, 0, stream, p));
    } else {
        PKV_CUDA(ctx, half ? launch_pdl(gather_pool_kernel<true>, blocks, block, 0, stream, p) : launch_pdl(gather_pool_kernel<false>, blocks, block, 0, stream, p));
    }
    return PATCHKV_OK;
}

}  // namespace
}  // namespace patchkv

using namespace patchkv;

extern "C" int patchkv_evict_select(patchkv_ctx* ctx, const patchkv_evict_args* args, void* stream) {
    if (!ctx) return PATCHKV_E_INVALID;
    std::lock_guard<std::mutex> lock(ctx->mu);
    return evict_select(ctx, args, static_cast<cudaStream_t>(stream));
}

extern "C" int patchkv_cache_gather(patchkv_ctx* ctx, const patchkv_geom* geom, const patchkv_pool* pool, const patchkv_qpool* cache,
                                    int layer, const patchkv_gather_args* args, void* stream) {
    if (!ctx) return PATCHKV_E_INVALID;
    std::lock_guard<std::mutex> lock(ctx->mu);
    return cache_gather(ctx, geom, pool, cache, layer, args, static_cast<cudaStream_t>(stream));
}
