// Cutting every request back to its budget: the lowest scores leave.
//
// The v-th smallest of a request's candidates is found digit by digit on keys that order like the scores (11, 11 and 10 bits:
// a histogram in shared memory, a scan, the digit that holds the rank), then the candidates below it -- and the last of those
// equal to it -- are listed in order.  v follows from lengths and budget alone, so every CTA works out for itself where its
// request's victims start, and one launch does it all.  Keys stay in shared memory as far as they fit; a long request is shared out
// over a cluster, whose CTAs read one another's histograms.
#include <atomic>

#include "attention.cuh"
#include "cluster.cuh"

namespace {

constexpr int SV_NT = 512, SV_WARPS = SV_NT / 32, SV_BINS = 2048, SV_KEYS = 16384, SV_MAX_CLUSTER = 8;

struct SelectArgs {
    const int32_t *num_requests;
    vtk_arr<const int32_t> tt_offsets, cache_ids, cache_len, budget, shared_len;
    vtk_arr<const float> scores;
    int32_t sinks, recent, max_requests, max_victims, keys;
    int64_t max_tokens;
    vtk_arr<int32_t> victim_req, victim_tok;
    int32_t *num_victims;
    uint32_t *flags;
};

struct Cut {                             // what a request loses
    int64_t base;                        // first cache (and table) entry
    int range, lo, hi, v;                // table entries; candidates are the cache entries [lo, hi); v of them leave
};

__device__ inline Cut look_up(const SelectArgs &a, int r, bool &clipped)
{
    Cut c;
    const int64_t t0 = a.tt_offsets[r], t1 = a.tt_offsets[r + 1];
    c.base = t0 < 0 ? 0 : (t0 > a.max_tokens ? a.max_tokens : t0);
    const int64_t end = t1 < c.base ? c.base : (t1 > a.max_tokens ? a.max_tokens : t1);
    c.range = (int)(end - c.base);
    const int want = a.cache_len[r], len = want < 0 ? 0 : (want > c.range ? c.range : want);
    clipped |= t0 != c.base || t1 != end || want != len;
    const int keep = a.budget[r] < 0 ? 0 : a.budget[r];
    int lo = a.shared_len.null() ? 0 : a.shared_len[r];
    lo = lo < 0 ? 0 : (lo > len ? len : lo);
    // ids ascend from 0 or above, so entry i >= sinks is no sink
    int n = a.sinks < len ? a.sinks : len;
    if (!a.cache_ids.null() && n > lo && a.cache_ids[c.base + n - 1] >= a.sinks) {
        int below = lo;                  // entries below are sinks, entries from n - 1 on are not
        --n;
        while (below < n) {
            const int mid = (below + n) >> 1;
            if (a.cache_ids[c.base + mid] < a.sinks) below = mid + 1; else n = mid;
        }
    }
    c.lo = n > lo ? n : lo;
    c.hi = a.recent < len ? len - a.recent : 0;
    const int most = c.hi > c.lo ? c.hi - c.lo : 0;
    if (most == 0) c.hi = c.lo;
    c.v = len > keep ? (len - keep < most ? len - keep : most) : 0;
    return c;
}

// ascending like the scores; NaN below everything, the two zeros alike
__device__ __forceinline__ uint32_t key_of(float x)
{
    if (x != x) return 0u;
    const uint32_t b = __float_as_uint(x + 0.f);
    return (b >> 31) ? ~b : b | 0x80000000u;
}

__device__ __forceinline__ uint32_t key_at(const SelectArgs &a, const Cut &c, int entry, int &id, bool &bad)
{
    id = a.cache_ids.null() ? entry : a.cache_ids[c.base + entry];
    if (id < 0 || id >= c.range) { bad = true; return 0u; }
    return key_of(a.scores[c.base + id]);
}

struct Shared {
    int hist[2 * SV_BINS + SV_BINS / 2]; // of the three digits
    int64_t sums[SV_WARPS];
    int warp_tot[32];
    uint64_t part[SV_WARPS], part_total; // keys below the threshold, equal ones << 32
    Cut cut;
    int bin, below, inside;
};

__device__ __forceinline__ void count_key(int *hist, int bin, bool there)
{
    // (many tokens that nothing has looked at: one bin for the whole warp)
    const unsigned who = __ballot_sync(0xffffffffu, there);
    if (who == 0) return;
    const int leader = __ffs(who) - 1, first = __shfl_sync(0xffffffffu, bin, leader);
    if (__all_sync(0xffffffffu, !there || bin == first)) {
        if (vtk_lane() == leader) atomicAdd(hist + first, __popc(who));
    } else if (there) {
        atomicAdd(hist + bin, 1);
    }
}

__global__ void __launch_bounds__(SV_NT) select_kernel(const __grid_constant__ SelectArgs a)
{
    __shared__ Shared sh;
    extern __shared__ uint32_t keys[];
    vtk_release_successor();
    vtk_wait_for_predecessor();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int C = vtk_cluster_size(), rank = vtk_cluster_rank(), clusters = gridDim.x / C;
    int R = *a.num_requests;
    bool clipped = R < 0 || R > a.max_requests, bad = false, dropped = false;
    R = R < 0 ? 0 : (R > a.max_requests ? a.max_requests : R);
    auto sync = [&]() { if (C > 1) vtk_cluster_sync(); else __syncthreads(); };
    if (R == 0 && blockIdx.x == 0 && tid == 0) *a.num_victims = 0;
    int64_t out = 0;                                         // victims of the requests in front
    int seen = 0;
    for (int r = blockIdx.x / C; r < R; r += clusters) {
        int64_t mine = 0;
        for (int i = seen + tid; i <= r; i += SV_NT) {
            const Cut c = look_up(a, i, clipped);
            if (i == r) sh.cut = c; else mine += c.v;
        }
        for (int i = tid; i < (int)(sizeof(sh.hist) / sizeof(int)); i += SV_NT) sh.hist[i] = 0;
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, d);
        if (lane == 0) sh.sums[warp] = mine;
        __syncthreads();
        for (int w = 0; w < SV_WARPS; ++w) out += sh.sums[w];
        const Cut c = sh.cut;
        seen = r + 1;
        if (r == R - 1 && rank == 0 && tid == 0) {
            const int64_t all = out + c.v;
            *a.num_victims = all > a.max_victims ? a.max_victims : (int)all;
            dropped = all > a.max_victims;
        }
        if (c.v > 0) {
            // this CTA's part of the candidates, a run of it for each warp
            const int n = c.hi - c.lo;
            const int part0 = (int)((int64_t)n * rank / C), part1 = (int)((int64_t)n * (rank + 1) / C), np = part1 - part0;
            const int per = ((np + SV_NT - 1) / SV_NT) * 32, w0 = warp * per < np ? warp * per : np, w1 = w0 + per < np ? w0 + per : np;
            uint32_t threshold = 0xffffffffu;                // above every key
            int less = c.v, keep_equal = 0;
            auto key = [&](int i, int &id) { return key_at(a, c, c.lo + part0 + i, id, bad); };
            const bool all = c.v == n;
            if (!all) {
                constexpr int U = 8;                         // independent loads a lane
                for (int i = w0; i < w1; i += 32 * U) {
                    uint32_t k[U];
                    int id;
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        const int at = i + 32 * u + lane;
                        k[u] = at < w1 ? key(at, id) : 0u;
                    }
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        const int at = i + 32 * u + lane;
                        if (at < w1 && at < a.keys) keys[at] = k[u];
                        count_key(sh.hist, (int)(k[u] >> 21), at < w1);
                    }
                }
                auto again = [&](int at) {
                    int id;
                    return at < a.keys ? keys[at] : key(at, id);
                };
                uint32_t prefix = 0;
                int rest = c.v - 1;                          // rank of the wanted key among those that share the prefix
                less = 0;
#pragma unroll
                for (int pass = 0; pass < 3; ++pass) {
                    constexpr int SHIFT[3] = {21, 10, 0}, BITS[3] = {11, 11, 10};
                    int *hist = sh.hist + pass * SV_BINS;
                    const int bins = 1 << BITS[pass];
                    if (pass > 0) {
                        for (int i = w0; i < w1; i += 32) {
                            const uint32_t k = i + lane < w1 ? again(i + lane) : 0u;
                            const bool there = i + lane < w1 && (k >> (SHIFT[pass] + BITS[pass])) == prefix;
                            count_key(hist, (int)((k >> SHIFT[pass]) & (uint32_t)(bins - 1)), there);
                        }
                    }
                    sync();
                    int h[4] = {0, 0, 0, 0}, sum = 0;
                    if (tid * 4 < bins) {
                        for (int p = 0; p < C; ++p)
#pragma unroll
                            for (int j = 0; j < 4; ++j) h[j] += C > 1 ? vtk_cluster_read(hist + tid * 4 + j, p) : hist[tid * 4 + j];
#pragma unroll
                        for (int j = 0; j < 4; ++j) sum += h[j];
                    }
                    const int in_warp = vtk_warp_incl_scan(sum);
                    if (lane == 31) sh.warp_tot[warp] = in_warp;
                    __syncthreads();
                    int before = in_warp - sum;
                    for (int w = 0; w < warp; ++w) before += sh.warp_tot[w];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        if (rest >= before && rest < before + h[j]) {
                            sh.bin = tid * 4 + j;
                            sh.below = before;
                            sh.inside = h[j];
                        }
                        before += h[j];
                    }
                    __syncthreads();
                    prefix = (prefix << BITS[pass]) | (uint32_t)sh.bin;
                    less += sh.below;
                    rest -= sh.below;
                    if (pass == 2) keep_equal = sh.inside - (c.v - less);
                    __syncthreads();
                }
                threshold = prefix;
            }
            // how many of each warp's run are below and equal, then the list
            auto value = [&](int at, int &id) {
                if (!all && at < a.keys) {
                    id = a.cache_ids.null() ? c.lo + part0 + at : a.cache_ids[c.base + c.lo + part0 + at];
                    return keys[at];
                }
                return key(at, id);
            };
            int lt = 0, eq = 0;
            if (all) {
                lt = w1 - w0;
            } else {
                for (int i = w0; i < w1; i += 32) {
                    int id;
                    const bool in = i + lane < w1;
                    const uint32_t k = in ? (i + lane < a.keys ? keys[i + lane] : key(i + lane, id)) : 0u;
                    lt += __popc(__ballot_sync(0xffffffffu, in && k < threshold));
                    eq += __popc(__ballot_sync(0xffffffffu, in && k == threshold));
                }
            }
            if (lane == 0) sh.part[warp] = (uint64_t)(uint32_t)lt | (uint64_t)(uint32_t)eq << 32;
            __syncthreads();
            uint64_t upto = 0, total = 0;
            for (int w = 0; w < SV_WARPS; ++w) {
                if (w < warp) upto += sh.part[w];
                total += sh.part[w];
            }
            if (C > 1) {
                if (tid == 0) sh.part_total = total;
                vtk_cluster_sync();
                for (int p = 0; p < rank; ++p) upto += vtk_cluster_read(&sh.part_total, p);
            }
            lt = (int)(uint32_t)upto;
            eq = (int)(upto >> 32);
            for (int i = w0; i < w1; i += 32) {
                int id = 0;
                const bool in = i + lane < w1;
                const uint32_t k = in ? value(i + lane, id) : 0u;
                const unsigned is_lt = __ballot_sync(0xffffffffu, in && k < threshold), is_eq = __ballot_sync(0xffffffffu, in && k == threshold);
                const unsigned before = (1u << lane) - 1u;
                const int my_lt = lt + __popc(is_lt & before), my_eq = eq + __popc(is_eq & before);
                if (in && (k < threshold || (k == threshold && my_eq >= keep_equal))) {
                    const int64_t at = out + my_lt + (my_eq > keep_equal ? my_eq - keep_equal : 0);
                    if (at < a.max_victims) {
                        a.victim_req[at] = r;
                        a.victim_tok[at] = id;
                    }
                }
                lt += __popc(is_lt);
                eq += __popc(is_eq);
            }
            out += c.v;
        }
        sync();                                              // the counts and keys are the next request's
    }
    if (clipped || dropped) atomicOr(a.flags, (uint32_t)VTOKEN_FLAG_CAPACITY);
    if (bad) atomicOr(a.flags, (uint32_t)VTOKEN_FLAG_BAD_VICTIM);
}

}  // namespace

extern "C" int vtoken_select_victims(vtoken_ctx *ctx, const vtoken_select_in *in, void *cuda_stream)
{
    if (!ctx || !in) return VTOKEN_EINVAL;
    if (!in->num_requests || !in->tt_offsets || !in->cache_len || !in->scores || !in->budget || !in->num_victims) return VTOKEN_EINVAL;
    if (in->max_victims < 0 || (in->max_victims > 0 && (!in->victim_req || !in->victim_tok))) return VTOKEN_EINVAL;
    if (in->sinks < 0 || in->recent < 0 || in->max_cache_len < 1) return VTOKEN_EINVAL;
    SelectArgs a;
    a.num_requests = in->num_requests;
    a.tt_offsets = VTK_ARR(ctx, in->tt_offsets, ctx->cfg.max_requests + 1);
    a.cache_ids = VTK_ARR(ctx, in->cache_ids, ctx->cfg.max_tokens);
    a.cache_len = VTK_ARR(ctx, in->cache_len, ctx->cfg.max_requests);
    a.budget = VTK_ARR(ctx, in->budget, ctx->cfg.max_requests);
    a.shared_len = VTK_ARR(ctx, in->shared_len, ctx->cfg.max_requests);
    a.scores = VTK_ARR(ctx, in->scores, ctx->cfg.max_tokens);
    a.sinks = in->sinks;
    a.recent = in->recent;
    a.max_requests = ctx->cfg.max_requests;
    a.max_victims = in->max_victims;
    a.max_tokens = ctx->cfg.max_tokens;
    a.victim_req = VTK_ARR(ctx, in->victim_req, in->max_victims);
    a.victim_tok = VTK_ARR(ctx, in->victim_tok, in->max_victims);
    a.num_victims = in->num_victims;
    a.flags = &ctx->rt_counts->error_flags;
    const int64_t longest = in->max_cache_len < ctx->cfg.max_tokens ? in->max_cache_len : ctx->cfg.max_tokens;
    int size = 1;
    while (size < SV_MAX_CLUSTER && longest > (int64_t)size * SV_KEYS) size *= 2;
    const int64_t keys = ((longest + size - 1) / size + 1023) / 1024 * 1024;
    a.keys = keys > SV_KEYS ? SV_KEYS : (int)keys;
    const int64_t most = (int64_t)ctx->num_sms * 8 / size;
    const int clusters = ctx->cfg.max_requests < most ? ctx->cfg.max_requests : (int)most;
    static std::atomic<int> allowed{-1};
    VTK_CUDA(ctx, vtk_allow_smem(ctx, allowed, (const void *)select_kernel, SV_KEYS * 4));
    VTK_CUDA(ctx, vtk_launch_clusters(ctx, select_kernel, size, dim3(clusters * size), dim3(SV_NT), a.keys * 4, (cudaStream_t)cuda_stream, a));
    VTK_CUDA(ctx, cudaGetLastError());
    return VTOKEN_OK;
}
