// Cutting every request back to its budget: the lowest scores leave.
//
// The v-th smallest of a request's candidates is found digit by digit on keys that order like the scores (11, 11 and 10 bits:
// a histogram in shared memory, a scan, the digit that holds the rank), then the candidates below it -- and the last of those
// equal to it -- are listed in order.  v follows from lengths and budget alone, so every CTA works out for itself where its
// request's victims start, and one launch does it all.  Keys stay in shared memory as far as they fit; a long request is shared out
// over a cluster, whose CTAs each add up a share of all their bins.
//
// Bound by instructions and barriers, not by what is read: 512 requests of 1.5 M tokens in all, 18 MB, take 24 us, where the longest
// request's CTA is waited for; six requests of 50 000 to 131 072 tokens 21 us on clusters of 16.  256 threads a request, so that four are
// resident on an SM (512 threads: 46 us); every CTA of a cluster reading all bins of all others: 41 us for the six.
#include <atomic>

#include "attention.cuh"
#include "cluster.cuh"

namespace {

constexpr int SV_BINS = 2048, SV_KEYS = 8192, SV_MAX_CLUSTER = 16;

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

struct Shared {
    alignas(16) int hist[2 * SV_BINS + SV_BINS / 2];         // of the three digits
    alignas(16) int slice[SV_BINS / 2];  // clusters: this CTA's share of the bins, of all CTAs
    int64_t sums[32];
    int warp_tot[32];
    uint64_t part[32], part_total; // keys below the threshold, equal ones << 32
    Cut cut;
    int bin, below, inside;
};

// of a lane's four keys those that begin with `prefix`, by their next digit (SHIFT: bits behind it; 0xffffffff: there is none)
template <int SHIFT>
__device__ __forceinline__ void count_keys(int *hist, const uint32_t (&k)[4], uint32_t prefix)
{
    constexpr int BITS = SHIFT == 0 ? 10 : 11;
    constexpr uint32_t MASK = (1u << BITS) - 1u;
    if (SHIFT == 21) {                   // tokens that nothing has looked at all have one key: one count for the warp
        const uint32_t first = __shfl_sync(0xffffffffu, k[0], 0);
        if (__all_sync(0xffffffffu, k[0] == first && k[1] == first && k[2] == first && k[3] == first)) {
            if (vtk_lane() == 0 && first != 0xffffffffu) atomicAdd(hist + (first >> SHIFT), 128);
            return;
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (SHIFT == 21 ? k[j] != 0xffffffffu : k[j] >> ((SHIFT + BITS) & 31) == prefix) atomicAdd(hist + ((k[j] >> SHIFT) & MASK), 1);      // (no score's key begins like 0xffffffff)
}

template <typename T, int U, typename F>
__device__ __forceinline__ void for_each(T (&x)[U][4], F f)
{
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int j = 0; j < 4; ++j) f(u, j, x[u][j]);
}

// NT: 256 threads, four requests an SM at a time; 1024 where clusters work on a request
template <int NT>
__global__ void __launch_bounds__(NT, 1024 / NT) select_kernel(const __grid_constant__ SelectArgs a)
{
    constexpr int WARPS = NT / 32;
    __shared__ Shared sh;
    extern __shared__ __align__(16) uint32_t keys[];
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
        for (int i = seen + tid; i <= r; i += NT) {
            const Cut c = look_up(a, i, clipped);
            if (i == r) sh.cut = c; else mine += c.v;
        }
        for (int i = tid; i < (int)(sizeof(sh.hist) / sizeof(int)); i += NT) sh.hist[i] = 0;
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, d);
        if (lane == 0) sh.sums[warp] = mine;
        __syncthreads();
        for (int w = 0; w < WARPS; ++w) out += sh.sums[w];
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
            const int per = ((np + 4 * NT - 1) / (4 * NT)) * 128, w0 = warp * per < np ? warp * per : np, w1 = w0 + per < np ? w0 + per : np;
            uint32_t threshold = 0xffffffffu;                // above every key
            int less = c.v, keep_equal = 0;
            const bool all = c.v == n;
            // the candidates i + lane, + 32, ..., 0xffffffff behind the last (no score has that key): from the tables, or kept
            const int32_t *id_at = a.cache_ids.null() ? nullptr : a.cache_ids.at(c.base + c.lo + part0, np);
            const float *score_at = a.scores.at(c.base, c.range);
            const int entry0 = c.lo + part0;
            auto fetch = [&](int i, auto &id, auto &k, auto whole) {
                constexpr bool WHOLE = decltype(whole)::value;       // no candidate of these lies behind the run
                for_each(id, [&](int u, int j, int &x) {
                    const int at = i + 128 * u + 32 * j + lane;
                    x = id_at != nullptr ? (WHOLE || at < w1 ? id_at[at] : 0) : entry0 + at;
                });
                for_each(k, [&](int u, int j, uint32_t &x) {
                    x = 0xffffffffu;
                    if (!WHOLE && i + 128 * u + 32 * j + lane >= w1) return;
                    const bool ok = (uint32_t)id[u][j] < (uint32_t)c.range;
                    bad |= !ok;
                    x = ok ? key_of(score_at[id[u][j]]) : 0u;
                });
            };
            auto kept = [&](int i, uint32_t (&k)[1][4]) {
                if (i + 128 <= a.keys) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) k[0][j] = keys[i + 32 * j + lane];
                } else {
                    int id[1][4];
                    fetch(i, id, k, std::false_type());
                }
            };
            if (!all) {
                constexpr int U = 3;                         // twelve independent loads a lane, twice
                auto count = [&](int i0, auto whole) {
                    uint32_t k[U][4];
                    int id[U][4];
                    fetch(i0, id, k, whole);
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        if (!decltype(whole)::value && i0 + 128 * u >= w1) break;    // (what is behind is another warp's)
                        if (i0 + 128 * (u + 1) <= a.keys)
#pragma unroll
                            for (int j = 0; j < 4; ++j) keys[i0 + 128 * u + 32 * j + lane] = k[u][j];
                        count_keys<21>(sh.hist, k[u], 0u);
                    }
                };
                int i0 = w0;
                for (; i0 + 128 * U <= w1; i0 += 128 * U) count(i0, std::true_type());
                for (; i0 < w1; i0 += 128 * U) count(i0, std::false_type());
                uint32_t prefix = 0;
                int rest = c.v - 1;                          // rank of the wanted key among those that share the prefix
                less = 0;
#pragma unroll
                for (int pass = 0; pass < 3; ++pass) {
                    constexpr int BITS[3] = {11, 11, 10};
                    int *hist = sh.hist + pass * SV_BINS;
                    const int bins = 1 << BITS[pass];
                    if (pass > 0) {
                        for (int i0 = w0; i0 < w1; i0 += 128) {
                            uint32_t k[1][4];
                            kept(i0, k);
                            if (pass == 1) count_keys<10>(hist, k[0], prefix);
                            else count_keys<0>(hist, k[0], prefix);
                        }
                    }
                    sync();
                    if (C > 1) {                             // every CTA adds up a share of the bins
                        const int share = bins / C;
                        for (int i = tid; i < share; i += NT) {
                            int x = 0;
#pragma unroll 8
                            for (int p = 0; p < C; ++p) x += vtk_cluster_read(hist + rank * share + i, p);
                            sh.slice[i] = x;
                        }
                        vtk_cluster_sync();
                    }
                    constexpr int PER = SV_BINS / NT;        // bins of a thread
                    int h[PER], sum = 0;
#pragma unroll
                    for (int j = 0; j < PER; ++j) h[j] = 0;
                    if (tid * PER < bins) {
                        if (C == 1) {
#pragma unroll
                            for (int j = 0; j < PER; ++j) h[j] = hist[tid * PER + j];
                        } else {
                            const int share = bins / C;      // (a power of two, 64 or more)
#pragma unroll
                            for (int j = 0; j < PER; j += 2) {
                                const int at = tid * PER + j;
                                const int2 x = vtk_cluster_read(reinterpret_cast<const int2 *>(sh.slice + at % share), at / share);
                                h[j] = x.x;
                                h[j + 1] = x.y;
                            }
                        }
#pragma unroll
                        for (int j = 0; j < PER; ++j) sum += h[j];
                    }
                    const int in_warp = vtk_warp_incl_scan(sum);
                    if (lane == 31) sh.warp_tot[warp] = in_warp;
                    __syncthreads();
                    int before = in_warp - sum;
                    for (int w = 0; w < warp; ++w) before += sh.warp_tot[w];
                    if (rest >= before && rest < before + sum) {
#pragma unroll
                        for (int j = 0; j < PER; ++j) {
                            if (rest >= before && rest < before + h[j]) {
                                sh.bin = tid * PER + j;
                                sh.below = before;
                                sh.inside = h[j];
                            }
                            before += h[j];
                        }
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
            int lt = 0, eq = 0;
            if (all) {
                lt = w1 - w0;
            } else {
                for (int i0 = w0; i0 < w1; i0 += 128) {
                    uint32_t k[1][4];
                    kept(i0, k);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        lt += k[0][j] < threshold;
                        eq += k[0][j] == threshold;
                    }
                }
                lt = __reduce_add_sync(0xffffffffu, lt);
                eq = __reduce_add_sync(0xffffffffu, eq);
            }
            if (lane == 0) sh.part[warp] = (uint64_t)(uint32_t)lt | (uint64_t)(uint32_t)eq << 32;
            __syncthreads();
            uint64_t upto = 0, total = 0;
            for (int w = 0; w < WARPS; ++w) {
                if (w < warp) upto += sh.part[w];
                total += sh.part[w];
            }
            if (C > 1) {
                if (tid == 0) sh.part_total = total;
                vtk_cluster_sync();
                for (int p = 0; p < rank; ++p) upto += vtk_cluster_read(&sh.part_total, p);
            }
            eq = (int)(upto >> 32);
            int64_t next = out + (uint32_t)upto + (eq > keep_equal ? eq - keep_equal : 0);       // where the run's victims go
            constexpr int U = 3;
            for (int i0 = w0; i0 < w1; i0 += 128 * U) {
                uint32_t k[U][4];
                int id[U][4];
                if (all || i0 + 128 * U > a.keys) {
                    fetch(i0, id, k, std::false_type());
                } else {
                    for_each(k, [&](int u, int j, uint32_t &x) {
                        const int at = i0 + 128 * u + 32 * j + lane;
                        x = at < w1 ? keys[at] : 0xffffffffu;
                    });
                    for_each(id, [&](int u, int j, int &x) {
                        const int at = i0 + 128 * u + 32 * j + lane;
                        x = entry0 + at;
                        if (id_at != nullptr && k[u][j] <= threshold && at < w1) x = id_at[at];
                    });
                }
                const unsigned before = (1u << lane) - 1u;
                for_each(k, [&](int u, int j, uint32_t &x) {
                    bool leaves = x < threshold;
                    if (!all) {
                        const unsigned eqs = __ballot_sync(0xffffffffu, x == threshold);
                        if (eqs) {
                            leaves |= x == threshold && eq + __popc(eqs & before) >= keep_equal;
                            eq += __popc(eqs);
                        }
                    }
                    const unsigned gone = __ballot_sync(0xffffffffu, leaves);
                    const int64_t to = next + __popc(gone & before);
                    if (leaves && to < a.max_victims) {
                        a.victim_req[to] = r;
                        a.victim_tok[to] = id[u][j];
                    }
                    next += __popc(gone);
                });
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
    cudaStream_t st = (cudaStream_t)cuda_stream;
    static std::atomic<int> allowed[2] = {{-1}, {-1}};       // the device that knows of the kernels' shared memory and clusters of 16
    if (size == 1) {
        VTK_CUDA(ctx, vtk_allow_smem(ctx, allowed[0], (const void *)select_kernel<256>, SV_KEYS * 4));
        VTK_CUDA(ctx, vtk_launch_clusters(ctx, select_kernel<256>, 1, dim3(clusters), dim3(256), a.keys * 4, st, a));
    } else {
        if (size > 8) VTK_CUDA(ctx, cudaFuncSetAttribute((const void *)select_kernel<1024>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
        VTK_CUDA(ctx, vtk_allow_smem(ctx, allowed[1], (const void *)select_kernel<1024>, SV_KEYS * 4));
        VTK_CUDA(ctx, vtk_launch_clusters(ctx, select_kernel<1024>, size, dim3(clusters * size), dim3(1024), a.keys * 4, st, a));
    }
    VTK_CUDA(ctx, cudaGetLastError());
    return VTOKEN_OK;
}
