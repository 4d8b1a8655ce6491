// Verification of drafted tokens: the first refusal, the row to draw from, the draw, the list of rejected drafts.
//
// Bound by the row of the vocabulary (two after a refusal) that the next token is drawn from.  A cluster works on a request; its
// warps take consecutive runs of the row and sum them in 64 bits, the CTAs exchange their sums, and the run that holds the drawn mass is
// cut up among its CTA's warps once more before one of them walks over what is left.  The drafts before it need two numbers each.  One more cluster tests the drafts of all
// requests and lists the rejected ones, so that a step is one launch.  200 requests, vocabulary 128 256: 44 us, 4.7 TB/s; one request of
// 32 000: 8 us, a chain of dependent loads.  (The forms that read 16 bytes at a time spill 224 bytes a thread at three CTAs an SM.)
#include "cluster.cuh"
#include "heads.cuh"

namespace {

constexpr int VD_NT = 256, VD_WARPS = VD_NT / 32, VD_LANES = 8;     // VD_LANES: threads that test the drafts of a request

struct VerifyArgs {
    const int32_t *num_requests;
    vtk_arr<const int32_t> draft_offsets, draft_tokens, first_id;
    const void *target, *draft;
    int64_t target_stride, draft_stride;
    vtk_arr<const float> accept_random, sample_random;
    vtk_arr<int32_t> accepted, next_tokens, out_tokens, victim_req, victim_tok;
    int32_t *num_victims;
    int32_t vocab, max_drafts, max_requests, max_victims;
    uint32_t *flags;
};

struct F32 {
    using type = float;
    static constexpr int VE = 4;
    static __device__ __forceinline__ float get(float x) { return x; }
    static __device__ __forceinline__ void unpack(uint4 w, float (&x)[4])
    {
        x[0] = __uint_as_float(w.x); x[1] = __uint_as_float(w.y); x[2] = __uint_as_float(w.z); x[3] = __uint_as_float(w.w);
    }
};
template <typename T>
struct Half {
    using type = uint16_t;
    static constexpr int VE = 8;
    static __device__ __forceinline__ float get(uint16_t x) { return T::unpack(x).x; }
    static __device__ __forceinline__ void unpack(uint4 w, float (&x)[8]) { vtk_unpack8<T>(w, x); }
};

// what a probability counts for
__device__ __forceinline__ float mass(float x) { return x > 0.f && x < INFINITY ? x : 0.f; }

struct Drafts { int d0, k; };
__device__ __forceinline__ Drafts drafts_of(const VerifyArgs &a, int r, bool &clipped)
{
    Drafts d;
    if (a.max_drafts == 0) { d.d0 = d.k = 0; return d; }
    const int o0 = a.draft_offsets[r], o1 = a.draft_offsets[r + 1];
    d.d0 = o0 < 0 ? 0 : (o0 > a.max_drafts ? a.max_drafts : o0);
    const int end = o1 < d.d0 ? d.d0 : (o1 > a.max_drafts ? a.max_drafts : o1);
    d.k = end - d.d0;
    clipped |= d.d0 != o0 || end != o1;
    return d;
}

template <typename P>
__device__ __forceinline__ bool refused(const VerifyArgs &a, int r, const Drafts &d, int i)
{
    using T = typename P::type;
    const int x = a.draft_tokens[d.d0 + i];
    float p = 0.f, q = a.draft == nullptr ? 1.f : 0.f;
    if (x >= 0 && x < a.vocab) {
        p = mass(P::get(static_cast<const T *>(a.target)[(int64_t)(d.d0 + r + i) * a.target_stride + x]));
        if (a.draft != nullptr) q = mass(P::get(static_cast<const T *>(a.draft)[(int64_t)(d.d0 + i) * a.draft_stride + x]));
    }
    return !((double)a.accept_random[d.d0 + i] * (double)q < (double)p);
}

// the row that a token is drawn from: p, or what p has more than q, or p without one token
template <typename P, bool VEC>
struct Row {
    using T = typename P::type;
    const T *p, *q;
    int without, vocab;
    // masses of the elements [at, at + VE), zero behind the vocabulary
    __device__ __forceinline__ void get(int at, float (&x)[P::VE], float (&y)[P::VE]) const
    {
        if (VEC && at + P::VE <= vocab) {
            P::unpack(*reinterpret_cast<const uint4 *>(p + at), x);
            if (q != nullptr) P::unpack(*reinterpret_cast<const uint4 *>(q + at), y);
        } else {
#pragma unroll
            for (int e = 0; e < P::VE; ++e) {
                x[e] = at + e < vocab ? P::get(p[at + e]) : 0.f;
                y[e] = q != nullptr && at + e < vocab ? P::get(q[at + e]) : 0.f;
            }
        }
    }
    __device__ __forceinline__ double value(int at, float x, float y) const
    {
        double v = (double)mass(x);
        if (q != nullptr) v = fmax(v - (double)mass(y), 0.0);
        return at == without ? 0.0 : v;
    }
    static constexpr int STEP = 32 * P::VE, U = 16 / P::VE;  // elements of a warp's load; independent loads
    // Of the elements [lo, hi) by a warp, in every lane.  CLEAN false: infinities are not taken out, a sum that is no finite number tells of
    // them.  There a difference p - q >= 0 is the 32-bit one and its rounding error, which 32 bits hold too (|p| >= |q|), so that one
    // conversion to 64 bits does where the definition has two and a comparison (conversions, at 16 a cycle and SM, bound the sum of a
    // row that way); the errors of 16 elements are added in 32 bits, 2^-45 of the sum.
    template <bool CLEAN, bool MINUS>
    __device__ __forceinline__ double sum_of(int lo, int hi) const
    {
        double s = 0.0;
        for (int i = lo + vtk_lane() * P::VE; i < hi; i += STEP * U) {
            float x[U][P::VE], y[U][P::VE], low = 0.f;
#pragma unroll
            for (int u = 0; u < U; ++u) get(i + u * STEP < hi ? i + u * STEP : vocab, x[u], y[u]);
            if (!CLEAN && !MINUS) {
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if ((uint32_t)(without - (i + u * STEP)) < (uint32_t)P::VE) {        // (one lane, once a row)
#pragma unroll
                        for (int e = 0; e < P::VE; ++e)
                            if (i + u * STEP + e == without) x[u][e] = 0.f;
                    }
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int e = 0; e < P::VE; ++e) {
                    if (CLEAN) {
                        s += value(i + u * STEP + e, x[u][e], y[u][e]);
                    } else if (MINUS) {
                        const float q0 = fmaxf(y[u][e], 0.f), p0 = fmaxf(x[u][e], q0), d = p0 - q0;
                        low += (p0 - d) - q0;
                        s += (double)d;
                    } else {
                        s += (double)fmaxf(x[u][e], 0.f);
                    }
                }
            s += (double)low;
        }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
        return s;
    }
    __device__ __forceinline__ double sum(int lo, int hi, bool clean) const
    {
        if (clean) return sum_of<true, true>(lo, hi);
        return q != nullptr ? sum_of<false, true>(lo, hi) : sum_of<false, false>(lo, hi);
    }
    // the first element of [lo, hi) at which the mass, `before` in front of it, exceeds `drawn`; else the last that has any; -1: none
    __device__ __forceinline__ int find(int lo, int hi, double before, double drawn) const
    {
        int any = -1;
        for (int i0 = lo; i0 < hi; i0 += STEP * U) {
            float x[U][P::VE], y[U][P::VE];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = i0 + u * STEP + vtk_lane() * P::VE;
                get(i < hi ? i : vocab, x[u], y[u]);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = i0 + u * STEP + vtk_lane() * P::VE;
                double v[P::VE], s = 0.0;
                int mine = -1;
#pragma unroll
                for (int e = 0; e < P::VE; ++e) {
                    v[e] = i < hi ? value(i + e, x[u][e], y[u][e]) : 0.0;
                    if (v[e] > 0.0) mine = i + e;
                    s += v[e];
                }
                const double incl = vtk_warp_incl_scan(s);
                double c = before + (incl - s);
                int found = -1;
#pragma unroll
                for (int e = 0; e < P::VE; ++e) {
                    c += v[e];
                    if (found < 0 && c > drawn && v[e] > 0.0) found = i + e;
                }
                const unsigned who = __ballot_sync(0xffffffffu, found >= 0);
                if (who) return __shfl_sync(0xffffffffu, found, __ffs(who) - 1);
                any = max(any, __reduce_max_sync(0xffffffffu, mine));
                before += __shfl_sync(0xffffffffu, incl, 31);
            }
        }
        return any;
    }
};

struct Shared {
    double warp_sum[VD_WARPS], again[VD_WARPS], cta_sum[2];
    int at;                              // first refusal, or the number of drafts
    int scan[VD_WARPS + 1];
};

// cluster `last` of the grid: every request's drafts, the rejected ones in a list
template <typename P>
__device__ void list_rejected(const VerifyArgs &a, Shared &sh, int R, bool &clipped)
{
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, sub = tid % VD_LANES;
    int64_t base = 0;
    for (int r0 = 0; r0 < R; r0 += VD_NT / VD_LANES) {
        const int r = r0 + tid / VD_LANES;
        Drafts d = {0, 0};
        if (r < R) d = drafts_of(a, r, clipped);
        int at = d.k;
        for (int i = sub; i < at; i += VD_LANES)
            if (refused<P>(a, r, d, i)) at = i;              // (the lane's first; the loop ends)
#pragma unroll
        for (int s = VD_LANES / 2; s > 0; s >>= 1) {
            const int o = __shfl_xor_sync(0xffffffffu, at, s);
            at = o < at ? o : at;
        }
        const int mine = sub == 0 ? d.k - at : 0, incl = vtk_warp_incl_scan(mine);
        if (lane == 31) sh.scan[warp] = incl;
        __syncthreads();
        int64_t before = base;
        for (int w = 0; w < VD_WARPS; ++w) {
            if (w < warp) before += sh.scan[w];
            base += sh.scan[w];
        }
        before += __shfl_sync(0xffffffffu, incl - mine, lane & ~(VD_LANES - 1));
        for (int i = at + sub; i < d.k; i += VD_LANES) {
            const int64_t to = before + (i - at);
            if (to < a.max_victims) {
                a.victim_req[to] = r;
                a.victim_tok[to] = a.first_id[r] + i;
            }
        }
        __syncthreads();
    }
    if (tid == 0) {
        *a.num_victims = base > a.max_victims ? a.max_victims : (int)base;
        clipped |= base > a.max_victims;
    }
}

template <typename P, bool VEC>
__global__ void __launch_bounds__(VD_NT, 3) verify_kernel(const __grid_constant__ VerifyArgs a, int row_clusters)
{
    using T = typename P::type;
    constexpr int STEP = Row<P, VEC>::STEP;
    __shared__ Shared sh;
    vtk_release_successor();
    vtk_wait_for_predecessor();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int C = vtk_cluster_size(), rank = vtk_cluster_rank(), cluster = blockIdx.x / C;
    int R = *a.num_requests;
    bool clipped = R < 0 || R > a.max_requests;
    R = R < 0 ? 0 : (R > a.max_requests ? a.max_requests : R);
    if (cluster >= row_clusters) {
        if (rank == 0) list_rejected<P>(a, sh, R, clipped);
        if (clipped) atomicOr(a.flags, (uint32_t)VTOKEN_FLAG_CAPACITY);
        return;
    }
    // the warp's run of every row
    const int per = ((a.vocab + C * VD_WARPS - 1) / (C * VD_WARPS) + STEP - 1) / STEP * STEP;
    const int64_t run0 = (int64_t)(rank * VD_WARPS + warp) * per;
    const int lo = run0 < a.vocab ? (int)run0 : a.vocab, hi = run0 + per < a.vocab ? (int)run0 + per : a.vocab;
    int turn = 0;
    for (int r = cluster; r < R; r += row_clusters) {
        const Drafts d = drafts_of(a, r, clipped);
        if (warp == 0) {
            int at = d.k;
            for (int i0 = 0; i0 < d.k && at == d.k; i0 += 32) {
                const unsigned no = __ballot_sync(0xffffffffu, i0 + lane < d.k && refused<P>(a, r, d, i0 + lane));
                if (no) at = i0 + __ffs(no) - 1;
            }
            if (lane == 0) sh.at = at;
        }
        __syncthreads();
        const int at = sh.at;
        Row<P, VEC> row;
        row.vocab = a.vocab;
        row.p = static_cast<const T *>(a.target) + (int64_t)(d.d0 + r + at) * a.target_stride;
        row.q = at < d.k && a.draft != nullptr ? static_cast<const T *>(a.draft) + (int64_t)(d.d0 + at) * a.draft_stride : nullptr;
        row.without = at < d.k && a.draft == nullptr ? a.draft_tokens[d.d0 + at] : -1;
        if (rank == 0) {
            if (tid == 0) a.accepted[r] = at;
            if (!a.out_tokens.null())
                for (int i = tid; i <= d.k; i += VD_NT)
                    if (i != at) a.out_tokens[d.d0 + r + i] = i < at ? a.draft_tokens[d.d0 + i] : -1;
        }
        double before, total;
        bool clean = false;
        for (;;) {
            const double sum = row.sum(lo, hi, clean);
            if (lane == 0) sh.warp_sum[warp] = sum;
            __syncthreads();
            if (tid == 0) {
                double s = 0.0;
                for (int w = 0; w < VD_WARPS; ++w) s += sh.warp_sum[w];
                sh.cta_sum[turn & 1] = s;
            }
            if (C > 1) vtk_cluster_sync(); else __syncthreads();
            before = total = 0.0;
            for (int c = 0; c < C; ++c) {
                if (c == rank) before = total;
                total += C > 1 ? vtk_cluster_read(&sh.cta_sum[turn & 1], c) : sh.cta_sum[turn & 1];
            }
            ++turn;
            if (!clean && !(total < INFINITY)) {             // (an infinity or what came of one: element by element)
                clean = true;
                continue;
            }
            if (total > 0.0 || (row.q == nullptr && row.without < 0)) break;
            row.q = nullptr;                                 // the draft's source has all that the target has
            row.without = -1;
        }
        // the run with the drawn mass: the first whose cumulated mass exceeds it, else the last that has any
        const float w0 = a.sample_random[r];
        const double drawn = (w0 > 0.f ? (double)w0 : 0.0) * total;
        int owner = -1, last = -1;
        double upto = 0.0;
        for (int c = 0; c < C; ++c) {
            const double s = C > 1 ? vtk_cluster_read(&sh.cta_sum[(turn - 1) & 1], c) : sh.cta_sum[(turn - 1) & 1];
            upto += s;
            if (s > 0.0) last = c;
            if (owner < 0 && upto > drawn) owner = c;
        }
        if (owner < 0) owner = last;
        if (owner == rank) {
            // which warp's run, which eighth of it, which element
            auto pick = [&](const double (&sums)[VD_WARPS], double &from) {
                int w = -1, with_mass = -1;
                double at_w = from, upto = from, at_mass = from;
                for (int i = 0; i < VD_WARPS; ++i) {
                    if (sums[i] > 0.0) { with_mass = i; at_mass = upto; }
                    if (w < 0 && upto + sums[i] > drawn) { w = i; at_w = upto; }
                    upto += sums[i];
                }
                from = w < 0 ? at_mass : at_w;
                return w < 0 ? with_mass : w;
            };
            double from = before;
            const int64_t r0 = (int64_t)(rank * VD_WARPS + pick(sh.warp_sum, from)) * per;
            const int piece = ((per + VD_WARPS - 1) / VD_WARPS + STEP - 1) / STEP * STEP;
            auto edge = [&](int w) {                         // of the pieces of the run
                const int64_t x = (int64_t)w * piece < per ? r0 + (int64_t)w * piece : r0 + per;
                return x < a.vocab ? (int)x : a.vocab;
            };
            const double sum = row.sum(edge(warp), edge(warp + 1), clean);
            if (lane == 0) sh.again[warp] = sum;
            __syncthreads();
            const int w = pick(sh.again, from);
            if (warp == w) {
                const int token = row.find(edge(w), edge(w + 1), from, drawn);
                if (lane == 0) {
                    a.next_tokens[r] = token;
                    if (!a.out_tokens.null()) a.out_tokens[d.d0 + r + at] = token;
                }
            }
        } else if (owner < 0 && rank == 0 && tid == 0) {
            a.next_tokens[r] = -1;
            if (!a.out_tokens.null()) a.out_tokens[d.d0 + r + at] = -1;
        }
        __syncthreads();                                     // the sums are the next request's
    }
    if (clipped) atomicOr(a.flags, (uint32_t)VTOKEN_FLAG_CAPACITY);
    if (C > 1) vtk_cluster_sync();                           // (a neighbour may still be reading here)
}

template <typename P>
int launch(vtoken_ctx *ctx, const VerifyArgs &a, bool vec, cudaStream_t st)
{
    // CTAs of a request: two for each SM in all, a CTA not below 2048 elements.  (Many requests: a cluster whose CTAs do not start
    // together waits for the last, 200 requests of 128 256 take 91 us with eight CTAs each and 44 with two.)  The number of requests is on the
    // device, so the context's capacity stands for it: one request of 128 256 takes 11.5 us in a context for up to 64, 33 in one for 512.
    int size = 1;
    while (size < 8 && a.vocab > size * VD_NT * 8 && (int64_t)a.max_requests * size < 2 * ctx->num_sms) size *= 2;
    const int64_t most = (int64_t)ctx->num_sms * 8 / size;
    const int rows = a.max_requests < most ? a.max_requests : (int)most, clusters = rows + (a.num_victims != nullptr ? 1 : 0);
    VTK_CUDA(ctx, vec ? vtk_launch_clusters(ctx, verify_kernel<P, true>, size, dim3(clusters * size), dim3(VD_NT), 0, st, a, rows)
                      : vtk_launch_clusters(ctx, verify_kernel<P, false>, size, dim3(clusters * size), dim3(VD_NT), 0, st, a, rows));
    VTK_CUDA(ctx, cudaGetLastError());
    return VTOKEN_OK;
}

}  // namespace

extern "C" int vtoken_verify_drafts(vtoken_ctx *ctx, const vtoken_verify_in *in, void *cuda_stream)
{
    if (!ctx || !in || !in->num_requests || !in->target_probs || !in->sample_random || !in->accepted || !in->next_tokens) return VTOKEN_EINVAL;
    if (in->max_drafts < 0 || in->vocab < 1 || in->vocab > (1 << 30)) return VTOKEN_EINVAL;
    if (in->max_drafts > 0 && (!in->draft_offsets || !in->draft_tokens || !in->accept_random)) return VTOKEN_EINVAL;
    if (in->prob_type != VTOKEN_PROB_BF16 && in->prob_type != VTOKEN_PROB_FP16 && in->prob_type != VTOKEN_PROB_F32) return VTOKEN_EINVAL;
    const int64_t ts = in->target_stride ? in->target_stride : in->vocab, ds = in->draft_stride ? in->draft_stride : in->vocab;
    if (ts < in->vocab || ds < in->vocab) return VTOKEN_EINVAL;
    const int size = in->prob_type == VTOKEN_PROB_F32 ? 4 : 2;
    if (((uintptr_t)in->target_probs | (uintptr_t)in->draft_probs) % size) return VTOKEN_EINVAL;
    const bool victims = in->victim_req || in->victim_tok || in->num_victims;
    if (in->max_victims < 0) return VTOKEN_EINVAL;
    if (victims && (!in->num_victims || !in->first_id || (in->max_victims > 0 && (!in->victim_req || !in->victim_tok)))) return VTOKEN_EINVAL;
    VerifyArgs a;
    const int64_t D = in->max_drafts, Q = ctx->cfg.max_requests;
    a.num_requests = in->num_requests;
    a.draft_offsets = VTK_ARR(ctx, in->draft_offsets, Q + 1);
    a.draft_tokens = VTK_ARR(ctx, in->draft_tokens, D);
    a.first_id = VTK_ARR(ctx, in->first_id, Q);
    a.target = in->target_probs;
    a.draft = in->draft_probs;
    a.target_stride = ts;
    a.draft_stride = ds;
    a.accept_random = VTK_ARR(ctx, in->accept_random, D);
    a.sample_random = VTK_ARR(ctx, in->sample_random, Q);
    a.accepted = VTK_ARR(ctx, in->accepted, Q);
    a.next_tokens = VTK_ARR(ctx, in->next_tokens, Q);
    a.out_tokens = VTK_ARR(ctx, in->out_tokens, D + Q);
    a.victim_req = VTK_ARR(ctx, in->victim_req, in->max_victims);
    a.victim_tok = VTK_ARR(ctx, in->victim_tok, in->max_victims);
    a.num_victims = victims ? in->num_victims : nullptr;
    a.vocab = in->vocab;
    a.max_drafts = in->max_drafts;
    a.max_requests = ctx->cfg.max_requests;
    a.max_victims = in->max_victims;
    a.flags = &ctx->rt_counts->error_flags;
    // rows that start on 16 bytes are read 16 bytes at a time
    const bool vec = (((uintptr_t)a.target | (uintptr_t)a.draft) & 15) == 0 && (ts * size) % 16 == 0 && (a.draft == nullptr || (ds * size) % 16 == 0);
    cudaStream_t st = (cudaStream_t)cuda_stream;
    switch (in->prob_type) {
        case VTOKEN_PROB_F32: return launch<F32>(ctx, a, vec, st);
        case VTOKEN_PROB_BF16: return launch<Half<VtkBf16>>(ctx, a, vec, st);
        default: return launch<Half<VtkFp16>>(ctx, a, vec, st);
    }
}
