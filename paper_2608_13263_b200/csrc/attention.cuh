// What the attention kernels share: arguments, the request's share of the slot cache, matrix instructions,
// rows of the pools in registers, and the exact recomputation of a row that a masked NaN reached.
#pragma once
#include <atomic>

#include "heads.cuh"

// A shared prefix as the planning kernel of attention_shared.cu leaves it in the workspace.
struct VtkPrefixGroup {
    int32_t q0, q1;                      // query rows of the group: those of consecutive requests
    int32_t base, len;                   // the prefix: cache entries [base, base + len)
    int32_t splits, tiles;               // parts that its tiles are cut into, tiles of a part
    int32_t first, end;                  // requests
    int64_t items;                       // items of the groups in front
    int64_t rows;                        // rows (query tokens times query heads) of several parts in the groups in front
};
struct VtkPrefixPlan {
    int64_t items;                       // of all groups: (256 query rows, part, key head)
    int64_t rows;                        // rows of several parts
    int32_t groups;
    int32_t query_tokens;                // of the call: parts are [splits][query_tokens][query heads]
};

struct VtkAttnArgs {
    const int32_t *num_requests;
    vtk_arr<const int32_t> q_offsets, positions, tt_offsets, cache_slots, cache_ids, cache_len;
    const uint16_t *q;
    uint16_t *out;
    float *lse;
    const uint8_t *k_rows, *v_rows;      // this layer's slabs
    int64_t q_stride, out_stride, row_bytes, slots_per_layer, max_tokens;
    int32_t max_requests, max_query_tokens, hq, hkv, group;
    float inv_group;
    int32_t window, sinks;
    float scale_log2;                    // sm_scale * log2(e) * 2^k_exponent
    float v_mul;                         // 2^v_exponent
    uint32_t *flags;
    uint32_t *counters;                  // workspace: arrivals of split rows, zero between calls
    float *part;                         // workspace: partial rows
    int32_t row_limit;                   // requests of more query rows (tokens times group) belong to attention_prompt.cu
    // shared prefixes only
    const VtkPrefixPlan *plan;
    const VtkPrefixGroup *groups;
    const int32_t *shared;               // per request: entries of its prefix
    float2 *pre_ml;                      // per part and row: running maximum (exponents of two) and sum of the prefix, joined in part 0 ...
    float *pre_o;                        // ... and the sum of its weighted values
};

// Ids are not negative.  A query at p sees the ids in (vtk_floor(p), p] and those below `sinks`.
__device__ __forceinline__ int vtk_floor(int p, int window) { return window == 0 || p < window ? -1 : p - window; }
__device__ __forceinline__ bool vtk_sees(int id, int p, int floor, int sinks) { return id <= p && (id > floor || id < sinks); }

// What a request's queries read of its slot cache: entries [0, n_sink) and [lo, lo + n - n_sink), numbered
// 0 .. n - 1 in that order ("virtual" indexes).  Behind a shared prefix the first of the two is [first, first + n_sink).
struct VtkRequest {
    int pmax, floor;                     // no query sees an id above pmax, nor one up to floor that is no sink
    int64_t base;                        // first cache entry
    int lo, n_sink, n, first;
    __device__ __forceinline__ int index(int v) const { return v < n_sink ? first + v : lo + (v - n_sink); }
    __device__ __forceinline__ int64_t entry(int v) const { return base + index(v); }
    // without the entries in front of `prefix`
    __device__ __forceinline__ void behind(int prefix)
    {
        const int hi = lo + (n - n_sink);
        first = n_sink > prefix ? prefix : 0;
        n_sink = n_sink > prefix ? n_sink - prefix : 0;
        lo = lo > prefix ? lo : prefix;
        n = n_sink + (hi > lo ? hi - lo : 0);
    }
};

__device__ __forceinline__ int vtk_clamp_offset(int x, int cap) { return x < 0 ? 0 : (x > cap ? cap : x); }

// the last id of [base, base + len): -1 when there is none
__device__ __forceinline__ int vtk_last_id(const VtkAttnArgs &a, int64_t base, int len)
{
    return len == 0 ? -1 : (a.cache_ids.null() ? len - 1 : a.cache_ids[base + len - 1]);
}

// entries of the ascending ids [base, base + len) that are <= p
__device__ inline int vtk_ids_up_to(const VtkAttnArgs &a, int64_t base, int len, int last, int p)
{
    if (last <= p) return len;
    if (p < 0) return 0;
    if (a.cache_ids.null()) return p + 1 < len ? p + 1 : len;
    int lo = 0, hi = len - 1;            // ids[hi] > p
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (a.cache_ids[base + mid] <= p) lo = mid + 1; else hi = mid;
    }
    return lo;
}

// Ids are strictly ascending from 0 or above, so ids[i] >= i: entry i >= sinks cannot be a sink, and of the
// entries with ids <= pmax at most (pmax - pmin) + window have an id > pmin - window.
__device__ inline VtkRequest vtk_request_span(const VtkAttnArgs &a, int64_t base, int len, int last, int pmin, int pmax)
{
    VtkRequest q;
    q.first = 0;
    q.pmax = pmax;
    q.floor = vtk_floor(pmin, a.window);
    q.base = base;
    const int hi = vtk_ids_up_to(a, base, len, last, pmax);
    int64_t lo = 0;
    if (a.window > 0) lo = (int64_t)hi - ((int64_t)pmax - pmin) - a.window;
    q.lo = lo > 0 ? (int)lo : 0;
    q.n_sink = a.sinks < q.lo ? a.sinks : q.lo;
    q.n = q.n_sink + (hi - q.lo);
    return q;
}

// rows and cache range of request r, clipped to what exists
__device__ inline void vtk_request_rows(const VtkAttnArgs &a, int r, int &q0, int &qn, int64_t &base, int &len, bool &clipped)
{
    const int a0 = a.q_offsets[r], a1 = a.q_offsets[r + 1];
    const int64_t t0 = a.tt_offsets[r], t1 = a.tt_offsets[r + 1];
    const int want = a.cache_len[r];
    q0 = vtk_clamp_offset(a0, a.max_query_tokens);
    const int q1 = vtk_clamp_offset(a1, a.max_query_tokens);
    qn = q1 > q0 ? q1 - q0 : 0;
    base = t0 < 0 ? 0 : (t0 > a.max_tokens ? a.max_tokens : t0);
    const int64_t end = t1 < base ? base : (t1 > a.max_tokens ? a.max_tokens : t1);
    len = want < 0 ? 0 : (want > end - base ? (int)(end - base) : want);
    clipped = a0 != q0 || a1 != q1 || q1 < q0 || t0 != base || t1 != end || want != len;
}

// ---- matrix instructions: 16 x 8 += 16 x 16 by 16 x 8, 32-bit accumulators ----------------------
template <typename M>
__device__ __forceinline__ void vtk_mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1);
template <>
__device__ __forceinline__ void vtk_mma<VtkBf16>(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void vtk_mma<VtkFp16>(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Softmax weights that go to half precision carry 2^7: next to a running maximum that may lag by 2^8 they end at 2^15, and what
// half precision rounds to zero is below 2^-32 of the largest, so n such tokens take at most n * 2^-32 of the largest |v| from an
// output whose sum of weights, in 32 bits, counts them (without the factor n * 2^-25: 2^-10 at 32 768 tokens).
template <typename M> __host__ __device__ constexpr float vtk_lift() { return M::kind == VTOKEN_KV_FP16 ? 7.f : 0.f; }

__device__ __forceinline__ float vtk_exp2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ uint4 vtk_ldg16(const void *p)
{
    uint4 w;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w.x), "=r"(w.y), "=r"(w.z), "=r"(w.w) : "l"(p));
    return w;
}

// ---- barriers in shared memory; every wait ends ----------------------------------------------------
__device__ __forceinline__ uint32_t vtk_smem_u32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void vtk_mbar_init(uint64_t *bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(vtk_smem_u32(bar)), "r"(count));
}
__device__ __forceinline__ void vtk_mbar_arrive(uint64_t *bar, uint32_t count = 1)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0], %1;" ::"r"(vtk_smem_u32(bar)), "r"(count) : "memory");
}
__device__ __forceinline__ bool vtk_mbar_try(uint64_t *bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}\n"
                 : "=r"(ok) : "r"(vtk_smem_u32(bar)), "r"(parity) : "memory");
    return ok != 0;
}
// without waiting at all (try_wait may sleep for a while)
__device__ __forceinline__ bool vtk_mbar_test(uint64_t *bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{\n .reg .pred p;\n mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}\n"
                 : "=r"(ok) : "r"(vtk_smem_u32(bar)), "r"(parity) : "memory");
    return ok != 0;
}
__device__ __forceinline__ uint64_t vtk_global_ns()
{
    uint64_t t;
    asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
    return t;
}
// (inlined: a call would keep the compiler from giving the roles of a kernel register counts of their own)
// false when the phase did not complete within the limit (`mark`, not zero, is left in `abort`), or another role has given up
static __device__ __forceinline__ bool vtk_mbar_wait_long(uint64_t *bar, uint32_t parity, uint64_t limit_ns, volatile int *abort, int mark)
{
    for (int i = 0; i < 2048; ++i)          // (the clock is far away: a wait that is over soon does not look at it)
        if (vtk_mbar_try(bar, parity)) return true;
    const uint64_t t0 = vtk_global_ns();
    for (;;) {
        for (int i = 0; i < 64; ++i)
            if (vtk_mbar_try(bar, parity)) return true;
        if (*abort) return false;
        if (vtk_global_ns() - t0 > limit_ns) { *abort = mark; return false; }
    }
}
__device__ __forceinline__ bool vtk_mbar_wait(uint64_t *bar, uint32_t parity, uint64_t limit_ns, int *abort, int mark)
{
    return vtk_mbar_try(bar, parity) || vtk_mbar_try(bar, parity) || vtk_mbar_wait_long(bar, parity, limit_ns, abort, mark);
}

// ---- one head of one pool row, `N` consecutive values from `d` on, as 32-bit values -------------
// (the value without 2^exponent)
template <int D, bool FP4, typename Act, int N>
__device__ __forceinline__ void vtk_row_values(const uint8_t *row, int hkv, int head, int d, float (&x)[N])
{
    if (!FP4) {
        const uint32_t *p = reinterpret_cast<const uint32_t *>(row + ((int64_t)head * D + d) * 2);
#pragma unroll
        for (int j = 0; j < N / 2; ++j) {
            const float2 v = Act::unpack(p[j]);
            x[2 * j] = v.x;
            x[2 * j + 1] = v.y;
        }
    } else {
        static_assert(N == 2 || N == 4, "one or two bytes of codes");
        const uint32_t two = *reinterpret_cast<const uint16_t *>(row + head * (D / 2) + (d / 4) * 2);
        const uint32_t codes = N == 4 ? two : two >> (4 * (d & 2));
        const uint32_t s2 = vtk_scales_to_half2(row[hkv * (D / 2) + head * (D / 16) + d / 16]);
        const float s = __half2float(__ushort_as_half((uint16_t)(s2 & 0xffffu)));
#pragma unroll
        for (int j = 0; j < N / 2; ++j) {
            const float2 v = VtkFp16::unpack(vtk_codes_to_half2(codes >> (8 * j)));
            x[2 * j] = v.x * s;
            x[2 * j + 1] = v.y * s;
        }
    }
}

// The matrix kernels multiply a masked token's value by a zero weight, so a NaN or an infinity there would reach rows that do not
// see the token.  (A masked key does not: its score is replaced.)  Rows whose result is not finite are looked at again, by a warp each.

// Does a token that the row at `pos` does not see, but that was fetched because another row does -- an id in (pos, pmax] or in
// (floor, vtk_floor(pos)] -- have a value that is not finite?  If not, the row is what the tokens it sees make it: a cache with NaN
// in it costs a look at these few tokens a row, and no row is worked on again for a value that it sees.
template <int D, bool FP4, typename Act>
__device__ __forceinline__ bool vtk_hidden_value(const VtkAttnArgs &a, int head, int pos, const VtkRequest &s, int len)
{
    constexpr int N = D / 32, AT_ONCE = 8;
    const int64_t base = s.base;
    const int last = vtk_last_id(a, base, len), kv = head / a.group;
    for (int part = 0; part < 2; ++part) {
        const int lo = vtk_ids_up_to(a, base, len, last, part ? s.floor : pos);
        const int hi = vtk_ids_up_to(a, base, len, last, part ? vtk_floor(pos, a.window) : s.pmax);
        for (int i = lo; i < hi; i += AT_ONCE) {
            bool odd = false;
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                const int64_t slot = i + u < hi ? a.cache_slots[base + i + u] : -1;
                if (slot < 0 || slot >= a.slots_per_layer) continue;
                float v[N];
                vtk_row_values<D, FP4, Act, N>(a.v_rows + slot * a.row_bytes, a.hkv, kv, vtk_lane() * N, v);
#pragma unroll
                for (int j = 0; j < N; ++j) odd |= !(fabsf(v[j]) < INFINITY);
            }
            if (__any_sync(0xffffffffu, odd)) return true;
        }
    }
    return false;
}

// One query row by one warp, token by token: the definition, of the tokens that the row sees alone.  Values come out as the lane's
// D / 32 consecutive dimensions; false when the row stands as it was stored, since no value that it does not see is at fault, or all
// in it that is not finite has turned out to be NaN.
template <int D, bool FP4, typename Act>
__device__ __noinline__ bool vtk_row_again(const VtkAttnArgs &a, int64_t q_row, int head, int pos, const VtkRequest &request, int len,
                                           float (&o)[D / 32], float &m, float &l)
{
    if (!vtk_hidden_value<D, FP4, Act>(a, head, pos, request, len)) return false;
    const int64_t base = request.base;
    constexpr int N = D / 32;
    const int lane = vtk_lane(), kv = head / a.group;
    float q[N];
    const uint32_t *qp = reinterpret_cast<const uint32_t *>(a.q + q_row * a.q_stride + (int64_t)head * D + lane * N);
#pragma unroll
    for (int j = 0; j < N / 2; ++j) {
        const float2 v = Act::unpack(qp[j]);
        q[2 * j] = v.x;
        q[2 * j + 1] = v.y;
    }
    m = -INFINITY;
    l = 0.f;
    const int floor = vtk_floor(pos, a.window);
#pragma unroll
    for (int j = 0; j < N; ++j) o[j] = 0.f;
    bool open[N];                        // dimensions in question
    const uint32_t *stored = reinterpret_cast<const uint32_t *>(a.out + q_row * a.out_stride + (int64_t)head * D + lane * N);
#pragma unroll
    for (int j = 0; j < N / 2; ++j) {
        const float2 v = Act::unpack(__ldcg(stored + j));
        open[2 * j] = !(fabsf(v.x) < INFINITY);
        open[2 * j + 1] = !(fabsf(v.y) < INFINITY);
    }
    for (int i = 0; i < len; ++i) {
        if (i % 32 == 31) {
            bool settled = true;
#pragma unroll
            for (int j = 0; j < N; ++j) settled &= !open[j] || o[j] != o[j];
            if (__all_sync(0xffffffffu, settled)) return false;
        }
        const int id = a.cache_ids.null() ? i : a.cache_ids[base + i];
        const int64_t slot = a.cache_slots[base + i];
        if (slot < 0 || slot >= a.slots_per_layer || !vtk_sees(id, pos, floor, a.sinks)) continue;
        float k[N], v[N];
        vtk_row_values<D, FP4, Act, N>(a.k_rows + slot * a.row_bytes, a.hkv, kv, lane * N, k);
        vtk_row_values<D, FP4, Act, N>(a.v_rows + slot * a.row_bytes, a.hkv, kv, lane * N, v);
        float s = 0.f;
#pragma unroll
        for (int j = 0; j < N; ++j) s += q[j] * k[j];
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
        s *= a.scale_log2;
        const float m2 = fmaxf(m, s), keep = m == m2 ? 1.f : (m == -INFINITY ? 0.f : exp2f(m - m2));
        const float p = s == -INFINITY ? 0.f : exp2f(s - m2);
        l = l * keep + p;
#pragma unroll
        for (int j = 0; j < N; ++j) o[j] = o[j] * keep + p * v[j];
        m = m2;
    }
    return true;
}

// the row's output and lse: the lane's N consecutive dimensions
template <int D, typename Act>
__device__ __forceinline__ void vtk_store_row(const VtkAttnArgs &a, int64_t q_row, int head, float (&o)[D / 32], float m, float l)
{
    constexpr int N = D / 32;
    const int lane = vtk_lane();
    const float r = l == 0.f ? 0.f : a.v_mul / l;
    uint32_t *p = reinterpret_cast<uint32_t *>(a.out + q_row * a.out_stride + (int64_t)head * D + lane * N);
    uint32_t w[N / 2];
#pragma unroll
    for (int j = 0; j < N / 2; ++j) w[j] = Act::pack(o[2 * j] * r, o[2 * j + 1] * r);
    if (N == 4) *reinterpret_cast<uint2 *>(p) = make_uint2(w[0], w[N / 2 - 1]);
    else p[0] = w[0];
    if (a.lse != nullptr && lane == 0) a.lse[q_row * a.hq + head] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
}

// host: large shared memory, asked for when a kernel first runs on a device (the call costs as much as a launch)
inline cudaError_t vtk_allow_smem(const vtoken_ctx *ctx, std::atomic<int> &allowed, const void *kernel, int bytes)
{
    if (allowed.load(std::memory_order_relaxed) == ctx->device) return cudaSuccess;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess) allowed.store(ctx->device, std::memory_order_relaxed);
    return e;
}

// host: 2^e
inline float vtk_two_to(int e)
{
    float x = 1.f;
    for (; e > 0; --e) x *= 2.f;
    for (; e < 0; ++e) x *= 0.5f;
    return x;
}

// host: the factor of the scores as an exponent of two, with that of the keys; false when it leaves 32 bits
inline bool vtk_score_scale(const vtoken_heads *heads, float sm_scale, float &scale)
{
    scale = sm_scale * 1.4426950408889634f * vtk_two_to(heads->k_exponent);
    return sm_scale > -1e30f && sm_scale < 1e30f && scale > -INFINITY && scale < INFINITY;
}

// host: the beginning of every workspace, zero between calls whichever they are: two tickets of the kernels for many query rows, then
// the arrivals that attention.cu counts, one for each head of a share (at most 16 a CTA).  What a call writes besides lies behind it.
constexpr int VTK_TICKET_BYTES = 16, VTK_CTA_SHARES = 16;
inline int64_t vtk_workspace_zeros(const vtoken_ctx *ctx) { return VTK_TICKET_BYTES + (int64_t)ctx->num_sms * VTK_CTA_SHARES * 4; }

// host: launchers of attention.cu and of attention_prompt.cu
int vtk_launch_attention_rows(vtoken_ctx *ctx, const vtoken_heads *heads, VtkAttnArgs a, int32_t max_query_len, bool shared, cudaStream_t st);
int vtk_launch_attention_prompt(vtoken_ctx *ctx, const vtoken_heads *heads, const VtkAttnArgs &a, uint32_t *tickets, bool prefix, cudaStream_t st);
int64_t vtk_attention_rows_workspace(const vtoken_ctx *ctx, const vtoken_heads *heads, VtkAttnArgs *a);
constexpr int VTK_ROW_LIMIT = 32;        // query rows (tokens times group) of a request up to which attention.cu works on it
// host: checks of a call and the kernels' arguments; VTOKEN_OK with max_query_tokens 0: nothing to do
int vtk_attention_args(vtoken_ctx *ctx, const vtoken_heads *heads, int32_t layer, const vtoken_attention_in *in, int64_t workspace_bytes, VtkAttnArgs &a);
