// Attention of requests whose caches begin with the same entries.
//
// Four kernels.  One CTA plans: the shortest prefix of each group, and the parts that the prefixes are cut into.  The prompt
// kernel takes the query rows of a whole group as if they were one request's -- they follow one another in q -- over the entries
// of the group's first request, so a prefix row is read once for up to 256 query rows, and leaves running maximum, sum and weighted
// values of each part; a warp for each row joins its parts.  The kernel for few rows goes on from there over the request's own entries: the state that a softmax over
// part of the tokens leaves is all that the other part needs, so nothing is rounded in between and there is nothing to join behind.
// Requests of many rows are left to the prompt kernel, which is bound by the products and not by what it reads.
//
// 64 requests behind 8192 tokens, 32 heads over 8: 113 us, of which own tokens (160 MB) take 50, the prefix 38 (10 until its first scores,
// 2.6 for each 256 rows and 128 tokens), planning and joining 15; without sharing the prefix would be 2.1 GB to read.
#include "attention.cuh"

namespace {

constexpr int AS_NT = 1024, AS_TILE = 128, AS_PAIR = 2 * AS_TILE, AS_MIN_TILES = 2, AS_GROUPS = 1024, AS_SIZED = 64, AS_SIZES = 256;

struct Args {
    VtkAttnArgs a;
    const int32_t *num_groups;
    vtk_arr<const int32_t> group_offsets, shared_len;
    VtkPrefixPlan *plan;
    VtkPrefixGroup *groups;
    int32_t *shared;
    int32_t *len, *readers;              // per group, where there are more than AS_GROUPS
    int64_t rows;                        // rows of the parts
    int32_t ctas;                        // of the prompt kernel
};

// (a 64-bit division is a subroutine of several hundred cycles)
__device__ __forceinline__ int64_t divide(int64_t x, int64_t y)
{
    return ((uint64_t)(x | y) >> 32) == 0 ? (int64_t)((uint32_t)x / (uint32_t)y) : x / y;
}

// warps: those that have something
__device__ __forceinline__ int64_t block_sum(int64_t x, int64_t *warp_sum, int warps)
{
    const int warp = threadIdx.x >> 5;
    if (warp < warps) {
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
        if (vtk_lane() == 0) warp_sum[warp] = x;
    }
    __syncthreads();
    int64_t sum = 0;
    for (int w = 0; w < warps; ++w) sum += warp_sum[w];
    __syncthreads();
    return sum;
}

__global__ void __launch_bounds__(AS_NT) shared_plan_kernel(const __grid_constant__ Args s)
{
    const VtkAttnArgs &a = s.a;
    __shared__ int64_t warp_sum[2][AS_NT / 32];
    __shared__ int edge[AS_GROUPS + 1], few_len[AS_GROUPS], few_readers[AS_GROUPS], few_units[AS_SIZED], group_tiles[AS_SIZED];
    vtk_release_successor();
    vtk_wait_for_predecessor();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int R = *a.num_requests, G = *s.num_groups;
    bool clipped = R < 0 || R > a.max_requests || G < 0 || G > a.max_requests;
    R = R < 0 ? 0 : (R > a.max_requests ? a.max_requests : R);
    G = G < 0 ? 0 : (G > a.max_requests ? a.max_requests : G);
    const bool few = G <= AS_GROUPS;
    int *group_len = few ? few_len : s.len, *group_readers = few ? few_readers : s.readers;
    for (int g = tid; g <= G; g += AS_NT) {
        if (few) edge[g] = s.group_offsets[g];
        if (g < G) {
            group_len[g] = INT32_MAX;
            group_readers[g] = 0;
        }
    }
    auto now = [](const int *p) { return *(const volatile int *)p; };      // (atomics have changed it, in shared or in global memory)
    auto offset = [&](int g) { return few ? edge[g] : s.group_offsets[g]; };
    __syncthreads();
    auto group_of = [&](int r) {                             // offset(lo) <= r < offset(hi)
        if (G == 0 || offset(0) > r || offset(G) <= r) return -1;
        int lo = 0, hi = G;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (offset(mid) <= r) lo = mid; else hi = mid;
        }
        return lo;
    };
    int first_group = -1;                                    // of the thread's first request, and its first group
    VtkPrefixGroup mine;
    mine.len = 0;
    for (int r = tid; r < R; r += AS_NT) {
        const int g = group_of(r);
        if (r == tid) first_group = g;
        if (g >= 0) {
            int q0, qn, len;
            int64_t base;
            bool c;
            const int want = s.shared_len[r];
            vtk_request_rows(a, r, q0, qn, base, len, c);
            atomicMin(&group_len[g], want < 0 ? 0 : (want > len ? len : want));
            if (qn > 0 && (int64_t)qn * a.group <= a.row_limit) atomicAdd(&group_readers[g], 1);
        }
        if (r != tid) s.shared[r] = g;
    }
    const int tokens = R > 0 ? vtk_clamp_offset(a.q_offsets[R], a.max_query_tokens) : 0;
    __syncthreads();
    // tiles in all, for parts of a size that gives every CTA one
    int64_t work = 0;
    for (int g = tid; g < G; g += AS_NT) {
        VtkPrefixGroup x;
        const int r0 = offset(g), r1 = offset(g + 1);
        x.first = r0 < 0 ? 0 : (r0 > R ? R : r0);
        x.end = r1 < x.first ? x.first : (r1 > R ? R : r1);
        clipped |= x.first != r0 || x.end != r1;
        x.len = now(&group_len[g]);
        x.q0 = vtk_clamp_offset(a.q_offsets[x.first], a.max_query_tokens);
        x.q1 = vtk_clamp_offset(a.q_offsets[x.end], a.max_query_tokens);
        const int64_t base = x.first < x.end ? a.tt_offsets[x.first] : 0;
        x.base = base < 0 ? 0 : (base > a.max_tokens ? (int)a.max_tokens : (int)base);
        // (one reader: nothing to gain)
        if (now(&group_readers[g]) < 2 || x.end <= x.first || x.q1 <= x.q0 || x.len == INT32_MAX) x.len = 0;
        group_len[g] = x.len;
        x.items = (((int64_t)(x.q1 - x.q0) * a.group + AS_PAIR - 1) >> 8) * a.hkv;
        x.tiles = (x.len + AS_TILE - 1) / AS_TILE;
        x.splits = 0;
        x.rows = 0;
        work += x.len > 0 ? x.items * x.tiles : 0;
        if (G <= AS_SIZED) {
            few_units[g] = x.len > 0 ? (int)x.items : 0;
            group_tiles[g] = x.tiles;
        }
        if (g == tid) mine = x;
        s.groups[g] = x;
    }
    const int warps = G < AS_NT ? (G + 31) / 32 : AS_NT / 32;               // that have groups
    work = block_sum(work, warp_sum[0], warps);
    const int64_t most = tokens > 0 ? divide(s.rows, (int64_t)tokens * a.hq) : 1;    // parts that there is room for
    // Tiles of a part.  A part costs about five tiles to start, and a CTA that gets one part more than the others is waited for: of sizes
    // upwards of one that gives every CTA its share the one with the fewest (rounds of parts) x (size + 5).
    int64_t size = divide(work + s.ctas - 1, s.ctas);
    size = size < AS_MIN_TILES ? AS_MIN_TILES : size;
    if (G <= AS_SIZED) {
        int64_t cost = INT64_MAX;
        const int64_t candidate = size / 4 + 1 + tid;
        if (tid < AS_SIZES) {
            if (candidate >= AS_MIN_TILES && candidate < (1 << 22)) {
                const float inverse = 1.f / (float)candidate;
                int64_t items = 0;
#pragma unroll 4
                for (int g = 0; g < G; ++g) items += (int64_t)few_units[g] * (int)(((float)group_tiles[g] - 0.5f) * inverse + 1.f);     // (parts: a quotient rounded up)
                cost = (divide(items + s.ctas - 1, s.ctas) * (candidate + 5)) << 24 | candidate;
            }
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) {
                const int64_t o = __shfl_xor_sync(0xffffffffu, cost, d);
                cost = o < cost ? o : cost;
            }
            if (lane == 0) warp_sum[0][warp] = cost;
        }
        __syncthreads();
        for (int w = 0; w < AS_SIZES / 32; ++w) cost = warp_sum[0][w] < cost ? warp_sum[0][w] : cost;
        __syncthreads();
        if (cost != INT64_MAX) size = cost & 0xffffff;
    }
    int64_t items_before = 0, rows_before = 0;
    for (int g0 = 0; g0 < G; g0 += AS_NT) {
        const int g = g0 + tid;
        int64_t items = 0, rows = 0;
        int tiles = 0, splits = 0;
        VtkPrefixGroup x = mine;
        if (g0 > 0 && g < G) x = s.groups[g];
        if (g < G && x.len > 0) {
            int64_t each = divide(x.tiles + most - 1, most);
            each = each < size ? size : each;
            splits = (int)divide(x.tiles + each - 1, each);
            tiles = (x.tiles + splits - 1) / splits;
            items = x.items * splits;
            rows = splits > 1 ? (int64_t)(x.q1 - x.q0) * a.hq : 0;
        }
        int64_t incl = 0, incl_rows = 0;
        if (warp < warps) {
            incl = vtk_warp_incl_scan(items);
            incl_rows = vtk_warp_incl_scan(rows);
            if (lane == 31) { warp_sum[0][warp] = incl; warp_sum[1][warp] = incl_rows; }
        }
        __syncthreads();
        int64_t in_front = items_before, rows_in_front = rows_before;
        for (int w = 0; w < warps; ++w) {
            if (w < warp) { in_front += warp_sum[0][w]; rows_in_front += warp_sum[1][w]; }
            items_before += warp_sum[0][w];
            rows_before += warp_sum[1][w];
        }
        if (g < G) {
            s.groups[g].items = in_front + incl - items;
            s.groups[g].rows = rows_in_front + incl_rows - rows;
            s.groups[g].tiles = tiles;
            s.groups[g].splits = splits;
        }
        __syncthreads();
    }
    for (int r = tid; r < R; r += AS_NT) {
        const int g = r == tid ? first_group : s.shared[r];
        s.shared[r] = g < 0 ? 0 : now(&group_len[g]);
    }
    if (tid == 0) {
        s.plan->items = items_before;
        s.plan->rows = rows_before;
        s.plan->groups = G;
        s.plan->query_tokens = tokens;
    }
    if (clipped) atomicOr(a.flags, (uint32_t)VTOKEN_FLAG_CAPACITY);
}

// The parts of a row, in their order, into part 0: a warp a row.
template <int D>
__global__ void __launch_bounds__(256) shared_join_kernel(const __grid_constant__ VtkAttnArgs a)
{
    constexpr int N = D / 32;
    vtk_release_successor();
    vtk_wait_for_predecessor();
    const int lane = vtk_lane();
    const int64_t stride = (int64_t)a.plan->query_tokens * a.hq, all = a.plan->rows, warps = (int64_t)gridDim.x * 8;
    const int G = a.plan->groups;
    for (int64_t row = blockIdx.x * 8 + (threadIdx.x >> 5); row < all; row += warps) {
        int lo = 0, hi = G;                  // the last group with rows up to this one (groups without rows have none in front of the next)
        while (hi - lo > 1) {
            const int step = (hi - lo + 31) / 32, probe = lo + lane * step;
            const int n = __popc(__ballot_sync(0xffffffffu, probe < hi && a.groups[probe].rows <= row));         // (lane 0's always is)
            const int next_hi = lo + n * step;
            lo += (n - 1) * step;
            if (next_hi < hi) hi = next_hi;
        }
        const int parts = a.groups[lo].splits;
        const int64_t at = (int64_t)a.groups[lo].q0 * a.hq + (row - a.groups[lo].rows);
        float top = -INFINITY, sum = 0.f, o[N];
#pragma unroll
        for (int j = 0; j < N; ++j) o[j] = 0.f;
        const float2 ml0 = lane < parts ? __ldcg(&a.pre_ml[lane * stride + at]) : make_float2(-INFINITY, 0.f);
        top = ml0.x;
        for (int k = 32 + lane; k < parts; k += 32) top = fmaxf(top, __ldcg(&a.pre_ml[k * stride + at]).x);
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
        for (int k0 = 0; k0 < parts; k0 += 32) {
            const float2 ml = k0 == 0 ? ml0 : (k0 + lane < parts ? __ldcg(&a.pre_ml[(k0 + lane) * stride + at]) : make_float2(-INFINITY, 0.f));
            const float mine = ml.x == -INFINITY ? 0.f : vtk_exp2(ml.x - top);
            const int n = parts - k0 < 32 ? parts - k0 : 32;
#pragma unroll 8
            for (int k = 0; k < n; ++k) {
                const float f = __shfl_sync(0xffffffffu, mine, k), l = __shfl_sync(0xffffffffu, ml.y, k);
                sum += f * l;
                const float *src = a.pre_o + ((k0 + k) * stride + at) * D + lane * N;
                float x[N];
                // (a part without a token that the row sees holds no values)
                if (N == 4) *reinterpret_cast<float4 *>(x) = f == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : __ldcg(reinterpret_cast<const float4 *>(src));
                else *reinterpret_cast<float2 *>(x) = f == 0.f ? make_float2(0.f, 0.f) : __ldcg(reinterpret_cast<const float2 *>(src));
#pragma unroll
                for (int j = 0; j < N; ++j) o[j] += f * x[j];
            }
        }
        float *dst = a.pre_o + at * D + lane * N;
        if (N == 4) *reinterpret_cast<float4 *>(dst) = make_float4(o[0], o[1], o[N - 2], o[N - 1]);
        else *reinterpret_cast<float2 *>(dst) = make_float2(o[0], o[1]);
        if (lane == 0) a.pre_ml[at] = make_float2(top, sum);
    }
}

// The workspace behind that of vtoken_attention.  Parts: a row for each query row, and enough for every CTA to have one of 256
// rows when the rows are few.
struct Layout { int64_t rows, plan, groups, shared, len, ml, o, bytes; };
Layout layout_of(const vtoken_ctx *ctx, const vtoken_heads *heads, int64_t max_query_tokens)
{
    Layout l;
    auto up = [](int64_t x) { return (x + 15) / 16 * 16; };
    const int64_t dense = max_query_tokens * heads->num_q_heads, least = (int64_t)ctx->num_sms * 2 * AS_PAIR;
    l.rows = dense > least ? dense : least;
    l.plan = up(vtk_attention_rows_workspace(ctx, heads, nullptr));
    l.groups = l.plan + up(sizeof(VtkPrefixPlan));
    l.shared = l.groups + up(ctx->cfg.max_requests * (int64_t)sizeof(VtkPrefixGroup));
    l.len = l.shared + up(ctx->cfg.max_requests * (int64_t)4);
    l.ml = l.len + up(ctx->cfg.max_requests * (int64_t)8);
    l.o = l.ml + up(l.rows * (int64_t)sizeof(float2));
    l.bytes = l.o + l.rows * heads->head_dim * 4;
    return l;
}

}  // namespace

extern "C" {

int64_t vtoken_attention_shared_workspace_bytes(const vtoken_ctx *ctx, const vtoken_heads *heads, int32_t max_query_tokens)
{
    if (!ctx || vtk_check_heads(ctx, heads, 0) != VTOKEN_OK || max_query_tokens < 0) return VTOKEN_EINVAL;
    return layout_of(ctx, heads, max_query_tokens).bytes;
}

int vtoken_attention_shared(vtoken_ctx *ctx, const vtoken_heads *heads, int32_t layer, const vtoken_attention_in *in,
                            const vtoken_shared_in *shared, void *cuda_stream)
{
    if (!ctx || !heads || !in || !shared || !shared->num_groups || !shared->group_offsets || !shared->shared_len) return VTOKEN_EINVAL;
    if (vtk_check_heads(ctx, heads, layer) != VTOKEN_OK || in->max_query_tokens < 0) return VTOKEN_EINVAL;
    const Layout l = layout_of(ctx, heads, in->max_query_tokens);
    Args s;
    VtkAttnArgs &a = s.a;
    int rc = vtk_attention_args(ctx, heads, layer, in, l.bytes, a);
    if (rc != VTOKEN_OK || in->max_query_tokens == 0) return rc;
    uint8_t *ws = (uint8_t *)in->workspace;
    s.num_groups = shared->num_groups;
    s.group_offsets = VTK_ARR(ctx, shared->group_offsets, ctx->cfg.max_requests + 1);
    s.shared_len = VTK_ARR(ctx, shared->shared_len, ctx->cfg.max_requests);
    s.plan = (VtkPrefixPlan *)(ws + l.plan);
    s.groups = (VtkPrefixGroup *)(ws + l.groups);
    s.shared = (int32_t *)(ws + l.shared);
    s.len = (int32_t *)(ws + l.len);
    s.readers = s.len + ctx->cfg.max_requests;
    s.rows = l.rows;
    s.ctas = ctx->num_sms;
    a.plan = s.plan;
    a.groups = s.groups;
    a.shared = s.shared;
    a.pre_ml = (float2 *)(ws + l.ml);
    a.pre_o = (float *)(ws + l.o);
    cudaStream_t st = (cudaStream_t)cuda_stream;
    const bool prompts = a.row_limit != INT32_MAX;
    VTK_CUDA(ctx, vtk_launch_dependent(ctx, shared_plan_kernel, dim3(1), dim3(AS_NT), 0, st, s));
    VTK_CUDA(ctx, cudaGetLastError());
    rc = vtk_launch_attention_prompt(ctx, heads, a, (uint32_t *)in->workspace, true, st);
    if (rc != VTOKEN_OK) return rc;
    const dim3 grid(ctx->num_sms * 4), block(256);
    VTK_CUDA(ctx, heads->head_dim == 128 ? vtk_launch_dependent(ctx, shared_join_kernel<128>, grid, block, 0, st, a)
                                         : vtk_launch_dependent(ctx, shared_join_kernel<64>, grid, block, 0, st, a));
    VTK_CUDA(ctx, cudaGetLastError());
    rc = vtk_launch_attention_rows(ctx, heads, a, prompts ? 1 : in->max_query_len, true, st);
    return rc == VTOKEN_OK && prompts ? vtk_launch_attention_prompt(ctx, heads, a, (uint32_t *)in->workspace, false, st) : rc;
}

}  // extern "C"
