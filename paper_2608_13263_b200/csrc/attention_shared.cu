// Attention of requests whose caches begin with the same entries.
//
// Three kernels.  One CTA plans: the shortest prefix of each group, and the parts that the prefixes are cut into.  The prompt
// kernel takes the query rows of a whole group as if they were one request's -- they follow one another in q -- over the entries
// of the group's first request, so a prefix row is read once for up to 256 query rows, and leaves running maximum, sum and weighted
// values of each part.  The kernel for few rows goes on from there over the request's own entries: the state that a softmax over
// part of the tokens leaves is all that the other part needs, so nothing is rounded in between and there is nothing to join behind.
// Requests of many rows are left to the prompt kernel, which is bound by the products and not by what it reads.
#include "attention.cuh"

namespace {

constexpr int AS_NT = 1024, AS_TILE = 128, AS_PAIR = 2 * AS_TILE, AS_MIN_TILES = 2;

struct Args {
    VtkAttnArgs a;
    const int32_t *num_groups;
    vtk_arr<const int32_t> group_offsets, shared_len;
    VtkPrefixPlan *plan;
    VtkPrefixGroup *groups;
    int2 *shared;
    int64_t rows;                        // rows of the parts
    int32_t ctas;                        // of the prompt kernel
};

__device__ __forceinline__ int64_t block_sum(int64_t x, int64_t *warp_sum)
{
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
    if (vtk_lane() == 0) warp_sum[threadIdx.x >> 5] = x;
    __syncthreads();
    int64_t sum = 0;
    for (int w = 0; w < AS_NT / 32; ++w) sum += warp_sum[w];
    __syncthreads();
    return sum;
}

__global__ void __launch_bounds__(AS_NT) shared_plan_kernel(const __grid_constant__ Args s)
{
    const VtkAttnArgs &a = s.a;
    __shared__ int64_t warp_sum[AS_NT / 32];
    vtk_release_successor();
    vtk_wait_for_predecessor();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int R = *a.num_requests, G = *s.num_groups;
    bool clipped = R < 0 || R > a.max_requests || G < 0 || G > a.max_requests;
    R = R < 0 ? 0 : (R > a.max_requests ? a.max_requests : R);
    G = G < 0 ? 0 : (G > a.max_requests ? a.max_requests : G);
    for (int g = tid; g < G; g += AS_NT) {
        s.groups[g].len = INT32_MAX;
        s.groups[g].members = 0;
    }
    __syncthreads();
    for (int r = tid; r < R; r += AS_NT) {
        int g = -1;
        if (G > 0 && s.group_offsets[0] <= r) {
            int lo = 0, hi = G;                              // group_offsets[lo] <= r < group_offsets[hi]
            if (r < s.group_offsets[G]) {
                while (hi - lo > 1) {
                    const int mid = (lo + hi) >> 1;
                    if (s.group_offsets[mid] <= r) lo = mid; else hi = mid;
                }
                g = lo;
            }
        }
        if (g >= 0) {
            int q0, qn, len;
            int64_t base;
            bool c;
            vtk_request_rows(a, r, q0, qn, base, len, c);
            int n = s.shared_len[r];
            n = n < 0 ? 0 : (n > len ? len : n);
            atomicMin(&s.groups[g].len, n);
            if (qn > 0 && (int64_t)qn * a.group <= a.row_limit) atomicAdd(&s.groups[g].members, 1);
        }
        s.shared[r] = make_int2(g, 0);
    }
    __syncthreads();
    // tiles in all, for parts of a size that gives every CTA one
    int64_t work = 0;
    for (int g = tid; g < G; g += AS_NT) {
        VtkPrefixGroup x;
        const int r0 = s.group_offsets[g], r1 = s.group_offsets[g + 1];
        x.first = r0 < 0 ? 0 : (r0 > R ? R : r0);
        x.end = r1 < x.first ? x.first : (r1 > R ? R : r1);
        clipped |= x.first != r0 || x.end != r1;
        x.len = __ldcg(&s.groups[g].len);
        x.members = __ldcg(&s.groups[g].members);
        x.q0 = vtk_clamp_offset(a.q_offsets[x.first], a.max_query_tokens);
        x.q1 = vtk_clamp_offset(a.q_offsets[x.end], a.max_query_tokens);
        const int64_t base = x.first < x.end ? a.tt_offsets[x.first] : 0;
        x.base = base < 0 ? 0 : (base > a.max_tokens ? (int)a.max_tokens : (int)base);
        if (x.members < 2 || x.end <= x.first || x.q1 <= x.q0 || x.len == INT32_MAX) x.len = 0;      // (one reader: nothing to gain)
        x.items = ((int64_t)(x.q1 - x.q0) * a.group + AS_PAIR - 1) / AS_PAIR * a.hkv;
        x.tiles = (x.len + AS_TILE - 1) / AS_TILE;
        x.splits = x.pad = 0;
        work += x.len > 0 ? x.items * x.tiles : 0;
        s.groups[g] = x;
    }
    work = block_sum(work, warp_sum);
    const int tokens = R > 0 ? vtk_clamp_offset(a.q_offsets[R], a.max_query_tokens) : 0;
    const int64_t most = tokens > 0 ? s.rows / ((int64_t)tokens * a.hq) : 1;      // parts that there is room for
    int64_t size = (work + s.ctas - 1) / s.ctas;
    size = size < AS_MIN_TILES ? AS_MIN_TILES : size;
    int64_t before = 0;
    for (int g0 = 0; g0 < G; g0 += AS_NT) {
        const int g = g0 + tid;
        int64_t items = 0;
        int tiles = 0, splits = 0;
        if (g < G && s.groups[g].len > 0) {
            const int all = s.groups[g].tiles;
            int64_t each = (all + most - 1) / most;
            each = each < size ? size : each;
            splits = (int)((all + each - 1) / each);
            tiles = (all + splits - 1) / splits;
            items = s.groups[g].items * splits;
        }
        const int64_t incl = vtk_warp_incl_scan(items);
        if (lane == 31) warp_sum[warp] = incl;
        __syncthreads();
        int64_t in_front = before;
        for (int w = 0; w < AS_NT / 32; ++w) {
            if (w < warp) in_front += warp_sum[w];
            before += warp_sum[w];
        }
        if (g < G) {
            s.groups[g].items = in_front + incl - items;
            s.groups[g].tiles = tiles;
            s.groups[g].splits = splits;
        }
        __syncthreads();
    }
    for (int r = tid; r < R; r += AS_NT) {
        const int g = s.shared[r].x;
        s.shared[r] = g < 0 ? make_int2(0, 0) : make_int2(s.groups[g].len, s.groups[g].splits);
    }
    if (tid == 0) {
        s.plan->items = before;
        s.plan->groups = G;
        s.plan->query_tokens = tokens;
    }
    if (clipped) atomicOr(a.flags, (uint32_t)VTOKEN_FLAG_CAPACITY);
}

// The workspace behind that of vtoken_attention.  Parts: a row for each query row, and enough for every CTA to have one of 256
// rows when the rows are few.
struct Layout { int64_t rows, plan, groups, shared, ml, o, bytes; };
Layout layout_of(const vtoken_ctx *ctx, const vtoken_heads *heads, int64_t max_query_tokens)
{
    Layout l;
    auto up = [](int64_t x) { return (x + 15) / 16 * 16; };
    const int64_t dense = max_query_tokens * heads->num_q_heads, least = (int64_t)ctx->num_sms * 2 * AS_PAIR;
    l.rows = dense > least ? dense : least;
    l.plan = up(vtk_attention_rows_workspace(ctx, heads, nullptr));
    l.groups = l.plan + up(sizeof(VtkPrefixPlan));
    l.shared = l.groups + up(ctx->cfg.max_requests * (int64_t)sizeof(VtkPrefixGroup));
    l.ml = l.shared + up(ctx->cfg.max_requests * (int64_t)sizeof(int2));
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
    s.shared = (int2 *)(ws + l.shared);
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
    if (rc == VTOKEN_OK) rc = vtk_launch_attention_rows(ctx, heads, a, prompts ? 1 : in->max_query_len, true, st);
    return rc == VTOKEN_OK && prompts ? vtk_launch_attention_prompt(ctx, heads, a, (uint32_t *)in->workspace, false, st) : rc;
}

}  // extern "C"
