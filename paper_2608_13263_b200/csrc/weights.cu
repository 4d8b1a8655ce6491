// Attention weight received by every cached token, few query rows per request (a decode step).
//
// w[t] = sum over query rows i and heads h of exp(s q_ih k_t - lse_ih): with the logarithms of the sums at hand every token stands by
// itself, so there is nothing to join.  Bound by HBM: each visible K row is read once.
//
// All caches are cut into chunks of 16 to 128 tokens (fewer when there are few chunks), and every CTA takes an equal run of chunks.
// Within a chunk a warp has a key head and tiles of 16 tokens: K fragments of mma.m16n8k16 come straight from the rows in HBM (8
// dimensions of one token are the B fragment of two instructions, see attention.cu), two tiles ahead, and the accumulator's columns
// are tokens, so that the sum over query rows is one over lanes.  The heads' sums of a token meet in shared memory, in the order of
// the heads.
#include "weights.cuh"

namespace {

constexpr int TW_NT = 256, TW_WARPS = TW_NT / 32, TW_CHUNK = 128, TW_CTAS = 2, TW_ROW_LIMIT = 32;

// ---- K fragments of 16 tokens of a head: lane (g, t) takes of tokens g and 8 + g the dimensions kdim(t, j) .. + 7, j < D / 32 ----
template <int D, typename Act>
struct Keys16 {
    static constexpr bool FP4 = false;
    using Mma = Act;
    static __device__ __forceinline__ int kdim(int t, int j) { return 32 * j + 8 * t; }
    uint4 w[2][D / 32];
    __device__ __forceinline__ void load(const VtkAttnArgs &a, int head, int t, int64_t s0, int64_t s1)
    {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int64_t s = u ? s1 : s0;
            const uint8_t *p = a.k_rows + (s < 0 ? 0 : s) * a.row_bytes + (head * D + 8 * t) * 2;
#pragma unroll
            for (int j = 0; j < D / 32; ++j) w[u][j] = s < 0 ? make_uint4(0, 0, 0, 0) : vtk_ldg16(p + 64 * j);
        }
    }
    __device__ __forceinline__ void get(int u, uint4 (&k)[D / 32]) const
    {
#pragma unroll
        for (int j = 0; j < D / 32; ++j) k[j] = w[u][j];
    }
};

template <int D>
struct Keys4 {
    static constexpr bool FP4 = true;
    using Mma = VtkFp16;
    static __device__ __forceinline__ int kdim(int t, int j) { return (D / 4) * t + 8 * j; }
    uint32_t w[2][D / 32], sc[2];
    __device__ __forceinline__ void load(const VtkAttnArgs &a, int head, int t, int64_t s0, int64_t s1)
    {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int64_t s = u ? s1 : s0;
#pragma unroll
            for (int j = 0; j < D / 32; ++j) w[u][j] = 0;
            sc[u] = 0;
            if (s < 0) continue;
            const uint8_t *row = a.k_rows + s * a.row_bytes, *codes = row + head * (D / 2) + t * (D / 8);
            const uint8_t *scales = row + a.hkv * (D / 2) + head * (D / 16) + t * (D / 64);
            if (D == 128) {
                const uint4 q = __ldg(reinterpret_cast<const uint4 *>(codes));
                w[u][0] = q.x; w[u][1] = q.y; w[u][D / 32 - 2] = q.z; w[u][D / 32 - 1] = q.w;
                sc[u] = __ldg(reinterpret_cast<const uint16_t *>(scales));
            } else {
                const uint2 q = __ldg(reinterpret_cast<const uint2 *>(codes));
                w[u][0] = q.x; w[u][1] = q.y;
                sc[u] = __ldg(scales);
            }
        }
    }
    __device__ __forceinline__ void get(int u, uint4 (&k)[D / 32]) const
    {
        const uint32_t two = vtk_scales_to_half2(sc[u]);
#pragma unroll
        for (int j = 0; j < D / 32; ++j) k[j] = vtk_expand8(w[u][j], __byte_perm(two, 0, j < 2 ? 0x1010 : 0x3232));
    }
};

// a request as the chunks see it
struct Known {
    int q0, qn, len, range;
    int64_t base;
};

__device__ inline Known look_up(const VtkAttnArgs &a, int r, bool &clipped)
{
    Known k;
    bool c;
    vtk_request_rows(a, r, k.q0, k.qn, k.base, k.len, c);
    clipped |= c;
    const int64_t t1 = a.tt_offsets[r + 1];
    k.range = (int)((t1 < k.base ? k.base : (t1 > a.max_tokens ? a.max_tokens : t1)) - k.base);
    if (k.qn * (int64_t)a.group > a.row_limit) k.qn = 0;
    return k;
}

__device__ __forceinline__ int64_t chunks_of(const Known &k, int chunk) { return k.qn > 0 ? ((int64_t)k.len + chunk - 1) / chunk : 0; }

struct Shared {
    int64_t prefix[TW_NT + 1];           // tokens, then chunks, in front of each thread's requests
    int64_t warp_sum[TW_WARPS];
    float part[2][TW_WARPS][TW_CHUNK];   // sums of a chunk's tokens over the rows of a warp's heads
};

template <int D, typename Keys, typename Act, int RH>
struct Rows {                            // 8 RH query rows of a head in registers: lane (g, t) holds rows g and 8 + g
    uint4 q[RH][D / 32];
    int pos[RH], floor[RH], pmin, pmax;
    float scale[RH], lse2[RH];
    bool none[RH];                       // the row is not there, or it saw nothing: it adds nothing, whatever the keys hold
    __device__ __forceinline__ void load(const VtkWeightsArgs &w, const Known &k, int rt, int head)
    {
        const VtkAttnArgs &a = w.at;
        const int lane = vtk_lane(), g = lane >> 2, t = lane & 3, rows = k.qn * a.group;
        pmin = INT32_MAX;
        pmax = -1;
#pragma unroll
        for (int h = 0; h < RH; ++h) {
            const int row = rt * 8 * RH + 8 * h + g;
            const bool have = row < rows;
            const int tok = have ? row / a.group : 0, qh = head * a.group + (have ? row % a.group : 0);
            const int64_t at = k.q0 + tok;
            pos[h] = have ? min(a.positions[at], INT32_MAX - 1) : -1;       // (INT32_MAX is the id of what is not there)
            floor[h] = vtk_floor(pos[h], a.window);
            const float l = have ? w.lse_in[at * a.hq + qh] : INFINITY;
            none[h] = !have || l == -INFINITY;
            lse2[h] = l * 1.4426950408889634f;
            scale[h] = a.scale_log2;
            if (have) {
                pmin = pos[h] < pmin ? pos[h] : pmin;
                pmax = pos[h] > pmax ? pos[h] : pmax;
            }
            const uint16_t *p = a.q + at * a.q_stride + (int64_t)qh * D;
#pragma unroll
            for (int j = 0; j < D / 32; ++j) q[h][j] = have ? *reinterpret_cast<const uint4 *>(p + Keys::kdim(t, j)) : make_uint4(0, 0, 0, 0);
            if (Keys::FP4 && Act::kind == VTOKEN_KV_BF16) {          // bf16 queries in half precision: see attention.cu
                float top = 0.f, x[8];
#pragma unroll
                for (int j = 0; j < D / 32; ++j) {
                    vtk_unpack8<VtkBf16>(q[h][j], x);
#pragma unroll
                    for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(x[e]));
                }
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                int e2 = (int)(__float_as_uint(top) >> 23) - 127;
                e2 = 14 - (e2 < -100 ? -100 : e2);
                const float up = __uint_as_float((uint32_t)(127 + e2) << 23);
                scale[h] *= __uint_as_float((uint32_t)(127 - e2) << 23);
#pragma unroll
                for (int j = 0; j < D / 32; ++j) {
                    vtk_unpack8<VtkBf16>(q[h][j], x);
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] *= up;
                    q[h][j] = vtk_pack8<VtkFp16>(x);
                }
            }
        }
        pmin = __reduce_min_sync(0xffffffffu, pmin);
        pmax = __reduce_max_sync(0xffffffffu, pmax);
    }
};

// RH: 8-row halves of the instruction that are used
template <int D, typename Keys, typename Act, int RH>
__global__ void __launch_bounds__(TW_NT, TW_CTAS) token_weights_kernel(const __grid_constant__ VtkWeightsArgs w)
{
    using Mma = typename Keys::Mma;
    const VtkAttnArgs &a = w.at;
    __shared__ Shared sh;
    vtk_release_successor();
    vtk_wait_for_predecessor();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    int R = *a.num_requests;
    bool clipped = R < 0 || R > a.max_requests;
    R = R < 0 ? 0 : (R > a.max_requests ? a.max_requests : R);
    const int seg = (R + TW_NT - 1) / TW_NT;

    // ---- the cut: chunks of a size at which every CTA gets some, counted in front of each thread's requests ----
    int chunk = TW_CHUNK;
    auto count = [&](int size, bool first) {
        int64_t n = 0;
        for (int r = tid * seg; r < (tid + 1) * seg && r < R; ++r) {
            bool c = false;
            n += chunks_of(look_up(a, r, c), size);
            if (first) clipped |= c;
        }
        const int64_t incl = vtk_warp_incl_scan(n);
        if (lane == 31) sh.warp_sum[warp] = incl;
        __syncthreads();
        int64_t before = 0;
        for (int v = 0; v < warp; ++v) before += sh.warp_sum[v];
        sh.prefix[tid + 1] = before + incl;
        if (tid == 0) sh.prefix[0] = 0;
        __syncthreads();
    };
    count(chunk, true);
    if (clipped && blockIdx.x == 0) atomicOr(a.flags, (uint32_t)VTOKEN_FLAG_CAPACITY);
    while (chunk > 16 && sh.prefix[TW_NT] < (int64_t)gridDim.x * 2) {
        chunk /= 2;
        count(chunk, false);
    }
    const int64_t W = sh.prefix[TW_NT], per = W / gridDim.x, more = W - per * gridDim.x;
    int64_t c0 = blockIdx.x * per + (blockIdx.x < more ? blockIdx.x : more);
    const int64_t c1 = c0 + per + (blockIdx.x < more ? 1 : 0);
    if (c0 >= c1) return;
    int lo = 0, hi = TW_NT;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (sh.prefix[mid] <= c0) lo = mid; else hi = mid;
    }
    int r = lo * seg;
    int64_t left = c0 - sh.prefix[lo];
    Known k;
    for (;; ++r) {
        bool c = false;
        k = look_up(a, r, c);
        const int64_t n = chunks_of(k, chunk);
        if (left < n) break;
        left -= n;
    }
    int at = (int)left * chunk;

    // ---- warps: heads side by side, and tiles of 16 tokens ----
    int heads = 1;
    while (heads < TW_WARPS && heads < a.hkv) heads <<= 1;
    const int lanes = TW_WARPS / heads, hl = warp / lanes, tw = warp % lanes, rounds = (a.hkv + heads - 1) / heads;
    Rows<D, Keys, Act, RH> q;
    int loaded_r = -1, loaded_head = -1, buffer = 0;
    bool bad_slot = false, bad_id = false;
    for (; c0 < c1; ++c0, buffer ^= 1) {
        const int n = k.len - at < chunk ? k.len - at : chunk, tiles = (n + 15) / 16;
        const int row_tiles = (k.qn * a.group + 8 * RH - 1) / (8 * RH);
        float *part = sh.part[buffer][warp];
        for (int round = 0; round < rounds; ++round) {
            const int head = round * heads + hl;
            if (head >= a.hkv) continue;
            if (loaded_r != r || loaded_head != head) {
                q.load(w, k, 0, head);
                loaded_r = r;
                loaded_head = head;
            }
            // slots of a tile's tokens two tiles ahead, their keys one ahead
            struct Tokens { int id[2], slot[2]; };
            auto look = [&](int tile) {
                Tokens x;
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int i = tile * 16 + 8 * u + g;
                    x.id[u] = INT32_MAX;
                    x.slot[u] = -1;
                    if (i < n) {
                        x.id[u] = a.cache_ids.null() ? at + i : a.cache_ids[k.base + at + i];
                        x.slot[u] = a.cache_slots[k.base + at + i];
                    }
                }
                return x;
            };
            auto fetch = [&](Tokens &x, Keys &keys) {
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    if ((int64_t)x.slot[u] >= a.slots_per_layer) {
                        bad_slot = true;
                        x.slot[u] = -1;
                    }
                    // (with more row tiles than one the rows' span is not known here)
                    if (row_tiles == 1 && !vtk_sees(x.id[u], q.pmax, vtk_floor(q.pmin, a.window), a.sinks)) x.slot[u] = -1;
                }
                keys.load(a, head, t, x.slot[0], x.slot[1]);
            };
            Tokens now = look(tw), next = look(tw + lanes);
            Keys keys, keys_next;
            fetch(now, keys);
            for (int tile = tw; tile < tiles; tile += lanes) {
                const Tokens after = look(tile + 2 * lanes);
                fetch(next, keys_next);
                float sum[2][2] = {{0.f, 0.f}, {0.f, 0.f}};          // of tokens 8 u + 2 t + e, over rows g (and 8 + g)
                if (__any_sync(0xffffffffu, now.slot[0] >= 0 || now.slot[1] >= 0)) {
                    for (int rt = 0; rt < row_tiles; ++rt) {
                        if (row_tiles > 1) q.load(w, k, rt, head);
                        const bool full = __all_sync(0xffffffffu, now.slot[0] >= 0 && now.slot[1] >= 0 &&
                                                     vtk_sees(now.id[0], q.pmin, vtk_floor(q.pmax, a.window), a.sinks) &&
                                                     vtk_sees(now.id[1], q.pmin, vtk_floor(q.pmax, a.window), a.sinks));
#pragma unroll
                        for (int u = 0; u < 2; ++u) {
                            float s[4] = {0.f, 0.f, 0.f, 0.f};
                            uint4 kf[D / 32];
                            keys.get(u, kf);
#pragma unroll
                            for (int j = 0; j < D / 32; ++j) {
                                vtk_mma<Mma>(s, q.q[0][j].x, RH == 2 ? q.q[RH - 1][j].x : 0u, q.q[0][j].y, RH == 2 ? q.q[RH - 1][j].y : 0u, kf[j].x, kf[j].y);
                                vtk_mma<Mma>(s, q.q[0][j].z, RH == 2 ? q.q[RH - 1][j].z : 0u, q.q[0][j].w, RH == 2 ? q.q[RH - 1][j].w : 0u, kf[j].z, kf[j].w);
                            }
                            int id[2] = {0, 0}, slot[2] = {0, 0};
                            if (!full) {
#pragma unroll
                                for (int e = 0; e < 2; ++e) {
                                    id[e] = __shfl_sync(0xffffffffu, now.id[u], 4 * (2 * t + e));
                                    slot[e] = __shfl_sync(0xffffffffu, now.slot[u], 4 * (2 * t + e));
                                }
                            }
#pragma unroll
                            for (int h = 0; h < RH; ++h)
#pragma unroll
                                for (int e = 0; e < 2; ++e) {
                                    float y = vtk_exp2(fmaf(s[2 * h + e], q.scale[h], -q.lse2[h]));
                                    if (q.none[h]) y = 0.f;
                                    if (!full && !(slot[e] >= 0 && vtk_sees(id[e], q.pos[h], q.floor[h], a.sinks))) y = 0.f;
                                    sum[u][e] += y;
                                }
                        }
                    }
                    if (row_tiles > 1) loaded_head = -1;
                }
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float y = sum[u][e];
                        y += __shfl_xor_sync(0xffffffffu, y, 4);
                        y += __shfl_xor_sync(0xffffffffu, y, 8);
                        y += __shfl_xor_sync(0xffffffffu, y, 16);
                        if (g == 0) {
                            float *p = part + tile * 16 + 8 * u + 2 * t + e;
                            *p = round == 0 ? y : *p + y;
                        }
                    }
                now = next;
                keys = keys_next;
                next = after;
            }
        }
        __syncthreads();                                     // (the next chunk's sums go to the other buffer)
        if (tid < n) {
            const int id = a.cache_ids.null() ? at + tid : a.cache_ids[k.base + at + tid];
            if (id >= 0 && id < k.range) {
                const int lane_of = tid / 16 % lanes;
                float y = 0.f;
                for (int h = 0; h < heads && h < a.hkv; ++h) y += sh.part[buffer][h * lanes + lane_of][tid];
                if (!w.prev.null()) y = fmaf(w.decay, w.prev[k.base + id], y);
                w.scores[k.base + id] = y;
            } else {
                bad_id = true;
            }
        }
        if (k.len - at > chunk) {
            at += chunk;
        } else if (c0 + 1 < c1) {
            bool c = false;
            do k = look_up(a, ++r, c); while (chunks_of(k, chunk) == 0);
            at = 0;
        }
    }
    if (bad_slot) atomicOr(a.flags, (uint32_t)VTOKEN_FLAG_BAD_SLOT);
    if (bad_id) atomicOr(a.flags, (uint32_t)VTOKEN_FLAG_BAD_VICTIM);
}

template <int D, typename Keys, typename Act>
int launch(vtoken_ctx *ctx, const VtkWeightsArgs &w, bool wide, cudaStream_t st)
{
    const dim3 grid(ctx->num_sms * TW_CTAS), block(TW_NT);
    VTK_CUDA(ctx, wide ? vtk_launch_dependent(ctx, token_weights_kernel<D, Keys, Act, 2>, grid, block, 0, st, w)
                       : vtk_launch_dependent(ctx, token_weights_kernel<D, Keys, Act, 1>, grid, block, 0, st, w));
    VTK_CUDA(ctx, cudaGetLastError());
    return VTOKEN_OK;
}

template <int D>
int launch_by_type(vtoken_ctx *ctx, const vtoken_heads *h, const VtkWeightsArgs &w, bool wide, cudaStream_t st)
{
    const bool bf = h->act_type == VTOKEN_KV_BF16;
    if (h->kv_type == VTOKEN_KV_FP4) return bf ? launch<D, Keys4<D>, VtkBf16>(ctx, w, wide, st) : launch<D, Keys4<D>, VtkFp16>(ctx, w, wide, st);
    return bf ? launch<D, Keys16<D, VtkBf16>, VtkBf16>(ctx, w, wide, st) : launch<D, Keys16<D, VtkFp16>, VtkFp16>(ctx, w, wide, st);
}

}  // namespace

extern "C" {

int64_t vtoken_token_weights_workspace_bytes(const vtoken_ctx *ctx, const vtoken_heads *heads, int32_t max_query_tokens)
{
    if (!ctx || vtk_check_heads(ctx, heads, 0) != VTOKEN_OK || max_query_tokens < 0) return VTOKEN_EINVAL;
    return vtk_weights_prompt_workspace(ctx, heads);
}

int vtoken_token_weights(vtoken_ctx *ctx, const vtoken_heads *heads, int32_t layer, const vtoken_weights_in *in, void *cuda_stream)
{
    if (!ctx || !heads || !in) return VTOKEN_EINVAL;
    if (vtk_check_heads(ctx, heads, layer) != VTOKEN_OK) return VTOKEN_EINVAL;
    if (!in->num_requests || !in->q_offsets || !in->tt_offsets || !in->cache_slots || !in->cache_len || !in->scores || !in->workspace) return VTOKEN_EINVAL;
    if (in->max_query_tokens != 0 && (!in->positions || !in->q || !in->lse)) return VTOKEN_EINVAL;     // (without elements: no address)
    if (in->max_query_tokens < 0 || in->max_query_len < 1 || in->window < 0 || in->sinks < 0) return VTOKEN_EINVAL;
    if (!(in->decay > -INFINITY && in->decay < INFINITY)) return VTOKEN_EINVAL;
    VtkWeightsArgs w;
    VtkAttnArgs &a = w.at;
    if (!vtk_score_scale(heads, in->sm_scale, a.scale_log2)) return VTOKEN_EINVAL;
    if ((((uintptr_t)in->q | (uintptr_t)in->workspace) & 15) || (((uintptr_t)in->lse | (uintptr_t)in->prev | (uintptr_t)in->scores) & 3)) return VTOKEN_EINVAL;
    a.q_stride = vtk_stride(in->q_stride, (int64_t)heads->num_q_heads * heads->head_dim);
    if (a.q_stride < 0) return VTOKEN_EINVAL;
    if (in->workspace_bytes < vtoken_token_weights_workspace_bytes(ctx, heads, in->max_query_tokens)) return VTOKEN_ECAPACITY;
    if (in->max_query_tokens == 0) return VTOKEN_OK;
    a.num_requests = in->num_requests;
    a.q_offsets = VTK_ARR(ctx, in->q_offsets, ctx->cfg.max_requests + 1);
    a.positions = VTK_ARR(ctx, in->positions, in->max_query_tokens);
    a.tt_offsets = VTK_ARR(ctx, in->tt_offsets, ctx->cfg.max_requests + 1);
    a.cache_slots = VTK_ARR(ctx, in->cache_slots, ctx->cfg.max_tokens);
    a.cache_ids = VTK_ARR(ctx, in->cache_ids, ctx->cfg.max_tokens);
    a.cache_len = VTK_ARR(ctx, in->cache_len, ctx->cfg.max_requests);
    a.q = (const uint16_t *)in->q;
    a.out = nullptr;
    a.lse = nullptr;
    a.k_rows = (const uint8_t *)ctx->cfg.k_pool + layer * ctx->layer_stride;
    a.v_rows = nullptr;
    a.out_stride = 0;
    a.row_bytes = ctx->row_bytes;
    a.slots_per_layer = ctx->slots_per_layer;
    a.max_tokens = ctx->cfg.max_tokens;
    a.max_requests = ctx->cfg.max_requests;
    a.max_query_tokens = in->max_query_tokens;
    a.hq = heads->num_q_heads;
    a.hkv = heads->num_kv_heads;
    a.group = heads->num_q_heads / heads->num_kv_heads;
    a.inv_group = 1.f / (float)a.group;
    a.window = in->window;
    a.sinks = in->window > 0 ? in->sinks : 0;
    a.v_mul = 1.f;
    a.flags = &ctx->rt_counts->error_flags;
    a.counters = nullptr;
    a.part = nullptr;
    w.lse_in = in->lse;
    w.prev = VTK_ARR(ctx, in->decay == 0.f ? (const float *)nullptr : in->prev, ctx->cfg.max_tokens);
    w.scores = VTK_ARR(ctx, in->scores, ctx->cfg.max_tokens);
    w.decay = in->decay;
    const bool prompts = (int64_t)in->max_query_len * a.group > TW_ROW_LIMIT;
    a.row_limit = prompts ? TW_ROW_LIMIT : INT32_MAX;
    const bool wide = (prompts ? 1 : (int64_t)in->max_query_len) * a.group > 8;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    const int rc = heads->head_dim == 128 ? launch_by_type<128>(ctx, heads, w, wide, st) : launch_by_type<64>(ctx, heads, w, wide, st);
    return rc == VTOKEN_OK && prompts ? vtk_launch_weights_prompt(ctx, heads, w, in->workspace, st) : rc;
}

}  // extern "C"
