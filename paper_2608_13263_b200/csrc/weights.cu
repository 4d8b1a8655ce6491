// Attention weight received by every cached token, few query rows per request (a decode step).
//
// w[t] = sum over query rows i and heads h of exp(s q_ih k_t - lse_ih): with the logarithms of the sums at hand every token stands by
// itself, so there is nothing to join.  Bound by HBM: each visible K row is read once.
//
// All caches are cut into chunks of 16 to 128 tokens (fewer when there are few chunks), and every CTA takes an equal run of chunks.
// Within a chunk a warp has a key head and tiles of 16 tokens (32 over 4-bit rows, where instructions count), copied several tiles ahead by cp.async into a ring of its own.  The
// product is taken as S^T = K Q^T, mma.m16n8k16 with the 16 tokens as rows and 8 query rows as columns: no row of the instruction is
// empty, a lane's accumulators belong to two tokens whose ids it holds, and the sum over query rows is one over four lanes.  (As
// S = Q K^T, with half of the instruction empty, twelve shuffles a tile and K one tile ahead in registers, 512 requests took 428 us,
// 256 over 4-bit rows 472.)  Up to 8 RH query rows of a head stay in registers; more are fetched again for every tile, which is right
// but slow (256 requests, 64 heads over 8, one to four query tokens: 184, 212, 663, 781 us; over 4-bit rows 139, 204, 857, 966).  The
// order of the contracted dimension is free, so 8 dimensions of a token, 16 bytes, are the fragments of two instructions, see
// attention.cu.  The heads' sums of a token meet in shared memory, in the order of the heads.
#include "weights.cuh"

namespace {

constexpr int TW_NT = 256, TW_WARPS = TW_NT / 32, TW_CHUNK = 128, TW_CTAS = 2, TW_ROW_LIMIT = 32;

__device__ __forceinline__ void cp_async16(uint32_t dst, const void *src, bool there)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// ---- K rows of a tile: lane (g, t) takes of tokens g and 8 + g the dimensions kdim(t, j) .. + 7, j < D / 32 ----
template <int D, typename Act>
struct Keys16 {
    static constexpr bool FP4 = false;
    using Mma = Act;
    static constexpr int TILE = 16, PITCH = D * 2, STAGE = TILE * PITCH, PIECES = D / 8, STAGES = D == 128 ? 3 : 5;
    static __device__ __forceinline__ int kdim(int t, int j) { return 32 * j + 8 * t; }
    // slot: lane i < TILE holds that of token i, negative = zeros
    static __device__ __forceinline__ void issue(uint32_t dst, const VtkAttnArgs &a, int head, int slot)
    {
        const int lane = vtk_lane(), c = lane % PIECES, sub = lane / PIECES;
        const uint32_t row_bytes = (uint32_t)a.row_bytes;
        const uint8_t *rows = a.k_rows + (head * (D * 2) + 16 * c);
        constexpr int PER = 32 / PIECES;
#pragma unroll
        for (int i = 0; i < TILE / PER; ++i) {
            const int tok = i * PER + sub, s = __shfl_sync(0xffffffffu, slot, tok);
            cp_async16(dst + tok * PITCH + ((c ^ ((tok & 1) << 2)) << 4), rows + (uint64_t)(uint32_t)(s < 0 ? 0 : s) * row_bytes, s >= 0);
        }
    }
    static __device__ __forceinline__ void get(const uint8_t *at, int, int u, int g, int t, uint4 (&k)[D / 32])
    {
#pragma unroll
        for (int j = 0; j < D / 32; ++j)
            k[j] = *reinterpret_cast<const uint4 *>(at + (8 * u + g) * PITCH + (((4 * j + t) ^ ((g & 1) << 2)) << 4));
    }
};

template <int D>
struct Keys4 {
    static constexpr bool FP4 = true;
    using Mma = VtkFp16;
    static constexpr int TILE = 32, PITCH = D / 2, CODES = TILE * PITCH, STAGE = CODES + TILE * 16, PIECES = D / 32, STAGES = 4;
    static __device__ __forceinline__ int kdim(int t, int j) { return (D / 4) * t + 8 * j; }
    static __device__ __forceinline__ void issue(uint32_t dst, const VtkAttnArgs &a, int head, int slot)
    {
        const int lane = vtk_lane(), c = lane % PIECES, sub = lane / PIECES;
        const uint32_t row_bytes = (uint32_t)a.row_bytes;
        const uint8_t *rows = a.k_rows + (head * PITCH + 16 * c), *scales = a.k_rows + (a.hkv * PITCH + ((head * (D / 16)) & ~15));
        constexpr int PER = 32 / PIECES;
#pragma unroll
        for (int i = 0; i < TILE / PER; ++i) {
            const int tok = i * PER + sub, s = __shfl_sync(0xffffffffu, slot, tok);
            cp_async16(dst + tok * PITCH + 16 * c, rows + (uint64_t)(uint32_t)(s < 0 ? 0 : s) * row_bytes, s >= 0);
        }
        // scales: the aligned 16 bytes that hold the head's
        cp_async16(dst + CODES + lane * 16, scales + (uint64_t)(uint32_t)(slot < 0 ? 0 : slot) * row_bytes, slot >= 0);
    }
    static __device__ __forceinline__ void get(const uint8_t *at, int head, int u, int g, int t, uint4 (&k)[D / 32])
    {
        const uint8_t *codes = at + (8 * u + g) * PITCH + t * (D / 8), *sc = at + CODES + (8 * u + g) * 16 + ((head * (D / 16)) & 15);
        uint32_t w[D / 32];
        if (D == 128) {
            const uint4 q = *reinterpret_cast<const uint4 *>(codes);
            w[0] = q.x; w[1] = q.y; w[D / 32 - 2] = q.z; w[D / 32 - 1] = q.w;
        } else {
            const uint2 q = *reinterpret_cast<const uint2 *>(codes);
            w[0] = q.x; w[1] = q.y;
        }
        const uint32_t two = vtk_scales_to_half2(D == 128 ? *reinterpret_cast<const uint16_t *>(sc + 2 * t) : sc[t]);
#pragma unroll
        for (int j = 0; j < D / 32; ++j) k[j] = vtk_expand8(w[j], __byte_perm(two, 0, j < 2 ? 0x1010 : 0x3232));
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

template <typename Keys>
struct Shared {
    alignas(128) uint8_t ring[TW_WARPS][Keys::STAGES][Keys::STAGE];
    int ids[TW_WARPS][Keys::STAGES][Keys::TILE];                // INT32_MAX: not there, or nobody sees it
    int64_t prefix[TW_NT + 1];           // chunks in front of each thread's requests
    int64_t warp_sum[TW_WARPS];
    float part[2][TW_WARPS][TW_CHUNK];   // sums of a chunk's tokens over the rows of a warp's heads
};

// 8 RH query rows of a head as columns of the products: lane (g, t) holds the dimensions of rows g (and 8 + g), and what the columns
// 2t, 2t + 1 (+ 8) need besides
template <int D, typename Keys, typename Act, int RH>
struct Rows {
    uint4 q[RH][D / 32];
    int pos[RH][2], pmin, pmax, rows;    // rows: of these columns, at most 8 RH
    float scale[RH][2], lse2[RH][2];
    bool none[RH][2];                    // the row is not there, or it saw nothing: it adds nothing, whatever the keys hold
    __device__ __forceinline__ void load(const VtkWeightsArgs &w, const Known &k, int rt, int head)
    {
        const VtkAttnArgs &a = w.at;
        const int lane = vtk_lane(), g = lane >> 2, t = lane & 3, all = k.qn * a.group;
        rows = all - rt * 8 * RH;
        pmin = INT32_MAX;
        pmax = -1;
#pragma unroll
        for (int h = 0; h < RH; ++h) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int row = rt * 8 * RH + 8 * h + 2 * t + e;
                const bool have = row < all;
                const int64_t at = k.q0 + (have ? row / a.group : 0);
                const float l = have ? w.lse_in[at * a.hq + head * a.group + row % a.group] : -INFINITY;
                pos[h][e] = have ? min(a.positions[at], INT32_MAX - 1) : -1;     // (INT32_MAX is the id of what is not there)
                none[h][e] = l == -INFINITY;
                lse2[h][e] = l * 1.4426950408889634f;
                scale[h][e] = a.scale_log2;
                if (have) {
                    pmin = pos[h][e] < pmin ? pos[h][e] : pmin;
                    pmax = pos[h][e] > pmax ? pos[h][e] : pmax;
                }
            }
            const int row = rt * 8 * RH + 8 * h + g;
            const bool have = row < all;
            const uint16_t *p = a.q + (k.q0 + (have ? row / a.group : 0)) * a.q_stride + (int64_t)(head * a.group + (have ? row % a.group : 0)) * D;
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
                const float up = __uint_as_float((uint32_t)(127 + e2) << 23), down = __uint_as_float((uint32_t)(127 - e2) << 23);
                scale[h][0] *= __shfl_sync(0xffffffffu, down, 8 * t);
                scale[h][1] *= __shfl_sync(0xffffffffu, down, 8 * t + 4);
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

// RH: columns of 8 query rows at a time
template <int D, typename Keys, typename Act, int RH>
__global__ void __launch_bounds__(TW_NT, TW_CTAS) token_weights_kernel(const __grid_constant__ VtkWeightsArgs w)
{
    using Mma = typename Keys::Mma;
    constexpr int ST = Keys::STAGES, TILE = Keys::TILE;
    const VtkAttnArgs &a = w.at;
    extern __shared__ __align__(128) uint8_t raw[];
    Shared<Keys> &sh = *reinterpret_cast<Shared<Keys> *>(raw);
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
    const int64_t enough = (int64_t)gridDim.x * 2, some = sh.prefix[TW_NT];
    if (some < enough) {
        while (chunk > TILE && some * (TW_CHUNK / chunk) < enough) chunk /= 2;
        __syncthreads();
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
    int at0 = (int)left * chunk;

    // ---- warps: heads side by side, and tiles of 16 tokens ----
    int heads = 1;
    while (heads < TW_WARPS && heads < a.hkv) heads <<= 1;
    const int lanes = TW_WARPS / heads, hl = warp / lanes, tw = warp % lanes, rounds = (a.hkv + heads - 1) / heads;
    const int turns = chunk / TILE > lanes ? chunk / TILE / lanes : 1;         // tiles of a warp in a chunk, for each of its heads
    const uint32_t ring = vtk_smem_u32(sh.ring[warp]);
    Rows<D, Keys, Act, RH> q;
    bool bad_slot = false, bad_id = false;
    int buffer = 0;
    // ---- runs of chunks in one request; the ring is filled across its chunks ----
    while (c0 < c1) {
        const int64_t here = chunks_of(k, chunk) - at0 / chunk;
        const int chunks = (int)(here < c1 - c0 ? here : c1 - c0);
        const int end = k.len - at0 > (int64_t)chunks * chunk ? at0 + chunks * chunk : k.len;
        const int row_tiles = (k.qn * a.group + 8 * RH - 1) / (8 * RH);
        int pmin = INT32_MAX, pmax = -1;                     // of all rows
        for (int i = lane; i < k.qn; i += 32) {
            const int p = min(a.positions[k.q0 + i], INT32_MAX - 1);
            pmin = p < pmin ? p : pmin;
            pmax = p > pmax ? p : pmax;
        }
        pmin = __reduce_min_sync(0xffffffffu, pmin);
        pmax = __reduce_max_sync(0xffffffffu, pmax);
        const int floor_min = vtk_floor(pmin, a.window);
        struct Place {                                       // the warp's next tile
            int c, round, turn;
        };
        auto advance = [&](Place &p) {
            if (++p.turn < turns) return;
            p.turn = 0;
            if (++p.round < rounds) return;
            p.round = 0;
            ++p.c;
        };
        Place get = {0, 0, 0};
        int issued = 0;
        struct Next { int slot, id, head; bool more; };
        auto look = [&]() {                                  // slots and ids of a tile's tokens, a step ahead of its copies
            Next n = {-1, INT32_MAX, get.round * heads + hl, get.c < chunks};
            const int tile = get.turn * lanes + tw, i = at0 + get.c * chunk + tile * TILE + lane;
            if (n.more && lane < TILE && tile * TILE < chunk && i < end && n.head < a.hkv) {
                n.slot = a.cache_slots[k.base + i];
                n.id = a.cache_ids.null() ? i : a.cache_ids[k.base + i];
            }
            advance(get);
            return n;
        };
        auto issue = [&](Next n) {
            if (n.more) {
                if ((int64_t)n.slot >= a.slots_per_layer) {
                    bad_slot = true;
                    n.slot = -1;
                }
                if (n.slot < 0 || !vtk_sees(n.id, pmax, floor_min, a.sinks)) {
                    n.slot = -1;
                    n.id = INT32_MAX;
                }
                const int stage = issued % ST;
                if (lane < TILE) sh.ids[warp][stage][lane] = n.id;
                if (__any_sync(0xffffffffu, n.slot >= 0)) Keys::issue(ring + stage * Keys::STAGE, a, n.head, n.slot);
                ++issued;
            }
            cp_commit();
        };
        Next next;
        {
            Next first[ST - 1];
#pragma unroll
            for (int i = 0; i < ST - 1; ++i) first[i] = look();
            next = look();
#pragma unroll
            for (int i = 0; i < ST - 1; ++i) issue(first[i]);
        }
        if (rounds == 1 && row_tiles == 1 && hl < a.hkv) q.load(w, k, 0, hl);
        int used = 0;
        for (int c = 0; c < chunks; ++c, buffer ^= 1) {
            const int at = at0 + c * chunk, n = end - at < chunk ? end - at : chunk;
            float *part = sh.part[buffer][warp];
            for (int round = 0; round < rounds; ++round) {
                const int head = round * heads + hl;
                if (rounds > 1 && row_tiles == 1 && head < a.hkv) q.load(w, k, 0, head);
                for (int turn = 0; turn < turns; ++turn, ++used) {
                    cp_wait<ST - 2>();
                    __syncwarp();
                    issue(next);
                    next = look();
                    const int tile = turn * lanes + tw;
                    if (head >= a.hkv || tile * TILE >= n) continue;
                    const int stage = used % ST;
#pragma unroll
                    for (int b = 0; b < TILE / 16; ++b) {
                        const int id[2] = {sh.ids[warp][stage][16 * b + g], sh.ids[warp][stage][16 * b + 8 + g]};
                        float sum[2] = {0.f, 0.f};           // of tokens g and 8 + g, over columns 2t and 2t + 1 (+ 8)
                        if (__any_sync(0xffffffffu, id[0] != INT32_MAX || id[1] != INT32_MAX)) {
                            uint4 kf[2][D / 32];
#pragma unroll
                            for (int u = 0; u < 2; ++u) Keys::get(sh.ring[warp][stage], head, 2 * b + u, g, t, kf[u]);
                            for (int rt = 0; rt < row_tiles; ++rt) {
                                if (row_tiles > 1) q.load(w, k, rt, head);
                                const int floor_max = vtk_floor(q.pmax, a.window);
                                const bool full = __all_sync(0xffffffffu, vtk_sees(id[0], q.pmin, floor_max, a.sinks) && vtk_sees(id[1], q.pmin, floor_max, a.sinks));
#pragma unroll
                                for (int h = 0; h < RH; ++h) {
                                    if (h == 1 && q.rows <= 8) break;    // (uniform)
                                    float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                                    for (int j = 0; j < D / 32; ++j) {
                                        vtk_mma<Mma>(s, kf[0][j].x, kf[1][j].x, kf[0][j].y, kf[1][j].y, q.q[h][j].x, q.q[h][j].y);
                                        vtk_mma<Mma>(s, kf[0][j].z, kf[1][j].z, kf[0][j].w, kf[1][j].w, q.q[h][j].z, q.q[h][j].w);
                                    }
                                    float y[2][2];
#pragma unroll
                                    for (int u = 0; u < 2; ++u)
#pragma unroll
                                        for (int e = 0; e < 2; ++e) {
                                            y[u][e] = vtk_exp2(fmaf(s[2 * u + e], q.scale[h][e], -q.lse2[h][e]));
                                            if (q.none[h][e]) y[u][e] = 0.f;
                                        }
                                    if (!full)
#pragma unroll
                                        for (int u = 0; u < 2; ++u)
#pragma unroll
                                            for (int e = 0; e < 2; ++e)
                                                if (!vtk_sees(id[u], q.pos[h][e], vtk_floor(q.pos[h][e], a.window), a.sinks)) y[u][e] = 0.f;
#pragma unroll
                                    for (int u = 0; u < 2; ++u) sum[u] += y[u][0] + y[u][1];
                                }
                            }
                        }
#pragma unroll
                        for (int u = 0; u < 2; ++u) {
                            sum[u] += __shfl_xor_sync(0xffffffffu, sum[u], 1);
                            sum[u] += __shfl_xor_sync(0xffffffffu, sum[u], 2);
                        }
                        if (t < 2) {
                            float *p = part + tile * TILE + 16 * b + 8 * t + g;
                            const float y = t == 0 ? sum[0] : sum[1];
                            *p = round == 0 ? y : *p + y;
                        }
                    }
                }
            }
            __syncthreads();                                 // (the next chunk's sums go to the other buffer)
            if (tid < n) {
                const int id = a.cache_ids.null() ? at + tid : a.cache_ids[k.base + at + tid];
                if (id >= 0 && id < k.range) {
                    const int lane_of = tid / TILE % lanes;
                    float y = 0.f;
                    for (int h = 0; h < heads && h < a.hkv; ++h) y += sh.part[buffer][h * lanes + lane_of][tid];
                    if (!w.prev.null()) y = fmaf(w.decay, w.prev[k.base + id], y);
                    w.scores[k.base + id] = y;
                } else {
                    bad_id = true;
                }
            }
        }
        cp_wait<0>();
        __syncwarp();
        c0 += chunks;
        if (c0 < c1) {
            bool c = false;
            do k = look_up(a, ++r, c); while (chunks_of(k, chunk) == 0);
            at0 = 0;
        }
    }
    if (bad_slot) atomicOr(a.flags, (uint32_t)VTOKEN_FLAG_BAD_SLOT);
    if (bad_id) atomicOr(a.flags, (uint32_t)VTOKEN_FLAG_BAD_VICTIM);
}

template <int D, typename Keys, typename Act>
int launch(vtoken_ctx *ctx, const VtkWeightsArgs &w, bool wide, cudaStream_t st)
{
    const dim3 grid(ctx->num_sms * TW_CTAS), block(TW_NT);
    constexpr int smem = (int)sizeof(Shared<Keys>);
    static_assert(TW_CTAS * (smem + 1024) <= 233472, "shared memory of an SM");
    static std::atomic<int> allowed[2] = {{-1}, {-1}};       // the device that knows of the kernels' shared memory
    auto kernel = wide ? token_weights_kernel<D, Keys, Act, 2> : token_weights_kernel<D, Keys, Act, 1>;
    VTK_CUDA(ctx, vtk_allow_smem(ctx, allowed[wide], (const void *)kernel, smem));
    VTK_CUDA(ctx, vtk_launch_dependent(ctx, kernel, grid, block, smem, st, w));
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
    return vtk_weights_prompt_workspace(ctx, heads, max_query_tokens);
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
    const bool prompts = (int64_t)in->max_query_len * a.group > TW_ROW_LIMIT && a.group <= 128;       // (a row tile holds whole query tokens)
    a.row_limit = prompts ? TW_ROW_LIMIT : INT32_MAX;
    const bool wide = (prompts ? 1 : (int64_t)in->max_query_len) * a.group > 8;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    const int rc = heads->head_dim == 128 ? launch_by_type<128>(ctx, heads, w, wide, st) : launch_by_type<64>(ctx, heads, w, wide, st);
    return rc == VTOKEN_OK && prompts ? vtk_launch_weights_prompt(ctx, heads, w, in->workspace, st) : rc;
}

}  // extern "C"
