// Attention weight received by every cached token from many query rows per request (prompts and chunks of prompts), on the fifth
// generation tensor cores.
//
// 2 D flops and one exponential a pair of query row and token.  The product is taken as S^T = K Q^T, tokens as the rows of the
// accumulator: a thread then owns a token and the sum over query rows is a sum over its registers, where S = Q K^T would need one over
// the lanes of a warp for every column.  256 x 128 pairs take 1024 cycles of the tensor pipe and 2048 of the 16 exponentials a
// cycle: the exponentials are the bound.
//
// An item is (request, 256 tokens, key head, chunk of row tiles): its K rows stay in shared memory while the tiles of Q that see any of
// them stream by, whole query tokens, 128 rows at most, a hardware copy each.  Sums of an item go to the workspace; a second small
// kernel adds them up in the order of chunks and heads and joins them with the scores before.  Roles, 24 warps:
//   0 .. 15          thread = token: exponentials of a row of S^T, summed.  Two groups of 8 warps take the row tiles in turn, each
//                    with an accumulator for the first and one for the second 128 tokens
//   16 .. 19         copies of K rows (by slot, once an item), 4-bit keys expanded on the way; bf16 queries over 4-bit keys converted
//   20, 21           products of the first and second 128 tokens, issued by one thread each, into the groups' accumulators in turn
//   22               draws items and finds the row tiles that see the item's tokens
//   23               positions and logarithms of a tile's rows, and the copy of its queries
// Each role goes from item to item on its own, handed on by barriers in shared memory.  Every wait is bounded (wait_limit_ms): where
// one runs out all roles leave and VTOKEN_FLAG_TIMEOUT is set.  (One warp that issued all products, four that copied the queries
// with cp.async and 128 arrivals a tile, and searches for row tiles between the tiles took 600 us for a prompt of 8192 tokens, 32 heads
// over 8; as it is, 453, with the exponentials' pipe taken 67 % of the time.  Over 4-bit rows fp16 queries take 445; bf16 queries, which the
// copying warps convert to half precision tile by tile, 993.)
#include <cuda.h>

#include "tensor.cuh"
#include "weights.cuh"

namespace {

constexpr int WP_NT = 768, WP_SUMS = 16, WP_COPY = WP_SUMS, WP_MMA = 20, WP_DRAW = 22, WP_ROWS = 23;
constexpr int WP_META = 4, WP_PAIR = 2 * TC_TILE, WP_JOIN_NT = 256, WP_WORDS = 32;
constexpr uint64_t WP_DRAIN_NS = 1000000000;

struct Args {
    VtkWeightsArgs w;
    uint32_t *tickets;                   // next item, CTAs that are done; zero between calls
    float *parts;                        // sums of the items, WP_PAIR each
    int64_t max_parts;
    int32_t row_limit;                   // requests of at most so many rows belong to weights.cu
    int32_t grid;                        // of the kernel that computes
    int32_t tokens;                      // query tokens of a row tile
    uint64_t limit_ns;
    int64_t stall;                       // (checked build) the item whose first rows never come
};

// a request in this kernel
struct Spread {
    int q0, qn, len;
    int64_t base, pairs, tiles;          // pairs of token tiles; row tiles
};

__device__ inline Spread spread_of(const Args &w, int r, bool &clipped)
{
    const VtkAttnArgs &a = w.w.at;
    Spread s;
    bool c;
    vtk_request_rows(a, r, s.q0, s.qn, s.base, s.len, c);
    clipped |= c;
    s.pairs = (int64_t)s.qn * a.group > w.row_limit ? ((int64_t)s.len + WP_PAIR - 1) / WP_PAIR : 0;
    s.tiles = ((int64_t)s.qn + w.tokens - 1) / w.tokens;
    return s;
}
__device__ __forceinline__ int64_t chunks_of(const Spread &s, int64_t chunk) { return (s.tiles + chunk - 1) / chunk; }

// The cut, the same in every CTA of both kernels: row tiles of a chunk, pairs and items in front of each thread's requests.
template <int NT>
struct Cut {
    int64_t pairs[NT + 1], items[NT + 1], warp_sum[2][NT / 32];
    int64_t chunk;
    int R, seg;
    template <typename F>
    __device__ void scan(const Args &w, F f, bool &clipped)  // f: request -> (pairs, items)
    {
        const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
        int64_t p = 0, n = 0;
        for (int64_t r = (int64_t)tid * seg; r < (int64_t)(tid + 1) * seg && r < R; ++r) {
            const Spread s = spread_of(w, (int)r, clipped);
            p += s.pairs;
            n += f(s);
        }
        const int64_t ip = vtk_warp_incl_scan(p), in = vtk_warp_incl_scan(n);
        if (lane == 31) { warp_sum[0][warp] = ip; warp_sum[1][warp] = in; }
        __syncthreads();
        int64_t bp = 0, bn = 0;
        for (int v = 0; v < warp; ++v) { bp += warp_sum[0][v]; bn += warp_sum[1][v]; }
        pairs[tid + 1] = bp + ip;
        items[tid + 1] = bn + in;
        if (tid == 0) pairs[0] = items[0] = 0;
        __syncthreads();
    }
    __device__ void make(const Args &w, bool &clipped)
    {
        const VtkAttnArgs &a = w.w.at;
        int n = *a.num_requests;
        clipped |= n < 0 || n > a.max_requests;
        n = n < 0 ? 0 : (n > a.max_requests ? a.max_requests : n);
        if (threadIdx.x == 0) { R = n; seg = (n + NT - 1) / NT; }
        __syncthreads();
        scan(w, [&](const Spread &s) { return s.pairs * s.tiles * a.hkv; }, clipped);
        // about eight items a CTA, of 4 to 32 row tiles, as many as the workspace has room for
        int64_t c = items[NT] / ((int64_t)w.grid * 8);
        c = c < 4 ? 4 : (c > 32 ? 32 : c);
        for (;; c = c * 2 > 32 * WP_WORDS ? 32 * WP_WORDS : c * 2) {
            bool again = false;
            scan(w, [&](const Spread &s) { return s.pairs * chunks_of(s, c) * a.hkv; }, again);
            if (items[NT] <= w.max_parts || c >= 32 * WP_WORDS) break;
        }
        if (threadIdx.x == 0) chunk = c;
        __syncthreads();
    }
    // the request of pair (or item) `i`, and what is left of i there
    __device__ int find(const Args &w, const int64_t (&prefix)[NT + 1], bool by_items, int64_t &i, int64_t &items_before, Spread &s) const
    {
        int lo = 0, hi = NT;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (prefix[mid] <= i) lo = mid; else hi = mid;
        }
        i -= prefix[lo];
        items_before = items[lo];
        for (int r = lo * seg;; ++r) {
            bool c = false;
            s = spread_of(w, r, c);
            const int64_t n = s.pairs * chunks_of(s, chunk) * w.w.at.hkv, here = by_items ? n : s.pairs;
            if (i < here) return r;
            i -= here;
            items_before += n;
        }
    }
};

struct Item {
    int none, kv, q0, qn, first, n;      // query tokens of the request; first cache entry and number of tokens
    int tile0, count;                    // first row tile of the chunk; how many see something
    int64_t base, ticket;
    uint32_t sees[WP_WORDS];             // which
};

struct Meta {                            // a tile of query rows
    int pmin, pmax, whole;               // whole: every row of the tile is there and saw something
    alignas(16) float lse2[TC_TILE];     // minus the logarithm to base 2
    alignas(16) int pos[TC_TILE];        // -1: the row adds nothing
    alignas(16) float scale[TC_TILE];    // bf16 queries over 4-bit keys: factor of the row's scores
};

// 16 columns of a thread's accumulator row: what token `id` gets from 16 query rows.  A row at p sees it when 0 <= p - id < reach.
template <bool SCALED, bool MASKED>
__device__ __forceinline__ void sum_columns(float c, const Meta &m, const uint32_t (&s)[16], const float4 (&l)[4], int col, int id, uint32_t reach, float2 (&sum)[2])
{
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
        float4 f = make_float4(c, c, c, c);
        if (SCALED) {
            f = *reinterpret_cast<const float4 *>(&m.scale[col + i]);
            f.x *= c; f.y *= c; f.z *= c; f.w *= c;
        }
        float2 y0 = fma2(make_float2(__uint_as_float(s[i]), __uint_as_float(s[i + 1])), make_float2(f.x, f.y), make_float2(l[i / 4].x, l[i / 4].y));
        float2 y1 = fma2(make_float2(__uint_as_float(s[i + 2]), __uint_as_float(s[i + 3])), make_float2(f.z, f.w), make_float2(l[i / 4].z, l[i / 4].w));
        y0.x = vtk_exp2(y0.x); y0.y = vtk_exp2(y0.y);
        y1.x = vtk_exp2(y1.x); y1.y = vtk_exp2(y1.y);
        if (MASKED) {
            const int4 p = *reinterpret_cast<const int4 *>(&m.pos[col + i]);
            y0.x = (uint32_t)p.x - (uint32_t)id < reach ? y0.x : 0.f;
            y0.y = (uint32_t)p.y - (uint32_t)id < reach ? y0.y : 0.f;
            y1.x = (uint32_t)p.z - (uint32_t)id < reach ? y1.x : 0.f;
            y1.y = (uint32_t)p.w - (uint32_t)id < reach ? y1.y : 0.f;
        }
        sum[0] = add2(sum[0], y0);
        sum[1] = add2(sum[1], y1);
    }
}

// The sum over a tile's query rows.  free: none of them needs a mask (the columns behind them do).  Two loops of two steps: a branch at
// every mask would keep the compiler from overlapping the chains of loads, products and exponentials (6500 cycles a tile instead of
// 3700, in an earlier form), and what is unrolled further is fetched for longer than short items last.
// release: called when the last columns are in registers, so that the next product need not wait for their exponentials.
template <bool SCALED, typename F>
__device__ __forceinline__ float row_sum(const VtkAttnArgs &a, const Meta &m, uint32_t src, int id, uint32_t reach, int rows, bool free, F release)
{
    float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
    uint32_t v[2][16];
    tc_ld16(src, v[0]);
    auto step = [&](int col, uint32_t (&now)[16], uint32_t (&then)[16], auto masked) {
        float4 l[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) l[i] = *reinterpret_cast<const float4 *>(&m.lse2[col + 4 * i]);
        tc_wait_ld(now);
        if (col + 16 < rows) tc_ld16(src + col + 16, then);
        else release();
        sum_columns<SCALED, decltype(masked)::value>(a.scale_log2, m, now, l, col, id, reach, sum);
    };
    int col = 0;
#pragma unroll 1
    for (; free && col + 32 <= rows; col += 32) {
        step(col, v[0], v[1], std::false_type());
        step(col + 16, v[1], v[0], std::false_type());
    }
#pragma unroll 1
    for (; col < rows; col += 32) {
        step(col, v[0], v[1], std::true_type());
        if (col + 16 < rows) step(col + 16, v[1], v[0], std::true_type());
    }
    sum[0] = add2(sum[0], sum[1]);
    return sum[0].x + sum[0].y;
}

template <int D>
struct Shared {
    static constexpr int Q = D == 128 ? 2 : 4;               // tiles of queries
    uint8_t k[2][2][D / 64][TC_TILE * 128];
    uint8_t q[Q][D / 64][TC_TILE * 128];
    Meta meta[WP_META];
    Item item[2];
    float other[2][WP_PAIR];             // the second group's sums of an item
    Cut<WP_NT> cut;
    uint64_t item_full[2], item_empty[2], meta_full[WP_META], meta_empty[WP_META], scale_full[WP_META], k_full[2], k_empty[2], other_full[2];
    uint64_t q_full[Q], q_empty[Q], s_full[2][2], s_empty[2][2], drain[2];                // scores: of 128 tokens, group
    uint32_t tmem;
    int abort;
};

template <int D, bool FP4, typename Act>
__global__ void __launch_bounds__(WP_NT, 1) weights_prompt_kernel(const __grid_constant__ Args w, const __grid_constant__ CUtensorMap queries)
{
    using Mma = typename std::conditional<FP4, VtkFp16, Act>::type;
    constexpr int PIECES = D / 8, PANEL = TC_TILE * 128, Q = Shared<D>::Q;
    constexpr bool SCALED = FP4 && Act::kind == VTOKEN_KV_BF16;
    const VtkAttnArgs &a = w.w.at;
    extern __shared__ uint8_t raw[];
    Shared<D> &sh = *reinterpret_cast<Shared<D> *>(raw + ((1024 - (vtk_smem_u32(raw) & 1023)) & 1023));
    vtk_release_successor();
    vtk_wait_for_predecessor();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid == 0) {
        for (int i = 0; i < 2; ++i) {
            vtk_mbar_init(&sh.item_full[i], 1); vtk_mbar_init(&sh.item_empty[i], WP_SUMS + 4 + 2 + 1);
            vtk_mbar_init(&sh.k_full[i], FP4 ? 4 : 128); vtk_mbar_init(&sh.k_empty[i], 2); vtk_mbar_init(&sh.other_full[i], 8); vtk_mbar_init(&sh.drain[i], 1);
            for (int b = 0; b < 2; ++b) { vtk_mbar_init(&sh.s_full[i][b], 1); vtk_mbar_init(&sh.s_empty[i][b], 4); }
        }
        for (int i = 0; i < WP_META; ++i) { vtk_mbar_init(&sh.meta_full[i], 1); vtk_mbar_init(&sh.meta_empty[i], 8 + (SCALED ? 4 : 0)); vtk_mbar_init(&sh.scale_full[i], 4); }
        for (int i = 0; i < Q; ++i) { vtk_mbar_init(&sh.q_full[i], SCALED ? 4 : 1); vtk_mbar_init(&sh.q_empty[i], 2); }
        sh.abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == WP_MMA) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(vtk_smem_u32(&sh.tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    bool clipped = false;
    sh.cut.make(w, clipped);
    if (blockIdx.x == 0 && (clipped || (tid == 0 && sh.cut.items[WP_NT] > w.max_parts))) atomicOr(a.flags, (uint32_t)VTOKEN_FLAG_CAPACITY);
    tc_before_sync();
    __syncthreads();
    tc_after_sync();
    const uint32_t tmem = sh.tmem;
    if (!SCALED && tid == WP_ROWS * 32) asm volatile("prefetch.tensormap [%0];" ::"l"(&queries) : "memory");
    const int rows = w.tokens * a.group;                     // of a tile
    constexpr uint32_t IDESC = (1u << 4) | ((Mma::kind == VTOKEN_KV_BF16 ? 1u : 0u) << 7) | ((Mma::kind == VTOKEN_KV_BF16 ? 1u : 0u) << 10) |
                               ((uint32_t)(TC_TILE >> 4) << 24) | ((uint32_t)(TC_TILE >> 3) << 17);
    auto wait_phase = [&](uint64_t *bar, uint32_t parity, uint64_t limit) {
        return (bool)__all_sync(0xffffffffu, vtk_mbar_wait(bar, parity, limit, &sh.abort, 1));
    };
    auto wait = [&](uint64_t *bar, uint32_t count, uint32_t ring) { return wait_phase(bar, (count / ring) & 1, w.limit_ns); };     // the count-th phase of a ring's barrier
    auto wait_empty = [&](uint64_t *bar, uint32_t count, uint32_t ring) { return wait_phase(bar, ((count / ring) & 1) ^ 1, w.limit_ns); };
    auto arrive = [&](uint64_t *bar) {
        __syncwarp();
        if (lane == 0) vtk_mbar_arrive(bar);
    };
    auto stalled = [&](const Item &it) {
#ifdef VTOKEN_CHECKED
        return it.ticket == w.stall;
#else
        return false;
#endif
    };

    // Every role runs over the items and, within one, over the row tiles that see something of it; the tiles are counted throughout.
    uint32_t n_item = 0, n_tile = 0, n_key = 0;
    auto each_item = [&](auto &&body) {
        for (;; ++n_item) {
            const int s = n_item & 1;
            if (!wait(&sh.item_full[s], n_item, 2)) return;
            const Item &it = sh.item[s];
            if (it.none || !body(it)) return;
            arrive(&sh.item_empty[s]);
            ++n_key;
        }
    };

    if (warp < WP_SUMS) {
        // ================= exponentials: thread = token =================
        const int group = warp >> 3, x = (warp >> 2) & 1, row = tid & 127, at = x * TC_TILE + row;
        const uint32_t src = tmem + ((uint32_t)(warp & 3) << 21) + (x * 2 + group) * TC_TILE;         // 32 lanes a warp
        uint32_t n_mine = 0;
        bool bad_slot = false;
        each_item([&](const Item &it) {
            int id = INT32_MAX;
            bool there = false;
            if (at < it.n) {
                const int64_t e = it.base + it.first + at, slot = a.cache_slots[e];
                there = slot >= 0 && slot < a.slots_per_layer;
                bad_slot |= slot >= a.slots_per_layer;
                if (there) id = a.cache_ids.null() ? it.first + at : a.cache_ids[e];
            }
            const bool every = __all_sync(0xffffffffu, there);
            const int id_lo = __reduce_min_sync(0xffffffffu, id), id_hi = __reduce_max_sync(0xffffffffu, there ? id : -1);
            const bool mine = x * TC_TILE < it.n;                                // (uniform)
            const uint32_t reach = a.window == 0 || id < a.sinks ? 0x80000000u : (uint32_t)a.window;
            const int count = it.count;
            float total = 0.f;
            for (int j = (int)((n_tile ^ group) & 1); j < count; j += 2) {       // (tiles of the other group pass by)
                const uint32_t n = n_tile + j, slot = n % WP_META;
                if (!wait(&sh.meta_full[slot], n, WP_META)) return false;
                const Meta &m = sh.meta[slot];
                if (mine) {
                    if (!wait(&sh.s_full[x][group], n_mine, 1)) return false;
                    if (SCALED && !wait(&sh.scale_full[slot], n, WP_META)) return false;
                    tc_after_sync();
                    const bool some = m.pmax >= id_lo && (a.window == 0 || id_hi > vtk_floor(m.pmin, a.window) || id_lo < a.sinks);
                    const bool full = every && m.whole && id_hi <= m.pmin && (id_lo > vtk_floor(m.pmax, a.window) || id_hi < a.sinks);
                    auto release = [&]() {
                        tc_before_sync();
                        arrive(&sh.s_empty[x][group]);
                    };
                    if (some) total += row_sum<SCALED>(a, m, src, id, reach, rows, full, release);
                    else release();
                    ++n_mine;
                }
                arrive(&sh.meta_empty[slot]);
            }
            n_tile += count;
            const int turn = n_item & 1;
            if (group == 1) {
                sh.other[turn][at] = total;
                arrive(&sh.other_full[turn]);
            } else {
                if (!wait(&sh.other_full[turn], n_item, 2)) return false;
                if (mine) w.parts[it.ticket * WP_PAIR + at] = total + sh.other[turn][at];
            }
            return true;
        });
        if (bad_slot) atomicOr(a.flags, (uint32_t)VTOKEN_FLAG_BAD_SLOT);
    } else if (warp < WP_COPY + 4) {
        // ================= copies =================
        const int pt = tid - WP_COPY * 32;
        each_item([&](const Item &it) {
            const int kb = n_key & 1;
            if (!wait_empty(&sh.k_empty[kb], n_key, 2)) return false;
            auto slot_of = [&](int at) {
                const int64_t slot = at < it.n ? a.cache_slots[it.base + it.first + at] : -1;
                return slot < a.slots_per_layer ? (int)slot : -1;
            };
            for (int x = 0; x < (it.n > TC_TILE ? 2 : 1); ++x) {
                const uint32_t dst = vtk_smem_u32(sh.k[kb][x]);
                if (!FP4) {
                    constexpr int ROWS = PIECES;             // PIECES threads a row, each with the same number of consecutive rows
                    const int piece = pt % PIECES, row0 = pt / PIECES * ROWS;
                    const uint8_t *base = a.k_rows + ((int64_t)it.kv * D + 8 * piece) * 2;
                    const int mine = slot_of(x * TC_TILE + pt);                  // (a warp's threads have 32 rows)
#pragma unroll
                    for (int i = 0; i < ROWS; ++i) {
                        const int slot = __shfl_sync(0xffffffffu, mine, lane / PIECES * ROWS + i);
                        cp_async16(dst + swizzled(row0 + i, piece), base + (int64_t)(slot < 0 ? 0 : slot) * a.row_bytes, slot >= 0);
                    }
                } else {
                    constexpr int QW = D / 32;               // four threads a token, a quarter of its codes and scales each
                    const int part = pt & 3;
                    uint32_t code[4][QW], sc[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int64_t slot = slot_of(x * TC_TILE + (pt >> 2) + 32 * i);
#pragma unroll
                        for (int k = 0; k < QW; ++k) code[i][k] = 0;
                        sc[i] = 0;
                        if (slot < 0) continue;
                        const uint8_t *src = a.k_rows + slot * a.row_bytes, *codes = src + it.kv * (D / 2) + part * (D / 8);
                        const uint8_t *scales = src + a.hkv * (D / 2) + it.kv * (D / 16) + part * (D / 64);
                        if (D == 128) {
                            const uint4 q4 = vtk_ldg16(codes);
                            code[i][0] = q4.x; code[i][1] = q4.y; code[i][QW - 2] = q4.z; code[i][QW - 1] = q4.w;
                            sc[i] = __ldg(reinterpret_cast<const uint16_t *>(scales));
                        } else {
                            const uint2 q2 = __ldg(reinterpret_cast<const uint2 *>(codes));
                            code[i][0] = q2.x; code[i][1] = q2.y;
                            sc[i] = __ldg(scales);
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t two_scales = vtk_scales_to_half2(sc[i]);
#pragma unroll
                        for (int k = 0; k < QW; ++k)
                            st_shared16(dst + swizzled((pt >> 2) + 32 * i, part * QW + k), vtk_expand8(code[i][k], __byte_perm(two_scales, 0, k < 2 ? 0x1010 : 0x3232)));
                    }
                }
            }
            if (!FP4) {
                cp_arrive(&sh.k_full[kb]);
            } else {
                async_proxy_fence();
                arrive(&sh.k_full[kb]);
            }
            if (!SCALED) return true;
            // bf16 queries in half precision: see attention.cu
            const int tok = pt / a.group, head = pt % a.group, words = (it.count > 0 ? WP_WORDS : 0);
            bool first = true;
            for (int word = 0; word < words; ++word)
                for (uint32_t left = it.sees[word]; left != 0; left &= left - 1, ++n_tile, first = false) {
                    const uint32_t slot = n_tile % WP_META, stage = n_tile % Q;
                    if (!wait(&sh.meta_full[slot], n_tile, WP_META)) return false;
                    const int64_t at = (int64_t)(it.tile0 + 32 * word + __ffs(left) - 1) * w.tokens + tok;
                    const bool there = pt < rows && at < it.qn;
                    const uint16_t *from = a.q;
                    if (there) from += (it.q0 + at) * a.q_stride + (int64_t)(it.kv * a.group + head) * D;
                    float top = 0.f, v[8];
                    for (int i = 0; i < PIECES; ++i) {
                        vtk_unpack8<VtkBf16>(there ? *reinterpret_cast<const uint4 *>(from + 8 * i) : make_uint4(0, 0, 0, 0), v);
#pragma unroll
                        for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(v[e]));
                    }
                    int e2 = (int)(__float_as_uint(top) >> 23) - 127;
                    e2 = 14 - (e2 < -100 ? -100 : e2);
                    const float up = __uint_as_float((uint32_t)(127 + e2) << 23);
                    sh.meta[slot].scale[pt] = __uint_as_float((uint32_t)(127 - e2) << 23);
                    arrive(&sh.scale_full[slot]);
                    arrive(&sh.meta_empty[slot]);
                    if (!wait_empty(&sh.q_empty[stage], n_tile, Q)) return false;
                    const uint32_t dst = vtk_smem_u32(sh.q[stage]);
                    for (int i = 0; i < PIECES; ++i) {
                        vtk_unpack8<VtkBf16>(there ? *reinterpret_cast<const uint4 *>(from + 8 * i) : make_uint4(0, 0, 0, 0), v);
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] *= up;
                        st_shared16(dst + swizzled(pt, i), vtk_pack8<VtkFp16>(v));
                    }
                    async_proxy_fence();
                    if (!(first && stalled(it)) || pt >= 32) arrive(&sh.q_full[stage]);
                }
            return true;
        });
        if (!FP4) cp_wait_all();
    } else if (warp < WP_MMA + 2) {
        // ================= products =================
        const bool one = tc_elect();
        const int x = warp - WP_MMA;
        uint32_t n_acc[2] = {0, 0};
        each_item([&](const Item &it) {
            const bool mine = x == 0 || it.n > TC_TILE;
            const int kb = n_key & 1, count = it.count;
            if (!wait(&sh.k_full[kb], n_key, 2)) return false;
            const uint64_t kd = operand(vtk_smem_u32(sh.k[kb][x]));
            for (int j = 0; j < count; ++j, ++n_tile) {
                const int stage = n_tile % Q, b = n_tile & 1;
                if (!wait(&sh.q_full[stage], n_tile, Q)) return false;           // (also where there is nothing to do: not to run ahead)
                if (mine) {
                    if (!wait_empty(&sh.s_empty[x][b], n_acc[b], 1)) return false;
                    async_proxy_fence();
                    tc_after_sync();
                    const uint64_t qd = operand(vtk_smem_u32(sh.q[stage]));
                    const uint32_t acc = tmem + (x * 2 + b) * TC_TILE;
#pragma unroll
                    for (int k = 0; k < D / 16; ++k) {
                        const uint32_t off = ((k / 4) * PANEL + (k % 4) * 32) >> 4;
                        tc_mma_ss(one, acc, kd + off, qd + off, IDESC, k > 0);
                    }
                    tc_commit(one, &sh.s_full[x][b]);
                    ++n_acc[b];
                }
                tc_commit(one, &sh.q_empty[stage]);
            }
            tc_commit(one, &sh.k_empty[kb]);
            return true;
        });
        // what was issued ends before the tensor memory goes
        tc_commit(one, &sh.drain[x]);
        const uint64_t t0 = vtk_global_ns();
        while (!vtk_mbar_try(&sh.drain[x], 0) && vtk_global_ns() - t0 < WP_DRAIN_NS) {}
        __syncwarp();
    } else if (warp == WP_DRAW) {
        // ================= items =================
        for (bool more = true; more; ++n_item) {
            Item it;                                         // (its words are written below)
            uint32_t mine = 0;                               // lane i: word i
            for (;;) {
                int64_t idx = 0;
                if (lane == 0) idx = (int64_t)atomicAdd(w.tickets, 1u);
                idx = __shfl_sync(0xffffffffu, idx, 0);
                it.none = 1;
                it.ticket = idx;
                it.count = 0;
                mine = 0;
                if (idx >= sh.cut.items[WP_NT] || idx >= w.max_parts) break;
                Spread sp;
                int64_t left = idx, before;
                sh.cut.find(w, sh.cut.items, true, left, before, sp);
                const int64_t chunks = chunks_of(sp, sh.cut.chunk);
                it.none = 0;
                it.kv = (int)(left % a.hkv);
                left /= a.hkv;
                const int64_t c = left % chunks, pair = left / chunks;
                it.tile0 = (int)(c * sh.cut.chunk);
                const int tiles = (int)((c + 1) * sh.cut.chunk < sp.tiles ? sh.cut.chunk : sp.tiles - c * sh.cut.chunk);
                it.q0 = sp.q0;
                it.qn = sp.qn;
                it.first = (int)(pair * WP_PAIR);
                it.n = sp.len - it.first < WP_PAIR ? sp.len - it.first : WP_PAIR;
                it.base = sp.base;
                const int id_lo = a.cache_ids.null() ? it.first : a.cache_ids[it.base + it.first];
                const int id_hi = a.cache_ids.null() ? it.first + it.n - 1 : a.cache_ids[it.base + it.first + it.n - 1];
                for (int word = 0; 32 * word < tiles; ++word) {
                    int pmin = INT32_MAX, pmax = INT32_MIN;
                    const int tile = 32 * word + lane;
                    if (tile < tiles) {
                        const int64_t t0 = (int64_t)(it.tile0 + tile) * w.tokens, t1 = t0 + w.tokens < it.qn ? t0 + w.tokens : it.qn;
                        const int32_t *pos = a.positions.at(it.q0 + t0, t1 - t0);
                        const int n = (int)(t1 - t0);
#pragma unroll 16
                        for (int t = 0; t < n; ++t) {
                            const int p = pos[t];
                            pmin = p < pmin ? p : pmin;
                            pmax = p > pmax ? p : pmax;
                        }
                    }
                    const bool sees = tile < tiles && pmax >= id_lo && (a.window == 0 || id_hi > vtk_floor(pmin, a.window) || id_lo < a.sinks);
                    const uint32_t found = __ballot_sync(0xffffffffu, sees);
                    it.count += __popc(found);
                    if (lane == word) mine = found;
                }
                if (it.count > 0) break;
                for (int i = lane; i < WP_PAIR; i += 32) w.parts[idx * WP_PAIR + i] = 0.f;       // nobody sees anything of it
            }
            more = !it.none;
            const int s = n_item & 1;
            // (an item's roles wait once a tile, and each of those waits has the limit)
            if (!wait_phase(&sh.item_empty[s], ((n_item / 2) & 1) ^ 1, w.limit_ns * (uint64_t)(sh.cut.chunk + 2))) break;
            Item &to = sh.item[s];
            to.sees[lane] = mine;
            if (lane == 0) {
                to.none = it.none; to.kv = it.kv; to.q0 = it.q0; to.qn = it.qn; to.first = it.first; to.n = it.n;
                to.tile0 = it.tile0; to.count = it.count; to.base = it.base; to.ticket = it.ticket;
            }
            arrive(&sh.item_full[s]);
        }
    } else {
        // ================= rows: positions, logarithms, queries =================
        static_assert(WP_WORDS == 32 && WP_ROWS == WP_NT / 32 - 1, "a lane a word; the last warp");
        int tok[4];                                          // of rows lane, lane + 32, ...; -1: there is none
        int64_t lse_of[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            tok[i] = 32 * i + lane < rows ? (32 * i + lane) / a.group : -1;
            lse_of[i] = (int64_t)(tok[i] < 0 ? 0 : tok[i]) * a.hq + (32 * i + lane) % a.group;
        }
        struct Values { float l[4]; int p[4]; };
        uint32_t started = 0, skipped = UINT32_MAX;          // copies, and one that was left out
        each_item([&](const Item &it) {
            const int count = it.count;
            int word = -1;
            uint32_t left = 0;
            auto next_tile = [&]() {                         // (`count` bits are set; the search ends whatever is found there)
                while (left == 0 && word + 1 < WP_WORDS) left = it.sees[++word];
                const int64_t t0 = (int64_t)(it.tile0 + (left == 0 ? 0 : 32 * word + __ffs(left) - 1)) * w.tokens;
                left &= left - 1;
                return t0;
            };
            auto fetch = [&](int64_t t0) {                   // (without a branch, so that all eight are on their way at once)
                Values v;
                const float *lse = w.w.lse_in + (it.q0 + t0) * a.hq + it.kv * a.group;
                const int32_t *pos = a.positions.at(it.q0 + t0);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const bool there = tok[i] >= 0 && t0 + tok[i] < it.qn;
                    v.l[i] = lse[there ? lse_of[i] : 0];
                    v.p[i] = pos[there ? tok[i] : 0];
                    if (!there) {
                        v.l[i] = -INFINITY;
                        v.p[i] = INT32_MIN;
                    }
                }
                return v;
            };
            int64_t t0 = next_tile();
            Values now = fetch(t0);
            for (int j = 0; j < count; ++j, ++n_tile) {
                const int64_t at = t0;
                Values then = now;
                if (j + 1 < count) {
                    t0 = next_tile();
                    then = fetch(t0);
                }
                const int stage = n_tile % Q, slot = n_tile % WP_META;
                if (!SCALED) {
                    if (!wait_empty(&sh.q_empty[stage], n_tile, Q)) return false;
                    if (j == 0 && stalled(it)) skipped = n_tile;
                    started = n_tile + 1;
                    if (lane == 0 && n_tile != skipped) {
                        asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(vtk_smem_u32(&sh.q_full[stage])), "r"(rows * D * 2) : "memory");
#pragma unroll
                        for (int panel = 0; panel < D / 64; ++panel)
                            asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                                         ::"r"(vtk_smem_u32(sh.q[stage][panel])), "l"(&queries), "r"(64 * panel), "r"(it.kv * a.group), "r"((int)(it.q0 + at)),
                                           "r"(vtk_smem_u32(&sh.q_full[stage])) : "memory");
                    }
                    __syncwarp();
                }
                int pmin = INT32_MAX, pmax = INT32_MIN;
                bool whole = true;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (tok[i] >= 0 && at + tok[i] < it.qn) pmin = now.p[i] < pmin ? now.p[i] : pmin;
                    pmax = now.p[i] > pmax ? now.p[i] : pmax;
                    whole &= tok[i] < 0 || now.l[i] != -INFINITY;
                }
                pmin = __reduce_min_sync(0xffffffffu, pmin);
                pmax = __reduce_max_sync(0xffffffffu, pmax);
                whole = __all_sync(0xffffffffu, whole);
                if (!wait_empty(&sh.meta_empty[slot], n_tile, WP_META)) return false;
                Meta &m = sh.meta[slot];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    m.lse2[32 * i + lane] = now.l[i] * -1.4426950408889634f;
                    m.pos[32 * i + lane] = now.l[i] == -INFINITY || now.p[i] < 0 ? -1 : (now.p[i] < INT32_MAX - 1 ? now.p[i] : INT32_MAX - 1);   // (INT32_MAX: what is not there)
                }
                if (lane == 0) {
                    m.pmin = pmin;
                    m.pmax = pmax;
                    m.whole = whole;
                }
                arrive(&sh.meta_full[slot]);
                now = then;
            }
            return true;
        });
        if (!SCALED) {                                       // (after an abort: copies in flight land before the memory goes)
            const uint64_t t0 = vtk_global_ns();
            for (uint32_t i = 0; i < (uint32_t)Q && i < started; ++i) {
                const uint32_t n = started - 1 - i;
                while (n != skipped && *(volatile int *)&sh.abort != 0 && !vtk_mbar_try(&sh.q_full[n % Q], (n / Q) & 1) && vtk_global_ns() - t0 < WP_DRAIN_NS) {}
            }
            __syncwarp();
        }
    }
    __syncthreads();
    if (tid == 0) {
        if (sh.abort) atomicOr(a.flags, (uint32_t)VTOKEN_FLAG_TIMEOUT);
        __threadfence();
        if (atomicAdd(w.tickets + 1, 1u) == gridDim.x - 1) { w.tickets[0] = 0; w.tickets[1] = 0; }
    }
    if (warp == WP_MMA) {
        tc_after_sync();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
    }
}

// sums of chunks and heads, in their order, and the scores before
__global__ void __launch_bounds__(WP_JOIN_NT) weights_join_kernel(const __grid_constant__ Args w)
{
    static_assert(WP_JOIN_NT == WP_PAIR, "thread = token");
    const VtkAttnArgs &a = w.w.at;
    __shared__ Cut<WP_JOIN_NT> cut;
    vtk_release_successor();
    vtk_wait_for_predecessor();
    bool clipped = false, bad_id = false;
    cut.make(w, clipped);
    for (int64_t p = blockIdx.x; p < cut.pairs[WP_JOIN_NT]; p += gridDim.x) {
        Spread s;
        int64_t pair = p, before;
        const int r = cut.find(w, cut.pairs, false, pair, before, s);
        const int64_t at = pair * WP_PAIR + threadIdx.x;
        if (at >= s.len) continue;
        const int id = a.cache_ids.null() ? (int)at : a.cache_ids[s.base + at];
        const int64_t t1 = a.tt_offsets[r + 1], end = t1 > a.max_tokens ? a.max_tokens : t1;
        if (id < 0 || id >= end - s.base) { bad_id = true; continue; }
        const int64_t n = chunks_of(s, cut.chunk) * a.hkv, first = before + pair * n;
        float y = 0.f;
        for (int64_t i = first; i < first + n && i < w.max_parts; ++i) y += __ldcg(w.parts + i * WP_PAIR + threadIdx.x);
        if (!w.w.prev.null()) y = fmaf(w.w.decay, w.w.prev[s.base + id], y);
        w.w.scores[s.base + id] = y;
    }
    if (bad_id) atomicOr(a.flags, (uint32_t)VTOKEN_FLAG_BAD_VICTIM);
}

// query tokens of a row tile: whole ones, so that a tile is one box of the queries
int tokens_of(const vtoken_heads *heads)
{
    const int group = heads->num_q_heads / heads->num_kv_heads;
    return group < TC_TILE ? TC_TILE / group : 1;
}

// what the items of a call can be: chunks of 32 * WP_WORDS row tiles everywhere, and some more where there are few
int64_t parts_of(const vtoken_ctx *ctx, const vtoken_heads *heads, int64_t max_query_tokens)
{
    const int64_t tiles = max_query_tokens / tokens_of(heads) + 1, chunks = (tiles + 32 * WP_WORDS - 1) / (32 * WP_WORDS);
    return ((ctx->cfg.max_tokens + WP_PAIR - 1) / WP_PAIR + ctx->cfg.max_requests) * heads->num_kv_heads * chunks + (int64_t)ctx->num_sms * 16;
}

// the queries as [tokens][heads][dimensions]; a box is 64 dimensions of a key head's query heads of a tile's tokens
cudaError_t map_queries(const VtkAttnArgs &a, int head_dim, bool bf16, int tokens, CUtensorMap *map)
{
    using Encode = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    static std::atomic<Encode> known{nullptr};
    Encode encode = known.load(std::memory_order_relaxed);
    if (encode == nullptr) {
        void *f = nullptr;
        cudaDriverEntryPointQueryResult found;
        const cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found);
        if (e != cudaSuccess) return e;
        if (found != cudaDriverEntryPointSuccess || f == nullptr) return cudaErrorNotSupported;
        encode = (Encode)f;
        known.store(encode, std::memory_order_relaxed);
    }
    const cuuint64_t size[3] = {(cuuint64_t)head_dim, (cuuint64_t)a.hq, (cuuint64_t)a.max_query_tokens};
    const cuuint64_t stride[2] = {(cuuint64_t)head_dim * 2, (cuuint64_t)a.q_stride * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)a.group, (cuuint32_t)tokens}, step[3] = {1, 1, 1};
    const CUresult r = encode(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<uint16_t *>(a.q), size, stride, box, step,
                              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

template <int D, bool FP4, typename Act>
int launch(vtoken_ctx *ctx, const Args &w, cudaStream_t st)
{
    constexpr int smem = (int)sizeof(Shared<D>) + 1024;
    static_assert(smem <= 232448, "shared memory of a CTA");
    constexpr bool bf = Act::kind == VTOKEN_KV_BF16;
    alignas(64) CUtensorMap map = {};
    if (!(FP4 && bf)) VTK_CUDA(ctx, map_queries(w.w.at, D, bf, w.tokens, &map));
    auto kernel = weights_prompt_kernel<D, FP4, Act>;
    static std::atomic<int> allowed{-1};                     // the device that knows of this kernel's shared memory
    VTK_CUDA(ctx, vtk_allow_smem(ctx, allowed, (const void *)kernel, smem));
    VTK_CUDA(ctx, vtk_launch_dependent(ctx, kernel, dim3(w.grid), dim3(WP_NT), smem, st, w, map));
    VTK_CUDA(ctx, vtk_launch_dependent(ctx, weights_join_kernel, dim3(ctx->num_sms * 2), dim3(WP_JOIN_NT), 0, st, w));
    VTK_CUDA(ctx, cudaGetLastError());
    return VTOKEN_OK;
}

template <int D>
int launch_by_type(vtoken_ctx *ctx, const vtoken_heads *h, const Args &w, cudaStream_t st)
{
    if (h->kv_type == VTOKEN_KV_FP4) return h->act_type == VTOKEN_KV_BF16 ? launch<D, true, VtkBf16>(ctx, w, st) : launch<D, true, VtkFp16>(ctx, w, st);
    return h->act_type == VTOKEN_KV_BF16 ? launch<D, false, VtkBf16>(ctx, w, st) : launch<D, false, VtkFp16>(ctx, w, st);
}

}  // namespace

int64_t vtk_weights_prompt_workspace(const vtoken_ctx *ctx, const vtoken_heads *heads, int32_t max_query_tokens)
{
    return vtk_workspace_zeros(ctx) + parts_of(ctx, heads, max_query_tokens) * WP_PAIR * 4;
}

int vtk_launch_weights_prompt(vtoken_ctx *ctx, const vtoken_heads *heads, const VtkWeightsArgs &weights, void *workspace, cudaStream_t st)
{
    Args w;
    w.w = weights;
    w.tickets = (uint32_t *)workspace;
    w.parts = (float *)((uint8_t *)workspace + vtk_workspace_zeros(ctx));     // (attention counts in front of them)
    w.max_parts = parts_of(ctx, heads, weights.at.max_query_tokens);
    w.row_limit = weights.at.row_limit;
    w.grid = ctx->num_sms;
    w.tokens = tokens_of(heads);
    w.limit_ns = (uint64_t)ctx->wait_limit_ns;
    w.stall = ctx->stall_item;
    return heads->head_dim == 128 ? launch_by_type<128>(ctx, heads, w, st) : launch_by_type<64>(ctx, heads, w, st);
}
