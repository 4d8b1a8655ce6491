// Attention of many query rows per request (prompts and chunks of prompts) over the slot cache, on the fifth
// generation tensor cores.
//
// 4 * D flops and one exponential per pair: 128 x 128 pairs of D 128 take the tensor pipe (8192 flops a cycle) as long as the
// SM's 16 exponentials a cycle, 2048 cycles for two row tiles and one of K and V.  Measured, those take about 5000, with no unit near
// its limit (4096 tokens: tensor pipe 34 %, exponentials 35 %, issue slots 33 %, DRAM 3 %): the bound is the chain of hand-overs from
// copy to scores to softmax to outputs to the free stage, and the barrier between items.  8192 tokens, 32 heads over 8: 655 to 687 us
// from machine to machine, 800 to 840 TFLOP/s; at an earlier step without exponentials, softmax, copies or most of the products each 640 to 700.
// One CTA per SM takes items (request, two tiles of 128 query rows, key head); the rows of a tile are the query
// tokens of the request times the heads of the group, so a K or V tile is read once for all of them, and the two
// row tiles share it again.  Roles, 16 warps:
//   0 .. 3, 4 .. 7   softmax of row tile 0 and 1, one thread a row: scores from tensor memory, running maximum (moved
//                    only when a score passes it by 2^8), exponentials, P as 16 bits back into the scores' columns (rounded once, as
//                    a second product for the rest would double the tensor work: error against 64 bits 0.0021 for 0.0016, bf16; behind
//                    shared prefixes, whose rows are not bound by it, twice)
//   8 .. 11          producers: rows of Q, K and V gathered by slot into 128-byte-swizzled tiles, 16 bytes a thread by
//                    cp.async, or 4-bit rows expanded to half precision in registers on the way
//   12               one thread issues every tcgen05.mma: S = Q K^T (both operands from shared memory, K-major),
//                    O += P V (P from tensor memory, V as it lies: token rows, the MN-major operand)
//   13               looks up the next item while this one runs
//   14, 15           look up the slots and ids of the tiles, and which rows of a tile see all of them
// While the softmax of one row tile runs, the products of the other keep the tensor pipe busy.
// Tensor memory: 2 x 128 columns of scores (P overwrites the first half of its own), 2 x D columns of output.
// Every wait is bounded (wait_limit_ms): where one runs out, the roles leave their loops, the tensor memory is freed
// and VTOKEN_FLAG_TIMEOUT is set.
#include "attention.cuh"
#include "tensor.cuh"

namespace {

constexpr int AP_REGS_SOFTMAX = 192, AP_REGS_LOAD = 80, AP_REGS_REST = 48;
static_assert(2 * AP_REGS_SOFTMAX + AP_REGS_LOAD + AP_REGS_REST <= 4 * 128, "the registers that the block is launched with");
constexpr int AP_NT = 512, AP_STAGES = 4, AP_TILE = TC_TILE, AP_META = 4;
constexpr uint64_t AP_DRAIN_NS = 1000000000;    // products in flight end by themselves: waited for whatever the caller's limit is

struct Item {                            // what one CTA works on
    int none, ticket;
    int kv, q0, first, rows, len;        // key head; first query row of the request; first row and rows of the pair of tiles
    int pmin[2], pmax[2];                // positions of the two row tiles
    int tile0, tiles;                    // tiles of 128 tokens
    int part;                            // shared prefixes: number of the part, -1: nobody reads these rows
    VtkRequest span;
};

struct Meta {                            // what the softmax needs of a tile's tokens
    int ids[AP_TILE];                    // ascending, INT32_MAX behind the last
    uint32_t every[2][4];                // bit: the token is seen by every row of the tile
    uint32_t there[4];                   // bit: the token has a slot in the pool
};

// entries of a tile's ascending ids that are <= p
__device__ __forceinline__ int ids_up_to(const int *ids, int p)
{
    int n = 0;
#pragma unroll
    for (int step = AP_TILE / 2; step > 0; step >>= 1)
        if (ids[n + step - 1] <= p) n += step;
    return n + (ids[n] <= p);            // (n is 127 at most here)
}
__device__ __forceinline__ uint32_t low_bits(int n) { return n >= 32 ? 0xffffffffu : (n <= 0 ? 0u : (1u << n) - 1u); }

template <int D>
struct Shared {
    uint8_t q[2][D / 64][AP_TILE * 128];
    uint8_t kv[AP_STAGES][D / 64][AP_TILE * 128];
    Meta meta[AP_META];
    alignas(16) int slots[AP_META][AP_TILE];     // what the producers copy: slot, -1 = zeros
    float row_scale[2][AP_TILE];
    Item item[2];
    int prefix[AP_NT + 1];
    int warp_sum[AP_NT / 32];
    uint64_t kv_full[AP_STAGES], kv_empty[AP_STAGES], meta_full[AP_META], meta_empty[AP_META], s_full[2], p_full[2][2], o_full[2], q_full, drain;
    uint32_t tmem;
    int abort;
};

// entries of the ascending ids [base, base + len) that are <= p, found by a warp: 32 probes a round
__device__ inline int ids_up_to_warp(const VtkAttnArgs &a, int64_t base, int len, int64_t p)
{
    if (p < 0) return 0;
    if (a.cache_ids.null()) return p + 1 < len ? (int)(p + 1) : len;
    int lo = 0, hi = len;                // ids below lo are <= p, ids from hi on are > p
    while (lo < hi) {
        const int step = (hi - lo + 31) / 32, probe = lo + vtk_lane() * step;
        const bool le = probe < hi && a.cache_ids[base + probe] <= p;
        const int n = __popc(__ballot_sync(0xffffffffu, le));
        const int next_hi = lo + n * step;
        if (n > 0) lo = lo + (n - 1) * step + 1;
        if (next_hi < hi) hi = next_hi < lo ? lo : next_hi;
    }
    return lo;
}

// The scheduler's work: ticket -> item.  Items of a request run from its last rows (the longest under a causal
// mask) to its first; all key heads of a pair of tiles follow one another.
template <int D>
__device__ void next_item(const VtkAttnArgs &a, Shared<D> &sh, Item &out, int R, int seg, uint32_t *tickets, int row_limit)
{
    const int lane = vtk_lane();
    int idx = 0;
    if (lane == 0) idx = (int)atomicAdd(tickets, 1u);
    idx = __shfl_sync(0xffffffffu, idx, 0);
    Item it;
    it.none = 1;
    it.ticket = idx;
    if (idx / a.hkv < sh.prefix[AP_NT]) {
        it.none = 0;
        it.kv = idx % a.hkv;
        const int pair = idx / a.hkv;
        int lo = 0, hi = AP_NT;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (sh.prefix[mid] <= pair) lo = mid; else hi = mid;
        }
        int left = pair - sh.prefix[lo], r = lo * seg, qn, pairs;
        int64_t base;
        bool clipped;
        for (;; ++r) {
            vtk_request_rows(a, r, it.q0, qn, base, it.len, clipped);
            pairs = qn * a.group > row_limit ? (qn * a.group + 2 * AP_TILE - 1) / (2 * AP_TILE) : 0;
            if (left < pairs) break;
            left -= pairs;
        }
        it.first = (pairs - 1 - left) * 2 * AP_TILE;
        it.rows = qn * a.group - it.first < 2 * AP_TILE ? qn * a.group - it.first : 2 * AP_TILE;
        int pmin = INT32_MAX, pmax = -1;
        for (int x = 0; x < 2; ++x) {
            int lo_p = INT32_MAX, hi_p = -1;
            const int r0 = it.first + x * AP_TILE, r1 = it.first + (it.rows < (x + 1) * AP_TILE ? it.rows : (x + 1) * AP_TILE);
            if (r0 < r1)
                for (int t = r0 / a.group + lane; t <= (r1 - 1) / a.group; t += 32) {
                    const int p = a.positions[it.q0 + t];
                    lo_p = p < lo_p ? p : lo_p;
                    hi_p = p > hi_p ? p : hi_p;
                }
            it.pmin[x] = __reduce_min_sync(0xffffffffu, lo_p);
            it.pmax[x] = __reduce_max_sync(0xffffffffu, hi_p);
            pmin = it.pmin[x] < pmin ? it.pmin[x] : pmin;
            pmax = it.pmax[x] > pmax ? it.pmax[x] : pmax;
        }
        it.span.pmax = pmax;
        it.span.floor = vtk_floor(pmin, a.window);
        it.span.base = base;
        it.span.first = 0;
        const int end = ids_up_to_warp(a, base, it.len, pmax);
        it.span.lo = a.window > 0 ? ids_up_to_warp(a, base, it.len, (int64_t)pmin - a.window) : 0;
        if (it.span.lo > end) it.span.lo = end;
        it.span.n_sink = a.sinks > 0 ? ids_up_to_warp(a, base, it.span.lo, (int64_t)a.sinks - 1) : 0;
        it.span.n = it.span.n_sink + end - it.span.lo;
        it.tile0 = it.part = 0;
        it.tiles = (it.span.n + AP_TILE - 1) / AP_TILE;
    }
    if (lane == 0) out = it;
}

// The same for shared prefixes: the rows of a group, the entries of its first request, a part of the tiles.
template <int D>
__device__ void next_prefix_item(const VtkAttnArgs &a, Item &out, uint32_t *tickets)
{
    const int lane = vtk_lane();
    int64_t idx = 0;
    if (lane == 0) idx = (int64_t)atomicAdd(tickets, 1u);
    idx = __shfl_sync(0xffffffffu, idx, 0);
    Item it;
    it.none = 1;
    it.ticket = (int)idx;
    if (idx < a.plan->items) {
        it.none = 0;
        int lo = 0, hi = a.plan->groups;     // the last group with items up to idx (groups without items have none in front of the next)
        while (hi - lo > 1) {
            const int step = (hi - lo + 31) / 32, probe = lo + vtk_lane() * step;
            const int n = __popc(__ballot_sync(0xffffffffu, probe < hi && a.groups[probe].items <= idx));    // (lane 0's always is)
            const int next_hi = lo + n * step;
            lo += (n - 1) * step;
            if (next_hi < hi) hi = next_hi;
        }
        const VtkPrefixGroup g = a.groups[lo];
        int64_t left = idx - g.items;
        it.kv = (int)(left % a.hkv);
        left /= a.hkv;
        it.part = (int)(left % g.splits);
        it.first = (int)(left / g.splits) * 2 * AP_TILE;
        it.q0 = g.q0;
        it.len = g.len;
        const int first_id = a.cache_ids.null() ? 0 : a.cache_ids[g.base], last_id = vtk_last_id(a, g.base, g.len);
        const int64_t rows = (int64_t)(g.q1 - g.q0) * a.group - it.first;
        it.rows = rows < 2 * AP_TILE ? (int)rows : 2 * AP_TILE;
        int pmin = INT32_MAX, pmax = -1;
        for (int x = 0; x < 2; ++x) {
            int lo_p = INT32_MAX, hi_p = -1;
            const int r0 = it.first + x * AP_TILE, r1 = it.first + (it.rows < (x + 1) * AP_TILE ? it.rows : (x + 1) * AP_TILE);
            if (r0 < r1)
                for (int t = r0 / a.group + lane; t <= (r1 - 1) / a.group; t += 32) {
                    const int p = a.positions[it.q0 + t];
                    lo_p = p < lo_p ? p : lo_p;
                    hi_p = p > hi_p ? p : hi_p;
                }
            it.pmin[x] = __reduce_min_sync(0xffffffffu, lo_p);
            it.pmax[x] = __reduce_max_sync(0xffffffffu, hi_p);
            pmin = it.pmin[x] < pmin ? it.pmin[x] : pmin;
            pmax = it.pmax[x] > pmax ? it.pmax[x] : pmax;
        }
        it.span.pmax = pmax;
        it.span.floor = vtk_floor(pmin, a.window);
        it.span.base = g.base;
        it.span.first = 0;
        // (searches are rounds of loads one behind the other: the ends are looked at first)
        const bool whole = last_id <= pmax, from_start = a.window == 0 || (int64_t)first_id > (int64_t)pmin - a.window;
        const int end = whole ? g.len : ids_up_to_warp(a, g.base, g.len, pmax);
        it.span.lo = from_start ? 0 : ids_up_to_warp(a, g.base, g.len, (int64_t)pmin - a.window);
        if (it.span.lo > end) it.span.lo = end;
        it.span.n_sink = a.sinks > 0 && it.span.lo > 0 ? ids_up_to_warp(a, g.base, it.span.lo < a.sinks ? it.span.lo : a.sinks, (int64_t)a.sinks - 1) : 0;
        it.span.n = it.span.n_sink + end - it.span.lo;
        const int all = (it.span.n + AP_TILE - 1) / AP_TILE;
        it.tile0 = it.part * g.tiles;
        it.tiles = all - it.tile0 < g.tiles ? (all > it.tile0 ? all - it.tile0 : 0) : g.tiles;
        // rows of one request that reads the prefix for itself
        int before = g.first, behind = g.end;
        const int t0 = it.q0 + it.first / a.group, t1 = it.q0 + (it.first + it.rows - 1) / a.group;
        if (a.row_limit == INT32_MAX) behind = before;       // (there are none)
        while (behind - before > 1) {        // q_offsets[before] <= t0 < q_offsets[behind]
            const int mid = (before + behind) >> 1;
            if (a.q_offsets[mid] <= t0) before = mid; else behind = mid;
        }
        if (behind > before && t1 < a.q_offsets[before + 1] && ((int64_t)a.q_offsets[before + 1] - a.q_offsets[before]) * a.group > a.row_limit) {
            it.part = -1;
            it.tiles = 0;
        }
    }
    if (lane == 0) out = it;
}

// One query row over the tokens [v0, v1) of a prefix by one warp, token by token (see vtk_row_again); false when it stands.
template <int D, bool FP4, typename Act>
__device__ __noinline__ bool prefix_row_again(const VtkAttnArgs &a, int64_t q_row, int head, int pos, const VtkRequest &span, int len, int v0, int v1,
                                              float (&o)[D / 32], float &m, float &l)
{
    if (!vtk_hidden_value<D, FP4, Act>(a, head, pos, span, len)) return false;
    constexpr int N = D / 32;
    const int lane = vtk_lane(), kv = head / a.group, floor = vtk_floor(pos, a.window);
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
#pragma unroll
    for (int j = 0; j < N; ++j) o[j] = 0.f;
    for (int i = v0; i < v1; ++i) {
        const int id = a.cache_ids.null() ? span.index(i) : a.cache_ids[span.entry(i)];
        const int64_t slot = a.cache_slots[span.entry(i)];
        if (slot < 0 || slot >= a.slots_per_layer || !vtk_sees(id, pos, floor, a.sinks)) continue;
        float k[N], v[N], s = 0.f;
        vtk_row_values<D, FP4, Act, N>(a.k_rows + slot * a.row_bytes, a.hkv, kv, lane * N, k);
        vtk_row_values<D, FP4, Act, N>(a.v_rows + slot * a.row_bytes, a.hkv, kv, lane * N, v);
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

// PREFIX: the rows of all requests of a group over their shared prefix, left as running maximum, sum and weighted values
template <int D, bool FP4, typename Act, bool PREFIX>
__global__ void __launch_bounds__(AP_NT, 1) attention_prompt_kernel(const __grid_constant__ VtkAttnArgs a, uint32_t *tickets, int row_limit,
                                                                    uint64_t limit_ns, float scale, int negate, int64_t stall)
{
    using Mma = typename std::conditional<FP4, VtkFp16, Act>::type;
    constexpr int PANEL = AP_TILE * 128, PIECES = D / 8;
    // Rows behind a prefix get the weights that the kernel for few rows would have given them, the sum of two 16-bit numbers (over 4-bit
    // rows with bf16 queries: one in half precision).  Scores are in registers when P is written, so the second number lies where the
    // other half of the scores was; the product over V is issued once more for it.  (One number: an error of up to 2^-8 of every bf16 weight,
    // as large as the output's own rounding.  Two cost 2 of 112 us a call behind 8192 tokens in bf16 and 10 of 160 behind 32
    // prefixes in fp16, where softmax warps are what is waited for.)
    constexpr bool SPLIT_P = PREFIX && !(FP4 && Act::kind == VTOKEN_KV_BF16);
    constexpr int P_LOW = AP_TILE / 2;                       // columns from the first number to the second
    extern __shared__ uint8_t raw[];
    Shared<D> &sh = *reinterpret_cast<Shared<D> *>(raw + ((1024 - (vtk_smem_u32(raw) & 1023)) & 1023));
    vtk_release_successor();
    vtk_wait_for_predecessor();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

    // ---- once per CTA: barriers, tensor memory, pairs of tiles per request ----
    if (tid == 0) {
        for (int i = 0; i < AP_STAGES; ++i) { vtk_mbar_init(&sh.kv_full[i], 128); vtk_mbar_init(&sh.kv_empty[i], 1); }
        for (int i = 0; i < AP_META; ++i) { vtk_mbar_init(&sh.meta_full[i], 2); vtk_mbar_init(&sh.meta_empty[i], 8); }
        for (int x = 0; x < 2; ++x) { vtk_mbar_init(&sh.s_full[x], 1); vtk_mbar_init(&sh.p_full[x][0], 4); vtk_mbar_init(&sh.p_full[x][1], 4); vtk_mbar_init(&sh.o_full[x], 1); }
        vtk_mbar_init(&sh.q_full, 128);
        vtk_mbar_init(&sh.drain, 1);
        sh.abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 12) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(vtk_smem_u32(&sh.tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    int R = *a.num_requests;
    bool clipped = R < 0 || R > a.max_requests;
    R = R < 0 ? 0 : (R > a.max_requests ? a.max_requests : R);
    const int seg = (R + AP_NT - 1) / AP_NT;
    int pairs = 0;
    for (int r = tid * seg; !PREFIX && r < (tid + 1) * seg && r < R; ++r) {
        int q0, qn, len;
        int64_t base;
        bool c;
        vtk_request_rows(a, r, q0, qn, base, len, c);
        clipped |= c;
        if (qn * a.group > row_limit) pairs += (qn * a.group + 2 * AP_TILE - 1) / (2 * AP_TILE);
    }
    if (clipped && blockIdx.x == 0) atomicOr(a.flags, (uint32_t)VTOKEN_FLAG_CAPACITY);
    const int incl = vtk_warp_incl_scan(pairs);
    if (lane == 31) sh.warp_sum[warp] = incl;
    tc_before_sync();
    __syncthreads();
    tc_after_sync();
    int before = 0;
    for (int w = 0; w < warp; ++w) before += sh.warp_sum[w];
    sh.prefix[tid + 1] = before + incl;
    if (tid == 0) sh.prefix[0] = 0;
    __syncthreads();
    const uint32_t tmem = sh.tmem;
    auto next = [&](Item &out) {
        if (PREFIX) next_prefix_item<D>(a, out, tickets);
        else next_item<D>(a, sh, out, R, seg, tickets, row_limit);
    };
    if (warp == 13) next(sh.item[0]);

    // running counts of the rings and barriers
    uint32_t kv_count = 0;               // K and V tiles loaded (producers) or used (mma)
    uint32_t s_count[2] = {0, 0}, item_count = 0, tile_count = 0, q_count = 0, o_count[2] = {0, 0};
    constexpr uint32_t IDESC = (1u << 4) | ((Mma::kind == VTOKEN_KV_BF16 ? 1u : 0u) << 7) | ((Mma::kind == VTOKEN_KV_BF16 ? 1u : 0u) << 10) |
                               ((uint32_t)(AP_TILE >> 4) << 24);
    const uint32_t idesc_s = IDESC | ((uint32_t)(AP_TILE >> 3) << 17) | ((uint32_t)negate << 13);
    constexpr uint32_t idesc_o = IDESC | ((uint32_t)(D >> 3) << 17) | (1u << 16);

    // Every role runs its own loop over the items, in step with the others at the items' ends.
    auto each_item = [&](auto &&body) {
        for (;; ++item_count) {
            asm volatile("barrier.cta.sync 0, 512;" ::: "memory");
            const Item &it = sh.item[item_count & 1];
            // Who gives up leaves the number of its item, from 1 on, so that the verdict is the same for all: a role that comes here late may
            // find the mark of one that has already given up in the item that starts now, and has to join it there, not leave.
            const int gave_up = *(volatile int *)&sh.abort;
            if (it.none || (gave_up != 0 && gave_up <= (int)item_count)) break;
            const int T = it.tiles;
            const bool two = it.rows > AP_TILE;
            body(it, T, two);
            kv_count += 2 * T;
            tile_count += T;
            s_count[0] += T;                                         // the second tile's barriers move only when there is one
            s_count[1] += two ? T : 0;
            if (T > 0) { ++q_count; ++o_count[0]; o_count[1] += two; }
        }
    };
    // (registers of the launch, 128 a thread, are shared out again: a softmax thread holds a row of scores)
    if (warp < 8) {
        // ================= softmax: thread = row =================
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(AP_REGS_SOFTMAX));
        each_item([&](const Item &it, int T, bool two) {
            const int x = warp >> 2, row = tid & 127;
            const uint32_t lanes = (uint32_t)(warp & 3) << 21;                   // 32 lanes a warp
            const uint32_t t_s = tmem + lanes + x * AP_TILE, t_o = tmem + lanes + 2 * AP_TILE + x * D;
            const bool have = x * AP_TILE + row < it.rows;
            const int at = it.first + x * AP_TILE + row;
            const int64_t tok = it.q0 + (have ? at / a.group : 0);
            const int head = it.kv * a.group + (have ? at % a.group : 0);
            const int pos = have ? a.positions[tok] : -1, floor = vtk_floor(pos, a.window);
            float m = -INFINITY, l = 0.f, c = scale;
            bool ok = true;
            // This warp is past a tile's ids and masks, and the producers are past its slots: the scores of the tile behind it (the
            // outputs, at the end) need rows that were copied after them.  Eight arrivals a tile: a lone row tile's warps count twice.
            auto done_with = [&](uint32_t tile) {
                if (lane == 0) vtk_mbar_arrive(&sh.meta_empty[tile % AP_META], two ? 1 : 2);
            };
            if (x == 0 || two) {
                if (FP4 && T > 0) {                                              // row scales come with the queries
                    ok = __all_sync(0xffffffffu, vtk_mbar_wait(&sh.q_full, q_count & 1, limit_ns, &sh.abort, item_count + 1));
                    c = scale * sh.row_scale[x][row];
                }
                for (int j = 0; j < T && ok; ++j) {
                    ok = __all_sync(0xffffffffu, vtk_mbar_wait(&sh.s_full[x], (s_count[x] + j) & 1, limit_ns, &sh.abort, item_count + 1));
                    if (!ok) break;
                    tc_after_sync();
                    const uint32_t cm = tile_count + j;
                    if (j > 0) done_with(cm - 1);
                    vtk_mbar_wait(&sh.meta_full[cm % AP_META], (cm / AP_META) & 1, limit_ns, &sh.abort, item_count + 1);       // (it is there)
                    const Meta &mt = sh.meta[cm % AP_META];
                    uint32_t vis[4];                                             // bit: this row sees the token
                    bool all = true;
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        vis[q] = mt.every[x][q];
                        if (vis[q] != 0xffffffffu) {
                            all = false;
                        }
                    }
                    if (!all) {                                                  // ids ascend: what the row sees is a range, and the sinks
                        const int hi = ids_up_to(mt.ids, pos), lo = floor < 0 ? 0 : ids_up_to(mt.ids, floor), sk = lo == 0 || a.sinks == 0 ? 0 : ids_up_to(mt.ids, a.sinks - 1);
#pragma unroll
                        for (int q = 0; q < 4; ++q) vis[q] = mt.there[q] & low_bits(hi - 32 * q) & (~low_bits(lo - 32 * q) | low_bits(sk - 32 * q));
                    }
                    uint32_t s[4][32];
#pragma unroll
                    for (int q = 0; q < 4; ++q) tc_ld32(t_s + 32 * q, s[q]);
                    float top4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        tc_wait_ld(s[q]);                                        // (the first waits for all four)
                        if (!all) {
#pragma unroll
                            for (int i = 0; i < 32; ++i)
                                if (!((vis[q] >> i) & 1u)) s[q][i] = 0xff800000u;
                        }
#pragma unroll
                        for (int i = 0; i < 32; i += 2) top4[(i >> 1) & 3] = max3(top4[(i >> 1) & 3], __uint_as_float(s[q][i]), __uint_as_float(s[q][i + 1]));
                    }
                    const float top = fmaxf(fmaxf(top4[0], top4[1]), fmaxf(top4[2], top4[3]));
                    const bool up = (top - m) * c > 8.f || (m == -INFINITY && top > -INFINITY);
                    if (__any_sync(0xffffffffu, up)) {
                        const float next = fmaxf(m, top);
                        const float f = m == -INFINITY ? 0.f : vtk_exp2((m - next) * c);
                        m = next;
                        l *= f;
                        if (j > 0) {                                             // the products up to j - 1 are complete: S j came after them
#pragma unroll
                            for (int q = 0; q < D / 16; ++q) {
                                uint32_t o[16];
                                tc_ld16(t_o + 16 * q, o);
                                tc_wait_ld(o);
#pragma unroll
                                for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                                tc_st16(t_o + 16 * q, o);
                            }
                        }
                    }
                    const float mc = (m == -INFINITY ? 0.f : m * c) - vtk_lift<Mma>();
                    float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
                    const float2 c2 = make_float2(c, c), mc2 = make_float2(-mc, -mc);
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        uint32_t p[16], low[16];
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            float2 y = fma2(make_float2(__uint_as_float(s[q][2 * i]), __uint_as_float(s[q][2 * i + 1])), c2, mc2);
                            y.x = vtk_exp2(y.x);
                            y.y = vtk_exp2(y.y);
                            sum[i & 1] = add2(sum[i & 1], y);
                            p[i] = Mma::pack(y.x, y.y);
                            if (SPLIT_P) {
                                const float2 r = Mma::unpack(p[i]);
                                low[i] = Mma::pack(y.x - r.x, y.y - r.y);
                            }
                        }
                        tc_st16(t_s + 16 * q, p);
                        if (SPLIT_P) tc_st16(t_s + P_LOW + 16 * q, low);
                        if (q & 1) {                                             // half of P: the product over it can start
                            tc_wait_st();
                            tc_before_sync();
                            __syncwarp();
                            if (lane == 0) vtk_mbar_arrive(&sh.p_full[x][q >> 1]);   // (arrivals are served one by one)
                        }
                    }
                    sum[0] = add2(sum[0], sum[1]);
                    l += sum[0].x + sum[0].y;
                }
                if (ok && T > 0) ok = __all_sync(0xffffffffu, vtk_mbar_wait(&sh.o_full[x], o_count[x] & 1, limit_ns, &sh.abort, item_count + 1));
                if (ok) {
                    if (T > 0) {
                        tc_after_sync();
                        done_with(tile_count + T - 1);
                    }
                    if (PREFIX) {
                        // as it is: the request's own tokens go on from here
                        const bool write = have && it.part >= 0;
                        const int64_t place = ((int64_t)it.part * a.plan->query_tokens + tok) * a.hq + head;
                        if (write) a.pre_ml[place] = make_float2(l == 0.f ? -INFINITY : m * c, l);
                        bool bad = false;
                        float *dst = a.pre_o + place * D;
#pragma unroll
                        for (int q = 0; q < D / 32; ++q) {
                            uint32_t o[32];
                            if (T > 0) {
                                tc_ld32(t_o + 32 * q, o);
                                tc_wait_ld(o);
#pragma unroll
                                for (int i = 0; i < 32; ++i) bad |= !(fabsf(__uint_as_float(o[i])) < INFINITY);
                                if (write && l != 0.f) {
#pragma unroll
                                    for (int i = 0; i < 8; ++i)
                                        *reinterpret_cast<uint4 *>(dst + 32 * q + 4 * i) = make_uint4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
                                }
                            }
                        }
                        unsigned again = __ballot_sync(0xffffffffu, write && bad && l != 0.f && fabsf(l) < INFINITY);
                        if (again) __syncwarp();                     // (other lanes write over what a row's own has just stored)
                        while (again) {
                            const int src = __ffs(again) - 1;
                            again &= again - 1;
                            const int64_t q_row = __shfl_sync(0xffffffffu, (int)tok, src), to = __shfl_sync(0xffffffffu, place, src);
                            const int h2 = __shfl_sync(0xffffffffu, head, src), p2 = __shfl_sync(0xffffffffu, pos, src);
                            const int v0 = it.tile0 * AP_TILE, v1 = (it.tile0 + T) * AP_TILE < it.span.n ? (it.tile0 + T) * AP_TILE : it.span.n;
                            float acc[D / 32], m2, l2;
                            if (prefix_row_again<D, FP4, Act>(a, q_row, h2, p2, it.span, it.len, v0, v1, acc, m2, l2)) {
                                const float lift = exp2f(vtk_lift<Mma>());
#pragma unroll
                                for (int j = 0; j < D / 32; ++j) a.pre_o[to * D + lane * (D / 32) + j] = acc[j] * lift;
                                if (lane == 0) a.pre_ml[to] = make_float2(m2, l2 * lift);
                            }
                        }
                        tc_before_sync();
                        return;
                    }
                    const float r = l == 0.f ? 0.f : a.v_mul / l;
                    const bool finite = fabsf(l) < INFINITY;         // (a sum that is not: the row sees a score that is not)
                    bool bad = false;
                    uint16_t *dst = a.out + tok * a.out_stride + (int64_t)head * D;
#pragma unroll
                    for (int q = 0; q < D / 32; ++q) {
                        uint32_t o[32];
                        if (T > 0) {
                            tc_ld32(t_o + 32 * q, o);
                            tc_wait_ld(o);
                        }
#pragma unroll
                        for (int i = 0; i < 32; ++i) {
                            const float y = T > 0 && l != 0.f ? __uint_as_float(o[i]) * r : 0.f;
                            bad |= T > 0 && !(fabsf(__uint_as_float(o[i])) < INFINITY);
                            o[i] = __float_as_uint(y);
                        }
                        if (have) {
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                uint4 w;
                                w.x = Act::pack(__uint_as_float(o[8 * i]), __uint_as_float(o[8 * i + 1]));
                                w.y = Act::pack(__uint_as_float(o[8 * i + 2]), __uint_as_float(o[8 * i + 3]));
                                w.z = Act::pack(__uint_as_float(o[8 * i + 4]), __uint_as_float(o[8 * i + 5]));
                                w.w = Act::pack(__uint_as_float(o[8 * i + 6]), __uint_as_float(o[8 * i + 7]));
                                *reinterpret_cast<uint4 *>(dst + 32 * q + 8 * i) = w;
                            }
                        }
                    }
                    if (have && a.lse != nullptr)
                        a.lse[tok * a.hq + head] = l == 0.f ? -INFINITY : (m * c + log2f(l) - vtk_lift<Mma>()) * 0.69314718055994531f;
                    // rows that a masked NaN may have reached: token by token
                    unsigned again = __ballot_sync(0xffffffffu, have && bad && finite);
                    if (again) __syncwarp();                         // (other lanes write over what a row's own has just stored)
                    while (again) {
                        const int src = __ffs(again) - 1;
                        again &= again - 1;
                        const int64_t q_row = __shfl_sync(0xffffffffu, (int)tok, src);
                        const int h2 = __shfl_sync(0xffffffffu, head, src), p2 = __shfl_sync(0xffffffffu, pos, src);
                        float acc[D / 32], m2, l2;
                        if (vtk_row_again<D, FP4, Act>(a, q_row, h2, p2, it.span, it.len, acc, m2, l2)) vtk_store_row<D, Act>(a, q_row, h2, acc, m2, l2);
                    }
                    tc_before_sync();
                }
            }
        });
    } else if (warp < 12) {
        // ================= producers =================
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(AP_REGS_LOAD));
        auto stalled = [&](const Item &it) {                       // the item whose wait for its queries has to run out (a test's)
#ifdef VTOKEN_CHECKED
            return it.ticket == stall;
#else
            return false;
#endif
        };
        each_item([&](const Item &it, int T, bool two) {
            if (T > 0) {
                const int pt = tid - 256;
                // queries, rows of both tiles (the rows of a prefix are fetched behind the first keys, which come from further away)
                auto queries = [&]() {
                    if (PREFIX && !FP4) {
                        // PIECES threads a row; a division for each thread, the 32 rows of its warp by shuffles
                        const int piece = pt % PIECES, row0 = pt / PIECES * PIECES;
                        for (int x = 0; x < (two ? 2 : 1); ++x) {
                            const int row = x * AP_TILE + pt, at = it.first + row;
                            int64_t mine = -1;
                            if (row < it.rows) mine = (it.q0 + at / a.group) * a.q_stride + (int64_t)(it.kv * a.group + at % a.group) * D;
#pragma unroll
                            for (int i = 0; i < PIECES; ++i) {
                                const int64_t from = __shfl_sync(0xffffffffu, mine, lane / PIECES * PIECES + i);
                                cp_async16(vtk_smem_u32(sh.q[x]) + swizzled(row0 + i, piece), a.q + (from < 0 ? 0 : from) + 8 * piece, from >= 0);
                            }
                        }
                        if (!stalled(it) || pt > 0) cp_arrive(&sh.q_full);
                    } else if (!FP4) {
                        const int rows = two ? 2 * AP_TILE : AP_TILE;
                        for (int i = pt; i < rows * PIECES; i += 128) {
                            const int row = i / PIECES, piece = i % PIECES, at = it.first + row;
                            const bool there = row < it.rows;
                            const uint16_t *src = a.q;
                            if (there) src += (it.q0 + at / a.group) * a.q_stride + (int64_t)(it.kv * a.group + at % a.group) * D + 8 * piece;
                            cp_async16(vtk_smem_u32(sh.q[row >> 7]) + swizzled(row & 127, piece), src, there);
                        }
                        if (!stalled(it) || pt > 0) cp_arrive(&sh.q_full);
                    } else {
                        for (int x = 0; x < (two ? 2 : 1); ++x) {
                            const int row = x * AP_TILE + pt, at = it.first + row;
                            const bool there = row < it.rows;
                            const uint16_t *src = a.q;
                            if (there) src += (it.q0 + at / a.group) * a.q_stride + (int64_t)(it.kv * a.group + at % a.group) * D;
                            float up = 1.f, down = 1.f;
                            if (Act::kind == VTOKEN_KV_BF16) {           // bf16 queries in half precision: see attention.cu
                                float top = 0.f, v[8];
                                for (int i = 0; i < PIECES; ++i) {
                                    vtk_unpack8<VtkBf16>(there ? *reinterpret_cast<const uint4 *>(src + 8 * i) : make_uint4(0, 0, 0, 0), v);
#pragma unroll
                                    for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(v[e]));
                                }
                                int e2 = (int)(__float_as_uint(top) >> 23) - 127;
                                e2 = 14 - (e2 < -100 ? -100 : e2);
                                up = __uint_as_float((uint32_t)(127 + e2) << 23);
                                down = __uint_as_float((uint32_t)(127 - e2) << 23);
                            }
                            sh.row_scale[x][pt] = down;
                            for (int i = 0; i < PIECES; ++i) {
                                uint4 w = there ? *reinterpret_cast<const uint4 *>(src + 8 * i) : make_uint4(0, 0, 0, 0);
                                if (Act::kind == VTOKEN_KV_BF16) {
                                    float v[8];
                                    vtk_unpack8<VtkBf16>(w, v);
#pragma unroll
                                    for (int e = 0; e < 8; ++e) v[e] *= up;
                                    w = vtk_pack8<VtkFp16>(v);
                                }
                                st_shared16(vtk_smem_u32(sh.q[x]) + swizzled(pt, i), w);
                            }
                        }
                        async_proxy_fence();
                        if (!stalled(it) || pt > 0) vtk_mbar_arrive(&sh.q_full);
                    }
                };
                if (!PREFIX) queries();
                auto wait_meta = [&](int j) {                      // the slots of tile j
                    const uint32_t c = tile_count + j;
                    return vtk_mbar_wait(&sh.meta_full[c % AP_META], (c / AP_META) & 1, limit_ns, &sh.abort, item_count + 1);
                };
                // 4-bit rows: four threads a token, a quarter of its codes and scales each, fetched one operand ahead
                constexpr int QW = D / 32;                         // words of 8 codes a thread
                struct Raw { uint32_t w[QW], sc; };
                Raw raw[2][4];                                     // K, V
                const int part = pt & 3;
                auto fetch_rows = [&](int which, int j) {
                    const uint8_t *rows = which ? a.v_rows : a.k_rows;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int64_t sl = sh.slots[(tile_count + j) % AP_META][(pt >> 2) + 32 * i];
                        Raw &r = raw[which][i];
#pragma unroll
                        for (int k = 0; k < QW; ++k) r.w[k] = 0;
                        r.sc = 0;
                        if (sl < 0) continue;
                        const uint8_t *src = rows + sl * a.row_bytes;
                        const uint8_t *codes = src + it.kv * (D / 2) + part * (D / 8);
                        const uint8_t *scales = src + a.hkv * (D / 2) + it.kv * (D / 16) + part * (D / 64);
                        if (D == 128) {
                            const uint4 q4 = vtk_ldg16(codes);
                            r.w[0] = q4.x; r.w[1] = q4.y; r.w[QW - 2] = q4.z; r.w[QW - 1] = q4.w;
                            r.sc = __ldg(reinterpret_cast<const uint16_t *>(scales));
                        } else {
                            const uint2 q2 = __ldg(reinterpret_cast<const uint2 *>(codes));
                            r.w[0] = q2.x; r.w[1] = q2.y;
                            r.sc = __ldg(scales);
                        }
                    }
                };
                auto deliver = [&](int stage) { async_proxy_fence(); vtk_mbar_arrive(&sh.kv_full[stage]); };
                for (int j = 0; j < T; ++j) {
                    const uint32_t c0 = kv_count + 2 * j, stage_k = c0 % AP_STAGES, stage_v = (c0 + 1) % AP_STAGES;
                    if (j == 0 || !FP4)
                        if (!wait_meta(j)) break;
                    if (FP4 && j == 0) fetch_rows(0, 0);
                    if (PREFIX && FP4 && j == 0) queries();
                    if (!vtk_mbar_wait(&sh.kv_empty[stage_k], ((c0 / AP_STAGES) & 1) ^ 1, limit_ns, &sh.abort, item_count + 1)) break;
                    bool ok = true;
#pragma unroll
                    for (int which = 0; which < 2; ++which) {
                        const uint32_t stage = which ? stage_v : stage_k;
                        if (which) {
                            ok = vtk_mbar_wait(&sh.kv_empty[stage_v], (((c0 + 1) / AP_STAGES) & 1) ^ 1, limit_ns, &sh.abort, item_count + 1);
                            if (ok && FP4 && j + 1 < T) ok = wait_meta(j + 1);
                            if (!ok) break;
                        }
                        const uint8_t *rows = which ? a.v_rows : a.k_rows;
                        const uint32_t dst = vtk_smem_u32(sh.kv[stage]);
                        if (!FP4) {
                            // PIECES threads a row, each with the same number of consecutive rows
                            constexpr int ROWS = PIECES;
                            const int piece = pt % PIECES, row0 = pt / PIECES * ROWS;
                            const uint8_t *base = rows + ((int64_t)it.kv * D + 8 * piece) * 2;
                            int sl[ROWS];
#pragma unroll
                            for (int i = 0; i < ROWS; i += 4) {
                                const int4 four = *reinterpret_cast<const int4 *>(&sh.slots[(tile_count + j) % AP_META][row0 + i]);
                                sl[i] = four.x; sl[i + 1] = four.y; sl[i + 2] = four.z; sl[i + 3] = four.w;
                            }
#pragma unroll
                            for (int i = 0; i < ROWS; ++i)
                                cp_async16(dst + swizzled(row0 + i, piece), base + (int64_t)(sl[i] < 0 ? 0 : sl[i]) * a.row_bytes, sl[i] >= 0);
                            cp_arrive(&sh.kv_full[stage]);
                            if (PREFIX && j == 0 && which == 0) queries();
                        } else {
                            if (which == 0) fetch_rows(1, j);
                            else if (j + 1 < T) fetch_rows(0, j + 1);
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const uint32_t two_scales = vtk_scales_to_half2(raw[which][i].sc);
#pragma unroll
                                for (int k = 0; k < QW; ++k)
                                    st_shared16(dst + swizzled((pt >> 2) + 32 * i, part * QW + k),
                                                vtk_expand8(raw[which][i].w[k], __byte_perm(two_scales, 0, k < 2 ? 0x1010 : 0x3232)));
                            }
                            deliver((int)stage);
                        }
                    }
                    if (!ok) break;
                }
                if (!FP4) cp_wait_all();                           // (they have: the products are done or, after an abort, waited for here)
            }
        });
    } else if (warp == 12) {
        // ================= products: one thread issues them =================
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(AP_REGS_REST));
        const bool one = tc_elect();
        const uint32_t q_addr = vtk_smem_u32(sh.q), kv_addr = vtk_smem_u32(sh.kv);
        each_item([&](const Item &it, int T, bool two) {
            (void)it;
            if (T == 0) return;
            const uint32_t k0 = kv_count;
            auto wait = [&](uint64_t *bar, uint32_t parity) { return (bool)__all_sync(0xffffffffu, vtk_mbar_wait(bar, parity, limit_ns, &sh.abort, item_count + 1)); };
            auto wait_tile = [&](uint32_t cc) { return wait(&sh.kv_full[cc % AP_STAGES], (cc / AP_STAGES) & 1); };
            auto come = [&](uint64_t *bar, uint32_t parity) { return (bool)__all_sync(0xffffffffu, vtk_mbar_test(bar, parity)); };
            auto tile_come = [&](uint32_t cc) { return come(&sh.kv_full[cc % AP_STAGES], (cc / AP_STAGES) & 1); };
            auto scores = [&](int x, uint32_t cc) {
                const uint64_t qd = operand(q_addr) + (uint64_t)(x * (D / 64) * PANEL >> 4);
                const uint64_t kd = operand(kv_addr) + (uint64_t)((cc % AP_STAGES) * (D / 64) * PANEL >> 4);
#pragma unroll
                for (int k = 0; k < D / 16; ++k) {
                    const uint32_t off = ((k / 4) * PANEL + (k % 4) * 32) >> 4;
                    tc_mma_ss(one, tmem + x * AP_TILE, qd + off, kd + off, idesc_s, k > 0);
                }
                tc_commit(one, &sh.s_full[x]);
            };
            auto outputs = [&](int x, uint32_t cc, int half, bool first) {
                const uint64_t vd = operand(kv_addr) + (uint64_t)((cc % AP_STAGES) * (D / 64) * PANEL >> 4);
#pragma unroll
                for (int i = 0; i < AP_TILE / 32; ++i) {
                    const int k = half * (AP_TILE / 32) + i;
                    tc_mma_ts(one, tmem + 2 * AP_TILE + x * D, tmem + x * AP_TILE + 8 * k, vd + (k * 16 * 128 >> 4), idesc_o, !first || k > 0);
                    if (SPLIT_P) tc_mma_ts(one, tmem + 2 * AP_TILE + x * D, tmem + x * AP_TILE + P_LOW + 8 * k, vd + (k * 16 * 128 >> 4), idesc_o, 1);
                }
            };
            bool ok = wait(&sh.q_full, q_count & 1) && wait_tile(k0);
            if (ok) {
                async_proxy_fence();
                tc_after_sync();
                scores(0, k0);
                if (two) scores(1, k0);
                tc_commit(one, &sh.kv_empty[k0 % AP_STAGES]);
            }
            // Whichever row tile has (half of) its P goes on: step 2 j of a row tile is the first half of its product over
            // V j, step 2 j + 1 the second half and the scores over K j + 1.
            int step[2] = {0, two ? 0 : 2 * T}, v_there = 0, k_there = 1;       // tiles of V and K that have come
            uint64_t idle = 0;
            uint32_t polls = 0;
            while (ok && (step[0] < 2 * T || step[1] < 2 * T)) {
                bool any = false;
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    if (step[x] >= 2 * T) continue;
                    const int j = step[x] >> 1, half = step[x] & 1;
                    const uint32_t ck = k0 + 2 * j, cv = ck + 1;
                    // (nothing waits here: the row tile that is ahead may need a stage that the other one has still to use)
                    if (!come(&sh.p_full[x][half], (s_count[x] + j) & 1)) continue;
                    if (half == 0 && v_there <= j) {
                        if (!tile_come(cv)) continue;
                        v_there = j + 1;
                        async_proxy_fence();
                    }
                    if (half == 1 && j + 1 < T && k_there <= j + 1) {
                        if (!tile_come(ck + 2)) continue;
                        k_there = j + 2;
                        async_proxy_fence();
                    }
                    any = true;
                    tc_after_sync();
                    outputs(x, cv, half, j == 0);
                    if (half == 1) {
                        const bool last = !two || step[x ^ 1] > step[x];        // the other row tile is past V j already
                        if (last) tc_commit(one, &sh.kv_empty[cv % AP_STAGES]);
                        if (j + 1 < T) {
                            scores(x, ck + 2);
                            if (last) tc_commit(one, &sh.kv_empty[(ck + 2) % AP_STAGES]);
                        } else {
                            tc_commit(one, &sh.o_full[x]);
                        }
                    }
                    ++step[x];
                }
                polls = any ? 0 : polls + 1;                            // (the clock is far away: looked at now and then)
                if (polls >= 4096 && polls % 256 == 0) {
                    const uint64_t now = vtk_global_ns();
                    if (polls == 4096) idle = now;
                    if (__any_sync(0xffffffffu, *(volatile int *)&sh.abort || now - idle > limit_ns)) {
                        *(volatile int *)&sh.abort = (int)item_count + 1;
                        ok = false;
                    }
                }
            }
            if (!ok) {                                               // what was issued ends before the tensor memory goes
                tc_commit(one, &sh.drain);
                const uint64_t t0 = vtk_global_ns();
                while (!vtk_mbar_try(&sh.drain, 0) && vtk_global_ns() - t0 < AP_DRAIN_NS) {}
            }
            __syncwarp();
        });
    } else {
        // ================= warp 13: the next item; 14 and 15: slots, ids and masks of the tiles =================
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(AP_REGS_REST));
        each_item([&](const Item &it, int T, bool two) {
            if (warp == 13) {
                next(sh.item[(item_count + 1) & 1]);
                return;
            }
            int slot[2], id[2];
            // VtkRequest::index, whose `first` is 0 in this kernel.  Left out over 16-bit rows: the register that it takes has others spilled (20
            // bytes; 8192 tokens 657 us instead of 653).  Over 4-bit rows the code with it is the faster one (268 us instead of 273).
            auto index = [&](int v) { return v < it.span.n_sink ? (FP4 ? it.span.first : 0) + v : it.span.lo + (v - it.span.n_sink); };
            auto fetch = [&](int j) {                              // this thread's two tokens of tile j
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int v = ((PREFIX ? it.tile0 : 0) + j) * AP_TILE + (warp - 14) * 64 + 32 * i + lane;
                    slot[i] = -1;
                    id[i] = INT32_MAX;
                    if (v < it.span.n) {
                        slot[i] = a.cache_slots[it.span.base + index(v)];
                        id[i] = a.cache_ids.null() ? index(v) : a.cache_ids[it.span.base + index(v)];
                    }
                }
            };
            if (T > 0) fetch(0);
            for (int j = 0; j < T; ++j) {
                // As far ahead of the copies as there are places.  The place has barriers of its own, whose next phase needs what is
                // written here: a phase of the stages' barriers could come and go unseen while these warps wait for slots.
                const uint32_t c = tile_count + j;
#ifdef VTOKEN_CHECKED
                for (int64_t left = stall - (1ll << 32); left >= 0; left -= 100000) __nanosleep(left < 100000 ? (unsigned)left + 1 : 100000u);
#endif
                if (!__all_sync(0xffffffffu, vtk_mbar_wait(&sh.meta_empty[c % AP_META], ((c / AP_META) & 1) ^ 1, limit_ns, &sh.abort, item_count + 1))) break;
                Meta &mt = sh.meta[c % AP_META];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int word = (warp - 14) * 2 + i, at = 32 * word + lane;
                    if (slot[i] >= a.slots_per_layer) {
                        atomicOr(a.flags, (uint32_t)VTOKEN_FLAG_BAD_SLOT);
                        slot[i] = -1;
                    }
                    mt.ids[at] = id[i];
                    sh.slots[c % AP_META][at] = vtk_sees(id[i], it.span.pmax, it.span.floor, a.sinks) ? slot[i] : -1;
                    const unsigned there = __ballot_sync(0xffffffffu, slot[i] >= 0);
                    const unsigned every0 = __ballot_sync(0xffffffffu, slot[i] >= 0 && vtk_sees(id[i], it.pmin[0], vtk_floor(it.pmax[0], a.window), a.sinks));
                    const unsigned every1 = __ballot_sync(0xffffffffu, slot[i] >= 0 && vtk_sees(id[i], it.pmin[1], vtk_floor(it.pmax[1], a.window), a.sinks));
                    if (lane == 0) {
                        mt.there[word] = there;
                        mt.every[0][word] = every0;
                        mt.every[1][word] = every1;
                    }
                }
                __syncwarp();
                if (lane == 0) vtk_mbar_arrive(&sh.meta_full[c % AP_META]);
                if (j + 1 < T) fetch(j + 1);
            }
        });
    }
    __syncthreads();
    if (tid == 0) {
        if (sh.abort) atomicOr(a.flags, (uint32_t)VTOKEN_FLAG_TIMEOUT);
        __threadfence();
        if (atomicAdd(tickets + 1, 1u) == gridDim.x - 1) { tickets[0] = 0; tickets[1] = 0; }
    }
    if (warp == 12) {
        tc_after_sync();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
    }
}

template <int D, bool FP4, typename Act, bool PREFIX>
int launch(vtoken_ctx *ctx, const VtkAttnArgs &a, uint32_t *tickets, cudaStream_t st)
{
    constexpr int smem = (int)sizeof(Shared<D>) + 1024;
    static_assert(smem <= 232448, "shared memory of a CTA");
    auto kernel = attention_prompt_kernel<D, FP4, Act, PREFIX>;
    static std::atomic<int> allowed{-1};                     // the device that knows of this kernel's shared memory
    VTK_CUDA(ctx, vtk_allow_smem(ctx, allowed, (const void *)kernel, smem));
    // the sign of the scores' factor goes into the product (a zero factor: one that no 32-bit score can be seen through)
    const float scale = a.scale_log2 == 0.f ? 7.9e-31f : (a.scale_log2 < 0.f ? -a.scale_log2 : a.scale_log2);
    VTK_CUDA(ctx, vtk_launch_dependent(ctx, kernel, dim3(ctx->num_sms), dim3(AP_NT), smem, st, a, tickets, a.row_limit,
                                       (uint64_t)ctx->wait_limit_ns, scale, (int)(a.scale_log2 < 0.f), ctx->stall_item));
    VTK_CUDA(ctx, cudaGetLastError());
    return VTOKEN_OK;
}

template <int D, bool PREFIX>
int launch_by_type(vtoken_ctx *ctx, const vtoken_heads *h, const VtkAttnArgs &a, uint32_t *tickets, cudaStream_t st)
{
    if (h->kv_type == VTOKEN_KV_FP4)
        return h->act_type == VTOKEN_KV_BF16 ? launch<D, true, VtkBf16, PREFIX>(ctx, a, tickets, st) : launch<D, true, VtkFp16, PREFIX>(ctx, a, tickets, st);
    return h->act_type == VTOKEN_KV_BF16 ? launch<D, false, VtkBf16, PREFIX>(ctx, a, tickets, st) : launch<D, false, VtkFp16, PREFIX>(ctx, a, tickets, st);
}

}  // namespace

int vtk_launch_attention_prompt(vtoken_ctx *ctx, const vtoken_heads *heads, const VtkAttnArgs &a, uint32_t *tickets, bool prefix, cudaStream_t st)
{
    if (prefix) return heads->head_dim == 128 ? launch_by_type<128, true>(ctx, heads, a, tickets, st) : launch_by_type<64, true>(ctx, heads, a, tickets, st);
    return heads->head_dim == 128 ? launch_by_type<128, false>(ctx, heads, a, tickets, st) : launch_by_type<64, false>(ctx, heads, a, tickets, st);
}
