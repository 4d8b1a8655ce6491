// Attention of few query rows per request (a decode step) over the slot cache.
//
// Bound by HBM: every visible K and V row is read once, 4 * D flops per row, head and query.
//
// The cut.  A segment is (request, tile of query rows, key head); its cache is numbered in tiles of 16 tokens (32 of
// the 4-bit cache), and
// all tiles of all segments in one row.  Teams of warps take equal shares of that row -- so every SM reads the same
// number of bytes whatever the lengths -- and every CTA (one per SM) works them out for itself from the tables.  A
// team is one warp when there are segments enough, the CTA's warps when there are few.  Its warps take the tiles of a
// segment in turn, each with a running maximum and sum per query row and the output accumulators in registers, and
// join in shared memory at the segment's end.  A segment that lies inside one share is finished there; at most the
// first and the last segment of a share are parts of longer ones: they leave a partial row, and the last team to
// arrive joins the parts in the order of the tables, so the sums do not depend on who came when.
//
// The stream.  Each warp copies its tiles (K and V rows of one head, gathered by slot) with cp.async into a ring of
// its own, several tiles ahead and across the ends of segments, so that about 100 KB per SM are in flight through
// joins, query loads and masks.  Pieces of 16 bytes are permuted within a row so that the reads below are free of
// bank conflicts.
//
// The products.  The heads of a group (and the query tokens of a request) are the rows of one matrix product, so a
// K or V row is read once for all of them.  The order of the contracted dimension is free as long as both operands
// agree, so mma.m16n8k16 gets its fragments with 16-byte loads:
//   S = Q K^T : 8 dimensions of one token are the B fragment of two instructions;
//   O^T = V^T P^T : 8 dimensions of four tokens, paired up to the A fragment by byte permutes; the accumulator layout
//   of S (rows = queries, columns = tokens) is the B fragment of P^T as it is.
// P is handed to the second product as the sum of two 16-bit values, so that its rounding does not add to that of
// the 16-bit output; over the 4-bit cache the products run in half precision, whose 11 bits are enough next to a
// bf16 output.  These legacy matrix instructions are enough here: 8 or 16 rows leave a 128-row tcgen05 tile mostly
// empty, and at full HBM rate the products need well under a third of the legacy tensor rate.
#include "attention.cuh"

namespace {

constexpr int AT_ROW_LIMIT = 32;         // query rows (tokens times group) of a request up to which it is worked on here
constexpr int AT_KNOWN = 8;              // requests of a share that are looked up together at the start
constexpr int AT_MIN_SHARE = 2;          // tiles of the smallest share, for each warp of its team
constexpr int AT_PARTS = 3;              // shares that a segment of mean length is cut into at most, about

__device__ __forceinline__ uint32_t smem_u32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
template <int BYTES>
__device__ __forceinline__ void cp_async(uint32_t dst, const void *src, bool there)
{
    if (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(dst), "l"(src), "n"(BYTES), "r"(there ? BYTES : 0) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// ---- a tile of tokens of one head in a warp's ring ---------------------------------------------
// K fragments of 16 tokens: lane (g, t) takes of tokens g and 8 + g the dimensions kdim(t, j) .. + 7, j < D / 32.
// V fragments: lane (g, t) takes of tokens 2t, 2t + 1, 2t + 8, 2t + 9 the dimensions vdim(g, x) .. + 7, x < D / 64.
template <int D, typename Act>
struct Rows16 {
    static constexpr bool FP4 = false;
    using Mma = Act;
    static constexpr int WARPS = 8, TILE = 16, PITCH = D * 2, HALF = TILE * PITCH, STAGE = 2 * HALF, PIECES = D / 8;
    static __device__ __forceinline__ int kdim(int t, int j) { return 32 * j + 8 * t; }
    static __device__ __forceinline__ int vdim(int g, int x) { return 64 * x + 8 * g; }
    // slot: lane i < TILE holds that of token i, negative = zeros
    static __device__ __forceinline__ void issue(uint32_t dst, const uint8_t *k_rows, const uint8_t *v_rows, int64_t row_bytes, int, int head, int slot)
    {
        const int lane = vtk_lane(), c = lane % PIECES, sub = lane / PIECES;
        constexpr int PER = 32 / PIECES;
        const int64_t off0 = (int64_t)head * (D * 2) + 16 * c;
#pragma unroll
        for (int i = 0; i < TILE / PER; ++i) {
            const int tok = i * PER + sub, s = __shfl_sync(0xffffffffu, slot, tok);
            const int64_t off = (s < 0 ? 0 : s) * row_bytes + off0;
            cp_async<16>(dst + tok * PITCH + ((c ^ ((tok & 1) << 2)) << 4), k_rows + off, s >= 0);
            cp_async<16>(dst + HALF + tok * PITCH + ((c ^ (((tok >> 1) & 3) << 1)) << 4), v_rows + off, s >= 0);
        }
    }
    const uint8_t *at;
    __device__ __forceinline__ void get_k(int b, int u, int g, int t, uint4 (&k)[D / 32]) const
    {
#pragma unroll
        for (int j = 0; j < D / 32; ++j)
            k[j] = *reinterpret_cast<const uint4 *>(at + (16 * b + 8 * u + g) * PITCH + (((4 * j + t) ^ ((g & 1) << 2)) << 4));
    }
    // of token 16 b + 2t + (i & 1) + 8 (i >> 1)
    __device__ __forceinline__ void get_v(int b, int i, int g, int t, uint4 (&v)[D / 64]) const
    {
#pragma unroll
        for (int x = 0; x < D / 64; ++x)
            v[x] = *reinterpret_cast<const uint4 *>(at + HALF + (16 * b + 2 * t + (i & 1) + 8 * (i >> 1)) * PITCH + (((8 * x + g) ^ (t << 1)) << 4));
    }
};

template <int D, int W>
struct Rows4 {
    static constexpr bool FP4 = true;
    using Mma = VtkFp16;
    static constexpr int WARPS = W, TILE = 32, PITCH = D / 2, HALF = TILE * PITCH, SCALES = D / 16, PIECES = D / 32;
    static constexpr int STAGE = 2 * HALF + 2 * TILE * SCALES;
    static __device__ __forceinline__ int kdim(int t, int j) { return (D / 4) * t + 8 * j; }
    static __device__ __forceinline__ int vdim(int g, int x) { return (D / 8) * g + 8 * x; }
    static __device__ __forceinline__ int vswizzle(int tok, int c) { return D == 128 ? c ^ ((tok >> 1) & 3) : c; }
    static __device__ __forceinline__ void issue(uint32_t dst, const uint8_t *k_rows, const uint8_t *v_rows, int64_t row_bytes, int hkv, int head, int slot)
    {
        const int lane = vtk_lane(), c = lane % PIECES, sub = lane / PIECES;
        constexpr int PER = 32 / PIECES;
#pragma unroll
        for (int i = 0; i < TILE / PER; ++i) {
            const int tok = i * PER + sub, s = __shfl_sync(0xffffffffu, slot, tok);
            const int64_t off = (s < 0 ? 0 : s) * row_bytes + head * PITCH + 16 * c;
            cp_async<16>(dst + tok * PITCH + 16 * c, k_rows + off, s >= 0);
            cp_async<16>(dst + HALF + tok * PITCH + 16 * vswizzle(tok, c), v_rows + off, s >= 0);
        }
        const int64_t off = (slot < 0 ? 0 : slot) * row_bytes + hkv * PITCH + head * SCALES;
        cp_async<SCALES>(dst + 2 * HALF + lane * SCALES, k_rows + off, slot >= 0);
        cp_async<SCALES>(dst + 2 * HALF + (TILE + lane) * SCALES, v_rows + off, slot >= 0);
    }
    const uint8_t *at;
    __device__ __forceinline__ void get_k(int b, int u, int g, int t, uint4 (&k)[D / 32]) const
    {
        const uint8_t *codes = at + (16 * b + 8 * u + g) * PITCH + t * (D / 8), *sc = at + 2 * HALF + (16 * b + 8 * u + g) * SCALES;
        if (D == 128) {                  // words 0, 1 belong to the first of the lane's two groups, 2, 3 to the second
            const uint4 w = *reinterpret_cast<const uint4 *>(codes);
            const uint32_t two = vtk_scales_to_half2(*reinterpret_cast<const uint16_t *>(sc + 2 * t));
            const uint32_t s0 = __byte_perm(two, 0, 0x1010), s1 = __byte_perm(two, 0, 0x3232);
            k[0] = vtk_expand8(w.x, s0);
            k[1] = vtk_expand8(w.y, s0);
            k[D / 32 - 2] = vtk_expand8(w.z, s1);
            k[D / 32 - 1] = vtk_expand8(w.w, s1);
        } else {
            const uint2 w = *reinterpret_cast<const uint2 *>(codes);
            const uint32_t s0 = __byte_perm(vtk_scales_to_half2(sc[t]), 0, 0x1010);
            k[0] = vtk_expand8(w.x, s0);
            k[1] = vtk_expand8(w.y, s0);
        }
    }
    __device__ __forceinline__ void get_v(int b, int i, int g, int t, uint4 (&v)[D / 64]) const
    {
        const int tok = 16 * b + 2 * t + (i & 1) + 8 * (i >> 1);
        const uint32_t s0 = __byte_perm(vtk_scales_to_half2(at[2 * HALF + (TILE + tok) * SCALES + (D == 128 ? g : g >> 1)]), 0, 0x1010);
        const uint8_t *codes = at + HALF + tok * PITCH;
        if (D == 128) {
            const uint2 w = *reinterpret_cast<const uint2 *>(codes + 16 * vswizzle(tok, g >> 1) + 8 * (g & 1));
            v[0] = vtk_expand8(w.x, s0);
            v[D / 64 - 1] = vtk_expand8(w.y, s0);
        } else {
            v[0] = vtk_expand8(*reinterpret_cast<const uint32_t *>(codes + 4 * g), s0);
        }
    }
};

// ring stages of a warp: what is left of 227 KB next to the join buffer, eight at most
template <int NR, typename Rows, int D> constexpr int at_stages()
{
    constexpr int NW = Rows::WARPS, room = (231000 - 128 - NW * NR * 8 - NW * NR * D * 4) / NW / (Rows::STAGE + Rows::TILE * 4);
    return room > 8 ? 8 : room;
}

template <int D, int NR, typename Rows>
struct Shared {
    static constexpr int ST = at_stages<NR, Rows, D>(), NW = Rows::WARPS, NT = NW * 32;
    alignas(128) uint8_t ring[NW][ST][Rows::STAGE];
    alignas(16) union {
        float o[NW][NR][D];        // join: 16-byte pieces of a row permuted by the row
        struct { int prefix[NT + 1]; int warp_sum[NW], warp_segments[NW]; int segments; } plan;
    };
    float2 ml[NW][NR];
    int ids[NW][ST][Rows::TILE];
    int last[NW];
};

// one request as the cut sees it
struct Known {
    int q0, qn, len, tiles, row_tiles;
    int pmax, floor;                     // no query sees an id above pmax, nor one up to floor that is no sink
    VtkRequest s;                        // (base, lo, n_sink, n)
};

template <int NR, int TILE>
__device__ inline Known look_up(const VtkAttnArgs &a, int r, bool &clipped)
{
    Known k;
    bool c;
    vtk_request_rows(a, r, k.q0, k.qn, k.s.base, k.len, c);
    clipped |= c;
    if (k.qn * (int64_t)a.group > a.row_limit) k.qn = 0;
    k.s.lo = k.s.n_sink = 0;
    k.s.n = k.len;
    k.pmax = INT32_MAX - 1;
    k.floor = -1;
    k.row_tiles = (k.qn * a.group + NR - 1) / NR;
    if (k.qn > 0 && k.qn <= 8) {         // few queries: only what one of them can see
        const int last = vtk_last_id(a, k.s.base, k.len);
        int pmin = a.positions[k.q0], pmax = pmin;
        for (int i = 1; i < k.qn; ++i) {
            const int p = a.positions[k.q0 + i];
            pmin = p < pmin ? p : pmin;
            pmax = p > pmax ? p : pmax;
        }
        k.pmax = pmax;
        k.floor = vtk_floor(pmin, a.window);
        k.s = vtk_request_span(a, k.s.base, k.len, last, pmin, pmax);
    }
    k.tiles = k.qn > 0 ? (k.s.n > 0 ? (k.s.n + TILE - 1) / TILE : 1) : 0;
    return k;
}

// A walk over the segments of a share; the request it is at is kept in the warp's shared memory.
template <int NR, int TILE>
struct Walk {
    Known *k;
    int r, rt, kv, t0, t1;               // segment and its tiles [t0, t1) inside the share
    int64_t f, f1;                       // next tile of the row of all tiles, end of the share
    __device__ __forceinline__ void clip() { t1 = k->tiles - t0 < f1 - f ? k->tiles : t0 + (int)(f1 - f); }
    __device__ __forceinline__ bool done() const { return f >= f1; }
    static __device__ __forceinline__ bool in_window(int r, int r_known) { return r >= r_known && r - r_known < AT_KNOWN; }
    __device__ __forceinline__ void next(const VtkAttnArgs &a, const Known *known, int r_known)
    {
        f += t1 - t0;
        t0 = t1 = 0;
        if (done()) return;
        if (++kv == a.hkv) {
            kv = 0;
            if (++rt == k->row_tiles) {
                rt = 0;
                bool c = false;
                int tiles;
                do {
                    ++r;
                    const Known n = in_window(r, r_known) ? known[r - r_known] : look_up<NR, TILE>(a, r, c);
                    tiles = n.tiles;
                    __syncwarp();
                    if (vtk_lane() == 0) *k = n;
                    __syncwarp();
                } while (tiles == 0);
            }
        }
        clip();
    }
};

// NR: query rows of a segment (8 or 16); SPLIT_P: P as a sum of two 16-bit values
template <int D, int NR, typename Rows, typename Act, bool SPLIT_P>
__global__ void __launch_bounds__(Rows::WARPS * 32, 1) attention_rows_kernel(const __grid_constant__ VtkAttnArgs a)
{
    using Mma = typename Rows::Mma;
    using Sh = Shared<D, NR, Rows>;
    constexpr int RH = NR / 8, MT = D / 16, N = D / 32, ST = Sh::ST, TILE = Rows::TILE, NW = Rows::WARPS, NT = NW * 32;
    extern __shared__ __align__(128) uint8_t raw[];
    Sh &sh = *reinterpret_cast<Sh *>(raw);
    __shared__ Known s_known[AT_KNOWN], s_get[NW], s_use[NW];
    vtk_release_successor();
    vtk_wait_for_predecessor();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;

    // ---- the share: tiles before each thread's requests, by two or three rounds of loads per request and a scan ----
    int R = *a.num_requests;
    bool clipped = R < 0 || R > a.max_requests;
    R = R < 0 ? 0 : (R > a.max_requests ? a.max_requests : R);
    const int seg = (R + NT - 1) / NT;
    int mine = 0, my_segments = 0;
    Known own;                                               // the thread's last request: its only one below 257 requests
    for (int r = tid * seg; r < (tid + 1) * seg && r < R; ++r) {
        own = look_up<NR, TILE>(a, r, clipped);
        mine += own.tiles * own.row_tiles;
        my_segments += own.tiles > 0 ? own.row_tiles : 0;
    }
    if (clipped && blockIdx.x == 0) atomicOr(a.flags, (uint32_t)VTOKEN_FLAG_CAPACITY);
    {
        const int incl = vtk_warp_incl_scan(mine);
        my_segments = __reduce_add_sync(0xffffffffu, my_segments);
        if (lane == 31) {
            sh.plan.warp_sum[warp] = incl;
            sh.plan.warp_segments[warp] = my_segments;
        }
        __syncthreads();
        int before = 0, all_segments = 0;
        for (int w = 0; w < warp; ++w) before += sh.plan.warp_sum[w];
        for (int w = 0; w < NW; ++w) all_segments += sh.plan.warp_segments[w];
        if (tid == 0) sh.plan.segments = all_segments;
        sh.plan.prefix[tid + 1] = before + incl;
        if (tid == 0) sh.plan.prefix[0] = 0;
        __syncthreads();
    }
    const int64_t W = (int64_t)sh.plan.prefix[NT] * a.hkv;
    // ---- teams: the fewer segments there are, the more warps share one ----
    const int64_t segments = (int64_t)sh.plan.segments * a.hkv, warps = (int64_t)gridDim.x * NW;
    int team = NW;                                           // warps of a team
    if (segments * AT_PARTS >= warps) team = 1;
    else if (segments * AT_PARTS * (NW / 4) >= warps) team = NW / 4;
    else if (segments * AT_PARTS * (NW / 2) >= warps) team = NW / 2;
    const int teams = NW / team, my_team = warp / team, tw = warp % team;
    // at least AT_MIN_SHARE tiles a warp: a segment that is cut finer costs more to join than it gains
    const int64_t most = (W + AT_MIN_SHARE * team - 1) / (AT_MIN_SHARE * team), G = most < (int64_t)gridDim.x * teams ? most : (int64_t)gridDim.x * teams;
    const bool packed = G == (int64_t)gridDim.x * teams;     // a CTA's shares side by side; few shares: on different SMs
    const int share0 = packed ? blockIdx.x * teams : blockIdx.x, share = packed ? share0 + my_team : my_team * gridDim.x + blockIdx.x;
    auto find = [&](int64_t f) {                             // thread segment that holds tile f
        const int at = (int)(f / a.hkv);                     // (in tiles of one key head)
        int lo = 0, hi = NT;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (sh.plan.prefix[mid] <= at) lo = mid; else hi = mid;
        }
        return lo;
    };
    Walk<NR, TILE> use;
    use.f = share < G ? W * share / G : 0;
    use.f1 = share < G ? W * (share + 1) / G : 0;
    use.k = &s_use[warp];
    int64_t left = 0;
    if (share < G) {
        const int lo = find(use.f);
        left = use.f - (int64_t)sh.plan.prefix[lo] * a.hkv;
        use.r = lo * seg;
    }
    const int known0 = G > 0 ? find(share0 < G ? W * share0 / G : 0) : 0;
    if (seg == 1 && tid >= known0 && tid < known0 + AT_KNOWN && tid < R) s_known[tid - known0] = own;
    const int r_known = seg == 1 ? known0 : INT32_MAX;
    __syncthreads();                                         // the plan's arrays become the join buffers
    if (share >= G) return;
    for (;; ++use.r) {
        bool c = false;
        const Known k = use.in_window(use.r, r_known) ? s_known[use.r - r_known] : look_up<NR, TILE>(a, use.r, c);
        const int64_t all = (int64_t)k.tiles * k.row_tiles * a.hkv;
        if (left < all) {
            if (lane == 0) s_use[warp] = s_get[warp] = k;
            __syncwarp();
            break;
        }
        left -= all;
    }
    use.rt = (int)(left / ((int64_t)use.k->tiles * a.hkv));
    left -= (int64_t)use.rt * use.k->tiles * a.hkv;
    use.kv = (int)(left / use.k->tiles);
    use.t0 = (int)(left - (int64_t)use.kv * use.k->tiles);
    use.clip();
    auto team_sync = [&]() {
        if (team == 1) __syncwarp();
        else asm volatile("barrier.cta.sync %0, %1;" ::"r"(1 + my_team), "r"(team * 32) : "memory");
    };

    // ---- the stream: this warp's tiles, ST - 1 ahead of their use, whatever segment they are of ----
    struct Next {                                            // a tile whose slots are on their way
        int slot, id, kv, pmax, floor;
        bool there;
    };
    Walk<NR, TILE> get = use;
    get.k = &s_get[warp];
    int tile = get.t0 + tw, issued = 0;
    bool more = true;
    auto meta = [&]() {                                      // the warp's next tile: slots and ids of its tokens
        while (more && tile >= get.t1) {
            get.next(a, s_known, r_known);
            more = !get.done();
            tile = get.t0 + tw;
        }
        Next n;
        n.slot = -1;
        n.id = INT32_MAX;
        n.pmax = n.floor = -1;
        n.kv = get.kv;
        n.there = more;
        const int v = tile * TILE + lane;
        if (more && lane < TILE && v < get.k->s.n) {
            n.slot = a.cache_slots[get.k->s.entry(v)];
            n.id = a.cache_ids.null() ? get.k->s.index(v) : a.cache_ids[get.k->s.entry(v)];
            n.pmax = get.k->pmax;
            n.floor = get.k->floor;
        }
        tile += team;
        return n;
    };
    auto issue = [&](Next n) {
        if (n.there) {
            if (n.slot >= 0 && (int64_t)n.slot >= a.slots_per_layer) {
                atomicOr(a.flags, (uint32_t)VTOKEN_FLAG_BAD_SLOT);
                n.slot = -1;
            }
            if (!vtk_sees(n.id, n.pmax, n.floor, a.sinks)) n.slot = -1;
            const int stage = issued % ST;
            if (lane < TILE) sh.ids[warp][stage][lane] = n.slot < 0 ? INT32_MAX : n.id;
            Rows::issue(smem_u32(sh.ring[warp][stage]), a.k_rows, a.v_rows, a.row_bytes, a.hkv, n.kv, n.slot);
            ++issued;
        }
        cp_commit();
    };
    Next next;
    {
        Next first[ST - 1];
#pragma unroll
        for (int i = 0; i < ST - 1; ++i) first[i] = meta();
        next = meta();
#pragma unroll
        for (int i = 0; i < ST - 1; ++i) issue(first[i]);
    }

    int used = 0;
    for (; !use.done(); use.next(a, s_known, r_known)) {
        const int kv = use.kv, rt = use.rt;
        const int rows = use.k->qn * a.group - rt * NR < NR ? use.k->qn * a.group - rt * NR : NR;
        // ---- queries: lane (g, t) holds of rows g and 8 + g the dimensions its K fragments hold ----
        uint4 q[RH][D / 32];
        int pos[RH], floor[RH];
        float scale[RH];
#pragma unroll
        for (int h = 0; h < RH; ++h) {
            const int row = g + 8 * h, at = rt * NR + row;
            pos[h] = floor[h] = -1;
            scale[h] = a.scale_log2;
            const uint16_t *p = nullptr;
            if (row < rows) {
                const int64_t tok = use.k->q0 + at / a.group;
                pos[h] = a.positions[tok];
                floor[h] = vtk_floor(pos[h], a.window);
                p = a.q + tok * a.q_stride + (int64_t)(kv * a.group + at % a.group) * D;
            }
#pragma unroll
            for (int j = 0; j < D / 32; ++j)
                q[h][j] = p != nullptr ? *reinterpret_cast<const uint4 *>(p + Rows::kdim(t, j)) : make_uint4(0, 0, 0, 0);
            if (Rows::FP4 && Act::kind == VTOKEN_KV_BF16) {
                // bf16 queries in half precision: the row times a power of two that puts its largest value at
                // 2^14 .. 2^15; what falls below half's range is 2^-38 of that
                float top = 0.f, x[8];
#pragma unroll
                for (int j = 0; j < D / 32; ++j) {
                    vtk_unpack8<VtkBf16>(q[h][j], x);
#pragma unroll
                    for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(x[e]));
                }
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                int e2 = (int)(__float_as_uint(top) >> 23) - 127;          // floor(log2), subnormals -127
                e2 = 14 - (e2 > 100 ? 100 : (e2 < -100 ? -100 : e2));
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
        int pmin = INT32_MAX, pmax = -1;
#pragma unroll
        for (int h = 0; h < RH; ++h) {
            if (g + 8 * h < rows) pmin = pos[h] < pmin ? pos[h] : pmin;
            pmax = pos[h] > pmax ? pos[h] : pmax;
        }
        pmin = __reduce_min_sync(0xffffffffu, pmin);
        pmax = __reduce_max_sync(0xffffffffu, pmax);
        const int floor_min = vtk_floor(pmin, a.window), floor_max = vtk_floor(pmax, a.window);

        float o[MT][RH][4], m[RH], l[RH];
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int h = 0; h < RH; ++h)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[i][h][e] = 0.f;
#pragma unroll
        for (int h = 0; h < RH; ++h) { m[h] = -INFINITY; l[h] = 0.f; }

        for (int tl = use.t0 + tw; tl < use.t1; tl += team, ++used) {
            cp_wait<ST - 2>();
            __syncwarp();
            issue(next);
            next = meta();
            const int stage = used % ST;
            Rows rows_now;
            rows_now.at = sh.ring[warp][stage];
            const int *ids = sh.ids[warp][stage];
            const int my_id = ids[lane & (TILE - 1)];
            if (!__any_sync(0xffffffffu, vtk_sees(my_id, pmax, floor_min, a.sinks))) continue;
            const bool full = __all_sync(0xffffffffu, vtk_sees(my_id, pmin, floor_max, a.sinks));
            constexpr int SUB = TILE / 16;
            float p[SUB][2][4], tile_max[RH];
#pragma unroll
            for (int b = 0; b < SUB; ++b)
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    p[b][u][0] = p[b][u][1] = p[b][u][2] = p[b][u][3] = 0.f;
                    uint4 k[D / 32];
                    rows_now.get_k(b, u, g, t, k);
#pragma unroll
                    for (int j = 0; j < D / 32; ++j) {
                        vtk_mma<Mma>(p[b][u], q[0][j].x, RH == 2 ? q[RH - 1][j].x : 0u, q[0][j].y, RH == 2 ? q[RH - 1][j].y : 0u, k[j].x, k[j].y);
                        vtk_mma<Mma>(p[b][u], q[0][j].z, RH == 2 ? q[RH - 1][j].z : 0u, q[0][j].w, RH == 2 ? q[RH - 1][j].w : 0u, k[j].z, k[j].w);
                    }
                }
#pragma unroll
            for (int h = 0; h < RH; ++h) tile_max[h] = -INFINITY;
#pragma unroll
            for (int b = 0; b < SUB; ++b)
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int e = 0; e < 2 * RH; ++e) p[b][u][e] *= scale[e >> 1];
            if (!full) {
#pragma unroll
                for (int b = 0; b < SUB; ++b)
#pragma unroll
                    for (int u = 0; u < 2; ++u)
#pragma unroll
                        for (int e = 0; e < 2 * RH; ++e)
                            if (!vtk_sees(ids[16 * b + 2 * t + (e & 1) + 8 * u], pos[e >> 1], floor[e >> 1], a.sinks)) p[b][u][e] = -INFINITY;
            }
#pragma unroll
            for (int b = 0; b < SUB; ++b)
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int e = 0; e < 2 * RH; ++e) tile_max[e >> 1] = fmaxf(tile_max[e >> 1], p[b][u][e]);
            // the running maximum moves only when a score passes it by 2^8: sums and P stay far inside 32 bits
            bool up = tile_max[0] > m[0] + 8.f;
            if (RH == 2) up |= tile_max[RH - 1] > m[RH - 1] + 8.f;
            if (__any_sync(0xffffffffu, up)) {
#pragma unroll
                for (int h = 0; h < RH; ++h) {
                    float x = tile_max[h];
                    x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
                    x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
                    x = fmaxf(x, m[h]);
                    const float f = m[h] == -INFINITY ? 0.f : vtk_exp2(m[h] - x);
                    m[h] = x;
                    l[h] *= f;
                    const float f0 = __shfl_sync(0xffffffffu, f, 8 * t), f1 = __shfl_sync(0xffffffffu, f, 8 * t + 4);
#pragma unroll
                    for (int i = 0; i < MT; ++i) {
                        o[i][h][0] *= f0; o[i][h][1] *= f1;
                        o[i][h][2] *= f0; o[i][h][3] *= f1;
                    }
                }
            }
#pragma unroll
            for (int b = 0; b < SUB; ++b) {
                uint32_t w[RH][2], w_lo[RH][2];
#pragma unroll
                for (int h = 0; h < RH; ++h) {
                    const float base = m[h] == -INFINITY ? 0.f : m[h];
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const float p0 = vtk_exp2(p[b][u][2 * h] - base), p1 = vtk_exp2(p[b][u][2 * h + 1] - base);
                        l[h] += p0 + p1;
                        w[h][u] = Mma::pack(p0, p1);
                        if (SPLIT_P) {
                            const float2 r = Mma::unpack(w[h][u]);
                            w_lo[h][u] = Mma::pack(p0 - r.x, p1 - r.y);
                        }
                    }
                }
                uint4 v[4][D / 64];
#pragma unroll
                for (int i = 0; i < 4; ++i) rows_now.get_v(b, i, g, t, v[i]);
#pragma unroll
                for (int x = 0; x < D / 64; ++x) {
                    const uint32_t w0[4] = {v[0][x].x, v[0][x].y, v[0][x].z, v[0][x].w}, w1[4] = {v[1][x].x, v[1][x].y, v[1][x].z, v[1][x].w};
                    const uint32_t w2[4] = {v[2][x].x, v[2][x].y, v[2][x].z, v[2][x].w}, w3[4] = {v[3][x].x, v[3][x].y, v[3][x].z, v[3][x].w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t a0 = __byte_perm(w0[i], w1[i], 0x5410), a1 = __byte_perm(w0[i], w1[i], 0x7632);
                        const uint32_t a2 = __byte_perm(w2[i], w3[i], 0x5410), a3 = __byte_perm(w2[i], w3[i], 0x7632);
#pragma unroll
                        for (int h = 0; h < RH; ++h) {
                            vtk_mma<Mma>(o[4 * x + i][h], a0, a1, a2, a3, w[h][0], w[h][1]);
                            if (SPLIT_P) vtk_mma<Mma>(o[4 * x + i][h], a0, a1, a2, a3, w_lo[h][0], w_lo[h][1]);
                        }
                    }
                }
            }
        }

        // ---- join the team's warps ----
        auto piece = [](int row, int c) { return ((c ^ (row & 7)) << 2); };      // 16-byte piece c of a row
#pragma unroll
        for (int h = 0; h < RH; ++h) {
            l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
            l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
            if (t == 0) sh.ml[warp][g + 8 * h] = make_float2(m[h], l[h]);
#pragma unroll
            for (int x = 0; x < D / 64; ++x)
#pragma unroll
                for (int e = 0; e < 2; ++e) {                // query row 2t + e: eight consecutive dimensions
                    const int row = 8 * h + 2 * t + e, c = Rows::vdim(g, x) / 4;
                    *reinterpret_cast<float4 *>(&sh.o[warp][row][piece(row, c)]) = make_float4(o[4 * x][h][e], o[4 * x][h][2 + e], o[4 * x + 1][h][e], o[4 * x + 1][h][2 + e]);
                    *reinterpret_cast<float4 *>(&sh.o[warp][row][piece(row, c + 1)]) = make_float4(o[4 * x + 2][h][e], o[4 * x + 2][h][2 + e], o[4 * x + 3][h][e], o[4 * x + 3][h][2 + e]);
                }
        }
        team_sync();
        const int w0 = my_team * team;
        const int64_t seg_lo = use.f - use.t0, seg_hi = seg_lo + use.k->tiles;
        const bool whole = use.t0 == 0 && use.t1 == use.k->tiles;
        // shares that hold parts of this segment, and where a share leaves its part
        const int first = (int)(((seg_lo + 1) * G - 1) / W), parts = (int)((seg_hi * G - 1) / W) - first + 1;
        auto part_at = [&](int i) { return a.part + (int64_t)(2 * i + (i == first)) * (NR * (D + 2)); };
        auto finish = [&](int row, float (&acc)[N], float mm, float ll) {
            const int at = rt * NR + row, head = kv * a.group + at % a.group;
            const int64_t tok = use.k->q0 + at / a.group;
            bool bad = !(fabsf(ll) < INFINITY);
#pragma unroll
            for (int j = 0; j < N; ++j) bad |= !(fabsf(acc[j]) < INFINITY);
            if (use.k->qn > 1 && __any_sync(0xffffffffu, bad))   // (one query token: what it does not see was not read)
                vtk_row_again<D, Rows::FP4, Act>(a, tok, head, a.positions[tok], use.k->s.base, use.k->len, acc, mm, ll);
            vtk_store_row<D, Act>(a, tok, head, acc, mm, ll);
        };
        for (int row = tw; row < rows; row += team) {
            float mm = -INFINITY, ll = 0.f, acc[N];
#pragma unroll
            for (int j = 0; j < N; ++j) acc[j] = 0.f;
            for (int w = w0; w < w0 + team; ++w) mm = fmaxf(mm, sh.ml[w][row].x);
#pragma unroll 4
            for (int w = w0; w < w0 + team; ++w) {
                const float2 ml = sh.ml[w][row];
                const float f = ml.x == -INFINITY ? 0.f : (ml.x == mm ? 1.f : vtk_exp2(ml.x - mm));
                ll += f * ml.y;
                const float *src = &sh.o[w][row][piece(row, lane * N / 4) + (lane * N) % 4];
#pragma unroll
                for (int j = 0; j < N; ++j) acc[j] += f * src[j];
            }
            if (!whole) {
                float *dst = part_at(share) + row * D + lane * N;
                if (N == 4) *reinterpret_cast<float4 *>(dst) = make_float4(acc[0], acc[1], acc[N - 2], acc[N - 1]);
                else *reinterpret_cast<float2 *>(dst) = make_float2(acc[0], acc[1]);
                if (lane == 0) *reinterpret_cast<float2 *>(part_at(share) + NR * D + 2 * row) = make_float2(mm, ll);
            } else {
                finish(row, acc, mm, ll);
            }
        }
        if (!whole) {
            __threadfence();
            team_sync();
            if (tw == 0 && lane == 0) {
                const bool last = atomicAdd(&a.counters[first], 1u) == (unsigned)(parts - 1);
                if (last) a.counters[first] = 0;             // ready for the next call
                sh.last[my_team] = last;
            }
            team_sync();
            if (*(volatile int *)&sh.last[my_team]) {
                __threadfence();
                for (int row = tw; row < rows; row += team) {
                    float mm = -INFINITY, ll = 0.f, acc[N];
#pragma unroll
                    for (int j = 0; j < N; ++j) acc[j] = 0.f;
                    for (int i = lane; i < parts; i += 32) mm = fmaxf(mm, __ldcg(part_at(first + i) + NR * D + 2 * row));
#pragma unroll
                    for (int d = 16; d > 0; d >>= 1) mm = fmaxf(mm, __shfl_xor_sync(0xffffffffu, mm, d));
#pragma unroll 8
                    for (int i = 0; i < parts; ++i) {
                        const float *src = part_at(first + i);
                        const float2 ml = __ldcg(reinterpret_cast<const float2 *>(src + NR * D + 2 * row));
                        const float f = ml.x == -INFINITY ? 0.f : (ml.x == mm ? 1.f : vtk_exp2(ml.x - mm));
                        ll += f * ml.y;
                        src += row * D + lane * N;
                        if (N == 4) {
                            const float4 x = __ldcg(reinterpret_cast<const float4 *>(src));
                            acc[0] += f * x.x; acc[1] += f * x.y; acc[N - 2] += f * x.z; acc[N - 1] += f * x.w;
                        } else {
                            const float2 x = __ldcg(reinterpret_cast<const float2 *>(src));
                            acc[0] += f * x.x; acc[1] += f * x.y;
                        }
                    }
                    finish(row, acc, mm, ll);
                }
            }
        }
        team_sync();                                         // the join buffers are used by the next segment
    }
}

template <int D, int NR, typename Rows, typename Act, bool SPLIT_P>
int launch(vtoken_ctx *ctx, const VtkAttnArgs &a, cudaStream_t st)
{
    auto kernel = attention_rows_kernel<D, NR, Rows, Act, SPLIT_P>;
    constexpr int smem = (int)sizeof(Shared<D, NR, Rows>);
    static_assert(Shared<D, NR, Rows>::ST >= 2 && smem + sizeof(Known) * (AT_KNOWN + 2 * Rows::WARPS) <= 232448, "shared memory of a CTA");
    VTK_CUDA(ctx, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
    VTK_CUDA(ctx, vtk_launch_dependent(ctx, kernel, dim3(ctx->num_sms), dim3(Rows::WARPS * 32), smem, st, a));
    VTK_CUDA(ctx, cudaGetLastError());
    return VTOKEN_OK;
}

template <int D, typename Act>
int launch_by_type(vtoken_ctx *ctx, bool fp4, bool wide, const VtkAttnArgs &a, cudaStream_t st)
{
    constexpr bool bf = Act::kind == VTOKEN_KV_BF16;
    if (fp4) return wide ? launch<D, 16, Rows4<D, 8>, Act, !bf>(ctx, a, st) : launch<D, 8, Rows4<D, 12>, Act, !bf>(ctx, a, st);
    return wide ? launch<D, 16, Rows16<D, Act>, Act, true>(ctx, a, st) : launch<D, 8, Rows16<D, Act>, Act, true>(ctx, a, st);
}

float two_to(int e)
{
    float x = 1.f;
    for (; e > 0; --e) x *= 2.f;
    for (; e < 0; ++e) x *= 0.5f;
    return x;
}

}  // namespace

// A share leaves at most two partial row tiles (8 rows a tile from up to 12 teams a CTA, or 16 from up to 8).
int64_t vtk_attention_rows_workspace(const vtoken_ctx *ctx, const vtoken_heads *heads, VtkAttnArgs *a)
{
    const int64_t shares = (int64_t)ctx->num_sms * 12;
    const int64_t counters = (shares * 4 + 15) / 16 * 16 + 16;       // and the prompt kernel's two tickets in front
    if (a) a->part = (float *)((uint8_t *)(a->counters - 4) + counters);
    return counters + shares * 2 * (16 * 8 / 12 + 1) * (heads->head_dim + 2) * 4;
}

int vtk_launch_attention_rows(vtoken_ctx *ctx, const vtoken_heads *heads, VtkAttnArgs a, int32_t max_query_len, cudaStream_t st)
{
    vtk_attention_rows_workspace(ctx, heads, &a);
    const bool fp4 = heads->kv_type == VTOKEN_KV_FP4, wide = (int64_t)a.group * max_query_len > 8;
    if (heads->head_dim == 128)
        return heads->act_type == VTOKEN_KV_BF16 ? launch_by_type<128, VtkBf16>(ctx, fp4, wide, a, st) : launch_by_type<128, VtkFp16>(ctx, fp4, wide, a, st);
    return heads->act_type == VTOKEN_KV_BF16 ? launch_by_type<64, VtkBf16>(ctx, fp4, wide, a, st) : launch_by_type<64, VtkFp16>(ctx, fp4, wide, a, st);
}

extern "C" {

int64_t vtoken_attention_workspace_bytes(const vtoken_ctx *ctx, const vtoken_heads *heads, int32_t max_query_tokens)
{
    if (!ctx || vtk_check_heads(ctx, heads, 0) != VTOKEN_OK || max_query_tokens < 0) return VTOKEN_EINVAL;
    return vtk_attention_rows_workspace(ctx, heads, nullptr);
}

int vtoken_attention(vtoken_ctx *ctx, const vtoken_heads *heads, int32_t layer, const vtoken_attention_in *in, void *cuda_stream)
{
    if (!ctx || !heads || !in) return VTOKEN_EINVAL;
    if (vtk_check_heads(ctx, heads, layer) != VTOKEN_OK) return VTOKEN_EINVAL;
    if (!in->num_requests || !in->q_offsets || !in->positions || !in->q || !in->tt_offsets || !in->cache_slots || !in->cache_len ||
        !in->out || !in->workspace)
        return VTOKEN_EINVAL;
    if (in->max_query_tokens < 0 || in->max_query_len < 1 || in->window < 0 || in->sinks < 0) return VTOKEN_EINVAL;
    if (!(in->sm_scale > -1e30f && in->sm_scale < 1e30f)) return VTOKEN_EINVAL;
    if (((uintptr_t)in->q | (uintptr_t)in->out | (uintptr_t)in->workspace) & 15) return VTOKEN_EINVAL;
    VtkAttnArgs a;
    const int64_t dense = (int64_t)heads->num_q_heads * heads->head_dim;
    a.q_stride = vtk_stride(in->q_stride, dense);
    a.out_stride = vtk_stride(in->out_stride, dense);
    if (a.q_stride < 0 || a.out_stride < 0) return VTOKEN_EINVAL;
    if (in->workspace_bytes < vtoken_attention_workspace_bytes(ctx, heads, in->max_query_tokens)) return VTOKEN_ECAPACITY;
    if (in->max_query_tokens == 0) return VTOKEN_OK;
    a.num_requests = in->num_requests;
    a.q_offsets = VTK_ARR(ctx, in->q_offsets, ctx->cfg.max_requests + 1);
    a.positions = VTK_ARR(ctx, in->positions, in->max_query_tokens);
    a.tt_offsets = VTK_ARR(ctx, in->tt_offsets, ctx->cfg.max_requests + 1);
    a.cache_slots = VTK_ARR(ctx, in->cache_slots, ctx->cfg.max_tokens);
    a.cache_ids = VTK_ARR(ctx, in->cache_ids, ctx->cfg.max_tokens);
    a.cache_len = VTK_ARR(ctx, in->cache_len, ctx->cfg.max_requests);
    a.q = (const uint16_t *)in->q;
    a.out = (uint16_t *)in->out;
    a.lse = in->lse;
    a.k_rows = (const uint8_t *)ctx->cfg.k_pool + layer * ctx->layer_stride;
    a.v_rows = (const uint8_t *)ctx->cfg.v_pool + layer * ctx->layer_stride;
    a.row_bytes = ctx->row_bytes;
    a.slots_per_layer = ctx->slots_per_layer;
    a.max_tokens = ctx->cfg.max_tokens;
    a.max_requests = ctx->cfg.max_requests;
    a.max_query_tokens = in->max_query_tokens;
    a.hq = heads->num_q_heads;
    a.hkv = heads->num_kv_heads;
    a.group = heads->num_q_heads / heads->num_kv_heads;
    a.window = in->window;
    a.sinks = in->window > 0 ? in->sinks : 0;
    a.scale_log2 = in->sm_scale * 1.4426950408889634f * two_to(heads->k_exponent);
    a.v_mul = two_to(heads->v_exponent);
    a.flags = &ctx->rt_counts->error_flags;
    a.counters = (uint32_t *)in->workspace + 4;
    a.part = nullptr;
    const bool prompts = (int64_t)in->max_query_len * a.group > AT_ROW_LIMIT;
    a.row_limit = prompts ? AT_ROW_LIMIT : INT32_MAX;
    const int rc = vtk_launch_attention_rows(ctx, heads, a, prompts ? 1 : in->max_query_len, (cudaStream_t)cuda_stream);
    return rc == VTOKEN_OK && prompts ? vtk_launch_attention_prompt(ctx, heads, a, (uint32_t *)in->workspace, (cudaStream_t)cuda_stream) : rc;
}

}  // extern "C"
