// Attention of few query rows per request (a decode step) over the slot cache.
//
// Bound by HBM: every visible K and V row is read once, 4 * D flops per row, head and query.  512 requests over 3.1 GB of
// 16-bit rows take 536 to 564 us from machine to machine (5.5 to 5.8 TB/s, 0.85 to 0.89 of the copy bandwidth).  256 requests over 650 MB of
// 4-bit rows take 238 us: there 63 % of the issue slots are taken (ALU 50 %, DRAM 33 %), by about 400 instructions for 16 tokens of
// a head to expand codes and scales, and the warps, four a scheduler, wait on their own chains of them; the instantiation with 512
// threads has 128 registers and spills (336 bytes of loads).  A small call takes 6 us of dependent loads (requests, lengths,
// positions, slots, rows); 64 requests over 137 MB take 44 us at 25 % of the issue slots: latency of the plan, of the first tiles and
// of the joins.
//
// The cut.  A segment is (request, tile of query rows, group of key heads); its cache is numbered in tiles of 16 tokens, and
// all tiles of all segments in one row.  Teams of warps take equal shares of that row -- so every SM reads the same
// number of bytes whatever the lengths -- and every CTA (one per SM) works them out for itself from the tables.  A
// team has a warp for each head of the group, and more of them per head, its lanes, when there are few segments.  The lanes take
// the tiles of a segment in turn, each with a running maximum and sum per query row and the output accumulators in
// registers, and join in shared memory at the segment's end.  A segment that lies inside one share is finished there; at most
// the first and the last segment of a share are parts of longer ones: they leave a partial row, and the last team to
// arrive joins the parts in the order of the tables, so the sums do not depend on who came when.
// Groups: one head over 16-bit rows (256 bytes of a row are read well by themselves, and more segments mean fewer parts), up
// to eight over 4-bit rows, whose 64 bytes of codes and 8 of scales would each cost a sector of DRAM when the heads of a row are
// read at different times (324 us with groups of one, 240 with eight, at that step, on the 256 requests).
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
// the 16-bit output (in half precision they carry 2^7, see vtk_lift); over the 4-bit cache the products run in half precision, whose 11 bits are enough next to a
// bf16 output.  These legacy matrix instructions are enough here: 8 or 16 rows leave a 128-row tcgen05 tile mostly
// empty, and at full HBM rate the products need well under a third of the legacy tensor rate.
#include "attention.cuh"

namespace {

constexpr int AT_ROW_LIMIT = 32;         // query rows (tokens times group) of a request up to which it is worked on here
constexpr int AT_KNOWN = 8;              // requests of a share that are looked up together at the start
constexpr int AT_MIN_SHARE = 2;          // tiles of the smallest share, for each warp of its team
constexpr int AT_PARTS = 3;              // shares that a segment of mean length is cut into at most, about

__device__ __forceinline__ void cp_async16(uint32_t dst, const void *src, bool there)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
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
    static constexpr int WARPS = 8, GROUP = 1, TILE = 16, PITCH = D * 2, HALF = TILE * PITCH, STAGE = 2 * HALF, PIECES = D / 8;
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
            cp_async16(dst + tok * PITCH + ((c ^ ((tok & 1) << 2)) << 4), k_rows + off, s >= 0);
            cp_async16(dst + HALF + tok * PITCH + ((c ^ (((tok >> 1) & 3) << 1)) << 4), v_rows + off, s >= 0);
        }
    }
    const uint8_t *at;
    __device__ __forceinline__ void set(const uint8_t *stage, int) { at = stage; }
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
    static constexpr int WARPS = W, GROUP = 8, TILE = 16, PITCH = D / 2, HALF = TILE * PITCH, SCALES = D / 16, PIECES = D / 32;
    static constexpr int STAGE = 2 * HALF + 2 * TILE * 16;
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
            cp_async16(dst + tok * PITCH + 16 * c, k_rows + off, s >= 0);
            cp_async16(dst + HALF + tok * PITCH + 16 * vswizzle(tok, c), v_rows + off, s >= 0);
        }
        // scales: the aligned 16 bytes that hold the head's; lanes 0 .. 15 of K, 16 .. 31 of V
        const int sl = __shfl_sync(0xffffffffu, slot, lane & 15);
        const int64_t off = (sl < 0 ? 0 : sl) * row_bytes + hkv * PITCH + ((head * SCALES) & ~15);
        cp_async16(dst + 2 * HALF + lane * 16, (lane < TILE ? k_rows : v_rows) + off, sl >= 0);
    }
    const uint8_t *at;
    int mine;                            // the head's scales in their 16 bytes
    __device__ __forceinline__ void set(const uint8_t *stage, int head) { at = stage; mine = (head * SCALES) & 15; }
    __device__ __forceinline__ void get_k(int b, int u, int g, int t, uint4 (&k)[D / 32]) const
    {
        const uint8_t *codes = at + (16 * b + 8 * u + g) * PITCH + t * (D / 8), *sc = at + 2 * HALF + (16 * b + 8 * u + g) * 16 + mine;
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
        const uint32_t s0 = __byte_perm(vtk_scales_to_half2(at[2 * HALF + (TILE + tok) * 16 + mine + (D == 128 ? g : g >> 1)]), 0, 0x1010);
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
    constexpr int NW = Rows::WARPS, room = (230900 - 128 - NW * NR * 8 - NW * NR * D * 4) / NW / (Rows::STAGE + Rows::TILE * 4);
    return room > 8 ? 8 : room;
}

template <int D, int NR, typename Rows>
struct Shared {
    static constexpr int ST = at_stages<NR, Rows, D>(), NW = Rows::WARPS, NT = NW * 32;
    alignas(128) uint8_t ring[NW][ST][Rows::STAGE];
    alignas(16) union {
        float o[NW][NR * D];             // join: a warp's accumulators, 16 bytes a lane
        struct { int64_t warp_sum[NW], before[NW]; int warp_segments[NW], start[NW]; } plan;
    };
    float2 ml[NW][NR];
    int ids[NW][ST][Rows::TILE];
    int last[NW], bad[NW];
};

// (a 64-bit division is a subroutine of several hundred cycles)
__device__ __forceinline__ int64_t divide(int64_t x, int64_t y)
{
    return ((uint64_t)(x | y) >> 32) == 0 ? (int64_t)((uint32_t)x / (uint32_t)y) : x / y;
}

// query row -> token and head of the group (an integer division is forty instructions; the quotient in 32-bit floating point
// is off by one at most)
__device__ __forceinline__ void split_row(const VtkAttnArgs &a, int row, int64_t &tok, int &head)
{
    int q = row < (1 << 22) ? __float2int_rz((float)row * a.inv_group) : row / a.group, r = row - q * a.group;
    if (r < 0) { --q; r += a.group; }
    if (r >= a.group) { ++q; r -= a.group; }
    tok = q;
    head = r;
}

// what a part counts for next to a maximum
__device__ __forceinline__ float weight(float m, float top) { return m == -INFINITY ? 0.f : (m == top ? 1.f : vtk_exp2(m - top)); }

// one request as the cut sees it
struct Known {
    int q0, qn, len, tiles, row_tiles;
    VtkRequest s;
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
    k.s.pmax = k.s.floor = -1;
    k.row_tiles = (k.qn * a.group + NR - 1) / NR;
    if (k.qn > 0) {                      // only what one of the queries can see
        const int last = vtk_last_id(a, k.s.base, k.len);
        int pmin = a.positions[k.q0], pmax = pmin;
#pragma unroll 4
        for (int i = 1; i < k.qn; ++i) {
            const int p = a.positions[k.q0 + i];
            pmin = p < pmin ? p : pmin;
            pmax = p > pmax ? p : pmax;
        }
        k.s = vtk_request_span(a, k.s.base, k.len, last, pmin, pmax);
    }
    k.tiles = k.qn > 0 ? (k.s.n > 0 ? (k.s.n + TILE - 1) / TILE : 1) : 0;
    return k;
}

// A walk over the segments of a share; the request it is at is kept in the warp's shared memory.
template <int NR, int TILE>
struct Walk {
    Known *k;
    int r, rt, hg, t0, t1;               // segment (hg: group of key heads) and its tiles [t0, t1) inside the share
    int64_t f, f1;                       // next tile of the row of all tiles, end of the share
    __device__ __forceinline__ void clip() { t1 = k->tiles - t0 < f1 - f ? k->tiles : t0 + (int)(f1 - f); }
    __device__ __forceinline__ bool done() const { return f >= f1; }
    static __device__ __forceinline__ bool in_window(int r, int r_known) { return r >= r_known && r - r_known < AT_KNOWN; }
    __device__ __forceinline__ void next(const VtkAttnArgs &a, int groups, const Known *known, int r_known)
    {
        f += t1 - t0;
        t0 = t1 = 0;
        if (done()) return;
        if (++hg == groups) {
            hg = 0;
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
    int64_t mine = 0;                                        // (a prompt that the hint did not tell of may have 2^31 of them by itself)
    int my_segments = 0;
    Known own;                                               // the thread's last request: its only one below 257 requests
    for (int r = tid * seg; r < (tid + 1) * seg && r < R; ++r) {
        own = look_up<NR, TILE>(a, r, clipped);
        mine += (int64_t)own.tiles * own.row_tiles;
        my_segments += own.tiles > 0 ? own.row_tiles : 0;
    }
    if (clipped && blockIdx.x == 0) atomicOr(a.flags, (uint32_t)VTOKEN_FLAG_CAPACITY);
    const int64_t incl = vtk_warp_incl_scan(mine);
    my_segments = __reduce_add_sync(0xffffffffu, my_segments);
    if (lane == 31) {
        sh.plan.warp_sum[warp] = incl;
        sh.plan.warp_segments[warp] = my_segments;
    }
    __syncthreads();
    int64_t before = 0, all_tiles = 0;
    int all_segments = 0;
    for (int w = 0; w < NW; ++w) {
        before += w < warp ? sh.plan.warp_sum[w] : 0;
        all_tiles += sh.plan.warp_sum[w];
        all_segments += sh.plan.warp_segments[w];
    }
    before += incl - mine;                                   // tiles of the requests in front of the thread's

    // ---- teams: the fewer segments there are, the more warps share one ----
    int group = Rows::GROUP, lanes = 1, groups;
    while (group > 1 && group / 2 >= a.hkv) group >>= 1;
    for (;;) {
        groups = (a.hkv + group - 1) / group;
        if ((int64_t)all_segments * groups * AT_PARTS >= (int64_t)gridDim.x * (NW / (group * lanes))) break;
        if (group * lanes < NW) lanes <<= 1;
        else if (group > 1) { group >>= 1; lanes <<= 1; }
        else break;
    }
    const int per_team = group * lanes, teams = NW / per_team, my_team = warp / per_team;
    const int hl = warp / lanes % group, tw = warp % lanes;  // head of the group, lane of tokens
    const int64_t W = all_tiles * groups;
    // at least AT_MIN_SHARE tiles a lane: a segment that is cut finer costs more to join than it gains
    const int64_t most = divide(W + AT_MIN_SHARE * lanes - 1, AT_MIN_SHARE * lanes), G = most < (int64_t)gridDim.x * teams ? most : (int64_t)gridDim.x * teams;
    const bool packed = G == (int64_t)gridDim.x * teams;     // a CTA's shares side by side; few shares: on different SMs
    auto share_at = [&](int team) { return packed ? blockIdx.x * teams + team : team * gridDim.x + blockIdx.x; };
    const int share = share_at(my_team);
    // the first `longer` shares have one tile more than the others
    const int64_t size = G > 0 ? divide(W, G) : 0, longer = W - size * G;
    auto start_of = [&](int64_t i) { return i * size + (i < longer ? i : longer); };
    auto share_of = [&](int64_t f) { return (int)(f < longer * (size + 1) ? divide(f, size + 1) : longer + divide(f - longer * (size + 1), size)); };
    for (int team = 0; team < teams; ++team) {               // the thread whose requests hold a share's first tile
        if (share_at(team) >= G) break;
        const int64_t f = start_of(share_at(team));
        if (f >= before * groups && f < (before + mine) * groups) {
            sh.plan.start[team] = tid;
            sh.plan.before[team] = before;
        }
    }
    __syncthreads();
    Walk<NR, TILE> use;
    use.f = share < G ? start_of(share) : 0;
    use.f1 = share < G ? start_of(share + 1) : 0;
    use.k = &s_use[warp];
    int64_t left = 0;
    if (share < G) {
        left = use.f - sh.plan.before[my_team] * groups;
        use.r = sh.plan.start[my_team] * seg;
    }
    const int known0 = G > share_at(0) ? sh.plan.start[0] : 0;
    if (seg == 1 && tid >= known0 && tid < known0 + AT_KNOWN && tid < R) s_known[tid - known0] = own;
    const int r_known = seg == 1 ? known0 : INT32_MAX;
    __syncthreads();                                         // the plan's arrays become the join buffers
    if (share >= G) return;
    for (;; ++use.r) {
        bool c = false;
        const Known k = use.in_window(use.r, r_known) ? s_known[use.r - r_known] : look_up<NR, TILE>(a, use.r, c);
        const int64_t all = (int64_t)k.tiles * k.row_tiles * groups;
        if (left < all) {
            if (lane == 0) s_use[warp] = s_get[warp] = k;
            __syncwarp();
            break;
        }
        left -= all;
    }
    use.rt = (int)divide(left, (int64_t)use.k->tiles * groups);
    left -= (int64_t)use.rt * use.k->tiles * groups;
    use.hg = (int)divide(left, use.k->tiles);
    use.t0 = (int)(left - (int64_t)use.hg * use.k->tiles);
    use.clip();
    auto team_sync = [&]() {
        if (lanes == 1) __syncwarp();
        else asm volatile("barrier.cta.sync %0, %1;" ::"r"(1 + warp / lanes), "r"(lanes * 32) : "memory");
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
            get.next(a, groups, s_known, r_known);
            more = !get.done();
            tile = get.t0 + tw;
        }
        Next n;
        n.slot = -1;
        n.id = INT32_MAX;
        n.pmax = n.floor = -1;
        n.kv = get.hg * group + hl;
        n.there = more;
        const int v = tile * TILE + lane;
        if (more && lane < TILE && v < get.k->s.n && n.kv < a.hkv) {
            n.slot = a.cache_slots[get.k->s.entry(v)];
            n.id = a.cache_ids.null() ? get.k->s.index(v) : a.cache_ids[get.k->s.entry(v)];
            n.pmax = get.k->s.pmax;
            n.floor = get.k->s.floor;
        }
        tile += lanes;
        return n;
    };
    auto issue = [&](Next n) {
        if (n.there) {
            const bool seen = vtk_sees(n.id, n.pmax, n.floor, a.sinks);           // (the span's ends are counted, not looked up)
            if (n.slot >= 0 && (int64_t)n.slot >= a.slots_per_layer) {
                if (seen) atomicOr(a.flags, (uint32_t)VTOKEN_FLAG_BAD_SLOT);
                n.slot = -1;
            }
            if (!seen) n.slot = -1;
            const int stage = issued % ST;
            if (lane < TILE) sh.ids[warp][stage][lane] = n.slot < 0 ? INT32_MAX : n.id;
            Rows::issue(vtk_smem_u32(sh.ring[warp][stage]), a.k_rows, a.v_rows, a.row_bytes, a.hkv, n.kv, n.slot);
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
    for (; !use.done(); use.next(a, groups, s_known, r_known)) {
        const int kv = use.hg * group + hl, rt = use.rt;
        const int rows = kv >= a.hkv ? 0 :              // (the last group may lack heads)
             use.k->qn * a.group - rt * NR < NR ? use.k->qn * a.group - rt * NR : NR;
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
                int64_t tok;
                int head;
                split_row(a, at, tok, head);
                tok += use.k->q0;
                pos[h] = min(a.positions[tok], INT32_MAX - 1);     // (INT32_MAX is the id of what is not there)
                floor[h] = vtk_floor(pos[h], a.window);
                p = a.q + tok * a.q_stride + (int64_t)(kv * a.group + head) * D;
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

        for (int tl = use.t0 + tw; tl < use.t1; tl += lanes, ++used) {
            cp_wait<ST - 2>();
            __syncwarp();
            issue(next);
            next = meta();
            const int stage = used % ST;
            Rows rows_now;
            rows_now.set(sh.ring[warp][stage], kv);
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
                    const float base = (m[h] == -INFINITY ? 0.f : m[h]) - vtk_lift<Mma>();
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

        // ---- join the team's warps, pair by pair: fragments as they are, 16 bytes a thread ----
#pragma unroll
        for (int h = 0; h < RH; ++h) {
            l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
            l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
        }
        for (int half = lanes / 2; half > 0; half >>= 1) {
            if (tw >= half && tw < 2 * half) {
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int h = 0; h < RH; ++h)
                        *reinterpret_cast<float4 *>(&sh.o[warp][((i * RH + h) * 32 + lane) * 4]) = make_float4(o[i][h][0], o[i][h][1], o[i][h][2], o[i][h][3]);
#pragma unroll
                for (int h = 0; h < RH; ++h)
                    if (t == 0) sh.ml[warp][g + 8 * h] = make_float2(m[h], l[h]);
            }
            team_sync();
            if (tw < half) {
                const int w = warp + half;
#pragma unroll
                for (int h = 0; h < RH; ++h) {
                    const float2 ml = sh.ml[w][g + 8 * h];
                    const float top = fmaxf(m[h], ml.x), f = weight(m[h], top), f2 = weight(ml.x, top);
                    l[h] = l[h] * f + ml.y * f2;
                    m[h] = top;
                    const float a0 = __shfl_sync(0xffffffffu, f, 8 * t), a1 = __shfl_sync(0xffffffffu, f, 8 * t + 4);
                    const float b0 = __shfl_sync(0xffffffffu, f2, 8 * t), b1 = __shfl_sync(0xffffffffu, f2, 8 * t + 4);
#pragma unroll
                    for (int i = 0; i < MT; ++i) {
                        const float4 x = *reinterpret_cast<const float4 *>(&sh.o[w][((i * RH + h) * 32 + lane) * 4]);
                        o[i][h][0] = o[i][h][0] * a0 + x.x * b0;
                        o[i][h][1] = o[i][h][1] * a1 + x.y * b1;
                        o[i][h][2] = o[i][h][2] * a0 + x.z * b0;
                        o[i][h][3] = o[i][h][3] * a1 + x.w * b1;
                    }
                }
            }
        }

        // ---- the rows: finished, or a part of a longer segment ----
        const int64_t seg_lo = use.f - use.t0, seg_hi = seg_lo + use.k->tiles;
        const bool whole = use.t0 == 0 && use.t1 == use.k->tiles;
        // shares that hold parts of this segment, and where a share leaves its part
        const int first = share_of(seg_lo), parts = share_of(seg_hi - 1) - first + 1;
        auto part_at = [&](int i) { return a.part + ((int64_t)(2 * i + (i == first)) * group + hl) * (NR * (D + 2)); };
        auto query = [&](int row, int64_t &tok, int &head) { split_row(a, rt * NR + row, tok, head); tok += use.k->q0; head += kv * a.group; };
        uint16_t *to[RH][2];                                 // rows 2t and 2t + 1 (+ 8) of the output, null: there is none
#pragma unroll
        for (int h = 0; h < RH; ++h)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                int64_t tok;
                int head;
                query(8 * h + 2 * t + e, tok, head);
                to[h][e] = 8 * h + 2 * t + e < rows ? a.out + tok * a.out_stride + (int64_t)head * D + Rows::vdim(g, 0) : nullptr;
            }
        // m-tile i of the rows 2t and 2t + 1 (+ 8): two dimensions each
        auto store = [&](int i, const float (&x)[RH][4], const float (&r)[RH][2]) {
#pragma unroll
            for (int h = 0; h < RH; ++h)
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    if (to[h][e] != nullptr)
                        *reinterpret_cast<uint32_t *>(to[h][e] + (Rows::vdim(0, i / 4) + 2 * (i % 4))) = Act::pack(x[h][e] * r[h][e], x[h][2 + e] * r[h][e]);
        };
        auto finite = [](const float (&x)[RH][4]) {
            bool ok = true;
#pragma unroll
            for (int h = 0; h < RH; ++h)
#pragma unroll
                for (int e = 0; e < 4; ++e) ok &= fabsf(x[h][e]) < INFINITY;
            return ok;
        };
        auto totals = [&](const float (&mm)[RH], const float (&ll)[RH], bool write, float (&r)[RH][2], bool &ok) {
#pragma unroll
            for (int h = 0; h < RH; ++h) {
                const float f = ll[h] == 0.f ? 0.f : a.v_mul / ll[h];
                ok &= fabsf(ll[h]) < INFINITY;
                r[h][0] = __shfl_sync(0xffffffffu, f, 8 * t);
                r[h][1] = __shfl_sync(0xffffffffu, f, 8 * t + 4);
                if (write && a.lse != nullptr && t == 0 && g + 8 * h < rows) {
                    int64_t tok;
                    int head;
                    query(g + 8 * h, tok, head);
                    a.lse[tok * a.hq + head] = ll[h] == 0.f ? -INFINITY : (mm[h] + log2f(ll[h]) - vtk_lift<Mma>()) * 0.69314718055994531f;
                }
            }
        };
        // rows that a masked NaN may have reached (with one query token what it does not see was not read)
        auto again = [&]() {
            for (int row = tw; row < rows; row += lanes) {
                int64_t tok;
                int head;
                query(row, tok, head);
                float acc[N], mm, ll;
                if (vtk_row_again<D, Rows::FP4, Act>(a, tok, head, a.positions[tok], use.k->s, use.k->len, acc, mm, ll))
                    vtk_store_row<D, Act>(a, tok, head, acc, mm, ll);
            }
        };
        bool bad = false;
        if (rows <= 0) {                                     // a head that is not there: its warps only keep step
            if (!whole) team_sync();
        } else if (whole) {
            if (tw == 0) {
                bool ok = true;
                float r[RH][2];
                totals(m, l, true, r, ok);
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    ok &= finite(o[i]);
                    store(i, o[i], r);
                }
                bad = !__all_sync(0xffffffffu, ok);
            }
        } else {
            if (tw == 0) {
                float *dst = part_at(share);
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int h = 0; h < RH; ++h)
                        __stcg(reinterpret_cast<float4 *>(dst + ((i * RH + h) * 32 + lane) * 4), make_float4(o[i][h][0], o[i][h][1], o[i][h][2], o[i][h][3]));
#pragma unroll
                for (int h = 0; h < RH; ++h)
                    if (t == 0) __stcg(reinterpret_cast<float2 *>(dst + NR * D + 2 * (g + 8 * h)), make_float2(m[h], l[h]));
                __syncwarp();
                if (lane == 0) {                             // (the warp's writes are released with the arrival, the others' acquired)
                    uint32_t *counter = a.counters + first * group + hl, seen;
                    asm volatile("atom.add.acq_rel.gpu.global.u32 %0, [%1], 1;" : "=r"(seen) : "l"(counter) : "memory");
                    const bool last = seen == (unsigned)(parts - 1);
                    if (last) *counter = 0;                  // ready for the next call
                    sh.last[warp] = last;
                }
            }
            team_sync();
            if (*(volatile int *)&sh.last[warp - tw]) {
                float mm[RH], ll[RH];
                float2 ml0[4][RH];                           // (nearly always all there are)
#pragma unroll
                for (int k = 0; k < 4; ++k)
#pragma unroll
                    for (int h = 0; h < RH; ++h)
                        ml0[k][h] = __ldcg(reinterpret_cast<const float2 *>(part_at(first + (k < parts ? k : 0)) + NR * D + 2 * (g + 8 * h)));
#pragma unroll
                for (int h = 0; h < RH; ++h) {
                    mm[h] = fmaxf(fmaxf(ml0[0][h].x, ml0[1][h].x), fmaxf(ml0[2][h].x, ml0[3][h].x));
                    ll[h] = 0.f;
                }
                for (int i = 4; i < parts; ++i)
#pragma unroll
                    for (int h = 0; h < RH; ++h) mm[h] = fmaxf(mm[h], __ldcg(part_at(first + i) + NR * D + 2 * (g + 8 * h)));
                // lane w of the head: the m-tiles w, w + lanes, ..., as many at a time as the registers hold
                bool ok = true, counted = false;
                float r[RH][2];
                constexpr int AT_ONCE = NR == 8 && NW == 8 ? 8 : 4;
                for (int i0 = tw; i0 < MT; i0 += AT_ONCE * lanes) {
                    float acc[AT_ONCE][RH][4];
#pragma unroll
                    for (int i = 0; i < AT_ONCE; ++i)
#pragma unroll
                        for (int h = 0; h < RH; ++h)
#pragma unroll
                            for (int e = 0; e < 4; ++e) acc[i][h][e] = 0.f;
#pragma unroll 3
                    for (int k = 0; k < parts; ++k) {
                        const float *src = part_at(first + k);
#pragma unroll
                        for (int h = 0; h < RH; ++h) {
                            const float2 ml = __ldcg(reinterpret_cast<const float2 *>(src + NR * D + 2 * (g + 8 * h)));
                            const float f = weight(ml.x, mm[h]);
                            if (!counted) ll[h] += f * ml.y;
                            const float f0 = __shfl_sync(0xffffffffu, f, 8 * t), f1 = __shfl_sync(0xffffffffu, f, 8 * t + 4);
#pragma unroll
                            for (int i = 0; i < AT_ONCE; ++i)
                                if (i0 + i * lanes < MT) {
                                    const float4 x = __ldcg(reinterpret_cast<const float4 *>(src + (((i0 + i * lanes) * RH + h) * 32 + lane) * 4));
                                    acc[i][h][0] += f0 * x.x;
                                    acc[i][h][1] += f1 * x.y;
                                    acc[i][h][2] += f0 * x.z;
                                    acc[i][h][3] += f1 * x.w;
                                }
                        }
                    }
                    if (!counted) totals(mm, ll, tw == 0, r, ok);
                    counted = true;
#pragma unroll
                    for (int i = 0; i < AT_ONCE; ++i)
                        if (i0 + i * lanes < MT) {
                            ok &= finite(acc[i]);
                            store(i0 + i * lanes, acc[i], r);
                        }
                }
                bad = !__all_sync(0xffffffffu, ok);
            }
        }
        if (use.k->qn > 1 && rows > 0) {
            if (lanes > 1) {                                 // one lane's finding is the head's
                if (lane == 0) sh.bad[warp] = bad;
                team_sync();
                bad = false;
                for (int w = warp - tw; w < warp - tw + lanes; ++w) bad |= *(volatile int *)&sh.bad[w] != 0;
            }
            if (bad) {
                __syncwarp();                                // (other lanes write over what this one has just stored)
                again();
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
    static std::atomic<int> allowed{-1};                     // the device that knows of this kernel's shared memory
    VTK_CUDA(ctx, vtk_allow_smem(ctx, allowed, (const void *)kernel, smem));
    VTK_CUDA(ctx, vtk_launch_dependent(ctx, kernel, dim3(ctx->num_sms), dim3(Rows::WARPS * 32), smem, st, a));
    VTK_CUDA(ctx, cudaGetLastError());
    return VTOKEN_OK;
}

template <int D, typename Act>
int launch_by_type(vtoken_ctx *ctx, bool fp4, bool wide, const VtkAttnArgs &a, cudaStream_t st)
{
    constexpr bool bf = Act::kind == VTOKEN_KV_BF16;
    if (fp4) return wide ? launch<D, 16, Rows4<D, 8>, Act, !bf>(ctx, a, st) : launch<D, 8, Rows4<D, 16>, Act, !bf>(ctx, a, st);
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

// A share leaves parts of at most two segments for each of its heads; shares times heads are at most 16 a CTA with 8
// rows, 8 with 16.
int64_t vtk_attention_rows_workspace(const vtoken_ctx *ctx, const vtoken_heads *heads, VtkAttnArgs *a)
{
    const int64_t shares = (int64_t)ctx->num_sms * 16, counters = shares * 4 + 16;       // (the prompt kernel's two tickets in front)
    if (a) a->part = (float *)((uint8_t *)(a->counters - 4) + counters);
    return counters + shares * 2 * 8 * (heads->head_dim + 2) * 4;
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
    if (!in->num_requests || !in->q_offsets || !in->tt_offsets || !in->cache_slots || !in->cache_len || !in->workspace) return VTOKEN_EINVAL;
    if (in->max_query_tokens != 0 && (!in->positions || !in->q || !in->out)) return VTOKEN_EINVAL;     // (without elements: no address)
    if (in->max_query_tokens < 0 || in->max_query_len < 1 || in->window < 0 || in->sinks < 0) return VTOKEN_EINVAL;
    const float scale = in->sm_scale * 1.4426950408889634f * two_to(heads->k_exponent);
    if (!(in->sm_scale > -1e30f && in->sm_scale < 1e30f) || !(scale > -INFINITY && scale < INFINITY)) return VTOKEN_EINVAL;
    if ((((uintptr_t)in->q | (uintptr_t)in->out | (uintptr_t)in->workspace) & 15) || ((uintptr_t)in->lse & 3)) return VTOKEN_EINVAL;
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
    a.inv_group = 1.f / (float)a.group;
    a.window = in->window;
    a.sinks = in->window > 0 ? in->sinks : 0;
    a.scale_log2 = scale;
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
