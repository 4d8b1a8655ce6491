// Attention of few query rows per request (a decode step) over the slot cache.
//
// Bound by HBM: every visible K and V row is read once, 4 * D flops per row, head and query.  The work is cut
// along the cache: an item is (request, tile of query rows, key head, chunk of the cache); one CTA takes an item,
// its warps the chunk's 16-token tiles in turn, with a running maximum and sum per query row and the output
// accumulators in registers.  A request of one chunk is finished by its CTA; of a longer one every CTA leaves a
// partial row and the last to arrive joins them in chunk order, so the order of the sums is that of the tables.
//
// The heads of a group (and the query tokens of a request) are the rows of one matrix product, so a K or V row is
// read once for all of them.  Both products take their operand from the cache straight from global memory into the
// registers where mma.m16n8k16 wants it, without a pass through shared memory: the order of the contracted
// dimension is free as long as both operands agree, so
//   S = Q K^T : a lane's 16-byte load of K (8 dimensions of one token) is the B fragment of two instructions;
//   O^T = V^T P^T : a lane loads 16 bytes (8 dimensions) of four tokens, byte permutes pair the tokens up to the
//   A fragment, and the accumulator layout of S (rows = queries, columns = tokens) is the B fragment of P^T as it is.
// P is handed to the second product as the sum of two 16-bit values, so that its rounding does not add to that of
// the 16-bit output; over the 4-bit cache the products run in half precision, whose 11 bits are enough next to a
// bf16 output.  These legacy matrix instructions are enough here: 8 or 16 rows leave a 128-row tcgen05 tile mostly
// empty, and at full HBM rate the products need well under a tenth of the tensor rate.
#include "attention.cuh"

namespace {

constexpr int AT_WARPS = 4, AT_NT = AT_WARPS * 32;
// CTAs per SM: what 168 (8 query rows) and 255 registers a thread leave room for
template <int NR> constexpr int AT_CTAS = NR == 8 ? 3 : 2;
// requests whose spans a CTA keeps in shared memory (below the 48 KB of static arrays)
constexpr int AT_ROW_LIMIT = 32;          // query rows (tokens times group) of a request up to which it is worked on here
template <int NR> constexpr int AT_KNOWN = NR == 8 ? 512 : 256;

// ---- 16 tokens of one head in registers --------------------------------------------------------
// K: lane (g, t) holds of tokens g and 8 + g the dimensions `kdim(j) .. + 7`, j < D / 32.
// V: lane (g, t) holds of tokens 2t, 2t + 1, 2t + 8, 2t + 9 the dimensions `vdim(x) .. + 7`, x < D / 64.
template <int D, typename Act>
struct Rows16 {
    static constexpr bool FP4 = false;
    using Mma = Act;
    uint4 k[2][D / 32], v[4][D / 64];
    static __device__ __forceinline__ int kdim(int t, int j) { return 32 * j + 8 * t; }
    static __device__ __forceinline__ int vdim(int g, int x) { return 64 * x + 8 * g; }
    __device__ __forceinline__ void load_k(int u, bool there, const uint8_t *row, int, int head, int t)
    {
#pragma unroll
        for (int j = 0; j < D / 32; ++j)
            k[u][j] = there ? vtk_ldg16(row + ((int64_t)head * D + kdim(t, j)) * 2) : make_uint4(0, 0, 0, 0);
    }
    __device__ __forceinline__ void load_v(int i, bool there, const uint8_t *row, int, int head, int g)
    {
#pragma unroll
        for (int x = 0; x < D / 64; ++x)
            v[i][x] = there ? vtk_ldg16(row + ((int64_t)head * D + vdim(g, x)) * 2) : make_uint4(0, 0, 0, 0);
    }
    __device__ __forceinline__ uint4 get_k(int u, int j) const { return k[u][j]; }
    __device__ __forceinline__ uint4 get_v(int i, int x) const { return v[i][x]; }
};

template <int D>
struct Rows4 {
    static constexpr bool FP4 = true;
    using Mma = VtkFp16;
    uint32_t k[2][D / 32], v[4][D / 64], ks[2], vs[4];
    static __device__ __forceinline__ int kdim(int t, int j) { return (D / 4) * t + 8 * j; }
    static __device__ __forceinline__ int vdim(int g, int x) { return (D / 8) * g + 8 * x; }
    __device__ __forceinline__ void load_k(int u, bool there, const uint8_t *row, int hkv, int head, int t)
    {
        const uint8_t *codes = row + head * (D / 2) + (D / 8) * t;
        const uint8_t *scales = row + hkv * (D / 2) + head * (D / 16) + (D / 64) * t;
        if (D == 128) {
            const uint4 w = there ? vtk_ldg16(codes) : make_uint4(0, 0, 0, 0);
            k[u][0] = w.x; k[u][1] = w.y; k[u][D / 32 - 2] = w.z; k[u][D / 32 - 1] = w.w;
            ks[u] = there ? __ldg(reinterpret_cast<const uint16_t *>(scales)) : 0;
        } else {
            const uint2 w = there ? __ldg(reinterpret_cast<const uint2 *>(codes)) : make_uint2(0, 0);
            k[u][0] = w.x; k[u][1] = w.y;
            ks[u] = there ? __ldg(scales) : 0;
        }
    }
    __device__ __forceinline__ void load_v(int i, bool there, const uint8_t *row, int hkv, int head, int g)
    {
        const uint8_t *codes = row + head * (D / 2) + (D / 16) * g;
        const uint8_t *scales = row + hkv * (D / 2) + head * (D / 16);
        if (D == 128) {
            const uint2 w = there ? __ldg(reinterpret_cast<const uint2 *>(codes)) : make_uint2(0, 0);
            v[i][0] = w.x; v[i][D / 64 - 1] = w.y;
            vs[i] = there ? __ldg(scales + g) : 0;
        } else {
            v[i][0] = there ? __ldg(reinterpret_cast<const uint32_t *>(codes)) : 0;
            vs[i] = there ? __ldg(scales + g / 2) : 0;
        }
    }
    static __device__ __forceinline__ uint4 expand(uint32_t w, uint32_t s)
    {
        return make_uint4(vtk_hmul2(vtk_codes_to_half2(w), s), vtk_hmul2(vtk_codes_to_half2(w >> 8), s),
                          vtk_hmul2(vtk_codes_to_half2(w >> 16), s), vtk_hmul2(vtk_codes_to_half2(w >> 24), s));
    }
    __device__ __forceinline__ uint4 get_k(int u, int j) const
    {
        // D 128: words 0, 1 belong to the first of the lane's two groups, 2, 3 to the second
        const uint32_t two = vtk_scales_to_half2(D == 128 ? (j < 2 ? (ks[u] & 0xffu) : (ks[u] >> 8)) : ks[u]);
        return expand(k[u][j], __byte_perm(two, 0, 0x1010));
    }
    __device__ __forceinline__ uint4 get_v(int i, int x) const
    {
        return expand(v[i][x], __byte_perm(vtk_scales_to_half2(vs[i]), 0, 0x1010));
    }
};

// a request as a CTA's shared memory keeps it
struct Known {
    int q0, qn, lo, n_sink, n, len;
    int64_t base;
};

__device__ inline Known look_up(const VtkAttnArgs &a, int r, bool &clipped)
{
    Known k;
    bool c;
    vtk_request_rows(a, r, k.q0, k.qn, k.base, k.len, c);
    clipped |= c;
    if (k.qn * (int64_t)a.group > a.row_limit) k.qn = 0;
    k.lo = k.n_sink = 0;
    k.n = k.len;
    if (k.qn > 0 && k.qn <= 8) {         // few queries: only what one of them can see
        int pmin = a.positions[k.q0], pmax = pmin;
        for (int i = 1; i < k.qn; ++i) {
            const int p = a.positions[k.q0 + i];
            pmin = p < pmin ? p : pmin;
            pmax = p > pmax ? p : pmax;
        }
        const VtkRequest s = vtk_request_span(a, k.base, k.len, pmin, pmax);
        k.lo = s.lo;
        k.n_sink = s.n_sink;
        k.n = s.n;
    }
    return k;
}

// NR: query rows of an item (8 or 16); SPLIT_P: P as a sum of two 16-bit values
template <int D, int NR, typename Rows, typename Act, bool SPLIT_P>
__global__ void __launch_bounds__(AT_NT, AT_CTAS<NR>) attention_rows_kernel(const __grid_constant__ VtkAttnArgs a)
{
    using Mma = typename Rows::Mma;
    constexpr int RH = NR / 8, MT = D / 16, N = D / 32;
    __shared__ __align__(16) float s_o[AT_WARPS][NR][D + 4];
    __shared__ float2 s_ml[AT_WARPS][NR];
    __shared__ Known s_known[AT_KNOWN<NR>];
    __shared__ int s_items[AT_NT + 1], s_splits[AT_NT + 1];
    __shared__ unsigned long long s_sum[AT_WARPS];
    __shared__ int s_last;
    vtk_release_successor();
    vtk_wait_for_predecessor();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;

    // ---- the cut: every CTA works it out for itself (one or two loads per request and two scans) ----
    int R = *a.num_requests;
    bool clipped = R < 0 || R > a.max_requests;
    R = R < 0 ? 0 : (R > a.max_requests ? a.max_requests : R);
    const int seg = (R + AT_NT - 1) / AT_NT, r_lo = tid * seg, r_hi = r_lo + seg < R ? r_lo + seg : R;
    unsigned long long total = 0;
    for (int r = r_lo; r < r_hi; ++r) {
        const Known k = look_up(a, r, clipped);
        if (r < AT_KNOWN<NR>) s_known[r] = k;
        total += (unsigned long long)k.n * ((k.qn * a.group + NR - 1) / NR);
    }
    if (clipped && blockIdx.x == 0) atomicOr(a.flags, (uint32_t)VTOKEN_FLAG_CAPACITY);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) total += __shfl_xor_sync(0xffffffffu, total, d);
    if (lane == 0) s_sum[warp] = total;
    __syncthreads();
    total = 0;
#pragma unroll
    for (int w = 0; w < AT_WARPS; ++w) total += s_sum[w];
    int64_t want = (int64_t)((total + a.target - 1) / a.target);
    want = want < a.min_chunk ? a.min_chunk : want;
    const int chunk = (int)((want + AT_WARPS * 16 - 1) / (AT_WARPS * 16)) * (AT_WARPS * 16);
    int items = 0, splits = 0;
    for (int r = r_lo; r < r_hi; ++r) {
        const Known k = r < AT_KNOWN<NR> ? s_known[r] : look_up(a, r, clipped);
        const int rt = (k.qn * a.group + NR - 1) / NR, nc = k.n > chunk ? (k.n + chunk - 1) / chunk : 1;
        items += rt * nc;
        if (nc > 1) splits += rt * nc;
    }
    {
        const int i_items = vtk_warp_incl_scan(items), i_splits = vtk_warp_incl_scan(splits);
        __shared__ int w_items[AT_WARPS], w_splits[AT_WARPS];
        if (lane == 31) { w_items[warp] = i_items; w_splits[warp] = i_splits; }
        __syncthreads();
        int b_items = 0, b_splits = 0;
        for (int w = 0; w < warp; ++w) { b_items += w_items[w]; b_splits += w_splits[w]; }
        s_items[tid + 1] = b_items + i_items;
        s_splits[tid + 1] = b_splits + i_splits;
        if (tid == 0) s_items[0] = s_splits[0] = 0;
        __syncthreads();
    }
    const int64_t all = (int64_t)s_items[AT_NT] * a.hkv;

    for (int64_t item = blockIdx.x; item < all; item += gridDim.x) {
        // ---- which: the heads of a chunk follow one another, so neighbouring CTAs read neighbouring bytes ----
        const int kv = (int)(item % a.hkv), idx = (int)(item / a.hkv);
        int lo = 0, hi = AT_NT;                              // s_items[lo] <= idx < s_items[hi]
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (s_items[mid] <= idx) lo = mid; else hi = mid;
        }
        int left = idx - s_items[lo], split0 = s_splits[lo], r = lo * seg, nc = 1;
        Known rq;
        for (;; ++r) {
            rq = r < AT_KNOWN<NR> ? s_known[r] : look_up(a, r, clipped);
            nc = rq.n > chunk ? (rq.n + chunk - 1) / chunk : 1;
            const int its = nc * ((rq.qn * a.group + NR - 1) / NR);
            if (left < its) break;
            left -= its;
            if (nc > 1) split0 += its;
        }
        const int rt = left / nc, c = left % nc;
        split0 += rt * nc;                                   // first partial of this row tile
        const int rows = rq.qn * a.group - rt * NR < NR ? rq.qn * a.group - rt * NR : NR;

        // ---- queries: lane (g, t) holds of rows g and 8 + g the dimensions its K fragments hold ----
        uint4 q[RH][D / 32];
        int pos[RH];
        float scale[RH];
#pragma unroll
        for (int h = 0; h < RH; ++h) {
            const int row = g + 8 * h, at = rt * NR + row;
            pos[h] = -1;
            scale[h] = a.scale_log2;
            const uint16_t *p = nullptr;
            if (row < rows) {
                const int64_t tok = rq.q0 + at / a.group;
                pos[h] = a.positions[tok];
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

        float o[MT][RH][4], m[RH], l[RH];
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int h = 0; h < RH; ++h)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[i][h][e] = 0.f;
#pragma unroll
        for (int h = 0; h < RH; ++h) { m[h] = -INFINITY; l[h] = 0.f; }

        // ---- the chunk: warp w takes tiles w, w + AT_WARPS, ... of 16 tokens ----
        const int v_end = c * chunk + chunk < rq.n ? c * chunk + chunk : rq.n;
        const int span = rq.n_sink;
        auto meta = [&](int v, int &slot, int &id) {         // lanes 0 .. 15: entry v + lane
            slot = -1;
            id = INT32_MAX;
            if (lane < 16 && v + lane < v_end) {
                const int i = v + lane < span ? v + lane : rq.lo + (v + lane - span);
                slot = a.cache_slots[rq.base + i];
                id = a.cache_ids.null() ? i : a.cache_ids[rq.base + i];
            }
        };
        int v = c * chunk + warp * 16, slot = -1, id = INT32_MAX, slot2, id2;
        unsigned some = 0, full = 0;
        Rows rows_now;
        auto judge = [&]() {
            if (slot >= 0 && (int64_t)slot >= a.slots_per_layer) {
                atomicOr(a.flags, (uint32_t)VTOKEN_FLAG_BAD_SLOT);
                slot = -1;
            }
            const bool any = slot >= 0 && id <= pmax && (a.window == 0 || id > (int64_t)pmin - a.window || id < a.sinks);
            const bool every = any && id <= pmin && (a.window == 0 || id > (int64_t)pmax - a.window || id < a.sinks);
            some = __ballot_sync(0xffffffffu, any);
            full = __ballot_sync(0xffffffffu, every);
        };
        auto load_k = [&]() {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int64_t s = __shfl_sync(0xffffffffu, slot, 8 * u + g);
                rows_now.load_k(u, (some >> (8 * u + g)) & 1u, a.k_rows + s * a.row_bytes, a.hkv, kv, t);
            }
        };
        auto load_v = [&]() {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int tok = 2 * t + (i & 1) + 8 * (i >> 1);
                const int64_t s = __shfl_sync(0xffffffffu, slot, tok);
                rows_now.load_v(i, (some >> tok) & 1u, a.v_rows + s * a.row_bytes, a.hkv, kv, g);
            }
        };
        auto advance = [&]() {                               // to the warp's next tile that some row sees
            while (v < v_end) {
                slot = slot2;
                id = id2;
                meta(v + AT_WARPS * 16, slot2, id2);
                judge();
                if (some) return;
                v += AT_WARPS * 16;
            }
            some = 0;
        };
        meta(v, slot2, id2);
        advance();
        if (some) { load_k(); load_v(); }
        while (some) {
            float s[2][4];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                s[u][0] = s[u][1] = s[u][2] = s[u][3] = 0.f;
#pragma unroll
                for (int j = 0; j < D / 32; ++j) {
                    const uint4 k = rows_now.get_k(u, j);
                    vtk_mma<Mma>(s[u], q[0][j].x, RH == 2 ? q[RH - 1][j].x : 0u, q[0][j].y, RH == 2 ? q[RH - 1][j].y : 0u, k.x, k.y);
                    vtk_mma<Mma>(s[u], q[0][j].z, RH == 2 ? q[RH - 1][j].z : 0u, q[0][j].w, RH == 2 ? q[RH - 1][j].w : 0u, k.z, k.w);
                }
            }
            // the tile's masks; then the next tile's K rows are on their way while this one is worked on
            const unsigned some_now = some, full_now = full;
            int ids[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) ids[i] = __shfl_sync(0xffffffffu, id, 2 * t + (i & 1) + 8 * (i >> 1));
            v += AT_WARPS * 16;
            advance();
            if (some) load_k();
            float p[2][4], tile_max[RH];
#pragma unroll
            for (int h = 0; h < RH; ++h) tile_max[h] = -INFINITY;
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int e = 0; e < 2 * RH; ++e) {
                    const int h = e >> 1, tok = 2 * t + (e & 1) + 8 * u;
                    float x = s[u][e] * scale[h];
                    if (full_now != 0xffffu) {
                        const bool see = ((full_now >> tok) & 1u) ||
                                         (((some_now >> tok) & 1u) && vtk_sees(ids[(e & 1) + 2 * u], pos[h], a.window, a.sinks));
                        x = see ? x : -INFINITY;
                    }
                    p[u][e] = x;
                    tile_max[h] = fmaxf(tile_max[h], x);
                }
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
            uint32_t b[RH][2], b_lo[RH][2];
#pragma unroll
            for (int h = 0; h < RH; ++h) {
                const float base = m[h] == -INFINITY ? 0.f : m[h];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const float p0 = vtk_exp2(p[u][2 * h] - base), p1 = vtk_exp2(p[u][2 * h + 1] - base);
                    l[h] += p0 + p1;
                    b[h][u] = Mma::pack(p0, p1);
                    if (SPLIT_P) {
                        const float2 r = Mma::unpack(b[h][u]);
                        b_lo[h][u] = Mma::pack(p0 - r.x, p1 - r.y);
                    }
                }
            }
#pragma unroll
            for (int x = 0; x < D / 64; ++x) {
                const uint4 v0 = rows_now.get_v(0, x), v1 = rows_now.get_v(1, x), v2 = rows_now.get_v(2, x), v3 = rows_now.get_v(3, x);
                const uint32_t w0[4] = {v0.x, v0.y, v0.z, v0.w}, w1[4] = {v1.x, v1.y, v1.z, v1.w};
                const uint32_t w2[4] = {v2.x, v2.y, v2.z, v2.w}, w3[4] = {v3.x, v3.y, v3.z, v3.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t a0 = __byte_perm(w0[i], w1[i], 0x5410), a1 = __byte_perm(w0[i], w1[i], 0x7632);
                    const uint32_t a2 = __byte_perm(w2[i], w3[i], 0x5410), a3 = __byte_perm(w2[i], w3[i], 0x7632);
#pragma unroll
                    for (int h = 0; h < RH; ++h) {
                        vtk_mma<Mma>(o[4 * x + i][h], a0, a1, a2, a3, b[h][0], b[h][1]);
                        if (SPLIT_P) vtk_mma<Mma>(o[4 * x + i][h], a0, a1, a2, a3, b_lo[h][0], b_lo[h][1]);
                    }
                }
            }
            if (some) load_v();
        }

        // ---- join the warps ----
#pragma unroll
        for (int h = 0; h < RH; ++h) {
            l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
            l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
            if (t == 0) s_ml[warp][g + 8 * h] = make_float2(m[h], l[h]);
#pragma unroll
            for (int x = 0; x < D / 64; ++x)
#pragma unroll
                for (int e = 0; e < 2; ++e) {                // query row 2t + e: eight consecutive dimensions
                    float *dst = &s_o[warp][8 * h + 2 * t + e][Rows::vdim(g, x)];
                    *reinterpret_cast<float4 *>(dst) = make_float4(o[4 * x][h][e], o[4 * x][h][2 + e], o[4 * x + 1][h][e], o[4 * x + 1][h][2 + e]);
                    *reinterpret_cast<float4 *>(dst + 4) = make_float4(o[4 * x + 2][h][e], o[4 * x + 2][h][2 + e], o[4 * x + 3][h][e], o[4 * x + 3][h][2 + e]);
                }
        }
        __syncthreads();
        float *part = nc > 1 ? a.part + ((int64_t)(split0 + c) * a.hkv + kv) * (NR * (D + 2)) : nullptr;
        auto finish = [&](int row, float (&acc)[N], float mm, float ll) {
            const int at = rt * NR + row, head = kv * a.group + at % a.group;
            const int64_t tok = rq.q0 + at / a.group;
            bool bad = !(fabsf(ll) < INFINITY);
#pragma unroll
            for (int j = 0; j < N; ++j) bad |= !(fabsf(acc[j]) < INFINITY);
            if (rq.qn > 1 && __any_sync(0xffffffffu, bad))   // (one query token: what it does not see was not read)
                vtk_row_again<D, Rows::FP4, Act>(a, tok, head, a.positions[tok], rq.base, rq.len, acc, mm, ll);
            vtk_store_row<D, Act>(a, tok, head, acc, mm, ll);
        };
        for (int row = warp; row < rows; row += AT_WARPS) {
            float mm = -INFINITY, ll = 0.f, acc[N];
#pragma unroll
            for (int j = 0; j < N; ++j) acc[j] = 0.f;
#pragma unroll
            for (int w = 0; w < AT_WARPS; ++w) mm = fmaxf(mm, s_ml[w][row].x);
#pragma unroll
            for (int w = 0; w < AT_WARPS; ++w) {
                const float2 ml = s_ml[w][row];
                const float f = ml.x == -INFINITY ? 0.f : (ml.x == mm ? 1.f : vtk_exp2(ml.x - mm));
                ll += f * ml.y;
#pragma unroll
                for (int j = 0; j < N; ++j) acc[j] += f * s_o[w][row][lane * N + j];
            }
            if (nc > 1) {
                float *dst = part + row * D + lane * N;
                if (N == 4) *reinterpret_cast<float4 *>(dst) = make_float4(acc[0], acc[1], acc[N - 2], acc[N - 1]);
                else *reinterpret_cast<float2 *>(dst) = make_float2(acc[0], acc[1]);
                if (lane == 0) *reinterpret_cast<float2 *>(part + NR * D + 2 * row) = make_float2(mm, ll);
            } else {
                finish(row, acc, mm, ll);
            }
        }
        if (nc > 1) {
            __threadfence();
            __syncthreads();
            uint32_t *counter = a.counters + (int64_t)split0 * a.hkv + kv;
            if (tid == 0) {
                s_last = atomicAdd(counter, 1u) == (unsigned)(nc - 1);
                if (s_last) *counter = 0;                    // ready for the next call
            }
            __syncthreads();
            if (s_last) {
                __threadfence();
                const float *first = a.part + ((int64_t)split0 * a.hkv + kv) * (NR * (D + 2));
                const int64_t step = (int64_t)a.hkv * (NR * (D + 2));
                for (int row = warp; row < rows; row += AT_WARPS) {
                    float mm = -INFINITY, ll = 0.f, acc[N];
#pragma unroll
                    for (int j = 0; j < N; ++j) acc[j] = 0.f;
                    for (int i = lane; i < nc; i += 32) mm = fmaxf(mm, __ldcg(first + i * step + NR * D + 2 * row));
#pragma unroll
                    for (int d = 16; d > 0; d >>= 1) mm = fmaxf(mm, __shfl_xor_sync(0xffffffffu, mm, d));
#pragma unroll 4
                    for (int i = 0; i < nc; ++i) {
                        const float2 ml = __ldcg(reinterpret_cast<const float2 *>(first + i * step + NR * D + 2 * row));
                        const float f = ml.x == -INFINITY ? 0.f : (ml.x == mm ? 1.f : vtk_exp2(ml.x - mm));
                        ll += f * ml.y;
                        const float *src = first + i * step + row * D + lane * N;
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
        __syncthreads();                                     // shared memory is reused by the next item
    }
}

template <int D, int NR, typename Rows, typename Act, bool SPLIT_P>
int launch(vtoken_ctx *ctx, const VtkAttnArgs &a, cudaStream_t st)
{
    VTK_CUDA(ctx, vtk_launch_dependent(ctx, attention_rows_kernel<D, NR, Rows, Act, SPLIT_P>, dim3(ctx->num_sms * AT_CTAS<NR>), dim3(AT_NT), 0, st, a));
    VTK_CUDA(ctx, cudaGetLastError());
    return VTOKEN_OK;
}

template <int D, typename Act>
int launch_by_type(vtoken_ctx *ctx, bool fp4, bool wide, const VtkAttnArgs &a, cudaStream_t st)
{
    constexpr bool bf = Act::kind == VTOKEN_KV_BF16;
    if (fp4) return wide ? launch<D, 16, Rows4<D>, Act, !bf>(ctx, a, st) : launch<D, 8, Rows4<D>, Act, !bf>(ctx, a, st);
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

// Items per key head, and the workspace that the cut can need: only requests of more than one chunk leave partial
// rows, at most 2 * target of them per key head (n > chunk gives ceil(n / chunk) < 2 n / chunk, and the sum of n
// over row tiles is at most target * chunk).
int64_t vtk_attention_rows_workspace(const vtoken_ctx *ctx, const vtoken_heads *heads, VtkAttnArgs *a)
{
    const int64_t items = (int64_t)ctx->num_sms * AT_CTAS<8> * 4;
    const int64_t target = (items + heads->num_kv_heads - 1) / heads->num_kv_heads;
    const int64_t splits = 2 * target * heads->num_kv_heads;
    if (a) {
        a->target = (int32_t)target;
        a->min_chunk = 64;
    }
    const int64_t counters = (splits * 4 + 15) / 16 * 16 + 16;           // and the prompt kernel's two tickets in front
    if (a && a->counters) a->part = (float *)((uint8_t *)(a->counters - 4) + counters);
    return counters + splits * 16 * (heads->head_dim + 2) * 4;
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
