// The step's tokens into the cache and back out of it: queries and keys normalised per head and rotated by
// position, keys and values written to their slots (16-bit rows, or quantised to 4 bits), all in one pass over
// the projections.
//
// The floor is HBM's: a token's q, k and v are read once, q and the two rows written once, about 8 flops a value.
// Layout: a lane holds 8 values of a head, D / 8 lanes a head, so the mean square is log2(D / 8) shuffles.  A warp
// takes four rounds of heads of one token: its loads are all requested before the first is used and the token's
// cosines and sines (32 bits each, four times the bytes of a head's values per lane) are loaded once for all of them.
#include "heads.cuh"

namespace {

constexpr int WT_WARPS = 4, WT_ROUNDS = 4;

struct WriteArgs {
    const int32_t *num_tokens;
    int32_t max_tokens;
    const void *q, *k, *v, *q_weight, *k_weight;
    int64_t q_stride, k_stride, v_stride, q_out_stride;
    vtk_arr<const int32_t> positions, slots;
    const float *cos_sin;
    float eps, k_mul, v_mul;             // k_mul, v_mul: 2^-exponent of the 4-bit rows
    int32_t max_position, rot, interleaved, hq, hkv, tasks;
    void *q_out;
    uint8_t *k_rows, *v_rows;            // this layer's slabs
    int64_t slots_per_layer, row_bytes;
    uint32_t *flags;
};

// 64-bit value rounded once to 16 bits: to 24 bits with the sticky bit kept in the last one, then to nearest
template <typename Act>
__device__ __forceinline__ float round_once(double y)
{
    float f = __double2float_rz(y);
    if ((double)f != y && f == f) f = __uint_as_float(__float_as_uint(f) | 1u);
    return Act::unpack(Act::pack(f, 0.f)).x;
}

// normalisation and rotation of the lane's 8 values; F: the arithmetic (float, or double for rows that a coarse
// grid follows: there a value on the wrong side of a tie would be a whole step off)
template <typename F, int LPH>
__device__ __forceinline__ void norm_rotate(F (&y)[8], bool normed, const float (&w)[8], F eps, int l, int rot, int interleaved,
                                            const float (&cs)[8], const float (&sn)[8])
{
    F ss = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) ss += y[j] * y[j];
#pragma unroll
    for (int d = LPH / 2; d > 0; d >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, d);
    if (normed) {
        const F r = (F)1 / sqrt(ss / (F)(LPH * 8) + eps);
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = y[j] * r * (F)w[j];
    }
    if (rot == 0) return;
    if (interleaved) {
        if (8 * l >= rot) return;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const F a = y[2 * j], b = y[2 * j + 1], c = cs[j], s = sn[j];
            y[2 * j] = a * c - b * s;
            y[2 * j + 1] = b * c + a * s;
        }
    } else {
        const int hl = rot / 16;                          // lanes per half of the rotated part
        const int other = (vtk_lane() & ~(LPH - 1)) + (l < hl ? l + hl : (l < 2 * hl ? l - hl : l));
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const F o = __shfl_sync(0xffffffffu, y[j], other);
            if (l < hl) y[j] = y[j] * (F)cs[j] - o * (F)sn[j];
            else if (l < 2 * hl) y[j] = y[j] * (F)cs[j] + o * (F)sn[j];
        }
    }
}

// The lane's 8 values (its neighbour holds the other 8 of the group), times a power of two, to codes and a scale.
// Thresholds of the grid are compared in effect with x / scale: the division is the IEEE one, x has 8 or 11
// significant bits and the scale 4, so a quotient lands on a tie only when it is one.  A multiple that leaves 32
// bits saturates like any other that is too large.
__device__ __forceinline__ void quantise(float (&x)[8], float mul, uint32_t &codes, uint32_t &scale)
{
    float top = 0.f;
    bool odd = false;                                      // a NaN or an infinity
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        odd |= !(fabsf(x[j]) < __int_as_float(0x7f800000));
        x[j] *= mul;
        top = fmaxf(top, fabsf(x[j]));
    }
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
    odd |= (bool)__shfl_xor_sync(0xffffffffu, (int)odd, 1);
    uint16_t sc;
    const float want = __fdiv_rn(top, 6.f);
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(sc) : "f"(0.f), "f"(want));
    scale = sc & 0xffu;
    const float s = __half2float(__ushort_as_half((uint16_t)(vtk_scales_to_half2(scale) & 0xffffu)));
    codes = 0;
    if (odd) {
        scale = 0x7f;
    } else if (s > 0.f) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float lo = __fdiv_rn(x[2 * j], s), hi = __fdiv_rn(x[2 * j + 1], s);
            uint32_t two;
            asm("{\n\t.reg .b8 c;\n\tcvt.rn.satfinite.e2m1x2.f32 c, %1, %2;\n\tmov.b32 %0, {c, 0, 0, 0};\n\t}"
                : "=r"(two) : "f"(hi), "f"(lo));
            codes |= two << (8 * j);
        }
    }
}

// ---- 16-bit rows: two 32-bit operations an instruction, partners of a rotation in one lane ------
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(*reinterpret_cast<uint64_t *>(&a)), "l"(*reinterpret_cast<uint64_t *>(&b)), "l"(*reinterpret_cast<uint64_t *>(&c)));
    return *reinterpret_cast<float2 *>(&d);
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b)
{
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(*reinterpret_cast<uint64_t *>(&a)), "l"(*reinterpret_cast<uint64_t *>(&b)));
    return *reinterpret_cast<float2 *>(&d);
}

// A lane holds 8 values of a head as two runs of four: runs whose dimensions are rotation partners where pairs are
// (i, i + rot / 2), neighbouring runs elsewhere -- so that no rotation needs a shuffle.  Measured with 8 consecutive values a
// lane, partners fetched by shuffles and one operation an instruction, 16 384 tokens of 36 heads took 104 us; now 85 (3.6 TB/s of the
// 6.5 of a copy).  Neither HBM (37 %) nor the issue slots (61 %) are full: with 76 registers a third of the warps are resident, and a
// warp has loads in flight only until it starts on them.
template <int D, typename Act>
__global__ void __launch_bounds__(WT_WARPS * 32, 6) write_rows_kernel(const __grid_constant__ WriteArgs a)
{
    vtk_release_successor();
    vtk_wait_for_predecessor();
    constexpr int LPH = D / 8, HPR = 32 / LPH;            // lanes per head, heads per round
    const uint32_t task = blockIdx.x * WT_WARPS + (threadIdx.x >> 5);            // (below 2^31)
    const int64_t token = task / (uint32_t)a.tasks;
    int n = a.max_tokens;
    if (a.num_tokens != nullptr) {
        n = *a.num_tokens;
        n = n < 0 ? 0 : (n > a.max_tokens ? a.max_tokens : n);
    }
    if (token >= n) return;
    const int lane = vtk_lane(), l = lane % LPH, half = a.rot / 2;
    const bool turned = 8 * l < a.rot, split = turned && !a.interleaved;
    const int d0 = split ? 4 * l : 8 * l, d1 = split ? d0 + half : d0 + 4;       // the two runs
    const int first = (int)(task % (uint32_t)a.tasks) * (WT_ROUNDS * HPR) + lane / LPH;
    const int heads = a.hq + 2 * a.hkv;

    const uint16_t *q_in = (const uint16_t *)a.q + token * a.q_stride;
    const uint16_t *k_in = (const uint16_t *)a.k + token * a.k_stride - a.hq * D, *v_in = (const uint16_t *)a.v + token * a.v_stride - (a.hq + a.hkv) * D;
    uint2 raw[WT_ROUNDS][2];
#pragma unroll
    for (int i = 0; i < WT_ROUNDS; ++i) {
        const int h = first + i * HPR;
        raw[i][0] = raw[i][1] = make_uint2(0, 0);
        if (h < heads) {
            const uint16_t *p = (h < a.hq ? q_in : (h < a.hq + a.hkv ? k_in : v_in)) + h * D;
            raw[i][0] = *reinterpret_cast<const uint2 *>(p + d0);
            raw[i][1] = *reinterpret_cast<const uint2 *>(p + d1);
        }
    }
    uint2 wq[2] = {make_uint2(0, 0), make_uint2(0, 0)}, wk[2] = {make_uint2(0, 0), make_uint2(0, 0)};
    if (a.q_weight != nullptr && first < a.hq) {
        wq[0] = *reinterpret_cast<const uint2 *>((const uint16_t *)a.q_weight + d0);
        wq[1] = *reinterpret_cast<const uint2 *>((const uint16_t *)a.q_weight + d1);
    }
    if (a.k_weight != nullptr && first < a.hq + a.hkv && first + WT_ROUNDS * HPR > a.hq) {
        wk[0] = *reinterpret_cast<const uint2 *>((const uint16_t *)a.k_weight + d0);
        wk[1] = *reinterpret_cast<const uint2 *>((const uint16_t *)a.k_weight + d1);
    }
    int64_t slot = a.slots[token];
    if (slot >= a.slots_per_layer) {
        slot = -1;
        if (lane == 0) atomicOr(a.flags, (uint32_t)VTOKEN_FLAG_BAD_SLOT);
    }
    // factors of the rotation: pair j of the lane is x (1, c) + partner (0, s)
    float2 c2[4], s2[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) { c2[j] = make_float2(1.f, 1.f); s2[j] = make_float2(0.f, 0.f); }
    if (a.rot > 0) {
        const int pos = a.positions[token];
        if (pos < 0 || pos >= a.max_position) {
            if (lane == 0) atomicOr(a.flags, (uint32_t)VTOKEN_FLAG_BAD_POSITION);
            return;                                        // the whole warp: one token
        }
        if (turned) {
            const float *c = a.cos_sin + (int64_t)pos * a.rot + 4 * l;
            const float4 cs = *reinterpret_cast<const float4 *>(c), sn = *reinterpret_cast<const float4 *>(c + half);
            if (a.interleaved) {
                c2[0] = make_float2(cs.x, cs.x); c2[1] = make_float2(cs.y, cs.y); c2[2] = make_float2(cs.z, cs.z); c2[3] = make_float2(cs.w, cs.w);
                s2[0] = make_float2(-sn.x, sn.x); s2[1] = make_float2(-sn.y, sn.y); s2[2] = make_float2(-sn.z, sn.z); s2[3] = make_float2(-sn.w, sn.w);
            } else {
                c2[0] = c2[2] = make_float2(cs.x, cs.y);
                c2[1] = c2[3] = make_float2(cs.z, cs.w);
                s2[0] = make_float2(-sn.x, -sn.y); s2[1] = make_float2(-sn.z, -sn.w);
                s2[2] = make_float2(sn.x, sn.y); s2[3] = make_float2(sn.z, sn.w);
            }
        }
    }
    uint16_t *q_to = (uint16_t *)a.q_out + token * a.q_out_stride;
    uint16_t *k_to = (uint16_t *)(a.k_rows + slot * a.row_bytes) - a.hq * D, *v_to = (uint16_t *)(a.v_rows + slot * a.row_bytes) - (a.hq + a.hkv) * D;


#pragma unroll
    for (int i = 0; i < WT_ROUNDS; ++i) {
        const int h = first + i * HPR;
        const bool is_q = h < a.hq, is_k = !is_q && h < a.hq + a.hkv;
        uint2 out0 = raw[i][0], out1 = raw[i][1];
        if (__any_sync(0xffffffffu, is_q || is_k)) {
            float2 x[4] = {Act::unpack(raw[i][0].x), Act::unpack(raw[i][0].y), Act::unpack(raw[i][1].x), Act::unpack(raw[i][1].y)};
            float2 ss = mul2(x[0], x[0]);
#pragma unroll
            for (int j = 1; j < 4; ++j) ss = fma2(x[j], x[j], ss);
            float sum = ss.x + ss.y;
#pragma unroll
            for (int d = LPH / 2; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
            if (is_q ? a.q_weight != nullptr : is_k && a.k_weight != nullptr) {
                const float r = rsqrtf(sum * (1.f / D) + a.eps);                 // (two ulp of 32 bits)
                const uint2 w0 = is_q ? wq[0] : wk[0], w1 = is_q ? wq[1] : wk[1];
                const float2 r2 = make_float2(r, r);
                x[0] = mul2(mul2(x[0], r2), Act::unpack(w0.x)); x[1] = mul2(mul2(x[1], r2), Act::unpack(w0.y));
                x[2] = mul2(mul2(x[2], r2), Act::unpack(w1.x)); x[3] = mul2(mul2(x[3], r2), Act::unpack(w1.y));
            }
            float2 y[4];
            if (a.interleaved) {
#pragma unroll
                for (int j = 0; j < 4; ++j) y[j] = fma2(make_float2(x[j].y, x[j].x), s2[j], mul2(x[j], c2[j]));
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) y[j] = fma2(x[j ^ 2], s2[j], mul2(x[j], c2[j]));
            }
            if (!turned) {                                 // (a NaN times the factor zero is one)
#pragma unroll
                for (int j = 0; j < 4; ++j) y[j] = x[j];
            }
            if (is_q || is_k) {
                out0 = make_uint2(Act::pack(y[0].x, y[0].y), Act::pack(y[1].x, y[1].y));
                out1 = make_uint2(Act::pack(y[2].x, y[2].y), Act::pack(y[3].x, y[3].y));
            }
        }
        uint16_t *to = h < a.hq ? q_to : (h < a.hq + a.hkv ? k_to : v_to);
        to += h * D;
        if (h < heads && (is_q || slot >= 0)) {
            *reinterpret_cast<uint2 *>(to + d0) = out0;
            *reinterpret_cast<uint2 *>(to + d1) = out1;
        }
    }
}

// ---- 4-bit rows: 8 consecutive values a lane, half a group ---------------------------------------
// (16 384 tokens of 48 heads: 377 us against 106 into 16-bit rows; the keys' arithmetic in 64 bits runs at a fraction of the rate)
template <int D, typename Act>
__global__ void __launch_bounds__(WT_WARPS * 32) write_codes_kernel(const __grid_constant__ WriteArgs a)
{
    vtk_release_successor();
    vtk_wait_for_predecessor();
    constexpr int LPH = D / 8, HPR = 32 / LPH;            // lanes per head, heads per round
    const uint32_t task = blockIdx.x * WT_WARPS + (threadIdx.x >> 5);            // (below 2^31)
    const int64_t token = task / (uint32_t)a.tasks;
    int n = a.max_tokens;
    if (a.num_tokens != nullptr) {
        n = *a.num_tokens;
        n = n < 0 ? 0 : (n > a.max_tokens ? a.max_tokens : n);
    }
    if (token >= n) return;
    const int lane = vtk_lane(), l = lane % LPH;
    const int first = (int)(task % (uint32_t)a.tasks) * (WT_ROUNDS * HPR) + lane / LPH;
    const int heads = a.hq + 2 * a.hkv;

    uint4 raw[WT_ROUNDS];
#pragma unroll
    for (int i = 0; i < WT_ROUNDS; ++i) {
        const int h = first + i * HPR;
        raw[i] = make_uint4(0, 0, 0, 0);
        const uint16_t *p = nullptr;
        if (h < a.hq) p = (const uint16_t *)a.q + token * a.q_stride + (int64_t)h * D;
        else if (h < a.hq + a.hkv) p = (const uint16_t *)a.k + token * a.k_stride + (int64_t)(h - a.hq) * D;
        else if (h < heads) p = (const uint16_t *)a.v + token * a.v_stride + (int64_t)(h - a.hq - a.hkv) * D;
        if (p != nullptr) raw[i] = *reinterpret_cast<const uint4 *>(p + 8 * l);
    }
    int64_t slot = a.slots[token];
    if (slot >= a.slots_per_layer) {
        slot = -1;
        if (lane == 0) atomicOr(a.flags, (uint32_t)VTOKEN_FLAG_BAD_SLOT);
    }
    float cs[8], sn[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) { cs[j] = 1.f; sn[j] = 0.f; }
    if (a.rot > 0) {
        const int pos = a.positions[token];
        if (pos < 0 || pos >= a.max_position) {
            if (lane == 0) atomicOr(a.flags, (uint32_t)VTOKEN_FLAG_BAD_POSITION);
            return;                                        // the whole warp: one token
        }
        if (8 * l < a.rot) {
            const float *c = a.cos_sin + (int64_t)pos * a.rot;
            const int half = a.rot / 2;
            c += a.interleaved ? 4 * l : (8 * l < half ? 8 * l : 8 * l - half);
            const float4 c0 = *reinterpret_cast<const float4 *>(c), s0 = *reinterpret_cast<const float4 *>(c + half);
            cs[0] = c0.x; cs[1] = c0.y; cs[2] = c0.z; cs[3] = c0.w;
            sn[0] = s0.x; sn[1] = s0.y; sn[2] = s0.z; sn[3] = s0.w;
            if (!a.interleaved) {
                const float4 c1 = *reinterpret_cast<const float4 *>(c + 4), s1 = *reinterpret_cast<const float4 *>(c + half + 4);
                cs[4] = c1.x; cs[5] = c1.y; cs[6] = c1.z; cs[7] = c1.w;
                sn[4] = s1.x; sn[5] = s1.y; sn[6] = s1.z; sn[7] = s1.w;
            }
        }
    }

#pragma unroll
    for (int i = 0; i < WT_ROUNDS; ++i) {
        const int h = first + i * HPR;
        const bool is_q = h < a.hq, is_k = !is_q && h < a.hq + a.hkv, is_v = !is_q && !is_k && h < heads;
        float x[8];
        vtk_unpack8<Act>(raw[i], x);
        if (__any_sync(0xffffffffu, is_q || is_k)) {
            const void *wp = is_q ? a.q_weight : (is_k ? a.k_weight : nullptr);
            float w[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
            if (wp != nullptr) vtk_unpack8<Act>(*reinterpret_cast<const uint4 *>((const uint16_t *)wp + 8 * l), w);
            float y[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = x[j];
            bool done = false;
            if (__any_sync(0xffffffffu, is_k)) {
                double z[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) z[j] = x[j];
                norm_rotate<double, LPH>(z, wp != nullptr, w, (double)a.eps, l, a.rot, a.interleaved, cs, sn);
#pragma unroll
                for (int j = 0; j < 8; ++j) y[j] = round_once<Act>(z[j]);
                done = true;
            }
            if (!done) norm_rotate<float, LPH>(y, wp != nullptr, w, a.eps, l, a.rot, a.interleaved, cs, sn);
            if (is_q) *reinterpret_cast<uint4 *>((uint16_t *)a.q_out + token * a.q_out_stride + (int64_t)h * D + 8 * l) = vtk_pack8<Act>(y);
            if (is_k) {
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = y[j];
            }
        }
        const int kvh = is_k ? h - a.hq : h - a.hq - a.hkv;
        uint8_t *row = (is_k ? a.k_rows : a.v_rows) + slot * a.row_bytes;
        if (__any_sync(0xffffffffu, is_k || is_v)) {
            uint32_t codes, scale;
            quantise(x, is_k ? a.k_mul : a.v_mul, codes, scale);
            if ((is_k || is_v) && slot >= 0) {
                *reinterpret_cast<uint32_t *>(row + kvh * (D / 2) + 4 * l) = codes;
                if ((l & 1) == 0) row[(int64_t)a.hkv * (D / 2) + kvh * (D / 16) + l / 2] = (uint8_t)scale;
            }
        }
    }
}

struct ReadArgs {
    const int32_t *num_tokens;
    int32_t max_tokens, hkv;
    vtk_arr<const int32_t> slots;
    const uint8_t *k_rows, *v_rows;
    void *out_k, *out_v;
    float k_mul, v_mul;                  // 2^exponent
    int64_t slots_per_layer, row_bytes;
    uint32_t *flags;
};

template <int D, bool FP4, typename Act>
__global__ void __launch_bounds__(256) read_tokens_kernel(ReadArgs a)
{
    vtk_release_successor();
    vtk_wait_for_predecessor();
    const int per = a.hkv * (D / 8);                      // 8 values a thread, K then V
    const uint32_t i = blockIdx.x * 256u + threadIdx.x;   // (below 2^31)
    const int64_t token = i / (uint32_t)(2 * per);
    int n = a.max_tokens;
    if (a.num_tokens != nullptr) {
        n = *a.num_tokens;
        n = n < 0 ? 0 : (n > a.max_tokens ? a.max_tokens : n);
    }
    if (token >= n) return;
    const int at = (int)(i % (uint32_t)(2 * per));
    const bool is_v = at >= per;
    const int j = is_v ? at - per : at;
    void *out = is_v ? a.out_v : a.out_k;
    if (out == nullptr) return;
    const int64_t slot = a.slots[token];
    uint4 w = make_uint4(0, 0, 0, 0);
    if (slot >= a.slots_per_layer) atomicOr(a.flags, (uint32_t)VTOKEN_FLAG_BAD_SLOT);
    if (slot >= 0 && slot < a.slots_per_layer) {
        const uint8_t *row = (is_v ? a.v_rows : a.k_rows) + slot * a.row_bytes;
        if (!FP4) {
            w = *reinterpret_cast<const uint4 *>(row + 16 * (int64_t)j);
        } else {
            const uint32_t codes = *reinterpret_cast<const uint32_t *>(row + 4 * j);
            const uint32_t s2 = vtk_scales_to_half2(row[a.hkv * (D / 2) + j / 2]);
            const float s = __half2float(__ushort_as_half((uint16_t)(s2 & 0xffffu))), mul = is_v ? a.v_mul : a.k_mul;
            float x[8];
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const float2 c = VtkFp16::unpack(vtk_codes_to_half2(codes >> (8 * b)));
                x[2 * b] = c.x * s * mul;
                x[2 * b + 1] = c.y * s * mul;
            }
            w = vtk_pack8<Act>(x);
        }
    }
    *reinterpret_cast<uint4 *>((uint16_t *)out + token * (int64_t)a.hkv * D + 8 * j) = w;
}

template <int D, bool FP4, typename Act>
int launch_write(vtoken_ctx *ctx, const WriteArgs &a, cudaStream_t st)
{
    const int64_t warps = (int64_t)a.max_tokens * a.tasks;
    auto kernel = FP4 ? write_codes_kernel<D, Act> : write_rows_kernel<D, Act>;
    VTK_CUDA(ctx, vtk_launch_dependent(ctx, kernel, dim3((unsigned)((warps + WT_WARPS - 1) / WT_WARPS)),
                                       dim3(WT_WARPS * 32), 0, st, a));
    VTK_CUDA(ctx, cudaGetLastError());
    return VTOKEN_OK;
}

template <int D, bool FP4, typename Act>
int launch_read(vtoken_ctx *ctx, const ReadArgs &a, cudaStream_t st)
{
    const int64_t threads = (int64_t)a.max_tokens * 2 * a.hkv * (D / 8);
    VTK_CUDA(ctx, vtk_launch_dependent(ctx, read_tokens_kernel<D, FP4, Act>, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, st, a));
    VTK_CUDA(ctx, cudaGetLastError());
    return VTOKEN_OK;
}

// the instantiation of F for a geometry
#define VTK_BY_HEADS(F, h, ...)                                                                              \
    ((h)->head_dim == 128                                                                                    \
         ? ((h)->act_type == VTOKEN_KV_BF16                                                                  \
                ? ((h)->kv_type == VTOKEN_KV_FP4 ? F<128, true, VtkBf16>(__VA_ARGS__) : F<128, false, VtkBf16>(__VA_ARGS__)) \
                : ((h)->kv_type == VTOKEN_KV_FP4 ? F<128, true, VtkFp16>(__VA_ARGS__) : F<128, false, VtkFp16>(__VA_ARGS__))) \
         : ((h)->act_type == VTOKEN_KV_BF16                                                                  \
                ? ((h)->kv_type == VTOKEN_KV_FP4 ? F<64, true, VtkBf16>(__VA_ARGS__) : F<64, false, VtkBf16>(__VA_ARGS__)) \
                : ((h)->kv_type == VTOKEN_KV_FP4 ? F<64, true, VtkFp16>(__VA_ARGS__) : F<64, false, VtkFp16>(__VA_ARGS__))))

bool misaligned(const void *p) { return ((uintptr_t)p & 15) != 0; }

float two_to(int e)
{
    float x = 1.f;
    for (; e > 0; --e) x *= 2.f;
    for (; e < 0; ++e) x *= 0.5f;
    return x;
}

}  // namespace

extern "C" {

int64_t vtoken_kv_row_bytes(const vtoken_heads *heads)
{
    const int64_t row = vtk_heads_row_bytes(heads);
    return row > 0 ? row : VTOKEN_EINVAL;
}

int vtoken_write_tokens(vtoken_ctx *ctx, const vtoken_heads *heads, int32_t layer, const vtoken_write_in *in, void *cuda_stream)
{
    if (!ctx || !heads || !in) return VTOKEN_EINVAL;
    if (vtk_check_heads(ctx, heads, layer) != VTOKEN_OK) return VTOKEN_EINVAL;
    if (in->max_tokens < 0) return VTOKEN_EINVAL;
    const bool none = in->max_tokens == 0;                   // (arrays without elements may have no address)
    if (!none && (!in->k || !in->v || !in->slots || (in->q && !in->q_out))) return VTOKEN_EINVAL;
    if (misaligned(in->q) || misaligned(in->k) || misaligned(in->v) || misaligned(in->q_weight) || misaligned(in->k_weight) ||
        misaligned(in->cos_sin) || misaligned(in->q_out))
        return VTOKEN_EINVAL;
    if (in->rot_dim < 0 || in->rot_dim > heads->head_dim || in->rot_dim % 16 != 0) return VTOKEN_EINVAL;
    if (in->rot_dim > 0 && (!in->cos_sin || (!none && !in->positions) || in->max_position < 1)) return VTOKEN_EINVAL;
    if ((in->q_weight || in->k_weight) && !(in->eps > 0.f && in->eps < 1e30f)) return VTOKEN_EINVAL;
    const int64_t dq = (int64_t)heads->num_q_heads * heads->head_dim, dk = (int64_t)heads->num_kv_heads * heads->head_dim;
    WriteArgs a;
    a.q_stride = vtk_stride(in->q_stride, dq);
    a.k_stride = vtk_stride(in->k_stride, dk);
    a.v_stride = vtk_stride(in->v_stride, dk);
    a.q_out_stride = vtk_stride(in->q_out_stride, dq);
    if (a.q_stride < 0 || a.k_stride < 0 || a.v_stride < 0 || a.q_out_stride < 0) return VTOKEN_EINVAL;
    if (in->q && in->q == in->q_out && a.q_stride != a.q_out_stride) return VTOKEN_EINVAL;
    if (none) return VTOKEN_OK;
    a.num_tokens = in->num_tokens;
    a.max_tokens = in->max_tokens;
    a.q = in->q; a.k = in->k; a.v = in->v;
    a.q_weight = in->q_weight; a.k_weight = in->k_weight;
    a.positions = VTK_ARR(ctx, in->positions, in->max_tokens);
    a.slots = VTK_ARR(ctx, in->slots, in->max_tokens);
    a.cos_sin = in->cos_sin;
    a.eps = in->eps;
    a.k_mul = two_to(-heads->k_exponent);
    a.v_mul = two_to(-heads->v_exponent);
    a.max_position = in->max_position;
    a.rot = in->rot_dim;
    a.interleaved = in->interleaved != 0;
    a.hq = in->q ? heads->num_q_heads : 0;
    a.hkv = heads->num_kv_heads;
    const int per_task = WT_ROUNDS * 32 / (heads->head_dim / 8);
    a.tasks = (a.hq + 2 * a.hkv + per_task - 1) / per_task;
    a.q_out = in->q_out;
    a.k_rows = (uint8_t *)ctx->cfg.k_pool + layer * ctx->layer_stride;
    a.v_rows = (uint8_t *)ctx->cfg.v_pool + layer * ctx->layer_stride;
    a.slots_per_layer = ctx->slots_per_layer;
    a.row_bytes = ctx->row_bytes;
    a.flags = &ctx->rt_counts->error_flags;
    if ((int64_t)a.max_tokens * a.tasks + WT_WARPS > INT32_MAX) return VTOKEN_ECAPACITY;
    return VTK_BY_HEADS(launch_write, heads, ctx, a, (cudaStream_t)cuda_stream);
}

int vtoken_read_tokens(vtoken_ctx *ctx, const vtoken_heads *heads, int32_t layer, const int32_t *num_tokens, int32_t max_tokens,
                       const int32_t *slots, void *out_k, void *out_v, void *cuda_stream)
{
    if (!ctx || !heads) return VTOKEN_EINVAL;
    if (vtk_check_heads(ctx, heads, layer) != VTOKEN_OK) return VTOKEN_EINVAL;
    if (max_tokens < 0 || (max_tokens > 0 && !slots) || misaligned(out_k) || misaligned(out_v)) return VTOKEN_EINVAL;
    if (max_tokens == 0 || (!out_k && !out_v)) return VTOKEN_OK;
    ReadArgs a;
    a.num_tokens = num_tokens;
    a.max_tokens = max_tokens;
    a.hkv = heads->num_kv_heads;
    a.slots = VTK_ARR(ctx, slots, max_tokens);
    a.k_rows = (const uint8_t *)ctx->cfg.k_pool + layer * ctx->layer_stride;
    a.v_rows = (const uint8_t *)ctx->cfg.v_pool + layer * ctx->layer_stride;
    a.out_k = out_k;
    a.out_v = out_v;
    a.k_mul = two_to(heads->k_exponent);
    a.v_mul = two_to(heads->v_exponent);
    a.slots_per_layer = ctx->slots_per_layer;
    a.row_bytes = ctx->row_bytes;
    a.flags = &ctx->rt_counts->error_flags;
    if ((int64_t)max_tokens * 2 * a.hkv * (heads->head_dim / 8) + 256 > INT32_MAX) return VTOKEN_ECAPACITY;
    return VTK_BY_HEADS(launch_read, heads, ctx, a, (cudaStream_t)cuda_stream);
}

}  // extern "C"
