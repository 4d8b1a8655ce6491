// Helpers shared by the kernels that look inside a pool row (token writes and reads, attention): the 16-bit
// types, the 4-bit rows, the checks of vtoken_heads.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "common.cuh"

// ---- 16-bit types: pairs as 32-bit words -------------------------------------------------------
struct VtkBf16 {
    static constexpr int kind = VTOKEN_KV_BF16;
    static __device__ __forceinline__ float2 unpack(uint32_t w)
    {
        return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    }
    static __device__ __forceinline__ uint32_t pack(float lo, float hi)
    {
        uint32_t w;
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(hi), "f"(lo));
        return w;
    }
};

struct VtkFp16 {
    static constexpr int kind = VTOKEN_KV_FP16;
    static __device__ __forceinline__ float2 unpack(uint32_t w)
    {
        return __half22float2(*reinterpret_cast<const __half2 *>(&w));
    }
    static __device__ __forceinline__ uint32_t pack(float lo, float hi)
    {
        uint32_t w;
        asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(hi), "f"(lo));
        return w;
    }
};

template <typename T>
__device__ __forceinline__ void vtk_unpack8(uint4 w, float (&x)[8])
{
    const float2 a = T::unpack(w.x), b = T::unpack(w.y), c = T::unpack(w.z), d = T::unpack(w.w);
    x[0] = a.x; x[1] = a.y; x[2] = b.x; x[3] = b.y; x[4] = c.x; x[5] = c.y; x[6] = d.x; x[7] = d.y;
}

template <typename T>
__device__ __forceinline__ uint4 vtk_pack8(const float (&x)[8])
{
    return make_uint4(T::pack(x[0], x[1]), T::pack(x[2], x[3]), T::pack(x[4], x[5]), T::pack(x[6], x[7]));
}

// ---- 4-bit rows --------------------------------------------------------------------------------
constexpr int VTK_FP4_GROUP = 16;        // values that share a scale

__host__ __device__ __forceinline__ int64_t vtk_fp4_row_bytes(int num_kv_heads, int head_dim)
{
    const int64_t n = (int64_t)num_kv_heads * (head_dim / 2 + head_dim / VTK_FP4_GROUP);
    return (n + 15) / 16 * 16;
}

// two 8-bit scales (low byte, high byte) as two halves; exact
__device__ __forceinline__ uint32_t vtk_scales_to_half2(uint32_t two_bytes)
{
    uint32_t h;
    const uint16_t b = (uint16_t)two_bytes;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(b));
    return h;
}

// the two codes of byte `b` (low half first) as two halves; exact
__device__ __forceinline__ uint32_t vtk_codes_to_half2(uint32_t b)
{
    uint32_t h;
    asm("{\n\t.reg .b8 c, d0, d1, d2;\n\tmov.b32 {c, d0, d1, d2}, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, c;\n\t}" : "=r"(h) : "r"(b));
    return h;
}

// the eight codes of a word, in order
__device__ __forceinline__ uint4 vtk_word_to_half2(uint32_t w)
{
    uint4 r;
    asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %4;\n\tcvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, c;\n\tcvt.rn.f16x2.e2m1x2 %3, d;\n\t}" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "r"(w));
    return r;
}

__device__ __forceinline__ uint32_t vtk_hmul2(uint32_t a, uint32_t b)
{
    const __half2 r = __hmul2(*reinterpret_cast<__half2 *>(&a), *reinterpret_cast<__half2 *>(&b));
    return *reinterpret_cast<const uint32_t *>(&r);
}

// eight codes times the scale of their group (a pair of equal halves)
__device__ __forceinline__ uint4 vtk_expand8(uint32_t w, uint32_t s)
{
    const uint4 c = vtk_word_to_half2(w);
    return make_uint4(vtk_hmul2(c.x, s), vtk_hmul2(c.y, s), vtk_hmul2(c.z, s), vtk_hmul2(c.w, s));
}

// ---- host: geometry ----------------------------------------------------------------------------
// row bytes of a supported geometry, -1 otherwise
inline int64_t vtk_heads_row_bytes(const vtoken_heads *h)
{
    if (!h || h->num_kv_heads < 1 || h->num_q_heads < h->num_kv_heads || h->num_q_heads % h->num_kv_heads != 0) return -1;
    if (h->num_q_heads > 4096) return -1;
    if (h->head_dim != 64 && h->head_dim != 128) return -1;
    if (h->act_type != VTOKEN_KV_BF16 && h->act_type != VTOKEN_KV_FP16) return -1;
    if (h->kv_type == VTOKEN_KV_FP4) {
        if (h->k_exponent < -60 || h->k_exponent > 60 || h->v_exponent < -60 || h->v_exponent > 60) return -1;
        return vtk_fp4_row_bytes(h->num_kv_heads, h->head_dim);
    }
    if (h->kv_type != h->act_type || h->k_exponent != 0 || h->v_exponent != 0) return -1;
    return (int64_t)h->num_kv_heads * h->head_dim * 2;
}

// VTOKEN_OK when the geometry is supported and fits the context's rows and layers
inline int vtk_check_heads(const vtoken_ctx *ctx, const vtoken_heads *h, int32_t layer)
{
    if (!ctx || !h) return VTOKEN_EINVAL;
    if (layer < 0 || layer >= ctx->cfg.num_layers) return VTOKEN_EINVAL;
    const int64_t row = vtk_heads_row_bytes(h);
    return row > 0 && row == ctx->row_bytes ? VTOKEN_OK : VTOKEN_EINVAL;
}

// a token stride in elements: 0 = dense; -1 when it cannot be used
inline int64_t vtk_stride(int64_t given, int64_t dense)
{
    if (given == 0) return dense;
    return given >= dense && given % 8 == 0 ? given : -1;
}
