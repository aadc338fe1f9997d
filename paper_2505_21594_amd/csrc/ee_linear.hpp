// ee_linear, ee_linear_grad: products of 16-bit matrices on the matrix cores, with bias, activation and residual.
//
//   forward   z = x W^T + b,  y = act(z) + residual;
//   backward  dz = dy act'(z),  dx = dz W,  dW = dz^T x,  db = sum over rows of dz.
#pragma once

#include "ee_vocab.hpp"

namespace ee {

typedef __attribute__((ext_vector_type(8))) _Float16 f16x8_t;

// C[i][j] = sum_c A(i, c) B(j, c): an operand lies in memory with the sum's index contiguous ([i][c]) or with the result's ([c][i]).
struct GemmDev {
    const uint16_t *A, *B;
    long long lda, ldb, plane;         // plane: from one term of A to the next
    int terms, I, J, K;
    const float *bias;                 // [J]
    const void *residual;
    void *y, *pre;
    long long res_stride, y_stride, pre_stride;
    int res_type, y_type, type, act;
    int ni, nj, splits, per;           // tiles, parts of the sum, and a part's length
    int far;                           // rows are too far apart for 32-bit offsets
    float *part;                       // [splits][I][part_ld]
    long long part_ld;
};

template <int TYPE>
__device__ __forceinline__ f32x4_t mfma16(const u32x4_t &a, const u32x4_t &b, const f32x4_t &c)
{
    if constexpr (TYPE == EE_BF16)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c, 0, 0, 0);
}

// fp32 activations and their derivatives: SiLU z / (1 + e^-z), GELU z Phi(z)
__device__ __forceinline__ float act_of(int act, float z)
{
    if (act == EE_ACT_SILU) return z / (1.f + expf(-z));
    if (act == EE_ACT_GELU) return 0.5f * z * (1.f + erff(z * 0.70710678f));
    return z;
}
__device__ __forceinline__ float act_slope(int act, float z)
{
    if (act == EE_ACT_SILU) {
        const float s = 1.f / (1.f + expf(-z));
        return s * (1.f + z * (1.f - s));
    }
    if (act == EE_ACT_GELU) return 0.5f * (1.f + erff(z * 0.70710678f)) + z * expf(-0.5f * z * z) * 0.39894228f;
    return 1.f;
}

// Four neighbouring results of a row: bias, activation, residual, one rounding.
__device__ __forceinline__ void finish4(const GemmDev &g, int i, int j, f32x4_t v)
{
    if (i >= g.I || j >= g.J) return;
    const int n = min(g.J - j, 4);
    if (g.bias)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < n) v[e] += as_global(g.bias)[j + e];
    if (g.pre) {
        const size_t at = (size_t)i * g.pre_stride + j;
        if (n == 4)
            store4(g.type, g.pre, at, v[0], v[1], v[2], v[3]);
        else
            for (int e = 0; e < n; ++e) store_one(g.type, g.pre, at + e, v[e]);
    }
    if (g.act != EE_ACT_NONE)
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = act_of(g.act, v[e]);
    if (g.residual)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < n) v[e] += logit_at(g.res_type, g.residual, (size_t)i * g.res_stride + j + e);
    const size_t at = (size_t)i * g.y_stride + j;
    if (n == 4)
        store4(g.y_type, g.y, at, v[0], v[1], v[2], v[3]);
    else
        for (int e = 0; e < n; ++e) store_one(g.y_type, g.y, at + e, v[e]);
}

}  // namespace ee
