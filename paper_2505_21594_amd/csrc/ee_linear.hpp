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
    long long lda, ldb, plane;         // plane: from one term of A to the next, the larger one (the sum of both is A; of fp16 the smaller one times 2^-11)
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

// (fp16: the matrix cores line a product with a subnormal operand up as one with 2^-14, so that a sum may be off by 2^-24 of the largest product taken that way: 2 products of 4e-5 and 0.06
// by 2^-40.)
template <int TYPE>
__device__ __forceinline__ f32x4_t mfma16(const u32x4_t &a, const u32x4_t &b, const f32x4_t &c)
{
    if constexpr (TYPE == EE_BF16)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c, 0, 0, 0);
}

// fp32 activations and their derivatives: SiLU z / (1 + e^-z), GELU z Phi(z).  The exponential as 2^(z log2 e) and the reciprocal are the hardware's (1 ulp, and the
// argument's rounding, |z| 2^-24 of e^-z): a few units in 2^-24 of z, of GELU's value too, its far side's relative to itself.
__device__ __forceinline__ float logistic(float z) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * -1.44269504f)); }
// Phi(z) as half of erfc(-z / sqrt 2): 1 + erf(z / sqrt 2) has next to nothing left of it below z = -4 (a twentieth off at -5, nothing at -6); it costs
// 2 % (2041 x 4096 x 11008 with GELU, bf16, 210 -> 215 us).
__device__ __forceinline__ float normal(float z) { return 0.5f * erfcf(z * -0.70710678f); }
__device__ __forceinline__ float act_of(int act, float z)
{
    if (act == EE_ACT_SILU) return z * logistic(z);
    if (act == EE_ACT_GELU) return z * normal(z);
    return z;
}
__device__ __forceinline__ float act_slope(int act, float z)
{
    if (fabsf(z) > 100.f) z = copysignf(100.f, z);                                       // (where the slope is 0 or 1: no infinity times 0; NaN stays)
    if (act == EE_ACT_SILU) {
        const float s = logistic(z);
        return s * (1.f + z * (1.f - s));
    }
    if (act == EE_ACT_GELU) return normal(z) + z * expf(-0.5f * z * z) * 0.39894228f;
    return 1.f;
}

// Four neighbouring elements of a row, `n` of which are there; rows start at multiples of 16 bytes.
__device__ __forceinline__ f32x4_t load4(int type, const void *p, size_t at, int n)
{
    f32x4_t v = {0.f, 0.f, 0.f, 0.f};
    if (n < 4) {
        for (int e = 0; e < n; ++e) v[e] = logit_at(type, p, at + e);
    } else if (type == EE_FP32) {
        v = *as_global(reinterpret_cast<const f32x4_t *>(static_cast<const float *>(p) + at));
    } else {
        const u32x2_t w = *as_global(reinterpret_cast<const u32x2_t *>(static_cast<const uint16_t *>(p) + at));
        const unsigned a = w[0], b = w[1];
        if (type == EE_BF16) {
            v = (f32x4_t){__uint_as_float(a << 16), __uint_as_float(a & 0xFFFF0000u), __uint_as_float(b << 16), __uint_as_float(b & 0xFFFF0000u)};
        } else {
            typedef __attribute__((ext_vector_type(2))) _Float16 f16x2_t;
            const f16x2_t x = __builtin_bit_cast(f16x2_t, a), y = __builtin_bit_cast(f16x2_t, b);
            v = (f32x4_t){(float)x[0], (float)x[1], (float)y[0], (float)y[1]};
        }
    }
    return v;
}
__device__ __forceinline__ void store4_of(int type, void *p, size_t at, int n, const f32x4_t &v)
{
    if (n >= 4)
        store4(type, p, at, v[0], v[1], v[2], v[3]);
    else
        for (int e = 0; e < n; ++e) store_one(type, p, at + e, v[e]);
}
__device__ __forceinline__ f32x4_t bias4(const float *p, int n)
{
    f32x4_t v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (e < n) v[e] = as_global(p)[e];
    return v;
}
__device__ __forceinline__ f32x4_t bias_at(const GemmDev &g, int j) { return g.bias && j < g.J ? bias4(g.bias + j, g.J - j) : (f32x4_t){0.f, 0.f, 0.f, 0.f}; }

// Four neighbouring results of each of N rows, `step` apart: bias, activation, residual, one rounding.
template <int N>
__device__ __forceinline__ void finish(const GemmDev &g, int i, int step, int j, const f32x4_t &bias, f32x4_t (&v)[N])
{
    const int n = g.J - j;
    f32x4_t res[N];
    if (g.residual)
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (i + e * step < g.I) res[e] = load4(g.res_type, g.residual, (size_t)(i + e * step) * g.res_stride + j, n);
#pragma unroll
    for (int e = 0; e < N; ++e) {
        const int row = i + e * step;
        if (row >= g.I) break;
        v[e] += bias;
        if (g.pre) store4_of(g.type, g.pre, (size_t)row * g.pre_stride + j, n, v[e]);
        if (g.act != EE_ACT_NONE)
#pragma unroll
            for (int c = 0; c < 4; ++c) v[e][c] = act_of(g.act, v[e][c]);
        if (g.residual) v[e] += res[e];
        store4_of(g.y_type, g.y, (size_t)row * g.y_stride + j, n, v[e]);
    }
}

}  // namespace ee
