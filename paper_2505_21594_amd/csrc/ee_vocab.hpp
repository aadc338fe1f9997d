// What the operators on rows over a vocabulary share (ee_accept_drafts, ee_score_tokens, ee_distill): loads at any alignment, sums
// over a wave in 64 bits, a row's logits in registers.
#pragma once

#include <type_traits>

#include "ee_ops.hpp"

namespace ee {

// Neighbouring elements at any alignment of the element type; past the end of the row: `fill`.
template <int N, typename T>
__device__ __forceinline__ void load_some(const T *p, int n, float fill, float (&x)[N])
{
    if (n >= N) {
        typedef T some_t __attribute__((ext_vector_type(N), aligned(sizeof(T))));
        const some_t e = *(const EE_GLOBAL some_t *)as_global(p);
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = (float)e[i];
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            x[i] = fill;
            if (i < n) x[i] = (float)as_global(p)[i];
        }
    }
}
__device__ __forceinline__ double join_d(unsigned lo, unsigned hi) { return __longlong_as_double((long long)((unsigned long long)hi << 32 | lo)); }
template <int CTRL, int ROWS = 0xF>
__device__ __forceinline__ double dpp_d(double x)
{
    const unsigned long long b = (unsigned long long)__double_as_longlong(x);
    return join_d((unsigned)dpp<CTRL, ROWS>(0, (int)(unsigned)b), (unsigned)dpp<CTRL, ROWS>(0, (int)(unsigned)(b >> 32)));
}
// sum over a wave, in every lane, always in the same order
__device__ __forceinline__ double wave_sum_d(double x)
{
    x += dpp_d<DPP_XOR1>(x);
    x += dpp_d<DPP_XOR2>(x);
    x += dpp_d<DPP_HALF_MIRROR>(x);
    x += dpp_d<DPP_MIRROR>(x);
    unsigned la, lb, ha, hb;
    unsigned long long b = (unsigned long long)__double_as_longlong(x);
    pair16((unsigned)b, la, lb);
    pair16((unsigned)(b >> 32), ha, hb);
    x = join_d(la, ha) + join_d(lb, hb);
    b = (unsigned long long)__double_as_longlong(x);
    pair32((unsigned)b, la, lb);
    pair32((unsigned)(b >> 32), ha, hb);
    return join_d(la, ha) + join_d(lb, hb);
}
__device__ __forceinline__ float wave_max_f(float x)
{
    x = fmaxf(x, __int_as_float(dpp<DPP_XOR1>(0, __float_as_int(x))));
    x = fmaxf(x, __int_as_float(dpp<DPP_XOR2>(0, __float_as_int(x))));
    x = fmaxf(x, __int_as_float(dpp<DPP_HALF_MIRROR>(0, __float_as_int(x))));
    x = fmaxf(x, __int_as_float(dpp<DPP_MIRROR>(0, __float_as_int(x))));
    return quads_max(x);
}
// inclusive sums over the lanes of a wave
__device__ __forceinline__ double wave_scan_d(double x)
{
    x += dpp_d<DPP_SHR + 1>(x);
    x += dpp_d<DPP_SHR + 2>(x);
    x += dpp_d<DPP_SHR + 4>(x);
    x += dpp_d<DPP_SHR + 8>(x);
    x += dpp_d<DPP_BCAST15, 0xA>(x);
    x += dpp_d<DPP_BCAST31, 0xC>(x);
    return x;
}

typedef uint32_t u32x4_at4_t __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x4_at2_t __attribute__((ext_vector_type(4), aligned(2)));

// Part of a row in a workgroup's registers, as it lies in memory: chunk c of thread t holds the elements (c * NT + t) * N .. + N - 1 behind the
// part's first, N of them in 16 bytes; -infinity behind the part's end.
template <int TYPE, int E, int NT>
struct RowPart {
    static constexpr int N = TYPE == EE_FP32 ? 4 : 8;      // elements of a chunk
    static constexpr int ROOM = E * NT * N;                // of a part at most
    u32x4_t raw[E];

    static __device__ __forceinline__ int offset(int c, int tid) { return (c * NT + tid) * N; }
    // the part of `n` elements at `p` (the same in every lane), which is aligned to the element type
    __device__ __forceinline__ void load(const void *p, int n, int tid)
    {
        constexpr uint32_t NOTHING = TYPE == EE_FP32 ? 0xFF800000u : TYPE == EE_BF16 ? 0xFF80FF80u : 0xFC00FC00u;
        typedef std::conditional_t<TYPE == EE_FP32, u32x4_at4_t, u32x4_at2_t> some_t;
        const EE_GLOBAL char *const base = (const EE_GLOBAL char *)as_global(static_cast<const char *>(p));
        const int mine = n - tid * N;
#pragma unroll
        for (int c = 0; c < E; ++c) {
            if (n >= (c + 1) * NT * N) {
                raw[c] = *(const EE_GLOBAL some_t *)(base + c * NT * 16 + (unsigned)tid * 16u);
            } else {
                raw[c] = (u32x4_t){NOTHING, NOTHING, NOTHING, NOTHING};
                if (mine >= c * NT * N + N) raw[c] = *(const EE_GLOBAL some_t *)(base + c * NT * 16 + (unsigned)tid * 16u);
            }
        }
        // the chunk that the part's end is in
        const int last = n / N;
        if (n % N != 0 && tid == last % NT) {
            uint32_t w[4] = {NOTHING, NOTHING, NOTHING, NOTHING};
            const EE_GLOBAL char *const q = base + (size_t)last * 16;
#pragma unroll
            for (int i = 0; i < N - 1; ++i)
                if (last * N + i < n) {
                    if constexpr (TYPE == EE_FP32)
                        w[i] = *(const EE_GLOBAL uint32_t *)(q + i * 4);
                    else
                        w[i / 2] = i % 2 ? (w[i / 2] & 0xFFFFu) | (uint32_t) * (const EE_GLOBAL uint16_t *)(q + i * 2) << 16 : (w[i / 2] & 0xFFFF0000u) | *(const EE_GLOBAL uint16_t *)(q + i * 2);
                }
#pragma unroll
            for (int c = 0; c < E; ++c)
                if (c == last / NT) raw[c] = (u32x4_t){w[0], w[1], w[2], w[3]};
        }
    }
    static __device__ __forceinline__ void values(const u32x4_t &r, float (&x)[N])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (TYPE == EE_FP32) {
                x[i] = __uint_as_float(r[i]);
            } else if constexpr (TYPE == EE_BF16) {
                x[2 * i] = __uint_as_float(r[i] << 16);
                x[2 * i + 1] = __uint_as_float(r[i] & 0xFFFF0000u);
            } else {
                typedef __attribute__((ext_vector_type(2))) _Float16 f16x2_t;
                const uint32_t w = r[i];                     // (bit_cast of a vector's element itself takes its first one)
                const f16x2_t h = __builtin_bit_cast(f16x2_t, w);
                x[2 * i] = (float)h[0];
                x[2 * i + 1] = (float)h[1];
            }
        }
    }
    __device__ __forceinline__ void chunk(int c, float (&x)[N]) const { values(raw[c], x); }
    // the elements of chunk c whose bits are set become -infinity
    __device__ __forceinline__ void drop(int c, uint32_t bits)
    {
        constexpr uint32_t NOTHING = TYPE == EE_FP32 ? 0xFF800000u : TYPE == EE_BF16 ? 0xFF80u : 0xFC00u;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t w = raw[c][i];
            if constexpr (TYPE == EE_FP32) {
                w = bits >> i & 1 ? NOTHING : w;
            } else {
                w = bits >> (2 * i) & 1 ? (w & 0xFFFF0000u) | NOTHING : w;
                w = bits >> (2 * i + 1) & 1 ? (w & 0xFFFFu) | NOTHING << 16 : w;
            }
            raw[c][i] = w;
        }
    }
    // Every element becomes less by m, an element of the type itself: exactly where the two are within a factor of two of each other (their difference is a multiple of the smaller
    // one's last place), and elsewhere rounded to the type.
    __device__ __forceinline__ void less(float m)
    {
        again(m);
#pragma unroll
        for (int c = 0; c < E; ++c) {
            float x[N];
            chunk(c, x);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                raw[c][i] = TYPE == EE_FP32 ? __float_as_uint(x[i] - m) : TYPE == EE_BF16 ? pack_bf16(x[N / 4 * i] - m, x[N / 4 * i + N / 4 - 1] - m) : pack_fp16(x[N / 4 * i] - m, x[N / 4 * i + N / 4 - 1] - m);
        }
    }
    // Between two walks over the part, the first of which gave `done` and `too`: the compiler takes the elements as others than before, and does not keep them all as floats
    // in the meantime (twice the registers).
    __device__ __forceinline__ void again(float done, float too = 0.f)
    {
#pragma unroll
        for (int c = 0; c < E; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t w = raw[c][i];
                asm volatile("" : "+v"(w) : "v"(done), "v"(too));
                raw[c][i] = w;
            }
    }
};

// The larger one; NaN where one is (what fmaxf does for NaN costs an instruction more for every value that comes from memory).
__device__ __forceinline__ float larger(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// Exponents z c (c = log2(e) / T) of fp32.  Up to BELOW a thread takes its exponentials relative to its own largest, r = z c rounded: what the rounding leaves is 2^6 at most, which
// an exponential holds.  A thread whose largest is below -BELOW (masked tokens: z of the type's lowest value, z c past fp32) takes them relative to 0, and has nothing.  That is
// wrong only where the whole part's largest is that low, or above FAR: there the sums are taken again, relative to the largest logit m itself, by 2^((z - m) c) (what z - m is
// rounded by, where it is, is nothing beside exponents of that size).
constexpr float BELOW = 0x1p30f, FAR = 0x1p29f;
__device__ __forceinline__ float reference_of(float r) { return r < -BELOW ? 0.f : r; }      // (NaN stays)
__device__ __forceinline__ double wave_max_d(double x)
{
    x = fmax(x, dpp_d<DPP_XOR1>(x));
    x = fmax(x, dpp_d<DPP_XOR2>(x));
    x = fmax(x, dpp_d<DPP_HALF_MIRROR>(x));
    x = fmax(x, dpp_d<DPP_MIRROR>(x));
    unsigned la, lb, ha, hb;
    unsigned long long b = (unsigned long long)__double_as_longlong(x);
    pair16((unsigned)b, la, lb);
    pair16((unsigned)(b >> 32), ha, hb);
    x = fmax(join_d(la, ha), join_d(lb, hb));
    b = (unsigned long long)__double_as_longlong(x);
    pair32((unsigned)b, la, lb);
    pair32((unsigned)(b >> 32), ha, hb);
    return fmax(join_d(la, ha), join_d(lb, hb));
}

// One element of a row.
__device__ __forceinline__ float logit_at(int type, const void *row, size_t i)
{
    return type == EE_FP32   ? as_global(static_cast<const float *>(row))[i]
           : type == EE_BF16 ? (float)as_global(static_cast<const __bf16 *>(row))[i]
                             : (float)as_global(static_cast<const _Float16 *>(row))[i];
}
__device__ __forceinline__ const void *row_at(const void *base, int type, size_t element)
{
    return static_cast<const unsigned char *>(base) + element * (type == EE_FP32 ? 4 : 2);
}

// Parts that the rows of a call are taken in: one for a workgroup that holds the whole row where rows alone fill the chip; where they do not, as many as give it
// `enough` workgroups, of `least` tokens or more.
struct RowSplit {
    int parts, length;       // of a part; a multiple of 8
};
inline RowSplit split_rows(int n_rows, int vocab, int room, int least, int enough)
{
    int parts = (vocab + room - 1) / room;
    const long long wanted = ((long long)enough + n_rows - 1) / std::max(n_rows, 1);
    parts = (int)std::max<long long>(parts, std::min<long long>(wanted, (vocab + least - 1) / least));
    RowSplit s;
    s.length = ((vocab + parts - 1) / parts + 7) / 8 * 8;
    s.parts = (vocab + s.length - 1) / s.length;
    return s;
}

// what lanes of a wave have written to LDS, read by others of it after this (the accesses themselves are in order)
__device__ __forceinline__ void wave_lds_order() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); __builtin_amdgcn_wave_barrier(); }

// Stores of N neighbouring elements at any alignment of the element type, and of one.
template <int N>
__device__ __forceinline__ void store_some(int type, void *base, size_t at, const float (&x)[N])
{
    if (type == EE_FP32) {
        typedef float some_t __attribute__((ext_vector_type(4), aligned(4)));
#pragma unroll
        for (int i = 0; i < N; i += 4) *(EE_GLOBAL some_t *)as_global_mut(static_cast<float *>(base) + at + i) = (some_t){x[i], x[i + 1], x[i + 2], x[i + 3]};
    } else {
        typedef uint32_t some_t __attribute__((ext_vector_type(N / 2), aligned(2)));
        some_t v;
#pragma unroll
        for (int i = 0; i < N / 2; ++i) v[i] = type == EE_BF16 ? pack_bf16(x[2 * i], x[2 * i + 1]) : pack_fp16(x[2 * i], x[2 * i + 1]);
        *(EE_GLOBAL some_t *)as_global_mut(static_cast<uint16_t *>(base) + at) = v;
    }
}
__device__ __forceinline__ void store_one(int type, void *base, size_t at, float x)
{
    if (type == EE_FP32)
        as_global_mut(static_cast<float *>(base))[at] = x;
    else
        as_global_mut(static_cast<uint16_t *>(base))[at] = (uint16_t)(type == EE_BF16 ? pack_bf16(x, x) : pack_fp16(x, x));
}

inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

}  // namespace ee
