// What the operators on device memory (ee_kv_append, ee_attend, ee_accept_drafts) share: the sequences of a batch as the
// kernels read them, element types, and the host's checks.
#pragma once

#include <math.h>

#include <algorithm>

#include "ee_host.hpp"
#include "ee_kernels.hpp"

namespace ee {

constexpr int OPS_MAX_GRID_Y = 65535;

// A cache and the new rows of its sequences, as a caller of the operators holds them.  Everything that is read from
// device memory is clamped to what the host knows, so that no value of it leads outside an array.
struct BatchDev {
    uint16_t *kpool, *vpool;
    const int *table, *row_start, *kv_len;
    int n_pages, n_seqs, n_rows, table_stride, n_kv_heads;

    // first row of sequence s (s <= n_seqs)
    __device__ __forceinline__ int start(int s) const { return min(max(as_global(row_start)[s], 0), n_rows); }
    // positions of sequence s that the cache has room for
    __device__ __forceinline__ int length(int s) const { return max(as_global(kv_len)[s], 0); }
    __device__ __forceinline__ int capacity() const { return min(table_stride, 0x7FFFFFF0 / KV_PAGE) * KV_PAGE; }
};

// Exchanges between lanes in the vector unit: a shuffle through LDS takes about 100 cycles, these 4 to 8.
template <int CTRL, int ROWS = 0xF>
__device__ __forceinline__ int dpp(int other, int x) { return __builtin_amdgcn_update_dpp(other, x, CTRL, ROWS, 0xF, false); }
constexpr int DPP_XOR1 = 0xB1, DPP_XOR2 = 0x4E, DPP_HALF_MIRROR = 0x141, DPP_MIRROR = 0x140, DPP_SHR = 0x110, DPP_BCAST15 = 0x142, DPP_BCAST31 = 0x143;

// the values of lanes l and l ^ 16, l and l ^ 32, in some order
__device__ __forceinline__ void pair16(unsigned x, unsigned &a, unsigned &b)
{
    const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    a = r[0];
    b = r[1];
}
__device__ __forceinline__ void pair32(unsigned x, unsigned &a, unsigned &b)
{
    const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    a = r[0];
    b = r[1];
}
// largest and sum over the lanes l, l ^ 16, l ^ 32, l ^ 48
__device__ __forceinline__ float quads_max(float x)
{
    unsigned a, b;
    pair16(__float_as_uint(x), a, b);
    x = fmaxf(__uint_as_float(a), __uint_as_float(b));
    pair32(__float_as_uint(x), a, b);
    return fmaxf(__uint_as_float(a), __uint_as_float(b));
}
__device__ __forceinline__ float quads_sum(float x)
{
    unsigned a, b;
    pair16(__float_as_uint(x), a, b);
    x = __uint_as_float(a) + __uint_as_float(b);
    pair32(__float_as_uint(x), a, b);
    return __uint_as_float(a) + __uint_as_float(b);
}
__device__ __forceinline__ unsigned quads_or(unsigned x)
{
    unsigned a, b;
    pair16(x, a, b);
    pair32(a | b, a, b);
    return a | b;
}

// inclusive sum over the lanes of a wave
__device__ __forceinline__ int wave_scan(int x)
{
    x += dpp<DPP_SHR + 1>(0, x);
    x += dpp<DPP_SHR + 2>(0, x);
    x += dpp<DPP_SHR + 4>(0, x);
    x += dpp<DPP_SHR + 8>(0, x);
    x += dpp<DPP_BCAST15, 0xA>(0, x);
    x += dpp<DPP_BCAST31, 0xC>(0, x);
    return x;
}

// smallest over a wave, in every lane
__device__ __forceinline__ int wave_min(int x)
{
    x = min(x, dpp<DPP_XOR1>(x, x));
    x = min(x, dpp<DPP_XOR2>(x, x));
    x = min(x, dpp<DPP_HALF_MIRROR>(x, x));
    x = min(x, dpp<DPP_MIRROR>(x, x));
    unsigned a, b;
    pair16((unsigned)x, a, b);
    pair32((unsigned)min((int)a, (int)b), a, b);
    return min((int)a, (int)b);
}

// Which of n things item `item` belongs to when thing i has count(i) items, and its place there; false past the last.  All
// lanes of a wave call it and get the same answer; 64 things a round.  Where there is no such item, *all is the number of items.
template <typename F>
__device__ __forceinline__ bool find_item(int n, int item, int lane, F count, int &index, int &place, int *all = nullptr)
{
    int before = 0;
    for (int base = 0; base < n; base += 64) {
        const int c = base + lane < n ? count(base + lane) : 0;
        const int incl = wave_scan(c), total = __builtin_amdgcn_readlane(incl, 63);
        if (item < total) {
            const int l = __builtin_ctzll(__ballot(incl > item));
            index = base + l;
            place = item - __builtin_amdgcn_readlane(incl - c, l);
            return true;
        }
        item -= total;
        before += total;
    }
    if (all) *all = before;
    return false;
}

// A kilobyte into LDS whose sixteen-byte pieces come from an address of each lane's: to LDS byte dst + 16 l.  As load_lds_kb, the caller waits.
__device__ __forceinline__ void load_lds_lanes(const void *src, unsigned dst)
{
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(src), "s"(dst) : "m0", "memory");
}

// eight neighbouring elements as floats; 16-byte aligned
template <int TYPE>
__device__ __forceinline__ void load8(const void *base, size_t at, float (&x)[8])
{
    if constexpr (TYPE == EE_FP32) {
        const f32x4_t *p = reinterpret_cast<const f32x4_t *>(static_cast<const float *>(base) + at);
        const f32x4_t a = as_global(p)[0], b = as_global(p)[1];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = a[i];
            x[4 + i] = b[i];
        }
    } else {
        const uint4 v = load_global16(static_cast<const uint16_t *>(base) + at);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (TYPE == EE_BF16) {
                x[2 * i] = __uint_as_float(w[i] << 16);
                x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
            } else {
                typedef __attribute__((ext_vector_type(2))) _Float16 f16x2_t;
                const f16x2_t h = __builtin_bit_cast(f16x2_t, w[i]);
                x[2 * i] = (float)h[0];
                x[2 * i + 1] = (float)h[1];
            }
        }
    }
}

__device__ __forceinline__ uint32_t pack_fp16(float a, float b)
{
    return (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)a) | (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)b) << 16;
}

// four neighbouring elements of the type, rounded once
__device__ __forceinline__ void store4(int type, void *base, size_t at, float a, float b, float c, float d)
{
    if (type == EE_FP32) {
        *as_global_mut(reinterpret_cast<f32x4_t *>(static_cast<float *>(base) + at)) = (f32x4_t){a, b, c, d};
    } else {
        const u32x2_t v = type == EE_BF16 ? (u32x2_t){pack_bf16(a, b), pack_bf16(c, d)} : (u32x2_t){pack_fp16(a, b), pack_fp16(c, d)};
        *as_global_mut(reinterpret_cast<u32x2_t *>(static_cast<uint16_t *>(base) + at)) = v;
    }
}

// eight neighbouring elements of the type, rounded once; 16-byte aligned
__device__ __forceinline__ void store8(int type, void *base, size_t at, const float (&x)[8])
{
    if (type == EE_FP32) {
        store4(type, base, at, x[0], x[1], x[2], x[3]);
        store4(type, base, at + 4, x[4], x[5], x[6], x[7]);
    } else {
        u32x4_t v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = type == EE_BF16 ? pack_bf16(x[2 * e], x[2 * e + 1]) : pack_fp16(x[2 * e], x[2 * e + 1]);
        *as_global_mut(reinterpret_cast<u32x4_t *>(static_cast<uint16_t *>(base) + at)) = v;
    }
}

// ------------------------------------------------------------------ host

inline size_t size_of_type(int type) { return type == EE_FP32 ? 4 : 2; }
inline bool aligned(const void *p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
// a stride of n rows or heads: its multiples keep 16-byte alignment (of one row or head it says nothing)
inline bool stride_ok(int64_t stride, int type, int n) { return n <= 1 || (stride >= 0 && stride < (int64_t)1 << 40 && stride * (int64_t)size_of_type(type) % 16 == 0); }

// The GPU that a call works on is current inside it, the caller's again after it.
struct DeviceScope {
    int before = -1;
    hipError_t status;
    explicit DeviceScope(int device)
    {
        status = hipGetDevice(&before);
        if (status == hipSuccess && before != device)
            status = hipSetDevice(device);
        else
            before = -1;
    }
    ~DeviceScope()
    {
        if (before >= 0) hipSetDevice(before);
    }
};

// What ee_kv_append and ee_attend demand of a cache and of the batch's rows.
int check_cache(const char *call, const ee_paged_cache *c, int n_rows, int n_heads, const void *row_start, const void *kv_len);
BatchDev batch_of(const ee_paged_cache &c, int n_rows, const int32_t *row_start, const int32_t *kv_len);

}  // namespace ee
