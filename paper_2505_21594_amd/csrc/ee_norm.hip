// ee_norm, ee_norm_grad: layer norm (center = 1) and RMS norm (0) of rows, and their gradients.
//
//   x^ = (x - mu) r,  mu = mean x (0 without center),  r = 1 / sqrt(mean (x - mu)^2 + eps),   y = x^ g + b;
//   u = dy g,   dx = r (u - mean u [center] - x^ mean(u x^)),   dg = sum over rows of dy x^,   db = sum over rows of dy.
//
// Bound by the rows' bytes (one MI355X, bf16: 8192 rows of 4096 forward 28.2 us, 4.8 TB/s, backward with all sums 48.7, 4.1 TB/s): a wave, or a workgroup, holds a
// row in registers, so that mean, squares about the mean (no difference of large sums) and result read memory once.  Backward, mean(u x^) is taken with u (x - mu),
// which needs no r: its sum travels with the squares'.  The gradients of gains and biases stay in registers while a workgroup goes over its rows; the workgroups'
// sums are added up in order by a second launch. Statistics and sums are fp32.
#include "ee_vocab.hpp"

namespace ee {

struct NormDev {
    const void *x, *dy;
    const float *gain, *bias;
    void *y;                           // dx in the backward pass
    float *part_gain, *part_bias;      // [workgroups][dim]
    long long x_stride, dy_stride, y_stride;
    int x_type, dy_type, y_type, n_rows, dim, center, groups;
    float eps, inv_dim;
};

// A row's elements as they lie in memory (eight of 16 bits in four words, of fp32 in eight): chunk c of lane l (of `lanes` that hold the row) holds elements
// 8 (c * lanes + l) .. + 7; 0 behind the row's end.  Loading converts nothing, so that nothing waits for it before the values are used.
template <int E, bool WIDE>
struct RawRow {
    u32x4_t w[E][WIDE ? 2 : 1];        // WIDE: fp32 too
};
template <int E, bool WIDE>
__device__ __forceinline__ void load_raw(int type, const void *base, size_t at, int n, int l, int lanes, RawRow<E, WIDE> &x)
{
    const EE_GLOBAL char *const p = (const EE_GLOBAL char *)as_global(static_cast<const char *>(row_at(base, type, at)));
#pragma unroll
    for (int c = 0; c < E; ++c) {
        const int from = (c * lanes + l) * 8, left = n - from;
#pragma unroll
        for (int h = 0; h < (WIDE ? 2 : 1); ++h) x.w[c][h] = (u32x4_t){0, 0, 0, 0};
        if (left >= 8) {
            if (WIDE && type == EE_FP32) {
#pragma unroll
                for (int h = 0; h < (WIDE ? 2 : 1); ++h) x.w[c][h] = *(const EE_GLOBAL u32x4_at4_t *)(p + (size_t)from * 4 + h * 16);
            } else {
                x.w[c][0] = *(const EE_GLOBAL u32x4_at2_t *)(p + (size_t)from * 2);
            }
        } else if (left > 0) {
            if (WIDE && type == EE_FP32) {
                const EE_GLOBAL uint32_t *const q = (const EE_GLOBAL uint32_t *)p + from;
                x.w[c][0][0] = q[0];
                if (left > 1) x.w[c][0][1] = q[1];
                if (left > 2) x.w[c][0][2] = q[2];
                if (left > 3) x.w[c][0][3] = q[3];
                if (left > 4) x.w[c][WIDE][0] = q[4];
                if (left > 5) x.w[c][WIDE][1] = q[5];
                if (left > 6) x.w[c][WIDE][2] = q[6];
            } else {
                const EE_GLOBAL uint16_t *const q = (const EE_GLOBAL uint16_t *)p + from;
                uint32_t a = q[0], b = 0, d = 0, e = 0;
                if (left > 1) a |= (uint32_t)q[1] << 16;
                if (left > 2) b = q[2];
                if (left > 3) b |= (uint32_t)q[3] << 16;
                if (left > 4) d = q[4];
                if (left > 5) d |= (uint32_t)q[5] << 16;
                if (left > 6) e = q[6];
                x.w[c][0] = (u32x4_t){a, b, d, e};
            }
        }
    }
}
template <int E, bool WIDE>
__device__ __forceinline__ void values_of(int type, const RawRow<E, WIDE> &r, float (&x)[E][8])
{
#pragma unroll
    for (int c = 0; c < E; ++c) {
        if (WIDE && type == EE_FP32) {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[c][i] = __uint_as_float(r.w[c][WIDE ? i / 4 : 0][i % 4]);
        } else if (type == EE_BF16) {
            RowPart<EE_BF16, 1, 64>::values(r.w[c][0], x[c]);
        } else {
            RowPart<EE_FP16, 1, 64>::values(r.w[c][0], x[c]);
        }
    }
}
template <int E>
__device__ __forceinline__ void load_row(int type, const void *base, size_t at, int n, int l, int lanes, float (&x)[E][8])
{
    RawRow<E, true> r;
    load_raw<E, true>(type, base, at, n, l, lanes, r);
    values_of<E, true>(type, r, x);
}
template <int E>
__device__ __forceinline__ void store_row(int type, void *base, size_t at, int n, int l, int lanes, const float (&x)[E][8])
{
#pragma unroll
    for (int c = 0; c < E; ++c) {
        const int from = (c * lanes + l) * 8;
        if (from + 8 <= n) {
            store_some<8>(type, base, at + from, x[c]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (from + i < n) store_one(type, base, at + from + i, x[c][i]);
        }
    }
}
template <int E>
__device__ __forceinline__ void load_gain(const float *gain, int n, int l, int lanes, float none, float (&g)[E][8])
{
#pragma unroll
    for (int c = 0; c < E; ++c) {
        const int from = (c * lanes + l) * 8;
        if (gain) {
            load_some<8>(gain + from, n - from, 0.f, g[c]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) g[c][i] = none;
        }
    }
}

__device__ __forceinline__ float wave_sum_f(float x)
{
    x += __int_as_float(dpp<DPP_XOR1>(0, __float_as_int(x)));
    x += __int_as_float(dpp<DPP_XOR2>(0, __float_as_int(x)));
    x += __int_as_float(dpp<DPP_HALF_MIRROR>(0, __float_as_int(x)));
    x += __int_as_float(dpp<DPP_MIRROR>(0, __float_as_int(x)));
    return quads_sum(x);
}
// Sums over the lanes that hold a row, a wave's or the workgroup's, in every one of them.  `turn` alternates between two halves of the exchange, so that one
// barrier is enough.
template <bool ONE, int COUNT>
__device__ __forceinline__ void row_sums(float (&v)[COUNT], float (*swap)[3][16], int &turn)
{
#pragma unroll
    for (int i = 0; i < COUNT; ++i) v[i] = wave_sum_f(v[i]);
    if constexpr (!ONE) {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
        if (lane == 0)
#pragma unroll
            for (int i = 0; i < COUNT; ++i) swap[turn][i][wave] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            // (the waves' sums by 16 lanes of each wave, added up in one order by every one)
            float s = (lane & 15) < waves ? swap[turn][i][lane & 15] : 0.f;
            s += __int_as_float(dpp<DPP_XOR1>(0, __float_as_int(s)));
            s += __int_as_float(dpp<DPP_XOR2>(0, __float_as_int(s)));
            s += __int_as_float(dpp<DPP_HALF_MIRROR>(0, __float_as_int(s)));
            s += __int_as_float(dpp<DPP_MIRROR>(0, __float_as_int(s)));
            v[i] = s;
        }
        turn ^= 1;
    }
}

// Sum / dim to the last place: elements that are all alike have themselves for a mean, and nothing left about it, where their sum is a number of fp32 (of 8 bits, up to 2^16 elements; of fp16's
// 11 up to 2^13).  With 1 / dim alone 1000 elements of 30000 are 0.002 off, times r = 316.
__device__ __forceinline__ float mean_of(float sum, const NormDev &a)
{
    const float m = sum * a.inv_dim;
    return fmaf(fmaf(-m, (float)a.dim, sum), a.inv_dim, m);
}

// ONE: a wave holds a row, a workgroup of 256 threads four of them; otherwise the workgroup, of as many waves as it takes.
template <int E, bool ONE>
__global__ void __launch_bounds__(ONE ? 256 : 512) ee_norm_kernel(NormDev a)
{
    __shared__ float swap[2][3][16];
    const int lanes = ONE ? 64 : blockDim.x, l = ONE ? threadIdx.x & 63 : threadIdx.x, row = ONE ? blockIdx.x * 4 + (threadIdx.x >> 6) : blockIdx.x;
    if (ONE && row >= a.n_rows) return;
    int turn = 0;
    float x[E][8], g[E][8], b[E][8];
    load_row<E>(a.x_type, a.x, (size_t)row * a.x_stride, a.dim, l, lanes, x);
    load_gain<E>(a.gain, a.dim, l, lanes, 1.f, g);
    load_gain<E>(a.bias, a.dim, l, lanes, 0.f, b);
    float mu = 0.f;
    if (a.center) {
        float v[1] = {0.f};
#pragma unroll
        for (int c = 0; c < E; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[0] += x[c][i];
        row_sums<ONE>(v, swap, turn);
        mu = mean_of(v[0], a);
    }
    float v[1] = {0.f};
#pragma unroll
    for (int c = 0; c < E; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x[c][i] = (c * lanes + l) * 8 + i < a.dim ? x[c][i] - mu : 0.f;
            v[0] += x[c][i] * x[c][i];
        }
    row_sums<ONE>(v, swap, turn);
    const float r = 1.f / sqrtf(v[0] * a.inv_dim + a.eps);
#pragma unroll
    for (int c = 0; c < E; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) x[c][i] = x[c][i] * r * g[c][i] + b[c][i];
    store_row<E>(a.y_type, a.y, (size_t)row * a.y_stride, a.dim, l, lanes, x);
}

// The next rows' loads (DEPTH of them) are on their way while a row is worked on: a compute unit has two workgroups, whose sums of gains' and biases' gradients are written once for
// all their rows (more workgroups write more of them).
template <int E, bool ONE, bool WIDE, int DEPTH>
__global__ void __launch_bounds__(ONE ? 256 : 1024, !ONE && E == 1 && !WIDE ? (DEPTH == 1 ? 6 : 5) : 1) ee_norm_grad_kernel(NormDev a)
{
    constexpr int ROWS = ONE ? 4 : 1;
    __shared__ float swap[2][3][16];
    __shared__ float sums[ONE ? 3 * E * 64 * 8 : 1];
    const int lanes = ONE ? 64 : blockDim.x, l = ONE ? threadIdx.x & 63 : threadIdx.x, sub = ONE ? threadIdx.x >> 6 : 0, step = gridDim.x * ROWS;
    int turn = 0;
    float dg[E][8], db[E][8], g[E][8];
    RawRow<E, WIDE> next_x[DEPTH], next_u[DEPTH];
#pragma unroll
    for (int c = 0; c < E; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) dg[c][i] = db[c][i] = 0.f;
    auto request = [&](int row, RawRow<E, WIDE> &x, RawRow<E, WIDE> &u) __attribute__((always_inline)) {
        if (row < a.n_rows) {
            load_raw<E, WIDE>(a.x_type, a.x, (size_t)row * a.x_stride, a.dim, l, lanes, x);
            load_raw<E, WIDE>(a.dy_type, a.dy, (size_t)row * a.dy_stride, a.dim, l, lanes, u);
        }
    };
    int row = blockIdx.x * ROWS + sub;
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) request(row + d * step, next_x[d], next_u[d]);
    load_gain<E>(a.gain, a.dim, l, lanes, 1.f, g);
    for (; row < a.n_rows; row += step) {
        float x[E][8], u[E][8];
        values_of<E, WIDE>(a.x_type, next_x[0], x);
        values_of<E, WIDE>(a.dy_type, next_u[0], u);
        if constexpr (DEPTH == 2) {
            next_x[0] = next_x[1];
            next_u[0] = next_u[1];
        }
        request(row + DEPTH * step, next_x[DEPTH - 1], next_u[DEPTH - 1]);
        float mu = 0.f;
        if (a.center) {
            float v[1] = {0.f};
#pragma unroll
            for (int c = 0; c < E; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) v[0] += x[c][i];
            row_sums<ONE>(v, swap, turn);
            mu = mean_of(v[0], a);
        }
        float v[3] = {0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < E; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                x[c][i] = (c * lanes + l) * 8 + i < a.dim ? x[c][i] - mu : 0.f;
                const float t = u[c][i] * g[c][i];
                v[0] += x[c][i] * x[c][i];
                v[1] += t;
                v[2] += t * x[c][i];
            }
        row_sums<ONE>(v, swap, turn);
        const float r = 1.f / sqrtf(v[0] * a.inv_dim + a.eps), mean = a.center ? v[1] * a.inv_dim : 0.f, along = v[2] * a.inv_dim * r;
#pragma unroll
        for (int c = 0; c < E; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float unit = x[c][i] * r, dy = u[c][i];
                dg[c][i] += dy * unit;
                db[c][i] += dy;
                x[c][i] = r * (dy * g[c][i] - mean - unit * along);
            }
        if (a.y) store_row<E>(a.y_type, a.y, (size_t)row * a.y_stride, a.dim, l, lanes, x);
    }
    auto combine = [&](float (&v)[E][8], float *out) {
        if constexpr (ONE) {
            __syncthreads();
            if (sub > 0)
#pragma unroll
                for (int c = 0; c < E; ++c)
#pragma unroll
                    for (int i = 0; i < 8; ++i) sums[(((sub - 1) * E + c) * 8 + i) * 64 + l] = v[c][i];
            __syncthreads();
            if (sub > 0) return;
#pragma unroll
            for (int c = 0; c < E; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    for (int w = 0; w < 3; ++w) v[c][i] += sums[((w * E + c) * 8 + i) * 64 + l];
        }
        store_row<E>(EE_FP32, out, (size_t)blockIdx.x * a.dim, a.dim, l, lanes, v);
    };
    if (a.part_gain) combine(dg, a.part_gain);
    if (a.part_bias) combine(db, a.part_bias);
}

constexpr int CS_COLS = 32, CS_ROWS = 16;
__global__ void __launch_bounds__(CS_COLS *CS_ROWS) ee_column_sums_kernel(const float *part, int parts, int n, float *out, const float *part2, float *out2)
{
    __shared__ float sums[CS_ROWS][CS_COLS];
    const int col = threadIdx.x % CS_COLS, r = threadIdx.x / CS_COLS, c = blockIdx.x * CS_COLS + col;
    if (blockIdx.y == 1) {
        part = part2;
        out = out2;
    }
    const int per = (parts + CS_ROWS - 1) / CS_ROWS, to = min((r + 1) * per, parts);
    float s = 0.f;
    if (c < n) {
#pragma unroll 8
        for (int p = r * per; p < to; ++p) s += as_global(part)[(size_t)p * n + c];
    }
    sums[r][col] = s;
    __syncthreads();
    if (r == 0 && c < n) {
        for (int i = 1; i < CS_ROWS; ++i) s += sums[i][col];
        as_global_mut(out)[c] = s;
    }
}
void launch_column_sums(const float *part, int parts, int n, float *out, const float *part2, float *out2, hipStream_t stream)
{
    if (!out) {
        out = out2;
        part = part2;
        out2 = nullptr;
    }
    if (out) hipLaunchKernelGGL(ee_column_sums_kernel, dim3((unsigned)((n + CS_COLS - 1) / CS_COLS), out2 ? 2 : 1), dim3(CS_COLS * CS_ROWS), 0, stream, part, parts, n, out, part2, out2);
}

typedef void (*norm_kernel_t)(NormDev);
struct NormShape {
    int chunks, threads;
    bool one;
    int rows() const { return one ? 4 : 1; }
};
// Forward, four waves for a row as long as four chunks a lane are enough: more of it on its way for every wave (8191 rows of 5120, bf16: ten waves of one chunk 45.1 us, four of three 41.8; 8192 of 4096: eight of one 29.1, four of two 28.2).
static NormShape norm_shape(int dim)
{
    const int pieces = (dim + 7) / 8;
    if (pieces <= 128) return {(pieces + 63) / 64, 256, true};
    const int threads = pieces <= 1024 ? 256 : 512;
    return {(pieces + threads - 1) / threads, threads, false};
}
// Backward, a chunk a lane, whose registers hold its part of the gains' and biases' gradients too; waves in fours, and few enough registers, so that a compute unit's SIMDs have room
// for a second workgroup (8191 rows of 5120: ten waves of 92 registers 83 us, twelve of 80 67.5, 12 bytes of them spilled; 8192 of 4096 by eight 48.7).  Two chunks a lane, with 52 bytes of
// spill (fp32 164): 2000 rows of 16384 90 us, fp32 173; with the gains loaded again for every row (40 and 176 bytes) 91 and 183.
static NormShape norm_grad_shape(int dim)
{
    const int pieces = (dim + 7) / 8;
    if (pieces <= 128) return {(pieces + 63) / 64, 256, true};
    const int chunks = pieces <= 1024 ? 1 : 2;
    return {chunks, ((pieces + chunks - 1) / chunks + 255) / 256 * 256, false};
}
static norm_kernel_t norm_kernel(const NormShape &s)
{
    if (s.one) return s.chunks == 1 ? ee_norm_kernel<1, true> : ee_norm_kernel<2, true>;
    return s.chunks == 1 ? ee_norm_kernel<1, false> : s.chunks == 2 ? ee_norm_kernel<2, false> : s.chunks == 3 ? ee_norm_kernel<3, false> : ee_norm_kernel<4, false>;
}
template <bool WIDE>
static norm_kernel_t norm_grad_kernel(const NormShape &s)
{
    if (s.one) return s.chunks == 1 ? ee_norm_grad_kernel<1, true, WIDE, 2> : ee_norm_grad_kernel<2, true, WIDE, 2>;
    return s.chunks == 1 ? (s.threads <= 512 ? ee_norm_grad_kernel<1, false, WIDE, 2> : ee_norm_grad_kernel<1, false, WIDE, 1>) : ee_norm_grad_kernel<2, false, WIDE, 1>;
}
// Workgroups of the backward pass: four rows for each at least where there are as many (each one's sums are written and read again), two for a compute unit at most.
static int norm_groups(int n_rows, const NormShape &s)
{
    const int n = (n_rows + s.rows() - 1) / s.rows();
    return std::min(std::max((n + 3) / 4, std::min(n, 128)), 512);
}

static int check_rows(const char *call, int device, int n_rows, int dim, int center, float eps)
{
    if (device < 0) return fail(EE_EINVAL, "%s: device %d", call, device);
    if (n_rows < 0 || n_rows > EE_NORM_MAX_ROWS) return fail(EE_EINVAL, "%s: n_rows %d not in [0,2^21]", call, n_rows);
    if (dim < 1 || dim > EE_NORM_MAX_DIM) return fail(EE_EINVAL, "%s: dim %d not in [1,%d]", call, dim, EE_NORM_MAX_DIM);
    if (center != 0 && center != 1) return fail(EE_EINVAL, "%s: center must be 0 or 1", call);
    if (!(eps >= 0.f) || !isfinite(eps)) return fail(EE_EINVAL, "%s: eps must be finite and not negative", call);
    return EE_OK;
}
static int check_array(const char *call, const char *what, const void *p, int type, int64_t stride, int n_rows, int dim)
{
    if (type < EE_BF16 || type > EE_FP32) return fail(EE_EINVAL, "%s: unknown element type %d", call, type);
    if (!p) return EE_OK;
    if (!aligned(p, size_of_type(type))) return fail(EE_EINVAL, "%s: %s is not aligned to its type", call, what);
    if (n_rows > 1 && (stride < dim || stride >= (int64_t)1 << 40)) return fail(EE_EINVAL, "%s: the row stride of %s is smaller than dim", call, what);
    return EE_OK;
}

}  // namespace ee

using namespace ee;

extern "C" int ee_norm(const ee_norm_args *p, void *stream)
{
    static const char *const call = "ee_norm";
    if (!p) return fail(EE_EINVAL, "%s: null argument", call);
    int rc = check_rows(call, p->device, p->n_rows, p->dim, p->center, p->eps);
    if (rc == EE_OK) rc = check_array(call, "x", p->x, p->dtype, p->x_stride, p->n_rows, p->dim);
    if (rc == EE_OK) rc = check_array(call, "y", p->y, p->out_dtype, p->y_stride, p->n_rows, p->dim);
    if (rc != EE_OK) return rc;
    if (p->n_rows == 0) return EE_OK;
    if (!p->x || !p->y) return fail(EE_EINVAL, "%s: null x or y", call);
    if (p->x == p->y && (p->dtype != p->out_dtype || (p->n_rows > 1 && p->x_stride != p->y_stride))) return fail(EE_EINVAL, "%s: y may be x only with the same type and stride", call);
    if (!aligned(p->gain, 4) || !aligned(p->bias, 4)) return fail(EE_EINVAL, "%s: fp32 arrays must be 4-byte aligned", call);
    NormDev a = {};
    a.x = p->x;
    a.gain = p->gain;
    a.bias = p->bias;
    a.y = p->y;
    a.x_stride = p->n_rows > 1 ? p->x_stride : 0;
    a.y_stride = p->n_rows > 1 ? p->y_stride : 0;
    a.x_type = p->dtype;
    a.y_type = p->out_dtype;
    a.n_rows = p->n_rows;
    a.dim = p->dim;
    a.center = p->center;
    a.eps = p->eps;
    a.inv_dim = 1.f / (float)p->dim;
    DeviceScope scope(p->device);
    HIP_TRY(scope.status);
    const NormShape s = norm_shape(p->dim);
    hipLaunchKernelGGL(norm_kernel(s), dim3((unsigned)((p->n_rows + s.rows() - 1) / s.rows())), dim3(s.threads), 0, static_cast<hipStream_t>(stream), a);
    HIP_TRY(hipGetLastError());
    return EE_OK;
}

static int check_norm_grad(const char *call, const ee_norm_grad_args *p)
{
    if (!p) return fail(EE_EINVAL, "%s: null argument", call);
    return check_rows(call, p->device, p->n_rows, p->dim, p->center, p->eps);
}
static size_t norm_grad_bytes(const ee_norm_grad_args *p) { return 2 * align256((size_t)norm_groups(p->n_rows, norm_grad_shape(p->dim)) * p->dim * sizeof(float)); }

extern "C" int ee_norm_grad_workspace(const ee_norm_grad_args *p, size_t *bytes)
{
    static const char *const call = "ee_norm_grad_workspace";
    if (!bytes) return fail(EE_EINVAL, "%s: null argument", call);
    *bytes = 0;
    int rc = check_norm_grad(call, p);
    if (rc == EE_OK) *bytes = norm_grad_bytes(p);
    return rc;
}

extern "C" int ee_norm_grad(const ee_norm_grad_args *p, void *workspace, size_t workspace_bytes, void *stream)
{
    static const char *const call = "ee_norm_grad";
    int rc = check_norm_grad(call, p);
    if (rc == EE_OK) rc = check_array(call, "x", p->x, p->dtype, p->x_stride, p->n_rows, p->dim);
    if (rc == EE_OK) rc = check_array(call, "dy", p->dy, p->dy_dtype, p->dy_stride, p->n_rows, p->dim);
    if (rc == EE_OK) rc = check_array(call, "dx", p->dx, p->dx_dtype, p->dx_stride, p->n_rows, p->dim);
    if (rc != EE_OK) return rc;
    if (!p->dx && !p->d_gain && !p->d_bias) return EE_OK;
    if (p->n_rows && (!p->x || !p->dy)) return fail(EE_EINVAL, "%s: null x or dy", call);
    if (p->dx && ((p->dx == p->x && (p->dtype != p->dx_dtype || (p->n_rows > 1 && p->x_stride != p->dx_stride))) ||
                  (p->dx == p->dy && (p->dy_dtype != p->dx_dtype || (p->n_rows > 1 && p->dy_stride != p->dx_stride)))))
        return fail(EE_EINVAL, "%s: dx may be x or dy only with the same type and stride", call);
    for (const void *x : {(const void *)p->gain, (const void *)p->d_gain, (const void *)p->d_bias})
        if (!aligned(x, 4)) return fail(EE_EINVAL, "%s: fp32 arrays must be 4-byte aligned", call);
    const size_t need = norm_grad_bytes(p);
    if (p->d_gain || p->d_bias)
        if (need > workspace_bytes || (need && (!workspace || !aligned(workspace, 256))))
            return fail(EE_EINVAL, "%s: the workspace has %zu bytes of %zu, or is not 256-byte aligned", call, workspace_bytes, need);
    const NormShape s = norm_grad_shape(p->dim);
    NormDev a = {};
    a.x = p->x;
    a.dy = p->dy;
    a.gain = p->gain;
    a.y = p->dx;
    a.part_gain = p->d_gain ? static_cast<float *>(workspace) : nullptr;
    a.part_bias = p->d_bias ? reinterpret_cast<float *>(static_cast<unsigned char *>(workspace) + need / 2) : nullptr;
    a.x_stride = p->n_rows > 1 ? p->x_stride : 0;
    a.dy_stride = p->n_rows > 1 ? p->dy_stride : 0;
    a.y_stride = p->n_rows > 1 ? p->dx_stride : 0;
    a.x_type = p->dtype;
    a.dy_type = p->dy_dtype;
    a.y_type = p->dx_dtype;
    a.n_rows = p->n_rows;
    a.dim = p->dim;
    a.center = p->center;
    a.eps = p->eps;
    a.inv_dim = 1.f / (float)p->dim;
    const int groups = norm_groups(p->n_rows, s);
    DeviceScope scope(p->device);
    HIP_TRY(scope.status);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (groups) hipLaunchKernelGGL(p->dtype == EE_FP32 || p->dy_dtype == EE_FP32 ? norm_grad_kernel<true>(s) : norm_grad_kernel<false>(s), dim3((unsigned)groups), dim3(s.threads), 0, st, a);
    HIP_TRY(hipGetLastError());
    launch_column_sums(a.part_gain, groups, p->dim, p->d_gain, a.part_bias, p->d_bias, st);
    HIP_TRY(hipGetLastError());
    return EE_OK;
}
