#include "ee_linear.hpp"

namespace ee {

// Eight neighbouring elements of row r at column c of an array of R rows and C columns; 0 outside it.  Rows start at multiples of 16 bytes.
__device__ __forceinline__ u32x4_t load_piece(const uint16_t *p, long long ld, int R, int C, int r, int c)
{
    u32x4_t v = {0, 0, 0, 0};
    if (r >= R || c >= C) return v;
    const uint16_t *q = p + (size_t)r * ld + c;
    if (c + 8 <= C) return *as_global(reinterpret_cast<const u32x4_t *>(q));
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (c + i < C) v[i / 2] |= (uint32_t)as_global(q)[i] << (i % 2 * 16);
    return v;
}

constexpr int GT = 128, GK = 32, GLD = GK + 8;     // tile of 128 x 128, 32 of the sum at a time

template <bool ALONG>
__device__ __forceinline__ void stage(const uint16_t *p, long long ld, int rows, int K, int r0, int k0, uint16_t (*to)[GLD], int tid)
{
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int piece = tid + h * 256;
        if (ALONG) {
            const int r = piece / 4, k = piece % 4 * 8;
            *reinterpret_cast<u32x4_t *>(&to[r][k]) = load_piece(p, ld, rows, K, r0 + r, k0 + k);
        } else {
            const int k = piece / 16, r = piece % 16 * 8;
            const u32x4_t v = load_piece(p, ld, K, rows, k0 + k, r0 + r);
#pragma unroll
            for (int i = 0; i < 8; ++i) to[r + i][k] = (uint16_t)(v[i / 2] >> (i % 2 * 16));
        }
    }
}

template <int TYPE, bool A_ALONG, bool B_ALONG>
__global__ void __launch_bounds__(256) ee_gemm16_kernel(GemmDev g)
{
    __shared__ __attribute__((aligned(16))) uint16_t as[GT][GLD], bs[GT][GLD];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, i0 = blockIdx.y * GT, j0 = blockIdx.x * GT;
    const int wi = (wave & 1) * 64, wj = (wave >> 1) * 64, r = lane & 15, quad = lane >> 4;
    f32x4_t acc[4][4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[j][i] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
    for (int t = 0; t < g.terms; ++t)
        for (int k = 0; k < g.K; k += GK) {
            __syncthreads();
            stage<A_ALONG>(g.A + t * g.plane, g.lda, g.I, g.K, i0, k, as, tid);
            stage<B_ALONG>(g.B, g.ldb, g.J, g.K, j0, k, bs, tid);
            __syncthreads();
            u32x4_t a[4], b[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                a[x] = *reinterpret_cast<const u32x4_t *>(&as[wi + x * 16 + r][quad * 8]);
                b[x] = *reinterpret_cast<const u32x4_t *>(&bs[wj + x * 16 + r][quad * 8]);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[j][i] = mfma16<TYPE>(b[j], a[i], acc[j][i]);
        }
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) finish4(g, i0 + wi + i * 16 + r, j0 + wj + j * 16 + quad * 4, acc[j][i]);
}

// dz = dy act'(z) as 16-bit terms, and sums of its columns over a part of the rows: a thread has eight columns.
struct SlopeDev {
    const uint16_t *dy, *pre;
    long long dy_stride, pre_stride, ldz, plane;
    uint16_t *dz;                      // [terms][rows][ldz], or null
    float *part;                       // [parts][n], or null
    int type, act, terms, rows, n, per;   // per: rows of a part
};
constexpr int SL_COLS = 32, SL_SUBS = 8;    // 256 columns of a workgroup, eight rows at a time
__global__ void __launch_bounds__(SL_COLS *SL_SUBS) ee_slope_kernel(SlopeDev a)
{
    __shared__ float sums[SL_SUBS][SL_COLS * 8];
    const int c = threadIdx.x % SL_COLS, sub = threadIdx.x / SL_COLS, col = (blockIdx.x * SL_COLS + c) * 8;
    const int from = blockIdx.y * a.per, to = min(from + a.per, a.rows);
    float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (col < a.n)
        for (int row = from + sub; row < to; row += SL_SUBS) {
            const u32x4_t v = load_piece(a.dy, a.dy_stride, a.rows, a.n, row, col);
            u32x4_t z = {0, 0, 0, 0};
            if (a.act != EE_ACT_NONE) z = load_piece(a.pre, a.pre_stride, a.rows, a.n, row, col);
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint16_t vb = (uint16_t)(v[i / 2] >> (i % 2 * 16)), zb = (uint16_t)(z[i / 2] >> (i % 2 * 16));
                x[i] = a.type == EE_BF16 ? bf16_to_f32(vb) : (float)__builtin_bit_cast(_Float16, vb);
                if (a.act != EE_ACT_NONE) x[i] *= act_slope(a.act, a.type == EE_BF16 ? bf16_to_f32(zb) : (float)__builtin_bit_cast(_Float16, zb));
                s[i] += x[i];
            }
            for (int t = 0; t < a.terms; ++t) {
                u32x4_t w;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    w[i] = a.type == EE_BF16 ? pack_bf16(x[2 * i], x[2 * i + 1]) : pack_fp16(x[2 * i], x[2 * i + 1]);
                    if (a.type == EE_BF16) {
                        x[2 * i] -= __uint_as_float(w[i] << 16);
                        x[2 * i + 1] -= __uint_as_float(w[i] & 0xFFFF0000u);
                    } else {
                        x[2 * i] -= (float)__builtin_bit_cast(_Float16, (uint16_t)w[i]);
                        x[2 * i + 1] -= (float)__builtin_bit_cast(_Float16, (uint16_t)(w[i] >> 16));
                    }
                }
                *as_global_mut(reinterpret_cast<u32x4_t *>(a.dz + t * a.plane + (size_t)row * a.ldz + col)) = w;
            }
        }
    if (!a.part) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) sums[sub][c * 8 + i] = s[i];
    __syncthreads();
    const int mine = blockIdx.x * SL_COLS * 8 + threadIdx.x;
    if (mine < a.n) {
        float all = 0.f;
#pragma unroll
        for (int i = 0; i < SL_SUBS; ++i) all += sums[i][threadIdx.x];
        as_global_mut(a.part)[(size_t)blockIdx.y * a.n + mine] = all;
    }
}

typedef void (*gemm16_kernel_t)(GemmDev);
static int launch_gemm16(const GemmDev &g, bool a_along, bool b_along, hipStream_t s)
{
    const gemm16_kernel_t k = g.type == EE_BF16 ? (a_along ? (b_along ? ee_gemm16_kernel<EE_BF16, true, true> : ee_gemm16_kernel<EE_BF16, true, false>) : ee_gemm16_kernel<EE_BF16, false, false>)
                                                : (a_along ? (b_along ? ee_gemm16_kernel<EE_FP16, true, true> : ee_gemm16_kernel<EE_FP16, true, false>) : ee_gemm16_kernel<EE_FP16, false, false>);
    hipLaunchKernelGGL(k, dim3((unsigned)((g.J + GT - 1) / GT), (unsigned)((g.I + GT - 1) / GT)), dim3(256), 0, s, g);
    HIP_TRY(hipGetLastError());
    return EE_OK;
}

static int check_sizes(const char *call, int device, int dtype, int act, int n_rows, int n_in, int n_out)
{
    if (device < 0) return fail(EE_EINVAL, "%s: device %d", call, device);
    if (dtype != EE_BF16 && dtype != EE_FP16) return fail(EE_EINVAL, "%s: operands must be bf16 or fp16 (type %d)", call, dtype);
    if (act < EE_ACT_NONE || act > EE_ACT_GELU) return fail(EE_EINVAL, "%s: unknown activation %d", call, act);
    if (n_rows < 0 || n_rows > EE_LINEAR_MAX) return fail(EE_EINVAL, "%s: n_rows %d not in [0,2^22]", call, n_rows);
    if (n_in < 1 || n_in > EE_LINEAR_MAX || n_out < 1 || n_out > EE_LINEAR_MAX) return fail(EE_EINVAL, "%s: n_in %d or n_out %d not in [1,2^22]", call, n_in, n_out);
    return EE_OK;
}
// rows of an array: 16-byte aligned, `width` elements at least from one to the next
static int check_matrix(const char *call, const char *what, const void *p, int type, int64_t stride, int n_rows, int width)
{
    if (!p) return EE_OK;
    if (type < EE_BF16 || type > EE_FP32) return fail(EE_EINVAL, "%s: unknown element type %d of %s", call, type, what);
    if (!aligned(p, 16)) return fail(EE_EINVAL, "%s: %s must be 16-byte aligned", call, what);
    if (!stride_ok(stride, type, n_rows)) return fail(EE_EINVAL, "%s: the row stride of %s keeps no 16-byte alignment", call, what);
    if (n_rows > 1 && stride < width) return fail(EE_EINVAL, "%s: the row stride of %s is smaller than its row", call, what);
    return EE_OK;
}

static int check_linear(const char *call, const ee_linear_args *p)
{
    if (!p) return fail(EE_EINVAL, "%s: null argument", call);
    return check_sizes(call, p->device, p->dtype, p->act, p->n_rows, p->n_in, p->n_out);
}

struct GradPlan {
    int terms_dx, terms_dw, terms;     // of dz, where it is formed
    int parts, per;                    // of the rows, for the bias's gradient and dz
    long long ldz;
    size_t dz_bytes, part_bytes;
    size_t bytes() const { return dz_bytes + part_bytes; }
};
static GradPlan plan_grad(const ee_linear_grad_args &p)
{
    GradPlan pl = {};
    // dz in one term for 16-bit results; for fp32 ones exactly enough: three terms of bf16 (2^-24), two of fp16 (2^-22)
    const int exact = p.dtype == EE_BF16 ? 3 : 2;
    pl.terms_dx = p.act != EE_ACT_NONE && p.dx_dtype == EE_FP32 ? exact : 1;
    pl.terms_dw = p.act != EE_ACT_NONE && p.dw_dtype == EE_FP32 ? exact : 1;
    pl.terms = p.act == EE_ACT_NONE ? 0 : std::max(pl.terms_dx, pl.terms_dw);
    pl.ldz = ((long long)p.n_out + 7) / 8 * 8;
    const int columns = (p.n_out + SL_COLS * 8 - 1) / (SL_COLS * 8);
    pl.per = std::max(SL_SUBS, (int)(((long long)p.n_rows * columns + 1023) / 1024 + SL_SUBS - 1) / SL_SUBS * SL_SUBS);
    pl.parts = (p.n_rows + pl.per - 1) / pl.per;
    pl.dz_bytes = align256((size_t)pl.terms * p.n_rows * pl.ldz * 2);
    pl.part_bytes = align256((size_t)pl.parts * p.n_out * sizeof(float));
    return pl;
}
static int check_linear_grad(const char *call, const ee_linear_grad_args *p)
{
    if (!p) return fail(EE_EINVAL, "%s: null argument", call);
    if (p->dx_dtype < EE_BF16 || p->dx_dtype > EE_FP32 || p->dw_dtype < EE_BF16 || p->dw_dtype > EE_FP32)
        return fail(EE_EINVAL, "%s: unknown element type %d or %d", call, p->dx_dtype, p->dw_dtype);
    return check_sizes(call, p->device, p->dtype, p->act, p->n_rows, p->n_in, p->n_out);
}

}  // namespace ee

using namespace ee;

extern "C" int ee_linear_workspace(const ee_linear_args *p, size_t *bytes)
{
    static const char *const call = "ee_linear_workspace";
    if (!bytes) return fail(EE_EINVAL, "%s: null argument", call);
    *bytes = 0;
    return check_linear(call, p);
}

extern "C" int ee_linear(const ee_linear_args *p, void *workspace, size_t workspace_bytes, void *stream)
{
    static const char *const call = "ee_linear";
    int rc = check_linear(call, p);
    if (rc == EE_OK) rc = check_matrix(call, "x", p->x, p->dtype, p->x_stride, p->n_rows, p->n_in);
    if (rc == EE_OK) rc = check_matrix(call, "weight", p->weight, p->dtype, p->weight_stride, p->n_out, p->n_in);
    if (rc == EE_OK) rc = check_matrix(call, "y", p->y, p->out_dtype, p->y_stride, p->n_rows, p->n_out);
    if (rc == EE_OK) rc = check_matrix(call, "residual", p->residual, p->residual_dtype, p->residual_stride, p->n_rows, p->n_out);
    if (rc == EE_OK) rc = check_matrix(call, "pre", p->pre, p->dtype, p->pre_stride, p->n_rows, p->n_out);
    if (rc != EE_OK) return rc;
    if (p->n_rows == 0) return EE_OK;
    if (!p->x || !p->weight || !p->y) return fail(EE_EINVAL, "%s: null x, weight or y", call);
    if (p->y == p->x || p->y == p->weight || p->pre == p->x || p->pre == p->y) return fail(EE_EINVAL, "%s: y and pre must be arrays of their own", call);
    if (p->residual == p->y && (p->residual_dtype != p->out_dtype || (p->n_rows > 1 && p->residual_stride != p->y_stride)))
        return fail(EE_EINVAL, "%s: y may be residual only with the same type and stride", call);
    if (!aligned(p->bias, 4)) return fail(EE_EINVAL, "%s: fp32 arrays must be 4-byte aligned", call);
    GemmDev g = {};
    g.A = static_cast<const uint16_t *>(p->x);
    g.B = static_cast<const uint16_t *>(p->weight);
    g.lda = p->n_rows > 1 ? p->x_stride : 0;
    g.ldb = p->n_out > 1 ? p->weight_stride : 0;
    g.terms = 1;
    g.I = p->n_rows;
    g.J = p->n_out;
    g.K = p->n_in;
    g.bias = p->bias;
    g.residual = p->residual;
    g.y = p->y;
    g.pre = p->pre;
    g.res_stride = p->n_rows > 1 ? p->residual_stride : 0;
    g.y_stride = p->n_rows > 1 ? p->y_stride : 0;
    g.pre_stride = p->n_rows > 1 ? p->pre_stride : 0;
    g.res_type = p->residual_dtype;
    g.y_type = p->out_dtype;
    g.type = p->dtype;
    g.act = p->act;
    DeviceScope scope(p->device);
    HIP_TRY(scope.status);
    return launch_gemm16(g, true, true, static_cast<hipStream_t>(stream));
}

extern "C" int ee_linear_grad_workspace(const ee_linear_grad_args *p, size_t *bytes)
{
    static const char *const call = "ee_linear_grad_workspace";
    if (!bytes) return fail(EE_EINVAL, "%s: null argument", call);
    *bytes = 0;
    int rc = check_linear_grad(call, p);
    if (rc == EE_OK) *bytes = plan_grad(*p).bytes();
    return rc;
}

extern "C" int ee_linear_grad(const ee_linear_grad_args *p, void *workspace, size_t workspace_bytes, void *stream)
{
    static const char *const call = "ee_linear_grad";
    int rc = check_linear_grad(call, p);
    if (rc == EE_OK) rc = check_matrix(call, "x", p->x, p->dtype, p->x_stride, p->n_rows, p->n_in);
    if (rc == EE_OK) rc = check_matrix(call, "weight", p->weight, p->dtype, p->weight_stride, p->n_out, p->n_in);
    if (rc == EE_OK) rc = check_matrix(call, "dy", p->dy, p->dtype, p->dy_stride, p->n_rows, p->n_out);
    if (rc == EE_OK) rc = check_matrix(call, "pre", p->pre, p->dtype, p->pre_stride, p->n_rows, p->n_out);
    if (rc == EE_OK) rc = check_matrix(call, "dx", p->dx, p->dx_dtype, p->dx_stride, p->n_rows, p->n_in);
    if (rc == EE_OK) rc = check_matrix(call, "d_weight", p->d_weight, p->dw_dtype, p->dw_stride, p->n_out, p->n_in);
    if (rc != EE_OK) return rc;
    if (!p->dx && !p->d_weight && !p->d_bias) return EE_OK;
    if (p->n_rows) {
        if (!p->dy) return fail(EE_EINVAL, "%s: null dy", call);
        if (p->act != EE_ACT_NONE && !p->pre) return fail(EE_EINVAL, "%s: an activation's gradient needs pre", call);
        if ((p->dx && !p->weight) || (p->d_weight && !p->x)) return fail(EE_EINVAL, "%s: dx needs weight, d_weight needs x", call);
    }
    for (const void *out : {(const void *)p->dx, (const void *)p->d_weight})
        if (out && (out == p->x || out == p->weight || out == p->dy || out == p->pre || (out == p->dx && out == p->d_weight)))
            return fail(EE_EINVAL, "%s: dx and d_weight must be arrays of their own", call);
    if (!aligned(p->d_bias, 4)) return fail(EE_EINVAL, "%s: fp32 arrays must be 4-byte aligned", call);
    const GradPlan pl = plan_grad(*p);
    if (pl.bytes() > workspace_bytes || (pl.bytes() && (!workspace || !aligned(workspace, 256))))
        return fail(EE_EINVAL, "%s: the workspace has %zu bytes of %zu, or is not 256-byte aligned", call, workspace_bytes, pl.bytes());
    DeviceScope scope(p->device);
    HIP_TRY(scope.status);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    uint16_t *const dz = static_cast<uint16_t *>(workspace);
    float *const part = reinterpret_cast<float *>(static_cast<unsigned char *>(workspace) + pl.dz_bytes);
    const long long plane = (long long)p->n_rows * pl.ldz;
    if (pl.parts && (p->d_bias || p->act != EE_ACT_NONE)) {
        SlopeDev a = {};
        a.dy = static_cast<const uint16_t *>(p->dy);
        a.pre = static_cast<const uint16_t *>(p->pre);
        a.dy_stride = p->n_rows > 1 ? p->dy_stride : 0;
        a.pre_stride = p->n_rows > 1 ? p->pre_stride : 0;
        a.ldz = pl.ldz;
        a.plane = plane;
        a.dz = dz;
        a.part = p->d_bias ? part : nullptr;
        a.type = p->dtype;
        a.act = p->act;
        a.terms = p->dx || p->d_weight ? pl.terms : 0;
        a.rows = p->n_rows;
        a.n = p->n_out;
        a.per = pl.per;
        hipLaunchKernelGGL(ee_slope_kernel, dim3((unsigned)((p->n_out + SL_COLS * 8 - 1) / (SL_COLS * 8)), (unsigned)pl.parts), dim3(SL_COLS * SL_SUBS), 0, s, a);
        HIP_TRY(hipGetLastError());
    }
    launch_column_sums(part, pl.parts, p->n_out, p->d_bias, nullptr, nullptr, s);
    HIP_TRY(hipGetLastError());
    GemmDev g = {};
    g.type = p->dtype;
    g.act = EE_ACT_NONE;
    g.plane = plane;
    g.A = p->act == EE_ACT_NONE ? static_cast<const uint16_t *>(p->dy) : dz;
    g.lda = p->act != EE_ACT_NONE ? pl.ldz : p->n_rows > 1 ? p->dy_stride : 0;
    if (p->dx && p->n_rows) {
        g.B = static_cast<const uint16_t *>(p->weight);
        g.ldb = p->n_out > 1 ? p->weight_stride : 0;
        g.terms = pl.terms_dx;
        g.I = p->n_rows;
        g.J = p->n_in;
        g.K = p->n_out;
        g.y = p->dx;
        g.y_type = p->dx_dtype;
        g.y_stride = p->n_rows > 1 ? p->dx_stride : 0;
        if ((rc = launch_gemm16(g, true, false, s)) != EE_OK) return rc;
    }
    if (p->d_weight) {
        g.B = static_cast<const uint16_t *>(p->x);
        g.ldb = p->n_rows > 1 ? p->x_stride : 0;
        g.terms = pl.terms_dw;
        g.I = p->n_out;
        g.J = p->n_in;
        g.K = p->n_rows;
        g.y = p->d_weight;
        g.y_type = p->dw_dtype;
        g.y_stride = p->n_out > 1 ? p->dw_stride : 0;
        if ((rc = launch_gemm16(g, false, false, s)) != EE_OK) return rc;
    }
    return EE_OK;
}
