// ee_kv_append: norms of queries and keys per head, rotation to their positions, keys and values into a paged cache.
//
// Bound by bytes (a row's queries, keys and values once in, once out) where there are many rows, by the chain of
// dependent loads (row -> sequence -> page -> data) where there are few.
// A block is up to 16 new rows of one sequence that lie on one page.  Its work is dealt to waves in units: a head of queries or keys of
// 64 / (HD / 16) rows, or a head of values (two of 64).  Queries and keys: a row's head is HD / 16 lanes, each with eight neighbouring elements of either
// half, so that the partners of a rotation (x_j and x_{j + HD/2}, or neighbours) are in one lane and every access is 16 bytes wide.  Values: the cache
// holds them transposed ([dim][position]), so a lane takes two dims of all 16 rows, and the wave turns its 64-byte pieces into whole kilobytes through
// LDS; pages that the new rows cover only partly are written position by position, so that the others stay as they are.
// (Units of four heads, which fetch a row's cosines and sines once for all: eight rounds of five rows 7.7 -> 10.1 us, 2041 rows of 32 heads 26.2 -> 28.8.)
#include "ee_ops.hpp"

namespace ee {

constexpr int APP_WAVES = 4;
constexpr int append_value_heads(int hd) { return 128 / hd; }   // heads of a unit of values: a lane has two dims

struct AppendDev {
    BatchDev b;
    const void *q, *k, *v;
    void *q_out;
    long long q_stride, q_head, k_stride, k_head, v_stride, v_head, o_stride, o_head;
    const float *q_gain, *k_gain, *rope;
    int n_heads, rope_len, rope_pairs, out_type;
    int q_units, k_units;         // units of a block before the keys' first, before the values' first
    int units;
    float eps;
};

// Where a block's rows lie: positions first .. first + 15, rows row0 + slot for the slots [lo, hi).
struct AppendBlock {
    int seq, page;                // page: place in the sequence's table (negative: in front of it)
    int row0, lo, hi;
    int usable;                   // slots from here on have no place (end of the tables), nor have those of negative positions
};

__device__ __forceinline__ bool append_block(const BatchDev &b, int block, int lane, int rope_len, AppendBlock &at)
{
    int seq, j;
    auto span = [&](int s, int &r0, int &p0, int &kv) {
        r0 = b.start(s);
        const int n = max(b.start(s + 1) - r0, 0);
        kv = b.length(s);
        p0 = kv - n;              // (may be negative: rows in front of position 0)
        return n;
    };
    if (!find_item(b.n_seqs, block, lane, [&](int s) {
            int r0, p0, kv;
            const int n = span(s, r0, p0, kv);
            return n > 0 ? ((kv - 1) >> 4) - (p0 >> 4) + 1 : 0;
        }, seq, j))
        return false;
    int r0, p0, kv;
    span(seq, r0, p0, kv);
    at.seq = seq;
    at.page = (p0 >> 4) + j;
    const int first = at.page << 4;
    at.lo = max(p0 - first, 0);
    at.hi = min(kv - first, KV_PAGE);
    at.row0 = r0 - p0 + first;
    at.usable = at.page < 0 ? 0 : max(min(min(b.capacity(), rope_len) - first, KV_PAGE), 0);
    return true;
}

template <int HD, int TERMS, int IN>
__device__ __forceinline__ void append_normed(const AppendDev &a, const AppendBlock &at, int page, bool is_k, int h, int it, int lane)
{
    constexpr int LANES = HD / 16, ROWS = 64 / LANES;
    const int sub = lane % LANES, i0 = sub * 8;
    const void *src = is_k ? a.k : a.q;
    const long long stride = is_k ? a.k_stride : a.q_stride, head = is_k ? a.k_head : a.q_head;
    const float *gain = is_k ? a.k_gain : a.q_gain;
    if (at.hi <= it || at.lo >= it + ROWS) return;
    float g[2][8];
    if (gain) {
        load8<EE_FP32>(gain, i0, g[0]);
        load8<EE_FP32>(gain, HD / 2 + i0, g[1]);
    }
    const int slot = it + lane / LANES;
    const bool row_ok = slot >= at.lo && slot < at.hi;
    const bool placed = row_ok && slot < at.usable;
    const int row = at.row0 + (row_ok ? slot : max(at.lo, it));          // (lanes without a row repeat one)
    float y[2][8];
    const size_t from = (size_t)row * stride + (size_t)h * head + i0;
    load8<IN>(src, from, y[0]);
    load8<IN>(src, from + HD / 2, y[1]);
    // cosines and sines: of pairs (j, j + HD/2) the lane has j = i0 .. i0 + 7; of neighbours i0 / 2 .. + 3 and HD / 4 more
    float cs[2][8];
    if (a.rope) {
        const int pos = placed ? (at.page << 4) + slot : 0;
        const float *t = a.rope + (size_t)pos * HD;
        const int c0 = a.rope_pairs ? i0 : 2 * i0, c1 = a.rope_pairs ? HD / 2 + i0 : 2 * i0 + 8;
        load8<EE_FP32>(t, c0, cs[0]);
        load8<EE_FP32>(t, c1, cs[1]);
    }
    if (gain) {
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) ss += y[0][e] * y[0][e] + y[1][e] * y[1][e];
#pragma unroll
        for (int d = 1; d < LANES; d <<= 1) ss += __shfl_xor(ss, d, 64);
        const float r = 1.0f / sqrtf(ss * (1.0f / HD) + a.eps);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            y[0][e] = y[0][e] * r * g[0][e];
            y[1][e] = y[1][e] * r * g[1][e];
        }
    }
    if (a.rope) {
        if (a.rope_pairs) {
#pragma unroll
            for (int p = 0; p < 2; ++p)
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    const float u = y[p][e], w = y[p][e + 1], c = cs[p][e], s = cs[p][e + 1];
                    y[p][e] = u * c - w * s;
                    y[p][e + 1] = w * c + u * s;
                }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float u = y[0][e], w = y[1][e], c = cs[e >> 2][2 * (e & 3)], s = cs[e >> 2][2 * (e & 3) + 1];
                y[0][e] = u * c - w * s;
                y[1][e] = w * c + u * s;
            }
        }
    }
    if (!is_k) {
        if (row_ok) {
            const size_t to = (size_t)row * a.o_stride + (size_t)h * a.o_head + i0;
#pragma unroll
            for (int p = 0; p < 2; ++p) {
#pragma unroll
                for (int e = 0; e < 8; ++e) y[p][e] = placed ? y[p][e] : 0.f;
                store8(a.out_type, a.q_out, to + p * (HD / 2), y[p]);
            }
        }
    } else if (placed && page >= 0) {
        uint16_t *rec = a.b.kpool + ((((size_t)page * a.b.n_kv_heads + h) * KV_PAGE + slot) * TERMS) * HD + i0;
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            uint32_t hi[4], lo[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) split_bf16(y[p][2 * e], y[p][2 * e + 1], hi[e], lo[e]);
            *as_global_mut(reinterpret_cast<u32x4_t *>(rec + p * (HD / 2))) = (u32x4_t){hi[0], hi[1], hi[2], hi[3]};
            if constexpr (TERMS == 2) *as_global_mut(reinterpret_cast<u32x4_t *>(rec + HD + p * (HD / 2))) = (u32x4_t){lo[0], lo[1], lo[2], lo[3]};
        }
    }
}

// two neighbouring elements
template <int IN>
__device__ __forceinline__ void load2(const void *base, size_t at, float &a, float &b)
{
    if constexpr (IN == EE_FP32) {
        typedef __attribute__((ext_vector_type(2))) float f32x2_t;
        const f32x2_t v = *as_global(reinterpret_cast<const f32x2_t *>(static_cast<const float *>(base) + at));
        a = v[0];
        b = v[1];
    } else {
        const uint32_t v = *as_global(reinterpret_cast<const uint32_t *>(static_cast<const uint16_t *>(base) + at));
        if constexpr (IN == EE_BF16) {
            a = __uint_as_float(v << 16);
            b = __uint_as_float(v & 0xFFFF0000u);
        } else {
            a = (float)__builtin_bit_cast(_Float16, (uint16_t)(v & 0xFFFF));
            b = (float)__builtin_bit_cast(_Float16, (uint16_t)(v >> 16));
        }
    }
}

template <int HD, int TERMS, int IN>
__device__ __forceinline__ void append_values(const AppendDev &a, const AppendBlock &at, int page, int h0, int lane, char *lds)
{
    constexpr int LANES = HD / 2;                                           // of a head: two dims each
    const int d0 = (lane % LANES) * 2, h = h0 + lane / LANES;
    const int lo = at.lo, hi = min(at.hi, at.usable);
    if (page < 0 || lo >= hi) return;
    float x[KV_PAGE][2];
#pragma unroll
    for (int r = 0; r < KV_PAGE; ++r) {
        const int row = at.row0 + min(max(r, lo), hi - 1);
        load2<IN>(a.v, (size_t)row * a.v_stride + (size_t)min(h, a.b.n_kv_heads - 1) * a.v_head + d0, x[r][0], x[r][1]);
    }
    uint16_t *const recs = a.b.vpool + ((size_t)page * a.b.n_kv_heads + h0) * (size_t)(TERMS * HD * KV_PAGE);
    uint32_t w[2][2][KV_PAGE / 2];
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int r = 0; r < KV_PAGE / 2; ++r) split_bf16(x[2 * r][e], x[2 * r + 1][e], w[0][e][r], w[1][e][r]);
#pragma unroll
    for (int t = 0; t < TERMS; ++t) {
        if (lo == 0 && hi == KV_PAGE) {
            // the lane's 64 bytes (two dims of 16 positions) -> the wave's four kilobytes, sixteen bytes a lane and turn
            u32x4_t *mine = reinterpret_cast<u32x4_t *>(lds) + lane * 4;
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int k = 0; k < 2; ++k)                                 // (turned by the lane, or all would meet in the same banks)
                    mine[(e * 2 + k + (lane >> 1)) & 3] = (u32x4_t){w[t][e][4 * k], w[t][e][4 * k + 1], w[t][e][4 * k + 2], w[t][e][4 * k + 3]};
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");              // (one wave's own LDS: no barrier)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int piece = k * 64 + lane, from = piece >> 2;         // of lane `from`
                const u32x4_t v = reinterpret_cast<const u32x4_t *>(lds)[from * 4 + ((piece + (from >> 1)) & 3)];
                const int head = from / LANES, in = piece - head * LANES * 4;
                if (h0 + head < a.b.n_kv_heads) *as_global_mut(reinterpret_cast<u32x4_t *>(recs + (size_t)head * (TERMS * HD * KV_PAGE) + t * HD * KV_PAGE) + in) = v;
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        } else if (h < a.b.n_kv_heads) {
            uint16_t *out = recs + (size_t)(lane / LANES) * (TERMS * HD * KV_PAGE) + (t * HD + d0) * KV_PAGE;
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int r = 0; r < KV_PAGE; r += 2) {
                    uint16_t *o = out + e * KV_PAGE + r;
                    const uint32_t two = w[t][e][r >> 1];
                    const bool first = r >= lo && r < hi, second = r + 1 >= lo && r + 1 < hi;
                    if (first && second)
                        *as_global_mut(reinterpret_cast<uint32_t *>(o)) = two;
                    else if (first)
                        as_global_mut(o)[0] = (uint16_t)two;
                    else if (second)
                        as_global_mut(o)[1] = (uint16_t)(two >> 16);
                }
        }
    }
}

template <int HD, int TERMS, int IN>
__global__ void __launch_bounds__(APP_WAVES * 64) ee_append_kernel(AppendDev a)
{
    __shared__ __align__(16) char lds[APP_WAVES][4096];
    constexpr int ROWS = 64 / (HD / 16), ROUNDS = KV_PAGE / ROWS;            // rows of a unit of queries or keys, units for a page
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int unit = blockIdx.y * APP_WAVES + wave;
    AppendBlock at;
    if (unit >= a.units || !append_block(a.b, blockIdx.x, lane, a.rope ? a.rope_len : 0x7FFFFFFF, at)) return;
    int page = -1;
    if (at.usable > 0) {
        page = as_global(a.b.table)[(size_t)at.seq * a.b.table_stride + at.page];
        if (page >= a.b.n_pages) page = -1;
    }
    if (unit < a.k_units) {
        const bool is_k = unit >= a.q_units;
        const int u = is_k ? unit - a.q_units : unit;
        append_normed<HD, TERMS, IN>(a, at, page, is_k, u / ROUNDS, u % ROUNDS * ROWS, lane);
    } else {
        append_values<HD, TERMS, IN>(a, at, page, (unit - a.k_units) * append_value_heads(HD), lane, lds[wave]);
    }
}

typedef void (*append_kernel_t)(AppendDev);
template <int HD, int TERMS>
static append_kernel_t append_kernel(int type)
{
    return type == EE_BF16 ? ee_append_kernel<HD, TERMS, EE_BF16> : type == EE_FP16 ? ee_append_kernel<HD, TERMS, EE_FP16> : ee_append_kernel<HD, TERMS, EE_FP32>;
}

int check_cache(const char *call, const ee_paged_cache *c, int n_rows, int n_heads, const void *row_start, const void *kv_len)
{
    if (c->device < 0) return fail(EE_EINVAL, "%s: device %d", call, c->device);
    if (c->head_dim != 64 && c->head_dim != 128) return fail(EE_EINVAL, "%s: head_dim %d is neither 64 nor 128", call, c->head_dim);
    if (c->terms != 1 && c->terms != 2) return fail(EE_EINVAL, "%s: terms %d is neither 1 nor 2", call, c->terms);
    if (c->n_kv_heads < 1 || c->n_kv_heads > 4096) return fail(EE_EINVAL, "%s: n_kv_heads %d not in [1,4096]", call, c->n_kv_heads);
    if (n_heads < 0 || n_heads > 4096 * 16 || n_heads % c->n_kv_heads)
        return fail(EE_EINVAL, "%s: n_heads %d is no multiple of n_kv_heads %d", call, n_heads, c->n_kv_heads);
    if (c->n_seqs < 0 || n_rows < 0 || n_rows > 1 << 24 || c->n_seqs > 1 << 20)
        return fail(EE_EINVAL, "%s: n_seqs %d or n_rows %d out of range", call, c->n_seqs, n_rows);
    if (c->n_pages < 1 || c->table_stride < 1) return fail(EE_EINVAL, "%s: n_pages %d, table_stride %d must be positive", call, c->n_pages, c->table_stride);
    if (c->n_seqs == 0 || n_rows == 0) return EE_OK;
    if (!c->k_pool || !c->v_pool || !c->page_table || !row_start || !kv_len) return fail(EE_EINVAL, "%s: null pool, page_table, row_start or kv_len", call);
    if (!aligned(c->k_pool, 16) || !aligned(c->v_pool, 16)) return fail(EE_EINVAL, "%s: the pools must be 16-byte aligned", call);
    if (!aligned(c->page_table, 4) || !aligned(row_start, 4) || !aligned(kv_len, 4)) return fail(EE_EINVAL, "%s: int32 arrays must be 4-byte aligned", call);
    return EE_OK;
}

BatchDev batch_of(const ee_paged_cache &c, int n_rows, const int32_t *row_start, const int32_t *kv_len)
{
    BatchDev b;
    b.kpool = static_cast<uint16_t *>(c.k_pool);
    b.vpool = static_cast<uint16_t *>(c.v_pool);
    b.table = c.page_table;
    b.row_start = row_start;
    b.kv_len = kv_len;
    b.n_pages = c.n_pages;
    b.n_seqs = c.n_seqs;
    b.n_rows = n_rows;
    b.table_stride = c.table_stride;
    b.n_kv_heads = c.n_kv_heads;
    return b;
}

}  // namespace ee

using namespace ee;

extern "C" int ee_kv_append(const ee_paged_cache *c, const ee_append_args *p, void *stream)
{
    static const char *const call = "ee_kv_append";
    if (!c || !p) return fail(EE_EINVAL, "%s: null argument", call);
    int rc = check_cache(call, c, p->n_rows, p->n_heads, p->row_start, p->kv_len);
    if (rc != EE_OK) return rc;
    if (p->dtype < EE_BF16 || p->dtype > EE_FP32 || p->q_out_dtype < EE_BF16 || p->q_out_dtype > EE_FP32)
        return fail(EE_EINVAL, "%s: unknown element type %d or %d", call, p->dtype, p->q_out_dtype);
    if (!(p->eps >= 0.f) || !isfinite(p->eps)) return fail(EE_EINVAL, "%s: eps must not be negative", call);
    if (p->rope_pairs != 0 && p->rope_pairs != 1) return fail(EE_EINVAL, "%s: rope_pairs %d is neither 0 nor 1", call, p->rope_pairs);
    if (p->rope && p->rope_len < 1) return fail(EE_EINVAL, "%s: rope_len %d", call, p->rope_len);
    const struct {
        int64_t stride;
        int type, n;
    } strides[8] = {{p->k_stride, p->dtype, p->n_rows},    {p->k_head_stride, p->dtype, c->n_kv_heads},    {p->v_stride, p->dtype, p->n_rows},
                    {p->v_head_stride, p->dtype, c->n_kv_heads}, {p->q_stride, p->dtype, p->n_rows},        {p->q_head_stride, p->dtype, p->n_heads},
                    {p->q_out_stride, p->q_out_dtype, p->n_rows}, {p->q_out_head_stride, p->q_out_dtype, p->n_heads}};
    for (int i = 0; i < (p->n_heads ? 8 : 4); ++i)
        if (!stride_ok(strides[i].stride, strides[i].type, strides[i].n))
            return fail(EE_EINVAL, "%s: stride %lld keeps no 16-byte alignment", call, (long long)strides[i].stride);
    if (c->n_seqs == 0 || p->n_rows == 0) return EE_OK;
    if (!p->k || !p->v || (p->n_heads && (!p->q || !p->q_out))) return fail(EE_EINVAL, "%s: null q, k, v or q_out", call);
    for (const void *x : {p->q, p->k, p->v, (const void *)p->q_out, (const void *)p->q_gain, (const void *)p->k_gain, (const void *)p->rope})
        if (!aligned(x, 16)) return fail(EE_EINVAL, "%s: q, k, v, q_out, gains and rope must be 16-byte aligned", call);
    if (p->n_heads && p->q == p->q_out && (p->dtype != p->q_out_dtype || (p->n_rows > 1 && p->q_stride != p->q_out_stride) ||
                                           (p->n_heads > 1 && p->q_head_stride != p->q_out_head_stride)))
        return fail(EE_EINVAL, "%s: q_out may be q only with the same type and strides", call);

    AppendDev a;
    a.b = batch_of(*c, p->n_rows, p->row_start, p->kv_len);
    a.q = p->q;
    a.k = p->k;
    a.v = p->v;
    a.q_out = p->q_out;
    a.q_stride = p->q_stride;
    a.q_head = p->q_head_stride;
    a.k_stride = p->k_stride;
    a.k_head = p->k_head_stride;
    a.v_stride = p->v_stride;
    a.v_head = p->v_head_stride;
    a.o_stride = p->q_out_stride;
    a.o_head = p->q_out_head_stride;
    a.q_gain = p->q_gain;
    a.k_gain = p->k_gain;
    a.rope = p->rope;
    a.n_heads = p->n_heads;
    a.rope_len = p->rope_len;
    a.rope_pairs = p->rope_pairs;
    a.out_type = p->q_out_dtype;
    a.eps = p->eps;
    // A sequence's n rows touch at most 1 + (n + 14) / 16 pages, one if there is one row: with T rows in s sequences, of which t have more
    // than one, at most s + (T - s + 15 t) / 16.
    const int s = std::min(c->n_seqs, p->n_rows), t = std::min(s, p->n_rows - s);
    const unsigned blocks = (unsigned)(s + (p->n_rows - s + 15 * t) / KV_PAGE);
    const int rounds = c->head_dim == 64 ? 1 : 2, of_values = append_value_heads(c->head_dim);
    a.q_units = p->n_heads * rounds;
    a.k_units = a.q_units + c->n_kv_heads * rounds;
    a.units = a.k_units + (c->n_kv_heads + of_values - 1) / of_values;
    const unsigned groups = (a.units + APP_WAVES - 1) / APP_WAVES;
    if (groups > OPS_MAX_GRID_Y) return fail(EE_EINVAL, "%s: %d heads are too many for a call", call, p->n_heads);
    DeviceScope scope(c->device);
    HIP_TRY(scope.status);
    append_kernel_t kernel = c->head_dim == 64 ? (c->terms == 1 ? append_kernel<64, 1>(p->dtype) : append_kernel<64, 2>(p->dtype))
                                               : (c->terms == 1 ? append_kernel<128, 1>(p->dtype) : append_kernel<128, 2>(p->dtype));
    hipLaunchKernelGGL(kernel, dim3(blocks, groups), dim3(APP_WAVES * 64), 0, static_cast<hipStream_t>(stream), a);
    HIP_TRY(hipGetLastError());
    return EE_OK;
}
