#include "ee_attend.hpp"

namespace ee {

// Pages that the members [s0, s1) of a group read together: the entries they have in common, as far as every new row of every
// member sees all of their positions.
__device__ __forceinline__ int common_pages(const AttendDev &a, int group, int s0, int s1, int lane, int &first_member)
{
    int pages = min(max(as_global(a.group_pages)[group], 0), a.b.table_stride);
    first_member = s1;
    for (int base = s0; base < s1; base += 64) {
        const int s = base + lane;
        int mine = 0x7FFFFFFF, has = 0;
        if (s < s1) {
            const int n = a.b.start(s + 1) - a.b.start(s);
            has = n > 0;
            if (has) mine = max(a.b.length(s) - n + 1, 0) >> 4;
        }
        if (const unsigned long long who = __ballot(has); who && first_member == s1) first_member = base + __builtin_ctzll(who);
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) mine = min(mine, __shfl_xor(mine, d, 64));
        pages = min(pages, mine);
    }
    pages = __builtin_amdgcn_readfirstlane(pages);
    return pages;
}

__device__ __forceinline__ int group_bound(const AttendDev &a, int g) { return min(max(as_global(a.group_start)[g], 0), a.b.n_seqs); }

// Group of sequence `seq`, or -1.
__device__ __forceinline__ int group_of(const AttendDev &a, int seq, int lane)
{
    for (int base = 0; base < a.n_groups; base += 64) {
        const int g = base + lane;
        const bool in = g < a.n_groups && group_bound(a, g) <= seq && seq < group_bound(a, g + 1);
        if (const unsigned long long who = __ballot(in)) return base + __builtin_ctzll(who);
    }
    return -1;
}

template <int HD, int TERMS, int QT, int RT>
__global__ void __launch_bounds__(ATT_W * 64) ee_attend_kernel(AttendDev a)
{
    extern __shared__ __align__(16) char lds_raw[];
    constexpr int KT = HD / 32, NT = HD / 16, LINES = RT * 16;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lm = lane & 15, quad = lane >> 4;
    const int G = a.per_key, kvh = blockIdx.y;
    const int shared_items = a.chunks_shared * a.parts_shared;
    int item = blockIdx.x;
    const bool shared = item < shared_items;
    const int parts = shared ? a.parts_shared : a.parts_own;
    if (!shared) item -= shared_items;
    const int chunk = item / parts, part = item - chunk * parts;

    AttendItem it;
    int row0, n_rows, seq, group = -1, place, slot, first_pos = 0;
    bool clear_shared = false;
    if (shared) {
        if (!find_item(a.n_groups, chunk, lane, [&](int g) {
                const int s0 = group_bound(a, g), s1 = max(group_bound(a, g + 1), s0);
                return (max(a.b.start(s1) - a.b.start(s0), 0) * G + LINES - 1) / LINES;
            }, group, place))
            return;
        const int s0 = group_bound(a, group), s1 = max(group_bound(a, group + 1), s0);
        row0 = a.b.start(s0);
        n_rows = a.b.start(s1) - row0;
        const int pages = common_pages(a, group, s0, s1, lane, seq);
        if (seq >= s1) return;                                              // (row_start decreases somewhere)
        it.pg_lo = (int)((long long)pages * part / parts);
        it.pg_hi = (int)((long long)pages * (part + 1) / parts);
        slot = part;
    } else {
        if (!find_item(a.b.n_seqs, chunk, lane, [&](int s) { return (max(a.b.start(s + 1) - a.b.start(s), 0) * G + LINES - 1) / LINES; }, seq, place)) return;
        row0 = a.b.start(seq);
        n_rows = a.b.start(seq + 1) - row0;
        first_pos = a.b.length(seq) - n_rows;                               // position of the first row
        int from = 0;
        if (a.n_groups) {
            group = group_of(a, seq, lane);
            int member;
            if (group >= 0)
                from = common_pages(a, group, group_bound(a, group), group_bound(a, group + 1), lane, member);
            else
                clear_shared = part == 0;
        }
        const int last_line = min(place * LINES + LINES, n_rows * G) - 1;
        const int visible = min(first_pos + last_line / G + 1, a.b.capacity());
        const int pages = max(((max(visible, 0) + KV_PAGE - 1) >> 4) - from, 0);
        it.pg_lo = from + (int)((long long)pages * part / parts);
        it.pg_hi = from + (int)((long long)pages * (part + 1) / parts);
        slot = a.parts_shared + part;
    }
    it.line0 = place * LINES;
    it.lines = min(LINES, n_rows * G - it.line0);
    it.n_pages = a.b.n_pages;
    it.table = a.b.table + (size_t)seq * a.b.table_stride;
    it.page_step = (size_t)a.b.n_kv_heads * KV_PAGE * TERMS * HD;
    it.k = a.b.kpool + (size_t)kvh * KV_PAGE * TERMS * HD;
    it.v = a.b.vpool + (size_t)kvh * KV_PAGE * TERMS * HD;

    // this lane's lines: row, head, last position seen
    int row[RT], head[RT], last[RT], max_last = 0x7FFFFFF0;
    bf16x8_t q[RT][KT][QT];
    const bool any = it.pg_hi > it.pg_lo;
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        const int line = it.line0 + min(t * 16 + lm, it.lines - 1), i = line / G;
        row[t] = row0 + i;
        head[t] = kvh * G + line - i * G;
        last[t] = shared ? 0x7FFFFFF0 : first_pos + i;
    }
    it.first_last = shared ? 0x7FFFFFF0 : first_pos + it.line0 / G;
    if (!shared) max_last = min(first_pos + (it.line0 + it.lines - 1) / G, a.b.capacity() - 1);
    AttendState<RT, NT> st;
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        st.mx[t] = -INFINITY;
        st.sum[t] = 0.f;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) st.o[t][nt] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
    }
    if (any) {
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            if (t * 16 >= it.lines) continue;
#pragma unroll
            for (int kt = 0; kt < KT; ++kt) {
                const size_t at = (size_t)row[t] * a.q_stride + (size_t)head[t] * a.q_head + kt * 32 + quad * 8;
                if constexpr (QT == 1) {
                    q[t][kt][0] = __builtin_bit_cast(bf16x8_t, load_global16(static_cast<const uint16_t *>(a.q) + at));
                } else {
                    float x[8];
                    if (a.q_type == EE_FP32)
                        load8<EE_FP32>(a.q, at, x);
                    else if (a.q_type == EE_FP16)
                        load8<EE_FP16>(a.q, at, x);
                    else
                        load8<EE_BF16>(a.q, at, x);
                    split_bf16x8((f32x4_t){x[0], x[1], x[2], x[3]}, (f32x4_t){x[4], x[5], x[6], x[7]}, q[t][kt][0], q[t][kt][1]);
                }
            }
        }
        attend_pages<HD, TERMS, QT, RT>(it, q, last, max_last, a.scale2, lane, wave, st);
        attend_join_waves<HD, RT>(st, reinterpret_cast<float *>(lds_raw), min(ATT_W, (it.pg_hi - it.pg_lo + 1) >> 1), a.scale2, lane, wave);
    }
    if (wave != 0) return;
    const int total = a.parts_shared + a.parts_own;
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        if (t * 16 + lm >= it.lines) continue;
        if (total == 1) {
            const float inv = st.sum[t] == 0.f ? 0.f : 1.0f / st.sum[t];    // (0: the line saw no position)
            const size_t to = (size_t)row[t] * a.o_stride + (size_t)head[t] * a.o_head + quad * 4;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) store4(a.out_type, a.out, to + nt * 16, st.o[t][nt][0] * inv, st.o[t][nt][1] * inv, st.o[t][nt][2] * inv, st.o[t][nt][3] * inv);
        } else {
            const size_t line = (size_t)row[t] * a.n_heads + head[t];
            if (st.mx[t] != -INFINITY) {                                    // (nothing is read of an empty part)
                float *o = a.part + (line * total + slot) * HD + quad * 4;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) *as_global_mut(reinterpret_cast<f32x4_t *>(o + nt * 16)) = st.o[t][nt];
            }
            if (quad == 0) {
                float *ml = a.part_ml + (line * total) * 2;
                as_global_mut(ml)[slot * 2] = st.mx[t];
                as_global_mut(ml)[slot * 2 + 1] = st.sum[t];
                if (clear_shared)
                    for (int s = 0; s < a.parts_shared; ++s) {
                        as_global_mut(ml)[s * 2] = -INFINITY;
                        as_global_mut(ml)[s * 2 + 1] = 0.f;
                    }
            }
        }
    }
}

// Joins the parts of every line, in order: thread = four dims of a line.
template <int HD>
__global__ void __launch_bounds__(256) ee_attend_join_kernel(AttendDev a)
{
    constexpr int TPL = HD / 4;                                             // threads of a line
    const long long line = (long long)blockIdx.x * (256 / TPL) + threadIdx.x / TPL;
    const int e = (threadIdx.x % TPL) * 4;
    const long long rows = a.b.start(a.b.n_seqs);
    if (line >= rows * a.n_heads) return;
    const int row = (int)(line / a.n_heads), head = (int)(line - (long long)row * a.n_heads);
    const int total = a.parts_shared + a.parts_own;
    const float *ml = a.part_ml + line * total * 2;
    const float *o = a.part + line * total * HD + e;
    float m = -INFINITY;
    bool bad = false;
    for (int p = 0; p < total; ++p) {
        const float mp = as_global(ml)[2 * p], lp = as_global(ml)[2 * p + 1];
        m = fmaxf(m, mp);
        bad |= mp == -INFINITY && lp != 0.f;                                // positions without a softmax
    }
    f32x4_t num = {0.f, 0.f, 0.f, 0.f};
    float den = 0.f;
    if (m != -INFINITY)
        for (int p = 0; p < total; ++p) {
            const float mp = as_global(ml)[2 * p];
            if (mp == -INFINITY) continue;
            const float f = __builtin_amdgcn_exp2f((mp - m) * a.scale2);
            const f32x4_t v = *as_global(reinterpret_cast<const f32x4_t *>(o + (size_t)p * HD));
#pragma unroll
            for (int r = 0; r < 4; ++r) num[r] += v[r] * f;
            den += as_global(ml)[2 * p + 1] * f;
        }
    const float inv = m != -INFINITY ? 1.0f / den : bad ? __builtin_nanf("") : 0.f;
    store4(a.out_type, a.out, (size_t)row * a.o_stride + (size_t)head * a.o_head + e, num[0] * inv, num[1] * inv, num[2] * inv, num[3] * inv);
}

typedef void (*attend_kernel_t)(AttendDev);
struct AttendKernel {
    attend_kernel_t f;
    size_t lds;
};
template <int HD, int TERMS, int QT>
static AttendKernel attend_of_tiles(int rt)
{
    if (rt == 1) return {ee_attend_kernel<HD, TERMS, QT, 1>, attend_lds<HD, 1>()};
    if constexpr (HD == 64)
        if (rt == 4) return {ee_attend_kernel<HD, TERMS, QT, 4>, attend_lds<HD, 4>()};
    return {ee_attend_kernel<HD, TERMS, QT, 2>, attend_lds<HD, 2>()};
}
static AttendKernel attend_kernel(int hd, int terms, int q_type, int rt)
{
    if (hd == 64) return terms == 2 ? attend_of_tiles<64, 2, 2>(rt) : q_type == EE_BF16 ? attend_of_tiles<64, 1, 1>(rt) : attend_of_tiles<64, 1, 2>(rt);
    return terms == 2 ? attend_of_tiles<128, 2, 2>(rt) : q_type == EE_BF16 ? attend_of_tiles<128, 1, 1>(rt) : attend_of_tiles<128, 1, 2>(rt);
}

// How a call is split; a function of what the host knows (sizes and the caller's bounds).
struct AttendPlan {
    int tiles;                        // tiles of 16 lines of an item
    int chunks_own, parts_own, chunks_shared, parts_shared;
    size_t part_floats, ml_floats;
};

// Chunks of `lines` lines that n things with T rows among them can have, each row `per_key` lines: one each, and one more for every `lines` lines behind
// its first row's (behind its first line, where rows do not fill chunks evenly).
static int most_chunks(int n, int T, int per_key, int lines)
{
    const long long things = std::min(n, T), all = (long long)T * per_key;
    const int first = lines % per_key == 0 ? per_key : per_key % lines == 0 ? lines : 1;
    return (int)(things + (all - things * first) / lines);
}

static AttendPlan plan_attend(const ee_paged_cache &c, const ee_attend_args &p)
{
    AttendPlan pl;
    const int T = p.n_rows, per_key = p.n_heads / c.n_kv_heads;
    const long long cap = std::min<long long>(c.table_stride, 0x7FFFFFF0 / KV_PAGE);
    const int pages = (int)std::min<long long>(cap, p.max_kv > 0 ? ((long long)p.max_kv + KV_PAGE - 1) / KV_PAGE : cap);
    const int shared_pages = p.n_groups == 0 ? 0 : (int)std::min<long long>(pages, p.max_shared > 0 ? p.max_shared / KV_PAGE : pages);
    const int seqs = std::min(c.n_seqs, T), groups = std::min(p.n_groups, seqs);
    const long long own_lines = (long long)T * per_key / seqs, shared_lines = groups ? (long long)T * per_key / groups : 0;
    const long long lines = std::max(own_lines, shared_lines);
    pl.tiles = lines <= 16 ? 1 : lines <= 32 || c.head_dim == 128 ? 2 : 4;
    pl.chunks_own = most_chunks(seqs, T, per_key, pl.tiles * 16);
    pl.chunks_shared = groups && shared_pages ? most_chunks(groups, T, per_key, pl.tiles * 16) : 0;
    const int own_pages = std::max(pages - shared_pages, 1);
    // Parts: enough for two workgroups a compute unit, as long as a part has 8 pages (a pair for each wave).
    const long long work = (long long)pl.chunks_own * own_pages + (long long)pl.chunks_shared * shared_pages;
    const long long per_part = std::max<long long>(8, work * c.n_kv_heads / 512);
    pl.parts_own = (int)std::min<long long>(std::max<long long>(own_pages / per_part, 1), 64);
    pl.parts_shared = pl.chunks_shared ? (int)std::min<long long>(std::max<long long>(shared_pages / per_part, 1), 64) : 0;
    const size_t total = (size_t)pl.parts_own + pl.parts_shared;
    const size_t all = (size_t)T * p.n_heads * total;
    pl.part_floats = total > 1 ? all * c.head_dim : 0;
    pl.ml_floats = total > 1 ? all * 2 : 0;
    return pl;
}

static int check_attend(const char *call, const ee_paged_cache *c, const ee_attend_args *p)
{
    if (!c || !p) return fail(EE_EINVAL, "%s: null argument", call);
    if (p->n_heads < 1) return fail(EE_EINVAL, "%s: n_heads %d", call, p->n_heads);
    int rc = check_cache(call, c, p->n_rows, p->n_heads, p->row_start, p->kv_len);
    if (rc != EE_OK) return rc;
    if (p->dtype < EE_BF16 || p->dtype > EE_FP32 || p->out_dtype < EE_BF16 || p->out_dtype > EE_FP32)
        return fail(EE_EINVAL, "%s: unknown element type %d or %d", call, p->dtype, p->out_dtype);
    if (!(p->scale > 0.f) || !isfinite(p->scale)) return fail(EE_EINVAL, "%s: scale must be positive and finite", call);
    if (p->n_groups < 0 || p->n_groups > c->n_seqs) return fail(EE_EINVAL, "%s: n_groups %d not in [0, n_seqs]", call, p->n_groups);
    if (p->max_kv < 0 || p->max_shared < 0) return fail(EE_EINVAL, "%s: negative max_kv or max_shared", call);
    return EE_OK;
}

}  // namespace ee

using namespace ee;

extern "C" int ee_attend_workspace(const ee_paged_cache *c, const ee_attend_args *p, size_t *bytes)
{
    static const char *const call = "ee_attend_workspace";
    if (!bytes) return fail(EE_EINVAL, "%s: null argument", call);
    *bytes = 0;
    if (!c || !p) return fail(EE_EINVAL, "%s: null argument", call);
    ee_paged_cache cs = *c;
    ee_attend_args ps = *p;
    // (sizes only: the arrays may not exist yet)
    static const int32_t there = 0;
    cs.page_table = ps.row_start = ps.kv_len = &there;
    cs.k_pool = cs.v_pool = reinterpret_cast<void *>((uintptr_t)256);
    int rc = check_attend(call, &cs, &ps);
    if (rc != EE_OK) return rc;
    if (c->n_seqs == 0 || p->n_rows == 0) return EE_OK;
    const AttendPlan pl = plan_attend(*c, *p);
    *bytes = (pl.part_floats + pl.ml_floats) * sizeof(float);
    return EE_OK;
}

extern "C" int ee_attend(const ee_paged_cache *c, const ee_attend_args *p, void *workspace, size_t workspace_bytes, void *stream)
{
    static const char *const call = "ee_attend";
    int rc = check_attend(call, c, p);
    if (rc != EE_OK) return rc;
    if (!stride_ok(p->q_stride, p->dtype) || !stride_ok(p->q_head_stride, p->dtype) || !stride_ok(p->out_stride, p->out_dtype) ||
        !stride_ok(p->out_head_stride, p->out_dtype))
        return fail(EE_EINVAL, "%s: a stride keeps no 16-byte alignment", call);
    if (c->n_seqs == 0 || p->n_rows == 0) return EE_OK;
    if (!p->q || !p->out || (p->n_groups && (!p->group_start || !p->group_pages))) return fail(EE_EINVAL, "%s: null q, out, group_start or group_pages", call);
    if (!aligned(p->q, 16) || !aligned(p->out, 16)) return fail(EE_EINVAL, "%s: q and out must be 16-byte aligned", call);
    if (!aligned(p->group_start, 4) || !aligned(p->group_pages, 4)) return fail(EE_EINVAL, "%s: int32 arrays must be 4-byte aligned", call);
    const AttendPlan pl = plan_attend(*c, *p);
    const size_t need = (pl.part_floats + pl.ml_floats) * sizeof(float);
    if (need > workspace_bytes || (need && (!workspace || !aligned(workspace, 256))))
        return fail(EE_EINVAL, "%s: the workspace has %zu bytes of %zu, or is not 256-byte aligned", call, workspace_bytes, need);
    if ((long long)pl.chunks_own * pl.parts_own + (long long)pl.chunks_shared * pl.parts_shared > 0x7FFFFFFF) return fail(EE_EINVAL, "%s: too many rows", call);

    AttendDev a;
    a.b = batch_of(*c, p->n_rows, p->row_start, p->kv_len);
    a.q = p->q;
    a.out = p->out;
    a.q_stride = p->q_stride;
    a.q_head = p->q_head_stride;
    a.o_stride = p->out_stride;
    a.o_head = p->out_head_stride;
    a.q_type = p->dtype;
    a.out_type = p->out_dtype;
    a.n_groups = pl.chunks_shared ? p->n_groups : 0;
    a.group_start = p->group_start;
    a.group_pages = p->group_pages;
    a.part = static_cast<float *>(workspace);
    a.part_ml = a.part + pl.part_floats;
    a.n_heads = p->n_heads;
    a.per_key = p->n_heads / c->n_kv_heads;
    a.parts_own = pl.parts_own;
    a.parts_shared = pl.parts_shared;
    a.chunks_shared = pl.chunks_shared;
    a.scale2 = p->scale * 1.44269504f;
    DeviceScope scope(c->device);
    HIP_TRY(scope.status);
    const AttendKernel k = attend_kernel(c->head_dim, c->terms, p->dtype, pl.tiles);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    hipLaunchKernelGGL(k.f, dim3(pl.chunks_own * pl.parts_own + pl.chunks_shared * pl.parts_shared, c->n_kv_heads), dim3(ATT_W * 64), k.lds, s, a);
    HIP_TRY(hipGetLastError());
    if (pl.part_floats) {
        const int per = 256 / (c->head_dim / 4);
        const unsigned blocks = (unsigned)(((size_t)p->n_rows * p->n_heads + per - 1) / per);
        hipLaunchKernelGGL(c->head_dim == 64 ? ee_attend_join_kernel<64> : ee_attend_join_kernel<128>, dim3(blocks), dim3(256), 0, s, a);
        HIP_TRY(hipGetLastError());
    }
    return EE_OK;
}
