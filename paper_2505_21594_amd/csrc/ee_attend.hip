#include "ee_attend.hpp"

namespace ee {

typedef void (*attend_kernel_t)(AttendDev);
struct AttendKernel {
    attend_kernel_t f;
    size_t lds;
};
template <int HD, int TERMS, int QT, int PT>
static AttendKernel attend_of_tiles(int tiles)
{
    if (tiles == 1) return {ee_attend_kernel<HD, TERMS, QT, PT, 1>, attend_lds<HD, QT, 1>()};
    if constexpr (TERMS == 1 || HD == 64)
        if (tiles == 2) return {ee_attend_kernel<HD, TERMS, QT, PT, 2>, attend_lds<HD, QT, 2>()};
    return {ee_attend_wide_kernel<HD, TERMS, QT, PT>, attend_wide_lds<HD, TERMS>()};
}
template <int HD>
static AttendKernel attend_kernel(int terms, int q_type, int out_type, int tiles)
{
    if (terms == 2) return attend_of_tiles<HD, 2, 3, 3>(tiles);
    if (out_type == EE_FP32) return q_type == EE_BF16 ? attend_of_tiles<HD, 1, 1, 3>(tiles) : attend_of_tiles<HD, 1, 3, 3>(tiles);
    if (q_type == EE_FP32) return attend_of_tiles<HD, 1, 3, 3>(tiles);
    if (q_type == EE_FP16) return attend_of_tiles<HD, 1, 2, 2>(tiles);
    return attend_of_tiles<HD, 1, 1, 2>(tiles);
}

// How a call is split; a function of what the host knows (sizes and the caller's bounds).
struct AttendPlan {
    int tiles;                        // tiles of 16 lines of an item; 8: the kernel for many lines
    int groups;                       // groups whose common pages are read once
    int quota, most_own, most_shared;
    long long items;
    size_t part_bytes, ml_bytes, lane_bytes;
    size_t bytes() const { return part_bytes + ml_bytes + lane_bytes; }
};

// Chunks of `lines` lines that n things with T rows among them can have, each row `per_key` lines: one each, and one more for every `lines` lines behind
// its first row's (behind its first line, where rows do not fill chunks evenly).
static long long most_chunks(int n, int T, int per_key, int lines)
{
    const long long things = std::min(n, T), all = (long long)T * per_key;
    const int first = lines % per_key == 0 ? per_key : per_key % lines == 0 ? lines : 1;
    return things + (all - things * first) / lines;
}

static size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// Pages of a part for the kernel for many lines: as many parts as give the least time by this estimate, the fewest of those within 5 %.  The largest
// item's pages, or all pages at two items for a compute unit; parts are written and read again at 1.25 MB a microsecond, behind a launch (at twice that where
// the new rows are all the positions: items then end one after the other).  us, heads of 128, bf16, 32 heads, 1 / 2 / about 5 parts: 350 rows
// 18.3 / 21.9 / 24.3, 500 22.5 / 25.8 / 27.8, 350 behind 2000 cached positions 72.4 / 47.0 / 44.9; one and two parts: 700 and 1000 rows behind 2000 84.1 / 70.0,
// 91.7 / 83.4, 1000 rows 37.3 / 37.9; 2041 rows of 16 heads 64.0 / 50.4.  (32 heads on 8, 350 and 700 rows behind 2000: three parts, which it takes, 51.5 and 73.9, the best
// number of them 45.5 and 72.4.)
static int wide_quota(const ee_paged_cache &c, const ee_attend_args &p, int own_pages, long long chunks, int seqs)
{
    const int step = c.terms == 1 ? 4 : 2;
    const double page = (c.terms == 2 ? 2.2 : p.dtype == EE_BF16 ? 0.44 : 1.1) * c.head_dim / 128;     // us a page
    const double all = (double)chunks * c.n_kv_heads * own_pages * (seqs == 1 ? 1.0 : 0.5) / 512;
    const double fresh = std::min(1.0, (double)p.n_rows / seqs / (16.0 * own_pages));
    const double part = (double)p.n_rows * p.n_heads * c.head_dim * 4 / 1.25e6 * (1 - 0.5 * fresh);
    int best_quota = 0;
    double best = 0;
    for (int n = 1; n <= 64; ++n) {
        const int quota = ((own_pages + n - 1) / n + step - 1) / step * step, parts = (own_pages + quota - 1) / quota;
        const double t = page * std::max<double>(quota, all) + (parts > 1 ? 3 + part * parts : 0);
        if (best_quota == 0 || t < 0.95 * best) {
            best_quota = quota;
            best = t;
        }
    }
    return best_quota;
}

static AttendPlan plan_attend(const ee_paged_cache &c, const ee_attend_args &p)
{
    AttendPlan pl = {};
    const int T = p.n_rows, per_key = p.n_heads / c.n_kv_heads;
    const long long cap = std::min<long long>(c.table_stride, 0x7FFFFFF0 / KV_PAGE);
    const int pages = (int)std::min<long long>(cap, p.max_kv > 0 ? ((long long)p.max_kv + KV_PAGE - 1) / KV_PAGE : cap);
    int shared_pages = p.n_groups == 0 ? 0 : (int)std::min<long long>(pages, p.max_shared > 0 ? p.max_shared / KV_PAGE : pages);
    const int seqs = std::min(c.n_seqs, T);
    const long long own_lines = (long long)T * per_key / seqs;
    // Many lines of a key head a sequence, on average over the call's: the kernel that reads keys and values for 128 of them at a time
    // (ee_attend_wide_kernel).  us, the others / it, heads of 128, one term, 8 sequences of 2000 positions, 32 heads on 8 / on 32: 32 lines 23.9 / 24.6,
    // 61.1 / 60.8, 48 lines 33.8 / 28.9, 64.8 / 66.5, 64 lines 33.1 / 26.7, 69.4 / 63.0, 128 lines 44.5 / 31.2, 126 / 71; one sequence of 8000: 32 lines 18.9 / 19.3,
    // 33.4 / 31.8, 48 lines 20.3 / 23.1, 46.7 / 38.6.  Two terms, 32 heads on 32: 48 lines 163 / 184, 64 lines 187 / 186, 96 lines 262 / 193; one sequence of 2000:
    // 64 lines 32 / 41, 96 lines 48 / 46.  (Prompts of 300, 500 and 900 rows alone, 32 on 32: 12.7 / 15.5, 16.6 / 21.9, 34.9 / 33.1.)
    // It reads common pages for every sequence: 8 sequences with 3840 of 4000 positions in common, once by the others / for every sequence by it, 8 and 32 key
    // heads: 48 lines 35.5 / 39.1, 92 / 101, 64 lines 40.0 / 40.7, 109 / 103, 128 lines 61 / 49, 204 / 119.
    // One kernel serves the whole call.  A prompt among single tokens behind 1000 positions, chosen / the prompt and the tokens in two calls: 900 rows and 31 tokens, 32
    // heads on 8 48.5 / 32.9 + 28.8, on 32 155 / 33.2 + 96.3 (by tiles of 32 lines; 129 by 128); 2041 and 100 146.8 / 69.4 + 86.4, 454 / 69.5 + 288.
    const bool wide = own_lines > (c.terms == 1 ? 32 : 64);
    pl.groups = wide || shared_pages == 0 ? 0 : std::min(p.n_groups, seqs);
    if (pl.groups == 0) shared_pages = 0;
    const long long lines = pl.groups ? std::max(own_lines, (long long)T * per_key / pl.groups) : own_lines;
    pl.tiles = wide ? 8 : lines <= 16 || (c.terms == 2 && c.head_dim == 128) ? 1 : 2;
    const long long chunks_own = most_chunks(seqs, T, per_key, pl.tiles * 16);
    const long long chunks_shared = pl.groups ? most_chunks(pl.groups, T, per_key, pl.tiles * 16) : 0;
    const int own_pages = std::max(pages - shared_pages, 1);
    const long long est_own = seqs * ((own_lines + pl.tiles * 16 - 1) / (pl.tiles * 16));
    if (wide) {
        pl.quota = wide_quota(c, p, own_pages, est_own, seqs);
    } else {
        // Parts: the fewest pages each (a pair for each wave at a time: multiples of 8) that leave the items as many as the chip holds at once, two for a
        // compute unit, if sequences are half the longest on average.  A second round costs more than longer parts: eight rounds of five rows of 32 heads
        // behind 576 common positions, parts of 16 / 24 pages (544 / 448 items) 21.6 / 16.8 us; 32 rows of 8 key heads behind 6000, parts of 40 / 56 / 80
        // pages (616 / 500 / 424 items) 33.9 / 27.3 / 32.4.  Where chunks alone are more than that, half as many parts again.
        const double room = std::max(512.0 / c.n_kv_heads, 1.5 * (double)(est_own + chunks_shared));
        pl.quota = 8;
        while (pl.quota < std::max(own_pages, shared_pages)) {
            const double own_parts = seqs == 1 ? (double)((own_pages + pl.quota - 1) / pl.quota) : std::max(1.0, 0.5 * own_pages / pl.quota + 0.5);
            const long long shared_parts = (shared_pages + pl.quota - 1) / pl.quota;
            if ((double)est_own * own_parts + (double)(chunks_shared * shared_parts) <= room && own_pages <= 64 * pl.quota && shared_pages <= 64 * pl.quota) break;
            pl.quota += std::max(8, pl.quota / 64 * 8);
        }
    }
    pl.most_own = std::min((own_pages + pl.quota - 1) / pl.quota, 64);
    pl.most_shared = std::min((shared_pages + pl.quota - 1) / pl.quota, 64);
    pl.items = chunks_own * pl.most_own + chunks_shared * pl.most_shared;
    const size_t most = (size_t)pl.most_own + pl.most_shared, all = (size_t)T * p.n_heads;
    if (most > 1) {
        pl.part_bytes = align256(all * most * c.head_dim * sizeof(float));
        pl.ml_bytes = align256(all * (most + 1) * sizeof(float2));
    }
    if (pl.groups && (c.n_seqs > 64 || p.n_groups > 64)) pl.lane_bytes = align256(((size_t)c.n_seqs + 2 * (size_t)p.n_groups) * sizeof(int));
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
    *bytes = plan_attend(*c, *p).bytes();
    return EE_OK;
}

extern "C" int ee_attend(const ee_paged_cache *c, const ee_attend_args *p, void *workspace, size_t workspace_bytes, void *stream)
{
    static const char *const call = "ee_attend";
    int rc = check_attend(call, c, p);
    if (rc != EE_OK) return rc;
    if (!stride_ok(p->q_stride, p->dtype, p->n_rows) || !stride_ok(p->q_head_stride, p->dtype, p->n_heads) || !stride_ok(p->out_stride, p->out_dtype, p->n_rows) ||
        !stride_ok(p->out_head_stride, p->out_dtype, p->n_heads))
        return fail(EE_EINVAL, "%s: a stride keeps no 16-byte alignment", call);
    if (c->n_seqs == 0 || p->n_rows == 0) return EE_OK;
    if (!p->q || !p->out || (p->n_groups && (!p->group_start || !p->group_pages))) return fail(EE_EINVAL, "%s: null q, out, group_start or group_pages", call);
    if (!aligned(p->q, 16) || !aligned(p->out, 16)) return fail(EE_EINVAL, "%s: q and out must be 16-byte aligned", call);
    if (!aligned(p->group_start, 4) || !aligned(p->group_pages, 4)) return fail(EE_EINVAL, "%s: int32 arrays must be 4-byte aligned", call);
    const AttendPlan pl = plan_attend(*c, *p);
    const size_t need = pl.bytes();
    if (need > workspace_bytes || (need && (!workspace || !aligned(workspace, 256))))
        return fail(EE_EINVAL, "%s: the workspace has %zu bytes of %zu, or is not 256-byte aligned", call, workspace_bytes, need);
    if (pl.items > 65535) return fail(EE_EINVAL, "%s: %lld chunks of rows and pages are too many for a call", call, pl.items);

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
    a.n_groups = pl.groups ? p->n_groups : 0;
    a.group_start = p->group_start;
    a.group_pages = p->group_pages;
    unsigned char *ws = static_cast<unsigned char *>(workspace);
    a.part = reinterpret_cast<float *>(ws);
    a.part_ml = reinterpret_cast<float2 *>(ws + pl.part_bytes);
    a.from = reinterpret_cast<int *>(ws + pl.part_bytes + pl.ml_bytes);
    a.common = a.from + c->n_seqs;
    a.member = a.common + p->n_groups;
    a.n_heads = p->n_heads;
    a.per_key = p->n_heads / c->n_kv_heads;
    a.quota = pl.quota;
    a.most_own = pl.most_own;
    a.most_shared = pl.most_shared;
    a.scale2 = p->scale * 1.44269504f;
    DeviceScope scope(c->device);
    HIP_TRY(scope.status);
    const AttendKernel k = c->head_dim == 64 ? attend_kernel<64>(c->terms, p->dtype, p->out_dtype, pl.tiles) : attend_kernel<128>(c->terms, p->dtype, p->out_dtype, pl.tiles);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (pl.lane_bytes) {
        hipLaunchKernelGGL(ee_attend_plan_kernel, dim3(c->n_seqs + p->n_groups), dim3(64), 0, s, a);
        HIP_TRY(hipGetLastError());
    }
    hipLaunchKernelGGL(k.f, dim3(c->n_kv_heads, (unsigned)pl.items), dim3(ATT_W * 64), k.lds, s, a);
    HIP_TRY(hipGetLastError());
    if (pl.part_bytes) {
        const int rows = 256 / (c->head_dim / 4), most = pl.most_own + pl.most_shared, spread = most <= 4 ? 1 : most <= 8 ? 4 : rows;
        const size_t lines = (size_t)p->n_rows * p->n_heads, per = (size_t)(rows / spread);
        hipLaunchKernelGGL(c->head_dim == 64 ? ee_attend_join_kernel<64> : ee_attend_join_kernel<128>, dim3((unsigned)((lines + per - 1) / per)), dim3(256), 0, s, a, spread);
        HIP_TRY(hipGetLastError());
    }
    return EE_OK;
}
