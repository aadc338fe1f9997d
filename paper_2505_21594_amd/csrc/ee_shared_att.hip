// Attention of a verify pass over sessions with pages in common: ee_attend's inner loop over the sessions' caches.
//
// An item is (head, up to 16 lines of one session's rows over its own pages, or of a group's rows over the common ones, a part of those pages); the
// parts of a row's head are joined by a second launch.  What bounds it: 8 sessions with 1024 positions in common, 32 heads of 128, are 46 MB in 25 us
// with the join's launch (53 us when every session's copy is read, 281 MB).  Results differ from ee_att_kernel's in the order of the fp32 sums only.
#include "ee_attend.hpp"

namespace ee {

template <int HD>
__global__ void __launch_bounds__(ATT_W * 64, 2) ee_shared_att_kernel(SharedAtt g)
{
    extern __shared__ __align__(16) char lds_raw[];
    constexpr int NT = HD / 16, TERMS = 2, QT = 3, PT = 3;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lm = lane & 15, quad = lane >> 4, head = blockIdx.x;
    int item = blockIdx.y, s, first_pos = 0, part, parts, slot, chunk = 0, n_lines, pg_lo = 0, pages;
    unsigned long long members = 0;
    const bool shared = item < g.group_items;
    if (shared) {
        int i = 0;
        for (;; ++i) {                                       // (at most ATT_MAX_GROUPS)
            const int n = (g.group[i].n * g.M + 15) / 16 * g.group[i].parts;
            if (item < n) break;
            item -= n;
        }
        parts = g.group[i].parts;
        members = g.group[i].members;
        chunk = item / parts;
        part = item - chunk * parts;
        slot = g.most_own + part;
        n_lines = g.group[i].n * g.M;
        pages = g.group[i].pages;
        s = (int)(members & 15);
    } else {
        item -= g.group_items;
        s = 0;
        while (s + 1 < g.n_sess && g.own[s + 1].first <= item) ++s;
        parts = g.own[s].parts;
        part = item - g.own[s].first;
        slot = part;
        n_lines = g.M;
        pg_lo = g.own[s].from;
    }
    const SessDev *const sd = g.sess + s;
    const int kv_len = as_global(&sd->kv_len)[0], n_pages = as_global(&sd->n_pages)[0];
    if (!shared) {
        first_pos = kv_len;
        pages = (kv_len + g.M + KV_PAGE - 1) / KV_PAGE - pg_lo;
    }
    AttendItem it;
    it.seq = 0;
    it.line0 = chunk * 16;
    it.lines = min(16, n_lines - it.line0);
    it.pg_lo = pg_lo + pages * part / parts;
    it.pg_hi = pg_lo + pages * (part + 1) / parts;
    AttendDev a;
    const size_t layer = (size_t)g.layer * n_pages * g.H * (KV_PAGE * TERMS * HD);
    a.b.kpool = (uint16_t *)as_global(&sd->kpool)[0] + layer;
    a.b.vpool = (uint16_t *)as_global(&sd->vpool)[0] + layer;
    a.b.table = as_global(&sd->page_table)[0];
    a.b.n_pages = a.b.table_stride = n_pages;
    a.b.n_kv_heads = g.H;
    a.q = g.q;
    a.q_stride = g.d;
    a.q_head = HD;
    a.q_type = EE_FP32;
    a.scale2 = g.scale2;
    const int line = it.line0 + min(lm, it.lines - 1), member = shared ? div_small(line, g.M) : 0, i = line - member * g.M;
    const int row[1] = {(shared ? (int)(members >> (4 * member) & 15) : s) * g.M + i}, heads[1] = {head}, last[1] = {shared ? ALL_SEEN : first_pos + i};
    AttendState<1, NT> st;
    attend_clear(st);
    if (it.pg_hi > it.pg_lo) {
        attend_pages<HD, TERMS, QT, PT, 1>(a, it, head, row, heads, last, shared ? ALL_SEEN : first_pos, shared ? ALL_SEEN : first_pos + g.M - 1, lane, wave,
                                           lds_raw + attend_join_lds<HD, 1>(), st);
        attend_join_waves<HD, 1>(st, reinterpret_cast<float *>(lds_raw), min(ATT_W, (it.pg_hi - it.pg_lo + 1) >> 1), lane, wave);
    }
    if (wave != 0 || lm >= it.lines) return;
    if (!shared && parts == 1 && g.own[s].group < 0) {       // the line's only part
        const float inv = 1.0f / st.sum[0];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const float v[4] = {st.o[0][nt][0] * inv, st.o[0][nt][1] * inv, st.o[0][nt][2] * inv, st.o[0][nt][3] * inv};
            store_split4(g.attn, g.rows, row[0], head * HD + nt * 16 + quad * 4, v);
        }
        return;
    }
    const size_t at = ((size_t)row[0] * g.H + head) * (g.most_own + g.most_shared) + slot;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) *as_global_mut(reinterpret_cast<f32x4_t *>(g.part + at * HD + nt * 16 + quad * 4)) = st.o[0][nt];
    if (quad == 0) {
        typedef __attribute__((ext_vector_type(2))) float f32x2_t;
        *as_global_mut(reinterpret_cast<f32x2_t *>(g.ml + at * 2)) = (f32x2_t){st.mx[0], st.sum[0]};
    }
}

// Joins the parts of every row's head, the own ones first, in order: thread = four dims.
template <int HD>
__global__ void __launch_bounds__(256) ee_shared_att_join_kernel(SharedAtt g)
{
    typedef __attribute__((ext_vector_type(2))) float f32x2_t;
    constexpr int TPL = HD / 4;
    const int line = blockIdx.x * (256 / TPL) + threadIdx.x / TPL, e = (threadIdx.x % TPL) * 4;
    if (line >= g.rows * g.H) return;
    const int row = line / g.H, head = line - row * g.H, s = row / g.M, group = g.own[s].group, own = g.own[s].parts;
    const int shared = group < 0 ? 0 : g.group[group].parts, most = g.most_own + g.most_shared;
    if (own == 1 && shared == 0) return;                     // written already
    const f32x2_t *ml = reinterpret_cast<const f32x2_t *>(g.ml) + (size_t)line * most;
    const float *o = g.part + (size_t)line * most * HD + e;
    f32x4_t num = {0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, den = 0.f;
    for (int base = 0; base < own + shared; base += 4) {     // (four parts' loads in flight together)
        f32x2_t x[4];
        f32x4_t v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int p = min(base + i, own + shared - 1), slot = p < own ? p : g.most_own + p - own;
            x[i] = as_global(ml)[slot];
            v[i] = *as_global(reinterpret_cast<const f32x4_t *>(o + (size_t)slot * HD));
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (base + i >= own + shared || x[i][0] == -INFINITY) continue;
            const float m_new = fmaxf(m, x[i][0]), f0 = __builtin_amdgcn_exp2f(m - m_new), f1 = __builtin_amdgcn_exp2f(x[i][0] - m_new);
            m = m_new;
            den = den * f0 + x[i][1] * f1;
#pragma unroll
            for (int r = 0; r < 4; ++r) num[r] = num[r] * f0 + v[i][r] * f1;
        }
    }
    const float inv = 1.0f / den;
    const float v[4] = {num[0] * inv, num[1] * inv, num[2] * inv, num[3] * inv};
    store_split4(g.attn, g.rows, row, head * HD + e, v);
}

void launch_shared_attention(const SharedAtt &a, int hd, int own_items, hipStream_t stream)
{
    const dim3 grid(a.H, a.group_items + own_items), joins((unsigned)((a.rows * a.H + 1024 / hd - 1) / (1024 / hd)));
    if (hd == 128) {
        hipLaunchKernelGGL(ee_shared_att_kernel<128>, grid, dim3(ATT_W * 64), (attend_lds<128, 3, 1>()), stream, a);
        hipLaunchKernelGGL(ee_shared_att_join_kernel<128>, joins, dim3(256), 0, stream, a);
    } else {
        hipLaunchKernelGGL(ee_shared_att_kernel<64>, grid, dim3(ATT_W * 64), (attend_lds<64, 3, 1>()), stream, a);
        hipLaunchKernelGGL(ee_shared_att_join_kernel<64>, joins, dim3(256), 0, stream, a);
    }
}

}  // namespace ee
