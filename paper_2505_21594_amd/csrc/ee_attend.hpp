// ee_attend: attention of new rows over paged caches, pages that sequences have in common read once for all of them.
//
//   out_i = sum_j softmax_j(scale q_i . k_j) v_j  over the positions a row sees, as one pass over the keys and values with a running
//   maximum m and sum l:  m' = max(m, s_j),  l' = l e^(m - m') + e^(s_j - m'),  o' = o e^(m - m') + e^(s_j - m') v_j;
//   parts of the positions join by the same rule.
//
// A line is a row's query head.  The lines that read one key head are taken in tiles of 16, an item is (key head, a chunk of lines of one sequence, or of
// one group over its common pages, a part of their pages) and goes to a workgroup.  Both products are v_mfma_f32_16x16x32_bf16, 32 positions (a
// pair of pages) at a time:
//   scores   S[position][line] = K . q^T    A = 16 positions x 32 values, B = q.  Row r of product p is position 8 (r >> 2) + 4 p + (r & 3) of the pair, so that
//            a lane's scores of both products are the eight positions 8 quad .. 8 quad + 7 (quad = lane >> 4, line = lane & 15) ...
//   output   O[dim][line] = V^T . P         ... which is the layout of the second product's B: P stays in its registers, and V, which a record holds
//            transposed, comes as one 16-byte access of eight positions.
// The output is kept transposed: a line's maximum, sum and output are in the lanes of its column, and rescaling needs no exchange.
//
// Precision: sums, maxima and outputs are fp32.  The products' operands are bf16 terms: K and V as the cache has them (TERMS), q in QT terms, exactly for bf16 (1) and
// fp16 (2) and to 2^-24 for fp32 (3); P in PT: 3 where the results are fp32 (2^-24), 2 (2^-16, a 256th of the result's own rounding) for results of 16 bits.
// (One term, 2^-8, for bf16 results of many lines: 2041 rows of 32 heads 60.3 us instead of 72.0, and 1.3 times the error of exact weights.)  Products of the smallest
// terms are left out (2^-24, or 2^-16 with 2 terms).
#pragma once

#include <type_traits>

#include "ee_ops.hpp"

namespace ee {

constexpr int ATT_W = 4;                       // waves of an item

struct AttendDev {
    BatchDev b;
    const void *q;
    void *out;
    long long q_stride, q_head, o_stride, o_head;
    const int *group_start, *group_pages;
    float *part;                               // [line of the batch][most_own + most_shared][HD]
    float2 *part_ml;                           // [line][1 + most_own + most_shared]: first (own parts, common parts) as integers, then maxima and sums
    int *from, *common, *member;               // per sequence / group, where ee_attend_plan_kernel works them out
    int q_type, out_type;
    int n_groups, n_heads, per_key;            // per_key: query heads of a key head
    int quota;                                 // pages of a part
    int most_own, most_shared;                 // parts at most
    float scale2;                              // scale * log2(e)
};

// What one item works on.
struct AttendItem {
    int seq;                                   // whose table is read
    int row0, rows;                            // rows the chunk's lines belong to: of the sequence, or of the group
    int line0, lines;                          // its lines among them
    int pg_lo, pg_hi;                          // its pages
    int first_pos;                             // position of row0; rows of a group: they see all pages of the item
    bool shared;
    int own_parts, common_parts, slot;         // parts of its lines, and which of them this is
};

constexpr int ALL_SEEN = 0x7FFFFFF0;

__device__ __forceinline__ int group_bound(const AttendDev &a, int g) { return min(max(as_global(a.group_start)[g], 0), a.b.n_seqs); }

// A sequence as its lane holds it.
struct SeqLane {
    int r0, n, len, from;                      // first row, rows, positions, pages that its group reads for it
};
__device__ __forceinline__ SeqLane seq_lane(const AttendDev &a, int s)
{
    SeqLane l = {0, 0, 0, 0};
    if (s < a.b.n_seqs) {
        l.r0 = a.b.start(s);
        l.n = max(a.b.start(s + 1) - l.r0, 0);
        l.len = a.b.length(s);
    }
    return l;
}
// pages of which every new row sees all positions
__device__ __forceinline__ int pages_seen(const SeqLane &l) { return l.n > 0 ? max(l.len - l.n + 1, 0) >> 4 : 0x7FFFFFFF; }

// Pages that a group reads together: the entries its members have in common, as far as every new row of every member sees all of
// their positions.  `member`: the first one with rows, whose table is read; s1 if there is none.
__device__ __forceinline__ int common_pages(const AttendDev &a, int group, int lane, int &member)
{
    const int s0 = group_bound(a, group), s1 = max(group_bound(a, group + 1), s0);
    int pages = min(max(as_global(a.group_pages)[group], 0), a.b.table_stride);
    member = s1;
    for (int base = s0; base < s1; base += 64) {
        SeqLane l = seq_lane(a, base + lane);
        if (base + lane >= s1) l.n = 0;
        if (const unsigned long long who = __ballot(l.n > 0); who && member == s1) member = base + __builtin_ctzll(who);
        pages = min(pages, wave_min(pages_seen(l)));
    }
    return member < s1 ? __builtin_amdgcn_readfirstlane(pages) : 0;
}

// Batches of more than 64 sequences: `from`, `common` and `member`, one wave each.
static __global__ void __launch_bounds__(64) ee_attend_plan_kernel(AttendDev a)
{
    const int lane = threadIdx.x, i = blockIdx.x;
    int member;
    if (i < a.n_groups) {
        const int pages = common_pages(a, i, lane, member);
        if (lane == 0) {
            as_global_mut(a.common)[i] = pages;
            as_global_mut(a.member)[i] = member;
        }
        return;
    }
    const int s = i - a.n_groups;
    int pages = 0;
    for (int base = 0; base < a.n_groups; base += 64) {
        const int g = base + lane;
        const bool in = g < a.n_groups && group_bound(a, g) <= s && s < group_bound(a, g + 1);
        if (const unsigned long long who = __ballot(in)) {
            pages = common_pages(a, base + __builtin_ctzll(who), lane, member);
            break;
        }
    }
    if (lane == 0) as_global_mut(a.from)[s] = pages;
}

__device__ __forceinline__ int own_parts(const AttendDev &a, int pages) { return min(max((pages + a.quota - 1) / a.quota, 1), a.most_own); }
__device__ __forceinline__ int common_parts(const AttendDev &a, int pages) { return min((pages + a.quota - 1) / a.quota, a.most_shared); }
__device__ __forceinline__ int table_pages(const AttendDev &a, int len) { return (min(max(len, 0), a.b.capacity()) + KV_PAGE - 1) >> 4; }

// Item `item` of the launch: the groups' chunks and parts first, then the sequences'.  All lanes get the same; false past the last.
template <int LINES>
__device__ __forceinline__ bool attend_item(const AttendDev &a, int item, int lane, AttendItem &it)
{
    const int G = a.per_key;
    const bool small = a.b.n_seqs <= 64 && a.n_groups <= 64;
    SeqLane mine = seq_lane(a, lane);
    int g_pages = 0, g_member = 0, g_r0 = 0, g_rows = 0;                    // of group `lane`
    auto group_rows = [&](int g, int &r0, int &rows) {
        const int s0 = group_bound(a, g), s1 = max(group_bound(a, g + 1), s0);
        r0 = a.b.start(s0);
        rows = max(a.b.start(s1) - r0, 0);
    };
    auto shared_count = [&](int pages, int rows) { return pages > 0 ? (rows * G + LINES - 1) / LINES * common_parts(a, pages) : 0; };
    if (a.n_groups > 0) {
        int g, place;
        if (small) {
            int s0 = 0, declared = 0;
            if (lane <= a.n_groups) s0 = group_bound(a, lane);
            if (lane < a.n_groups) {
                declared = min(max(as_global(a.group_pages)[lane], 0), a.b.table_stride);
                group_rows(lane, g_r0, g_rows);
            }
            const int seen = pages_seen(mine);
            for (int i = 0; i < a.n_groups; ++i) {
                const int lo = __builtin_amdgcn_readlane(s0, i), hi = i == 63 ? group_bound(a, 64) : __builtin_amdgcn_readlane(s0, i + 1);
                const bool in = lane >= lo && lane < hi;
                const unsigned long long who = __ballot(in && mine.n > 0);
                const int pages = who ? min(__builtin_amdgcn_readlane(declared, i), wave_min(in ? seen : 0x7FFFFFFF)) : 0;
                if (in) mine.from = pages;
                if (lane == i) {
                    g_pages = pages;
                    g_member = who ? __builtin_ctzll(who) : 0;
                }
            }
            const int c = shared_count(g_pages, g_rows), incl = wave_scan(c), total = __builtin_amdgcn_readlane(incl, 63);
            if (item < total) {
                g = __builtin_ctzll(__ballot(incl > item));
                place = item - __builtin_amdgcn_readlane(incl - c, g);
                it.seq = __builtin_amdgcn_readlane(g_member, g);
                it.row0 = __builtin_amdgcn_readlane(g_r0, g);
                it.rows = __builtin_amdgcn_readlane(g_rows, g);
                g_pages = __builtin_amdgcn_readlane(g_pages, g);
                it.shared = true;
            } else {
                item -= total;
                it.shared = false;
            }
        } else {
            int total = 0;
            it.shared = find_item(a.n_groups, item, lane, [&](int i) {
                int r0, rows;
                group_rows(i, r0, rows);
                return shared_count(as_global(a.common)[i], rows);
            }, g, place, &total);
            if (it.shared) {
                group_rows(g, it.row0, it.rows);
                g_pages = as_global(a.common)[g];
                it.seq = as_global(a.member)[g];
            } else {
                item -= total;
            }
        }
        if (it.shared) {
            const int parts = common_parts(a, g_pages), chunk = place / parts, part = place - chunk * parts;
            it.line0 = chunk * LINES;
            it.lines = min(LINES, it.rows * G - it.line0);
            it.pg_lo = (int)((long long)g_pages * part / parts);
            it.pg_hi = (int)((long long)g_pages * (part + 1) / parts);
            it.first_pos = ALL_SEEN;
            it.own_parts = it.common_parts = 2;                             // (never the only part)
            it.slot = a.most_own + part;
            return true;
        }
    }
    it.shared = false;
    auto own_count = [&](const SeqLane &l) { return l.n > 0 ? (l.n * G + LINES - 1) / LINES * own_parts(a, table_pages(a, l.len) - l.from) : 0; };
    for (int base = 0;; base += 64) {
        if (base > 0) mine = seq_lane(a, base + lane);
        if (!small && a.n_groups > 0 && base + lane < a.b.n_seqs) mine.from = as_global(a.from)[base + lane];
        const int c = own_count(mine), incl = wave_scan(c), total = __builtin_amdgcn_readlane(incl, 63);
        if (item < total) {
            const int l = __builtin_ctzll(__ballot(incl > item)), place = item - __builtin_amdgcn_readlane(incl - c, l);
            it.seq = base + l;
            it.row0 = __builtin_amdgcn_readlane(mine.r0, l);
            it.rows = __builtin_amdgcn_readlane(mine.n, l);
            const int len = __builtin_amdgcn_readlane(mine.len, l), from = __builtin_amdgcn_readlane(mine.from, l);
            const int parts = own_parts(a, table_pages(a, len) - from);
            // the last lines first: they see the most positions
            const int chunks = (it.rows * G + LINES - 1) / LINES, c_up = place / parts, part = place - c_up * parts;
            it.line0 = (chunks - 1 - c_up) * LINES;
            it.lines = min(LINES, it.rows * G - it.line0);
            it.first_pos = len - it.rows;
            const int pages = max(table_pages(a, it.first_pos + (it.line0 + it.lines - 1) / G + 1) - from, 0);
            it.pg_lo = from + (int)((long long)pages * part / parts);
            it.pg_hi = from + (int)((long long)pages * (part + 1) / parts);
            it.own_parts = parts;
            it.common_parts = from > 0 ? common_parts(a, from) : 0;
            it.slot = part;
            return true;
        }
        item -= total;
        if (base + 64 >= a.b.n_seqs) return false;
    }
}

template <int RT, int NT>
struct AttendState {
    f32x4_t o[RT][NT];
    float mx[RT], sum[RT];                     // of the scores times scale2; the sums are the lane's own until the end
    unsigned hollow;                           // bit t: this lane saw positions of its line of tile t, but no score above -infinity yet
};

template <int RT, int NT>
__device__ __forceinline__ void attend_clear(AttendState<RT, NT> &st)
{
    st.hollow = 0;
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        st.mx[t] = -INFINITY;
        st.sum[t] = 0.f;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) st.o[t][nt] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
    }
}

// Bits 15 and 31 are set where the low and the high element are infinite or NaN (a full exponent carries out of its field); other bits are anything.
__device__ __forceinline__ uint32_t nonfinite_carry(uint32_t w) { return (w & 0x7F807F80u) + 0x00800080u; }
__device__ __forceinline__ uint32_t nonfinite_carry(uint4 v) { return nonfinite_carry(v.x) | nonfinite_carry(v.y) | nonfinite_carry(v.z) | nonfinite_carry(v.w); }
__device__ __forceinline__ bool nonfinite(uint32_t carries) { return (carries & 0x80008000u) != 0; }
// bits of the first `keep` of two elements
__device__ __forceinline__ uint32_t keep_mask(int keep) { return keep >= 2 ? 0xFFFFFFFFu : keep == 1 ? 0xFFFFu : 0u; }
__device__ __forceinline__ uint4 keep_first(uint4 v, int keep)
{
    return make_uint4(v.x & keep_mask(keep), v.y & keep_mask(keep - 2), v.z & keep_mask(keep - 4), v.w & keep_mask(keep - 6));
}
// bits of the elements that are infinite or NaN
__device__ __forceinline__ uint32_t nonfinite_bits(uint32_t w) { return (nonfinite_carry(w) >> 15 & 0x00010001u) * 0xFFFFu; }
__device__ __forceinline__ uint4 nonfinite_bits(uint4 v) { return make_uint4(nonfinite_bits(v.x), nonfinite_bits(v.y), nonfinite_bits(v.z), nonfinite_bits(v.w)); }

// eight values as N bf16 terms
template <int N>
__device__ __forceinline__ void split_terms(const float (&x)[8], bf16x8_t (&t)[N])
{
    uint32_t w[N][4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        float a = x[2 * e], b = x[2 * e + 1];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            w[i][e] = pack_bf16(a, b);
            if (i + 1 < N) {
                a -= __uint_as_float(w[i][e] << 16);
                b -= __uint_as_float(w[i][e] & 0xFFFF0000u);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) t[i] = __builtin_bit_cast(bf16x8_t, make_uint4(w[i][0], w[i][1], w[i][2], w[i][3]));
}

// What a pair of pages leaves to be seen: positions of either page that exist for any line of the wave (uniform), whether
// anything of the pair is hidden from any line, and how many of the lane's positions 8 quad .. of the pair exist.
struct PairMask {
    int lim0, lim1;
    bool masked;
    __device__ __forceinline__ int keep(int quad) const { return min(max((quad < 2 ? lim0 : lim1) - (quad & 1) * 8, 0), 8); }
};
__device__ __forceinline__ PairMask pair_mask(int pos0, int id0, int id1, int first_last, int max_last)
{
    PairMask m;
    m.lim0 = id0 >= 0 ? min(max(max_last + 1 - pos0, 0), KV_PAGE) : 0;
    m.lim1 = id1 >= 0 ? min(max(max_last + 1 - pos0 - KV_PAGE, 0), KV_PAGE) : 0;
    m.masked = m.lim0 < KV_PAGE || m.lim1 < KV_PAGE || first_last < pos0 + 2 * KV_PAGE - 1;
    return m;
}

// Scores of a tile -> weights in z, with the running maximum and sum brought up to date.  Any number near the maximum serves as well: it is
// moved (and the output rescaled) only where some line's scores exceed it by ATT_SLACK powers of two, after which weights are at most 2^ATT_SLACK.
// The scores are therefore taken relative to the number in use right away, and the largest is found among those.
constexpr float ATT_SLACK = 8.f;
__device__ __forceinline__ float attend_base(float mx) { return mx == -INFINITY ? 0.f : mx; }
template <int NP, int RT, int NT>
__device__ __forceinline__ void attend_raise(AttendState<RT, NT> &st, int t, float local, float (&z)[NP][8])
{
    const float base = attend_base(st.mx[t]), m = fmaxf(st.mx[t], base + local), up = m == -INFINITY ? 0.f : m - base;
    const float f = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(st.mx[t] - m);
    st.mx[t] = m;
    st.sum[t] *= f;
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
        for (int e = 0; e < 8; ++e) z[p][e] -= up;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int r = 0; r < 4; ++r) st.o[t][nt][r] *= f;
}
template <int PT, int NP, int RT, int NT>
__device__ __forceinline__ void attend_exps(AttendState<RT, NT> &st, int t, float (&z)[NP][8], bf16x8_t (&P)[NP][PT])
{
#pragma unroll
    for (int p = 0; p < NP; ++p) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            z[p][e] = __builtin_amdgcn_exp2f(z[p][e]);
            st.sum[t] += z[p][e];
        }
        split_terms<PT>(z[p], P[p]);
    }
}

// A tile's scores of NP pairs, times scale2 and relative to the running maximum, as the lane's eights.  MASKED: those that its line does not see are
// nothing; keep: of the lane's positions of a pair, those that exist.  Returns the largest, and in `up` whether the maximum has to move.
template <bool MASKED, int NP, int RT, int NT>
__device__ __forceinline__ float attend_scores(AttendState<RT, NT> &st, int t, const f32x4_t (&S)[NP][2], const int (&keep)[NP], int pos0, int last, int quad, float scale2,
                                               float (&z)[NP][8], bool &up)
{
    bool sees = false;
    const float base = attend_base(st.mx[t]);
    float local = -INFINITY;
#pragma unroll
    for (int p = 0; p < NP; ++p) {
        const int seen = min(keep[p], last - pos0 - p * 32 - quad * 8 + 1);
        sees |= seen > 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            z[p][e] = fmaf(S[p][e >> 2][e & 3], scale2, -base);
            if constexpr (MASKED) z[p][e] = e < seen ? z[p][e] : -INFINITY;
        }
#pragma unroll
        for (int e = 0; e < 8; e += 2) local = fmaxf(fmaxf(local, z[p][e]), z[p][e + 1]);
    }
    local = quads_max(local);
    up |= local > (st.mx[t] == -INFINITY ? -INFINITY : ATT_SLACK);
    if (local == -INFINITY && (!MASKED || sees)) st.hollow |= 1u << t;     // (counts only where the maximum stays there)
    return local;
}

// A pair of which some lines see a position that others do not, and in which V holds an infinity or NaN: 0 * V would be NaN for the
// others.  Such elements leave the product (for both of their terms) and make NaN of the lines that see them.  v: the lane's
// elements of dim nt * 16 + lm.
template <int TERMS, int RT, int NT>
__device__ __forceinline__ void attend_odd(AttendState<RT, NT> &st, int nt, uint4 (&v)[TERMS], int pos0, const int (&last)[RT], int quad)
{
    uint4 odd = nonfinite_bits(v[0]);
    if constexpr (TERMS == 2) {
        const uint4 o = nonfinite_bits(v[1]);
        odd = make_uint4(odd.x | o.x, odd.y | o.y, odd.z | o.z, odd.w | o.w);
    }
#pragma unroll
    for (int u = 0; u < TERMS; ++u) v[u] = make_uint4(v[u].x & ~odd.x, v[u].y & ~odd.y, v[u].z & ~odd.z, v[u].w & ~odd.w);
    const uint32_t w[4] = {odd.x, odd.y, odd.z, odd.w};
    int first = ALL_SEEN + 1;                                               // first such position of the dim
#pragma unroll
    for (int e = 7; e >= 0; --e)
        if (w[e >> 1] >> 16 * (e & 1) & 1) first = pos0 + quad * 8 + e;
    first = min(first, __shfl_xor(first, 16, 64));
    first = min(first, __shfl_xor(first, 32, 64));
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int at = __shfl(first, quad * 4 + r, 64);
#pragma unroll
        for (int t = 0; t < RT; ++t)
            if (last[t] >= at) st.o[t][nt][r] = __builtin_nanf("");
    }
}

// A pair's V where something of the pair is hidden: what no line sees may hold anything, and what some lines see and others do not, infinities and NaN.
template <int TERMS, int RT, int NT>
__device__ __forceinline__ void attend_clean_v(AttendState<RT, NT> &st, uint4 (&v)[NT][TERMS], const PairMask &mask, int keep, int pos0, const int (&last)[RT], int quad)
{
    if constexpr (TERMS == 2) {                                             // (registers are short there: one dim tile after the other)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            v[nt][0] = keep_first(v[nt][0], keep);
            v[nt][1] = keep_first(v[nt][1], keep);
            if (__any(nonfinite(nonfinite_carry(v[nt][0]) | nonfinite_carry(v[nt][1])))) attend_odd<TERMS>(st, nt, v[nt], pos0, last, quad);
        }
    } else {
        if (mask.lim0 < KV_PAGE || mask.lim1 < KV_PAGE) {                   // (uniform)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) v[nt][0] = keep_first(v[nt][0], keep);
        }
        uint32_t odd = 0;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) odd |= nonfinite_carry(v[nt][0]);
        if (__any(nonfinite(odd))) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) attend_odd<TERMS>(st, nt, v[nt], pos0, last, quad);
        }
    }
}

// A lane's q of a line as operands: values 32 kt + 8 quad .. + 7.
template <int QT>
__device__ __forceinline__ void attend_load_q(const AttendDev &a, int row, int head, int kt, int quad, bf16x8_t (&q)[QT])
{
    const size_t at = (size_t)row * a.q_stride + (size_t)head * a.q_head + kt * 32 + quad * 8;
    if constexpr (QT == 1) {
        q[0] = __builtin_bit_cast(bf16x8_t, load_global16(static_cast<const uint16_t *>(a.q) + at));
    } else {
        float x[8];
        if (a.q_type == EE_FP32)
            load8<EE_FP32>(a.q, at, x);
        else if (a.q_type == EE_FP16)
            load8<EE_FP16>(a.q, at, x);
        else
            load8<EE_BF16>(a.q, at, x);
        split_terms<QT>(x, q);
    }
}

// One line's result: the output where this is its only part, a part of it otherwise.
template <int RT, int NT>
__device__ __forceinline__ void attend_store(const AttendDev &a, const AttendItem &it, const AttendState<RT, NT> &st, int t, int row, int head, int quad)
{
    constexpr int HD = NT * 16;
    const size_t line = (size_t)row * a.n_heads + head;
    const int most = a.most_own + a.most_shared;
    const bool alone = it.own_parts == 1 && it.common_parts == 0;
    if (alone) {
        const float inv = st.sum[t] == 0.f ? 0.f : 1.0f / st.sum[t];        // (0: the line saw no position)
        const size_t to = (size_t)row * a.o_stride + (size_t)head * a.o_head + quad * 4;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) store4(a.out_type, a.out, to + nt * 16, st.o[t][nt][0] * inv, st.o[t][nt][1] * inv, st.o[t][nt][2] * inv, st.o[t][nt][3] * inv);
    } else if (st.mx[t] != -INFINITY) {                                     // (nothing is read of an empty part)
        float *o = a.part + (line * most + it.slot) * HD + quad * 4;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) *as_global_mut(reinterpret_cast<f32x4_t *>(o + nt * 16)) = st.o[t][nt];
    }
    if (quad == 0 && most > 1) {
        typedef __attribute__((ext_vector_type(2))) float f32x2_t;
        f32x2_t *ml = reinterpret_cast<f32x2_t *>(a.part_ml + line * (most + 1));
        if (!alone) as_global_mut(ml)[1 + it.slot] = (f32x2_t){st.mx[t], st.sum[t]};
        if (it.slot == 0) as_global_mut(ml)[0] = (f32x2_t){__int_as_float(alone ? 0 : it.own_parts), __int_as_float(it.common_parts)};
    }
}

// The sums of a line's lanes, and NaN where it saw positions but no score above -infinity: it has no softmax.  Scores of NaN have left NaN in the sum,
// but no maximum: with any maximum the part counts, and the line becomes NaN.
template <int RT, int NT>
__device__ __forceinline__ void attend_finish(AttendState<RT, NT> &st)
{
    st.hollow = quads_or(st.hollow);
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        st.sum[t] = quads_sum(st.sum[t]);
        if (st.mx[t] != -INFINITY) continue;
        if (st.sum[t] != st.sum[t])
            st.mx[t] = 0.f;
        else if (st.hollow >> t & 1)
            st.sum[t] = __builtin_nanf("");
    }
}

// Two parts' sums as one: 0 where a part saw no position, NaN where it saw none with a score above -infinity (which says nothing
// beside a part with one).
__device__ __forceinline__ float join_sums(float m, float m1, float l1, float f1, float m2, float l2, float f2)
{
    if (m == -INFINITY) return l1 + l2;
    return (m1 == -INFINITY ? 0.f : l1 * f1) + (m2 == -INFINITY ? 0.f : l2 * f2);
}

// ------------------------------------------------------------------ few lines: bound by the cache's bytes
//
// The waves take the item's pairs of pages in turn, K and V straight from the records into registers: K of the next pair is requested when this
// one's scores are done, V when its product is.  q of 128 values and several terms or tiles is in LDS: in registers it would leave
// room for one workgroup a compute unit instead of two.

template <int HD, int QT, int RT>
constexpr bool attend_q_in_lds() { return HD == 128 && (QT > 1 || RT > 1); }

template <int HD, int TERMS, int QT, int PT, int RT>
__device__ __forceinline__ void attend_pages(const AttendDev &a, const AttendItem &it, int kvh, const int (&row)[RT], const int (&head)[RT], const int (&last)[RT], int first_last,
                                             int max_last, int lane, int wave, char *q_lds, AttendState<RT, HD / 16> &st)
{
    constexpr bool Q_LDS = attend_q_in_lds<HD, QT, RT>();
    constexpr int KT = HD / 32, NT = HD / 16, ID_PAIRS = 32;
    const int lm = lane & 15, quad = lane >> 4;
    const int pairs = (it.pg_hi - it.pg_lo + 1) >> 1, tiles = (it.lines + 15) >> 4;
    const size_t page_step = (size_t)a.b.n_kv_heads * KV_PAGE * TERMS * HD;
    const int *table = a.b.table + (size_t)it.seq * a.b.table_stride;
    int pr = wave;
    // ids of the wave's next 32 pairs, one page a lane; -1 outside the pools and past the item's last page
    int ids, ids_from = pr;
    auto load_ids = [&]() __attribute__((always_inline)) {
        const int pg = it.pg_lo + 2 * (ids_from + (lane >> 1) * ATT_W) + (lane & 1);
        ids = pg < it.pg_hi ? as_global(table)[pg] : -1;
        if (ids >= a.b.n_pages) ids = -1;
    };
    int id0, id1;
    auto find_ids = [&](int p) __attribute__((always_inline)) {
        const int i = (p - ids_from) / ATT_W * 2;
        id0 = __builtin_amdgcn_readlane(ids, i);
        id1 = __builtin_amdgcn_readlane(ids, i + 1);
    };
    // operand rows of K: page lm >> 3, position 8 ((lm >> 2) & 1) + 4 p + (lm & 3) of it; V: page quad >> 1, positions 8 (quad & 1) .. + 7
    const uint16_t *k0 = a.b.kpool + (size_t)kvh * KV_PAGE * TERMS * HD + ((lm >> 2 & 1) * 8 + (lm & 3)) * (TERMS * HD) + quad * 8;
    const uint16_t *v0 = a.b.vpool + (size_t)kvh * KV_PAGE * TERMS * HD + lm * KV_PAGE + (quad & 1) * 8;
    uint4 kf[2][TERMS][KT], vf[NT][TERMS];
    auto request_k = [&]() __attribute__((always_inline)) {
        const uint16_t *kb = k0 + (size_t)max(lm < 8 ? id0 : id1, 0) * page_step;
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int u = 0; u < TERMS; ++u)
#pragma unroll
                for (int kt = 0; kt < KT; ++kt) kf[p][u][kt] = load_global16(kb + p * 4 * TERMS * HD + u * HD + kt * 32);
    };
    auto request_v = [&]() __attribute__((always_inline)) {
        const uint16_t *vb = v0 + (size_t)max(quad < 2 ? id0 : id1, 0) * page_step;
#pragma unroll
        for (int u = 0; u < TERMS; ++u)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) vf[nt][u] = load_global16(vb + (u * HD + nt * 16) * KV_PAGE);
    };
    bf16x8_t q[Q_LDS ? 1 : RT][Q_LDS ? 1 : KT][QT];
    if constexpr (Q_LDS) {
        // wave w prepares values 32 w .. of all lines
        static_assert(KT == ATT_W, "a wave for each 32 values");
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            if (t >= tiles) continue;
            attend_load_q<QT>(a, row[t], head[t], wave, quad, q[0][0]);
#pragma unroll
            for (int i = 0; i < QT; ++i) *reinterpret_cast<bf16x8_t *>(q_lds + (((t * KT + wave) * QT + i) * 64 + lane) * 16) = q[0][0][i];
        }
    } else {
#pragma unroll
        for (int t = 0; t < RT; ++t)
            if (t < tiles) {
#pragma unroll
                for (int kt = 0; kt < KT; ++kt) attend_load_q<QT>(a, row[t], head[t], kt, quad, q[t][kt]);
            }
    }
    if (pr < pairs) {
        load_ids();
        find_ids(pr);
        request_k();
        request_v();
    }
    if constexpr (Q_LDS) lds_barrier();
    if (pr >= pairs) return;
    for (;;) {
        if constexpr (Q_LDS) asm volatile("" ::: "memory");                 // (or the loop's reads of q would move in front of it, into registers)
        const int pos0 = (it.pg_lo + 2 * pr) * KV_PAGE;
        const PairMask mask = pair_mask(pos0, id0, id1, first_last, max_last);
        f32x4_t S[RT][1][2];
#pragma unroll
        for (int t = 0; t < RT; ++t) S[t][0][0] = S[t][0][1] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                if (t >= tiles) continue;
                bf16x8_t x[QT];
#pragma unroll
                for (int i = 0; i < QT; ++i) x[i] = Q_LDS ? *reinterpret_cast<const bf16x8_t *>(q_lds + (((t * KT + kt) * QT + i) * 64 + lane) * 16) : q[Q_LDS ? 0 : t][Q_LDS ? 0 : kt][i];
#pragma unroll
                for (int p = 0; p < 2; ++p)
#pragma unroll
                    for (int u = 0; u < TERMS; ++u)
#pragma unroll
                        for (int i = 0; i < QT - u; ++i) S[t][0][p] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, kf[p][u][kt]), x[i], S[t][0][p], 0, 0, 0);
            }
        pr += ATT_W;
        const bool more = pr < pairs;
        if (more) {
            if (pr - ids_from >= ID_PAIRS * ATT_W) {
                ids_from = pr;
                load_ids();
            }
            find_ids(pr);
            request_k();
        }
        auto multiply = [&](auto masked) __attribute__((always_inline)) {
            constexpr bool MASKED = decltype(masked)::value;
            const int keep[1] = {mask.keep(quad)};
            bf16x8_t P[RT][1][PT];
            float s[RT][1][8], local[RT];
            bool up = false;
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                local[t] = -INFINITY;
                if (t < tiles) local[t] = attend_scores<MASKED, 1>(st, t, S[t], keep, pos0, last[t], quad, a.scale2, s[t], up);
            }
            if (__any(up)) {
#pragma unroll
                for (int t = 0; t < RT; ++t)
                    if (t < tiles) attend_raise(st, t, local[t], s[t]);
            }
#pragma unroll
            for (int t = 0; t < RT; ++t)
                if (t < tiles) attend_exps<PT, 1>(st, t, s[t], P[t]);
            if constexpr (MASKED)
                if (mask.masked) attend_clean_v<TERMS>(st, vf, mask, keep[0], pos0, last, quad);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int u = 0; u < TERMS; ++u) {
                    const bf16x8_t v = __builtin_bit_cast(bf16x8_t, vf[nt][u]);
#pragma unroll
                    for (int t = 0; t < RT; ++t) {
                        if (t >= tiles) continue;
#pragma unroll
                        for (int i = 0; i < PT - u; ++i) st.o[t][nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, P[t][0][i], st.o[t][nt], 0, 0, 0);
                    }
                }
        };
        // (two copies of this, but for two-term caches, where they need more registers than two workgroups a compute unit leave)
        if (TERMS == 2 || mask.masked)
            multiply(std::true_type{});
        else
            multiply(std::false_type{});
        if (!more) break;
        request_v();
    }
    attend_finish(st);
}

// floats per lane that a wave hands over
template <int HD, int RT>
constexpr int attend_lds_floats() { return RT * (HD / 16) * 4 + 2 * RT; }
template <int HD, int RT>
constexpr size_t attend_join_lds() { return (size_t)(ATT_W / 2) * 64 * attend_lds_floats<HD, RT>() * sizeof(float); }
template <int HD, int QT, int RT>
constexpr size_t attend_lds()
{
    constexpr size_t bytes = attend_join_lds<HD, RT>() + (attend_q_in_lds<HD, QT, RT>() ? RT * (HD / 32) * QT * 1024 : 0);
    static_assert(bytes <= 65536, "what a launch gets without asking for more");
    return bytes;
}

// Joins the waves' results into wave 0's, halves of them at a time; `active`: waves that had pages.
template <int HD, int RT>
__device__ __forceinline__ void attend_join_waves(AttendState<RT, HD / 16> &st, float *lds, int active, int lane, int wave)
{
    constexpr int NT = HD / 16;
#pragma unroll
    for (int half = ATT_W / 2; half >= 1; half >>= 1) {
        if (active <= half) continue;                                       // (uniform over the workgroup)
        float *slot = lds + (size_t)((wave & (half - 1)) * attend_lds_floats<HD, RT>()) * 64 + lane * 4;
        float *ml = lds + (size_t)((wave & (half - 1)) * attend_lds_floats<HD, RT>() + RT * NT * 4) * 64 + lane;
        if (wave >= half && wave < 2 * half) {
#pragma unroll
            for (int t = 0; t < RT; ++t) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) *reinterpret_cast<f32x4_t *>(slot + (t * NT + nt) * 256) = st.o[t][nt];
                ml[(2 * t) * 64] = st.mx[t];
                ml[(2 * t + 1) * 64] = st.sum[t];
            }
        }
        __syncthreads();
        if (wave < half) {
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                const float m2 = ml[(2 * t) * 64], l2 = ml[(2 * t + 1) * 64];
                const float m = fmaxf(st.mx[t], m2), base = m == -INFINITY ? 0.f : m;
                const float f1 = __builtin_amdgcn_exp2f(st.mx[t] - base), f2 = __builtin_amdgcn_exp2f(m2 - base);
                st.sum[t] = join_sums(m, st.mx[t], st.sum[t], f1, m2, l2, f2);
                st.mx[t] = m;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const f32x4_t o2 = *reinterpret_cast<const f32x4_t *>(slot + (t * NT + nt) * 256);
#pragma unroll
                    for (int r = 0; r < 4; ++r) st.o[t][nt][r] = st.o[t][nt][r] * f1 + o2[r] * f2;
                }
            }
        }
        __syncthreads();
    }
}

template <int HD, int TERMS, int QT, int PT, int RT>
__global__ void __launch_bounds__(ATT_W * 64, 2) ee_attend_kernel(AttendDev a)
{
    extern __shared__ __align__(16) char lds_raw[];
    constexpr int NT = HD / 16;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lm = lane & 15, quad = lane >> 4, kvh = blockIdx.x;
    AttendItem it;
    if (!attend_item<RT * 16>(a, blockIdx.y, lane, it)) return;
    // this lane's lines: row, head, last position seen
    int row[RT], head[RT], last[RT];
    const int i0 = it.line0 / a.per_key, l0 = it.line0 - i0 * a.per_key;    // row of the chunk's first line, and which of its lines that is
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        const int l = l0 + min(t * 16 + lm, it.lines - 1), i = div_small(l, a.per_key);
        row[t] = it.row0 + i0 + i;
        head[t] = kvh * a.per_key + l - i * a.per_key;
        last[t] = it.shared ? ALL_SEEN : it.first_pos + i0 + i;
    }
    AttendState<RT, NT> st;
    attend_clear(st);
    if (it.pg_hi > it.pg_lo) {
        const int first_last = it.shared ? ALL_SEEN : it.first_pos + i0;
        const int max_last = it.shared ? ALL_SEEN : min(it.first_pos + i0 + __builtin_amdgcn_readfirstlane(div_small(l0 + it.lines - 1, a.per_key)), a.b.capacity() - 1);
        attend_pages<HD, TERMS, QT, PT, RT>(a, it, kvh, row, head, last, first_last, max_last, lane, wave, lds_raw + attend_join_lds<HD, RT>(), st);
        attend_join_waves<HD, RT>(st, reinterpret_cast<float *>(lds_raw), min(ATT_W, (it.pg_hi - it.pg_lo + 1) >> 1), lane, wave);
    }
    if (wave != 0) return;
#pragma unroll
    for (int t = 0; t < RT; ++t)
        if (t * 16 + lm < it.lines) attend_store(a, it, st, t, row[t], head[t], quad);
}

// ------------------------------------------------------------------ many lines: bound by the matrix cores
//
// Four waves have 32 lines each; K and V of a step of 64 positions (32 of a two-term cache) go through LDS for all of them, straight from the
// records into operand order, the next step's on their way while this one is multiplied.  Two workgroups share a compute unit where the registers allow it:
// one fills the matrix cores while the other has its exponentials.  (Heads of 128 spill 40 bytes for that: the results' places, stored before the loop
// and loaded behind it.)

constexpr int ATT_WIDE = 128;                  // lines of an item
template <int TERMS>
constexpr int attend_wide_pairs() { return TERMS == 1 ? 2 : 1; }
template <int HD, int TERMS>
constexpr int attend_wide_pair() { return 32 * TERMS * HD * 4; }                                    // bytes of a pair's K and V
template <int HD, int TERMS>
constexpr size_t attend_wide_lds()
{
    static_assert(2 * attend_wide_pairs<TERMS>() * attend_wide_pair<HD, TERMS>() <= 65536, "what a launch gets without asking for more");
    return (size_t)2 * attend_wide_pairs<TERMS>() * attend_wide_pair<HD, TERMS>();
}

template <int HD, int TERMS, int QT, int PT>
__global__ void __launch_bounds__(256, QT == 1 ? 2 : 1) ee_attend_wide_kernel(AttendDev a)
{
    extern __shared__ __align__(16) char lds[];
    constexpr int KT = HD / 32, NT = HD / 16, RT = 2, NP = attend_wide_pairs<TERMS>();
    constexpr int PAIR = attend_wide_pair<HD, TERMS>(), STAGE = NP * PAIR;
    static_assert(KT == NT / 2, "K of a product is as much as half of V");
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lm = lane & 15, quad = lane >> 4, kvh = blockIdx.x;
    AttendItem it;
    if (!attend_item<ATT_WIDE>(a, blockIdx.y, lane, it)) return;
    const int lines = min(max(it.lines - wave * 32, 0), 32);
    const int i0 = it.line0 / a.per_key, l0 = it.line0 - i0 * a.per_key;    // row of the chunk's first line, and which of its lines that is
    int row[RT], head[RT], last[RT];
    bf16x8_t q[RT][KT][QT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        const int l = l0 + min(wave * 32 + t * 16 + lm, it.lines - 1), i = div_small(l, a.per_key);
        row[t] = it.row0 + i0 + i;
        head[t] = kvh * a.per_key + l - i * a.per_key;
        last[t] = it.first_pos + i0 + i;
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) attend_load_q<QT>(a, row[t], head[t], kt, quad, q[t][kt]);
    }
    const int first_last = it.first_pos + i0 + __builtin_amdgcn_readfirstlane(div_small(l0 + wave * 32, a.per_key));   // of the wave
    const int wave_last = lines > 0 ? min(it.first_pos + i0 + __builtin_amdgcn_readfirstlane(div_small(l0 + wave * 32 + lines - 1, a.per_key)), a.b.capacity() - 1) : -1;
    const int n_pg = it.pg_hi - it.pg_lo, steps = (n_pg + 2 * NP - 1) / (2 * NP);
    const int *table = a.b.table + (size_t)it.seq * a.b.table_stride;
    const unsigned lds0 = lds_offset(lds);
    // ids of 64 pages in the lanes, from page ids_from of the item on
    int ids = -1, ids_from = -64;
    auto load_ids = [&](int pg) __attribute__((always_inline)) {
        if (pg < ids_from + 64) return;
        ids_from = pg;
        ids = pg + lane < n_pg ? as_global(table)[it.pg_lo + pg + lane] : -1;
        if (ids >= a.b.n_pages) ids = -1;
    };
    // A pair in LDS is kilobytes in operand order, every lane's 16 bytes in turn, so that all reads are contiguous: K of product h, values kt, term u at
    // (h KT + kt) TERMS + u, behind them V of dims nt, term u at nt TERMS + u.  Waves 0 and 1 bring K of their product, 2 and 3 a half of V.
    const bool is_v = wave >= 2;
    const uint16_t *const src = (is_v ? a.b.vpool : a.b.kpool) + (size_t)kvh * KV_PAGE * TERMS * HD +
                                (is_v ? ((wave & 1) * HD / 2 + lm) * KV_PAGE + (quad & 1) * 8 : ((lm >> 2 & 1) * 8 + wave * 4 + (lm & 3)) * TERMS * HD + quad * 8);
    const bool second = is_v ? quad >= 2 : lm >= 8;          // which of the pair's pages the lane's 16 bytes are on
    const size_t page_step = (size_t)a.b.n_kv_heads * KV_PAGE * TERMS * HD;
    auto request = [&](int step, int slot, int (&id)[2 * NP]) __attribute__((always_inline)) {
        load_ids(2 * NP * step);
#pragma unroll
        for (int i = 0; i < 2 * NP; ++i) id[i] = __builtin_amdgcn_readlane(ids, 2 * NP * step + i - ids_from);
#pragma unroll
        for (int n = 0; n < NP; ++n) {
            const uint16_t *p = src + (size_t)max(second ? id[2 * n + 1] : id[2 * n], 0) * page_step;
            const unsigned dst = lds0 + slot * STAGE + n * PAIR + wave * (PAIR / 4);
            if (is_v) {
#pragma unroll
                for (int nt = 0; nt < NT / 2; ++nt)
#pragma unroll
                    for (int u = 0; u < TERMS; ++u) load_lds_lanes(p + (u * HD + nt * 16) * KV_PAGE, dst + (nt * TERMS + u) * 1024);
            } else {
#pragma unroll
                for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                    for (int u = 0; u < TERMS; ++u) load_lds_lanes(p + u * HD + kt * 32, dst + (kt * TERMS + u) * 1024);
            }
        }
    };
    AttendState<RT, NT> st;
    attend_clear(st);
    wait_vmem();
    int next[2 * NP] = {};
    if (steps > 0) request(0, 0, next);
    for (int step = 0; step < steps; ++step) {
        int id[2 * NP];
#pragma unroll
        for (int i = 0; i < 2 * NP; ++i) id[i] = next[i];
        wait_pending<0>();
        lds_barrier();                                       // this step is there for all waves, the last one has been read by all
        if (step + 1 < steps) request(step + 1, (step + 1) & 1, next);
        const int pos0 = (it.pg_lo + 2 * NP * step) * KV_PAGE;
        if (pos0 > wave_last) continue;
        const char *buf = lds + (step & 1) * STAGE + lane * 16;
        PairMask mask[NP];
        bool hidden = false;
#pragma unroll
        for (int n = 0; n < NP; ++n) {
            mask[n] = pair_mask(pos0 + n * 32, id[2 * n], id[2 * n + 1], first_last, wave_last);
            hidden |= mask[n].masked;
        }
        auto multiply = [&](auto masked) __attribute__((always_inline)) {
            constexpr bool MASKED = decltype(masked)::value;
            int keep[NP];
            f32x4_t S[RT][NP][2];
#pragma unroll
            for (int n = 0; n < NP; ++n) {
                keep[n] = mask[n].keep(quad);
#pragma unroll
                for (int t = 0; t < RT; ++t) S[t][n][0] = S[t][n][1] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int u = 0; u < TERMS; ++u) {
                            const bf16x8_t k = *reinterpret_cast<const bf16x8_t *>(buf + n * PAIR + ((h * KT + kt) * TERMS + u) * 1024);
#pragma unroll
                            for (int t = 0; t < RT; ++t)
#pragma unroll
                                for (int i = 0; i < QT - u; ++i) S[t][n][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[t][kt][i], S[t][n][h], 0, 0, 0);
                        }
            }
            float s[RT][NP][8], local[RT];
            bool up = false;
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                local[t] = attend_scores<MASKED, NP>(st, t, S[t], keep, pos0, last[t], quad, a.scale2, s[t], up);
            }
            if (__any(up)) {
#pragma unroll
                for (int t = 0; t < RT; ++t) attend_raise(st, t, local[t], s[t]);
            }
            bf16x8_t P[RT][NP][PT];
#pragma unroll
            for (int t = 0; t < RT; ++t) attend_exps<PT, NP>(st, t, s[t], P[t]);
#pragma unroll
            for (int n = 0; n < NP; ++n) {
                uint4 v[NT][TERMS];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int u = 0; u < TERMS; ++u) v[nt][u] = *reinterpret_cast<const uint4 *>(buf + n * PAIR + PAIR / 2 + (nt * TERMS + u) * 1024);
                if constexpr (MASKED) attend_clean_v<TERMS>(st, v, mask[n], keep[n], pos0 + n * 32, last, quad);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int u = 0; u < TERMS; ++u)
#pragma unroll
                        for (int t = 0; t < RT; ++t)
#pragma unroll
                            for (int i = 0; i < PT - u; ++i)
                                st.o[t][nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, v[nt][u]), P[t][n][i], st.o[t][nt], 0, 0, 0);
            }
        };
        if (hidden)
            multiply(std::true_type{});
        else
            multiply(std::false_type{});
    }
    attend_finish(st);
#pragma unroll
    for (int t = 0; t < RT; ++t)
        if (t * 16 + lm < lines) attend_store(a, it, st, t, row[t], head[t], quad);
}

// ------------------------------------------------------------------ parts
//
// Joins the parts of every line that has several, in order.  thread = four dims of a line and every 256 / (HD / 4)-th of its parts where there are many
// (`spread` of them side by side), of several lines otherwise.
template <int HD>
__global__ void __launch_bounds__(256) ee_attend_join_kernel(AttendDev a, int spread)
{
    constexpr int TPL = HD / 4, ROWS = 256 / TPL;
    typedef __attribute__((ext_vector_type(2))) float f32x2_t;
    __shared__ f32x4_t nums[ROWS][TPL];
    __shared__ float dens[ROWS], maxs[ROWS], bads[ROWS];
    const int tr = threadIdx.x / TPL, td = threadIdx.x % TPL, sub = tr % spread;
    const long long line = (long long)blockIdx.x * (ROWS / spread) + tr / spread;
    const int most = a.most_own + a.most_shared;
    const bool there = line < (long long)a.b.n_rows * a.n_heads;
    const f32x2_t *ml = reinterpret_cast<const f32x2_t *>(a.part_ml + (there ? line : 0) * (most + 1));
    const float *o = a.part + (there ? line : 0) * most * HD + td * 4;
    f32x4_t num = {0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, den = 0.f, bad = 0.f;
    int own = 0, shared = 0;
    // four slots at a time, the first four together with the counts that say which of them are in use
    for (int base = sub; base < most; base += 4 * spread) {
        f32x2_t x[4];
        f32x4_t v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int slot = min(base + i * spread, most - 1);
            x[i] = as_global(ml)[1 + slot];
            v[i] = *as_global(reinterpret_cast<const f32x4_t *>(o + (size_t)slot * HD));
        }
        if (base == sub) {
            const f32x2_t n = as_global(ml)[0];
            const long long from = a.b.start(0), rows = a.b.start(a.b.n_seqs);   // (no item has written counts of a row outside)
            if (line >= from * a.n_heads && line < rows * a.n_heads) {
                own = __float_as_int(n[0]);
                shared = own ? __float_as_int(n[1]) : 0;                    // (own 0: written already)
            }
            if (own == 0) break;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int slot = base + i * spread;
            if (!(slot < a.most_own ? slot < own : slot - a.most_own < shared) || slot >= most) continue;
            if (x[i][0] == -INFINITY) {
                bad = x[i][1] != 0.f ? 1.f : bad;                           // positions without a softmax
                continue;
            }
            const float m_new = fmaxf(m, x[i][0]), f0 = __builtin_amdgcn_exp2f(m - m_new), f1 = __builtin_amdgcn_exp2f(x[i][0] - m_new);
            m = m_new;
            den = den * f0 + x[i][1] * f1;
#pragma unroll
            for (int r = 0; r < 4; ++r) num[r] = num[r] * f0 + v[i][r] * f1;
        }
    }
    if (spread > 1) {
        nums[tr][td] = num;
        if (td == 0) {
            dens[tr] = den;
            maxs[tr] = m;
            bads[tr] = bad;
        }
        __syncthreads();
        if (sub != 0) return;
        for (int i = 1; i < spread; ++i) {
            const float m2 = maxs[tr + i];
            bad = fmaxf(bad, bads[tr + i]);
            if (m2 == -INFINITY) continue;
            const float m_new = fmaxf(m, m2), f0 = __builtin_amdgcn_exp2f(m - m_new), f1 = __builtin_amdgcn_exp2f(m2 - m_new);
            m = m_new;
            den = den * f0 + dens[tr + i] * f1;
            const f32x4_t v = nums[tr + i][td];
#pragma unroll
            for (int r = 0; r < 4; ++r) num[r] = num[r] * f0 + v[r] * f1;
        }
    }
    if (own == 0) return;
    const int row = (int)(line / a.n_heads), head = (int)(line - (long long)row * a.n_heads);
    const float inv = m != -INFINITY ? 1.0f / den : bad != 0.f ? __builtin_nanf("") : 0.f;
    store4(a.out_type, a.out, (size_t)row * a.o_stride + (size_t)head * a.o_head + td * 4, num[0] * inv, num[1] * inv, num[2] * inv, num[3] * inv);
}

}  // namespace ee
