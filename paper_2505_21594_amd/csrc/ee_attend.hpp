// ee_attend: attention of new rows over paged caches, pages that sequences have in common read once for all of them.
//
//   out_i = sum_j softmax_j(scale q_i . k_j) v_j  over the positions a row sees, as one pass over the keys and values with a running
//   maximum m and sum l:  m' = max(m, s_j),  l' = l e^(m - m') + e^(s_j - m'),  o' = o e^(m - m') + e^(s_j - m') v_j;
//   parts of the positions join by the same rule.
//
// Bound by the cache's bytes with few rows (64 flops a byte of a one-term cache with 16 lines), by the matrix cores with
// many.  A line is a row's query head; the lines that read one key head are taken RT tiles of 16 at a time.  An item is (key head, up to 16 RT
// lines of one sequence, or of one group over its common pages, a part of their pages) and goes to a workgroup of ATT_W waves,
// which take pairs of pages in turn; every wave keeps q, the running maximum and sum, and the output in registers:
//   scores   S[position][line] = K . q^T    v_mfma_f32_16x16x32_bf16, A = 16 positions x 32 values straight from a page's record, B = q
//   output   O[dim][line] = V^T . P         the same instruction over the pair's 32 positions: its k index may run over them in any order
//            that both operands share, so P stays in the registers that the scores came in (lane: line l & 15, positions (l >> 4) 4 .. + 3 of
//            either page), and V, which a record holds transposed, comes as a lane's 4 positions of either page.
// q of 16 bits beyond bf16 and P are two bf16 terms each (x = hi + lo to 2^-17), products of two lo terms are left out (2^-18); sums are fp32.
// The waves' results are joined through LDS; where a line has several parts, they go to memory and ee_attend_join_kernel
// joins them in order, so that results do not depend on who is first.
#pragma once

#include "ee_ops.hpp"

namespace ee {

constexpr int ATT_W = 4;                       // waves of an item
constexpr int ATT_ID_PAIRS = 32;               // pairs of pages whose ids a wave holds in its lanes

struct AttendDev {
    BatchDev b;
    const void *q;
    void *out;
    long long q_stride, q_head, o_stride, o_head;
    const int *group_start, *group_pages;
    float *part;                               // [line of the batch][parts][HD], then [line][parts][2] maxima and sums
    float *part_ml;
    int q_type, out_type;
    int n_groups, n_heads, per_key;            // per_key: query heads of a key head
    int parts_own, parts_shared, chunks_shared;
    float scale2;                              // scale * log2(e)
};

// What one item works on.
struct AttendItem {
    const uint16_t *k, *v;                     // record of page 0 for the key head
    size_t page_step;                          // elements from a page's record to the next page's
    const int *table;
    int n_pages;
    int pg_lo, pg_hi;                          // its pages
    int lines, line0;                          // its lines: line0 .. line0 + lines - 1 of the chunk's rows x heads
    int first_last;                            // last position that its first line sees (the others see as many or more)
};

template <int RT, int NT>
struct AttendState {
    f32x4_t o[RT][NT];
    float mx[RT], sum[RT];
};

__device__ __forceinline__ bool nonfinite_bf16(uint32_t w) { return (w & 0x7F80u) == 0x7F80u || (w & 0x7F800000u) == 0x7F800000u; }

// The pages [pg_lo, pg_hi) of an item, pairs of them in turn over the waves.  last[t]: last position that this lane's line of tile t sees.
template <int HD, int TERMS, int QT, int RT>
__device__ __forceinline__ void attend_pages(const AttendItem &it, const bf16x8_t (&q)[RT][HD / 32][QT], const int (&last)[RT], int max_last, float scale2, int lane,
                                             int wave, AttendState<RT, HD / 16> &st)
{
    constexpr int KT = HD / 32, NT = HD / 16;
    const int lm = lane & 15, quad = lane >> 4;
    const int pairs = (it.pg_hi - it.pg_lo + 1) >> 1;
    const int tiles = (it.lines + 15) >> 4;
    int pr = wave;
    if (pr >= pairs) return;
    int ids = -1, ids_from = pr;
    auto load_ids = [&]() __attribute__((always_inline)) {
        const int pg = it.pg_lo + 2 * (ids_from + (lane >> 1) * ATT_W) + (lane & 1);
        ids = pg < it.pg_hi ? as_global(it.table)[pg] : -1;
        if (ids >= it.n_pages) ids = -1;
    };
    unsigned hollow = 0;              // bit t: this lane's line of tile t saw positions, but no score above -infinity yet
    uint4 kf[2][TERMS][KT];
    uint2 vf[2][TERMS][NT];
    int id[2];
    auto find_ids = [&](int p) __attribute__((always_inline)) {
        const int i = (p - ids_from) / ATT_W * 2;
        id[0] = __builtin_amdgcn_readlane(ids, i);
        id[1] = __builtin_amdgcn_readlane(ids, i + 1);
    };
    auto request_k = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint16_t *kb = it.k + (size_t)max(id[h], 0) * it.page_step + lm * (TERMS * HD) + quad * 8;
#pragma unroll
            for (int t = 0; t < TERMS; ++t)
#pragma unroll
                for (int kt = 0; kt < KT; ++kt) kf[h][t][kt] = load_global16(kb + t * HD + kt * 32);
        }
    };
    auto request_v = [&](const int (&of)[2]) __attribute__((always_inline)) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint16_t *vb = it.v + (size_t)max(of[h], 0) * it.page_step + lm * KV_PAGE + quad * 4;
#pragma unroll
            for (int t = 0; t < TERMS; ++t)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) vf[h][t][nt] = load_global8(vb + (t * HD + nt * 16) * KV_PAGE);
        }
    };
    load_ids();
    find_ids(pr);
    request_k();
    request_v(id);
    for (;;) {
        const int pos0 = (it.pg_lo + 2 * pr) * KV_PAGE;
        // positions of either page that any line of the item may see
        int lim[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) lim[h] = id[h] < 0 || it.pg_lo + 2 * pr + h >= it.pg_hi ? 0 : min(max(max_last + 1 - pos0 - h * KV_PAGE, 0), KV_PAGE);
        const bool masked = lim[0] < KV_PAGE || lim[1] < KV_PAGE || it.first_last < pos0 + 2 * KV_PAGE - 1;
        f32x4_t S[RT][2];
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int h = 0; h < 2; ++h) S[t][h] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int kt = 0; kt < KT; ++kt) {
                const bf16x8_t kh = __builtin_bit_cast(bf16x8_t, kf[h][0][kt]);
#pragma unroll
                for (int t = 0; t < RT; ++t) {
                    if (t >= tiles) continue;
                    S[t][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kh, q[t][kt][0], S[t][h], 0, 0, 0);
                    if constexpr (QT == 2) S[t][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kh, q[t][kt][1], S[t][h], 0, 0, 0);
                    if constexpr (TERMS == 2)
                        S[t][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, kf[h][1][kt]), q[t][kt][0], S[t][h], 0, 0, 0);
                }
            }
        pr += ATT_W;
        const bool more = pr < pairs;
        if (more) {
            if (pr - ids_from >= ATT_ID_PAIRS * ATT_W) {
                ids_from = pr;
                load_ids();
            }
            find_ids(pr);
            request_k();
        }
        if (masked) {
            // what no line sees is taken out of V (it may hold anything), what a line does not see out of its scores
#pragma unroll
            for (int h = 0; h < 2; ++h)
                if (lim[h] < KV_PAGE) {
                    const int keep = min(max(lim[h] - quad * 4, 0), 4);
                    const uint32_t m0 = keep >= 2 ? 0xFFFFFFFFu : keep == 1 ? 0xFFFFu : 0u, m1 = keep >= 4 ? 0xFFFFFFFFu : keep == 3 ? 0xFFFFu : 0u;
#pragma unroll
                    for (int t = 0; t < TERMS; ++t)
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            vf[h][t][nt].x &= m0;
                            vf[h][t][nt].y &= m1;
                        }
                }
#pragma unroll
            for (int t = 0; t < RT; ++t)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int in_page = quad * 4 + r;
                        if (in_page >= lim[h] || pos0 + h * KV_PAGE + in_page > last[t]) S[t][h][r] = -INFINITY;
                    }
        }
        bf16x8_t Ph[RT], Pl[RT];
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            if (t >= tiles) continue;
            float m = st.mx[t];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int r = 0; r < 4; ++r) m = fmaxf(m, S[t][h][r]);
            m = fmaxf(m, __shfl_xor(m, 16, 64));
            m = fmaxf(m, __shfl_xor(m, 32, 64));
            const float base = m == -INFINITY ? 0.f : m;
            const float f = __builtin_amdgcn_exp2f((st.mx[t] - base) * scale2);
            st.mx[t] = m;
            if (m == -INFINITY && ((lim[0] > 0 && pos0 <= last[t]) || (lim[1] > 0 && pos0 + KV_PAGE <= last[t]))) hollow |= 1u << t;
            float sum = 0.f;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    S[t][h][r] = __builtin_amdgcn_exp2f((S[t][h][r] - base) * scale2);
                    sum += S[t][h][r];
                }
            st.sum[t] = st.sum[t] * f + sum;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int r = 0; r < 4; ++r) st.o[t][nt][r] *= f;
            split_bf16x8(S[t][0], S[t][1], Ph[t], Pl[t]);
        }
        if (masked) {
            // An infinity or NaN of V in a place that some lines see and others do not: 0 * V would be NaN for those.  A page with such
            // elements goes position by position, each for the lines that see it, and leaves the product of the pair.
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                bool odd = false;
#pragma unroll
                for (int t = 0; t < TERMS; ++t)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) odd |= nonfinite_bf16(vf[h][t][nt].x) || nonfinite_bf16(vf[h][t][nt].y);
                if (!__any(odd)) continue;
#pragma clang loop unroll(disable)
                for (int j = 0; j < lim[h]; ++j) {
                    const int mine = quad == j >> 2 ? j & 3 : 4;
                    const uint32_t m0 = mine == 0 ? 0xFFFFu : mine == 1 ? 0xFFFF0000u : 0u, m1 = mine == 2 ? 0xFFFFu : mine == 3 ? 0xFFFF0000u : 0u;
#pragma unroll
                    for (int t = 0; t < RT; ++t) {
                        if (t >= tiles) continue;
                        const bool sees = pos0 + h * KV_PAGE + j <= last[t];
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            f32x4_t o = st.o[t][nt];
#pragma unroll
                            for (int u = 0; u < TERMS; ++u) {
                                const uint32_t x = vf[h][u][nt].x & m0, y = vf[h][u][nt].y & m1;
                                const bf16x8_t v = __builtin_bit_cast(bf16x8_t, h == 0 ? make_uint4(x, y, 0u, 0u) : make_uint4(0u, 0u, x, y));
                                o = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, Ph[t], o, 0, 0, 0);
                                if (u == 0) o = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, Pl[t], o, 0, 0, 0);
                            }
#pragma unroll
                            for (int r = 0; r < 4; ++r) st.o[t][nt][r] = sees ? o[r] : st.o[t][nt][r];
                        }
                    }
                }
#pragma unroll
                for (int t = 0; t < TERMS; ++t)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) vf[h][t][nt] = make_uint2(0u, 0u);
            }
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const bf16x8_t vh = __builtin_bit_cast(bf16x8_t, make_uint4(vf[0][0][nt].x, vf[0][0][nt].y, vf[1][0][nt].x, vf[1][0][nt].y));
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                if (t >= tiles) continue;
                st.o[t][nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vh, Ph[t], st.o[t][nt], 0, 0, 0);
                st.o[t][nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vh, Pl[t], st.o[t][nt], 0, 0, 0);
                if constexpr (TERMS == 2) {
                    const bf16x8_t vl = __builtin_bit_cast(bf16x8_t, make_uint4(vf[0][1][nt].x, vf[0][1][nt].y, vf[1][1][nt].x, vf[1][1][nt].y));
                    st.o[t][nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vl, Ph[t], st.o[t][nt], 0, 0, 0);
                }
            }
        }
        if (!more) break;
        request_v(id);
    }
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        st.sum[t] += __shfl_xor(st.sum[t], 16, 64);
        st.sum[t] += __shfl_xor(st.sum[t], 32, 64);
        if (st.mx[t] == -INFINITY && (hollow >> t & 1)) st.sum[t] = __builtin_nanf("");
    }
}

// Two parts' sums as one: 0 where a part saw no position, NaN where it saw none with a score above -infinity (which says nothing
// beside a part with one).
__device__ __forceinline__ float join_sums(float m, float m1, float l1, float f1, float m2, float l2, float f2)
{
    if (m == -INFINITY) return l1 + l2;
    return (m1 == -INFINITY ? 0.f : l1 * f1) + (m2 == -INFINITY ? 0.f : l2 * f2);
}

// floats per lane that a wave hands over
template <int HD, int RT>
constexpr int attend_lds_floats() { return RT * (HD / 16) * 4 + 2 * RT; }
template <int HD, int RT>
constexpr size_t attend_lds()
{
    constexpr size_t bytes = (size_t)(ATT_W / 2) * 64 * attend_lds_floats<HD, RT>() * sizeof(float);
    static_assert(bytes <= 65536, "what a launch gets without asking for more");
    return bytes;
}

// Joins the waves' results into wave 0's, halves of them at a time; `active`: waves that had pages.
template <int HD, int RT>
__device__ __forceinline__ void attend_join_waves(AttendState<RT, HD / 16> &st, float *lds, int active, float scale2, int lane, int wave)
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
                const float f1 = __builtin_amdgcn_exp2f((st.mx[t] - base) * scale2), f2 = __builtin_amdgcn_exp2f((m2 - base) * scale2);
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

}  // namespace ee
