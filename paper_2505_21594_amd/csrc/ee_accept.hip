// ee_accept_drafts: how many drafted tokens of every sequence its rows' logits keep, and which token follows.
//
// Bound by the logits' bytes (read once) where rows are many, by two dependent launches where they are few.  Probabilities,
// sums and comparisons are in 64 bits: a draw is decided by where v * sum falls among the vocabulary's partial sums, and sums of fp32 terms
// would move those borders by more than rare tokens are wide.  In parts of ACC_PART tokens:
//   1. stats: every row's part: largest logit m (at temperature 0 also the lowest token that has it) and sum exp((z - m) / T);
//   2. draw: with a row's parts joined (Z), the keep tests; of the row that ends the round, every part's sum of max(q - p, 0); the
//      sequence's workgroup that arrives last finds the part in which the sum over the parts passes v * sum, and in it the token.
// All sums are taken in one order whatever the launch: results do not depend on timing.
#include "ee_ops.hpp"

namespace ee {

constexpr int ACC_PART = 4096;                                       // tokens of a workgroup
constexpr int ACC_THREADS = 256, ACC_EACH = 16;                      // ... of the first launch
constexpr int ACC_DRAW = 512, ACC_DRAW_EACH = 8, ACC_WAVES = ACC_DRAW / 64;   // ... of the second, with a wave for each of eight rows
static_assert(ACC_THREADS * ACC_EACH == ACC_PART && ACC_DRAW * ACC_DRAW_EACH == ACC_PART, "a part is a workgroup's");

struct AcceptRow {                     // one part of one row
    double sum;                        // sum of exp((z - m) / T)
    float m;
    int best;
};
struct RowStats {                      // a row's parts as one
    double Z;
    float m;
    int best;
};

struct AcceptDev {
    const void *logits;
    const float *probs, *u, *v, *temperature;
    const int *row_start, *drafts;
    int *accept_len, *next_token;
    long long z_stride, p_stride;
    AcceptRow *rows;                   // [n_rows][parts]
    unsigned long long *weights;       // [n_seqs][parts]  the ending row's sums of weights (bits of doubles)
    int *arrived;                      // [n_seqs]  parts delivered
    int type, n_seqs, n_rows, V, parts;

    __device__ __forceinline__ int start(int s) const { return min(max(as_global(row_start)[s], 0), n_rows); }
};

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
template <int N>
__device__ __forceinline__ void load_logits(const AcceptDev &a, int row, int first, float (&z)[N])
{
    const size_t at = (size_t)row * a.z_stride + first;
    const int n = a.V - first;
    if (a.type == EE_FP32)
        load_some<N>(static_cast<const float *>(a.logits) + at, n, -INFINITY, z);
    else if (a.type == EE_BF16)
        load_some<N>(static_cast<const __bf16 *>(a.logits) + at, n, -INFINITY, z);
    else
        load_some<N>(static_cast<const _Float16 *>(a.logits) + at, n, -INFINITY, z);
}

// 2^y of y <= 0 in 64 bits: y = n + r with |r| <= 1/2, and the series of 2^r = e^(r ln 2) up to r^12 ln2^12 / 12! (what follows is below 2.2e-16).  The
// vector unit bounds the first launch of many rows: two thirds of the instructions of the library's exp.  Below -1020: 0.
__device__ __forceinline__ double exp2_down(double y)
{
    constexpr double MAGIC = 6755399441055744.0;         // 1.5 * 2^52: the sum's last bits are y rounded to an integer
    const double t = y + MAGIC, r = y - (t - MAGIC);
    double e = 2.5678435993488206e-11;
    e = fma(e, r, 4.4455382718708116e-10);
    e = fma(e, r, 7.054911620801123e-09);
    e = fma(e, r, 1.01780860092397e-07);
    e = fma(e, r, 1.321548679014431e-06);
    e = fma(e, r, 1.5252733804059841e-05);
    e = fma(e, r, 0.0001540353039338161);
    e = fma(e, r, 0.0013333558146428443);
    e = fma(e, r, 0.009618129107628477);
    e = fma(e, r, 0.05550410866482158);
    e = fma(e, r, 0.24022650695910072);
    e = fma(e, r, 0.6931471805599453);
    e = fma(e, r, 1.0);
    const unsigned long long b = (unsigned long long)__double_as_longlong(e);
    const int n = (int)(unsigned)(unsigned long long)__double_as_longlong(t);
    e = __longlong_as_double((long long)(b + ((unsigned long long)(unsigned)(n << 20) << 32)));
    return y < -1020.0 ? 0.0 : e;
}
// exp((z - m) / T) as 2^((z - m) c), c = log2(e) / T
struct Scale {
    double c, m;
};
__device__ __forceinline__ Scale scale_of(float t, float m)
{
    Scale s;
    s.c = 1.4426950408889634 / (double)t;
    s.m = m == -INFINITY ? 0.0 : (double)m;
    return s;
}
__device__ __forceinline__ double term(const Scale &s, float z) { return exp2_down(((double)z - s.m) * s.c); }

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
// Rule by a sequence's temperature: 0: sampled, 1: greedy, 2: nothing is kept or drawn.
__device__ __forceinline__ int rule_of(float t) { return t == 0.f ? 1 : t > 0.f && t < INFINITY ? 0 : 2; }

// Sequence of a row and its temperature, 64 sequences at a time; n_seqs where no sequence has the row.
__device__ __forceinline__ int seq_of(const AcceptDev &a, int row, int lane, float &t)
{
    for (int base = 0; base < a.n_seqs; base += 64) {
        const int s = min(base + lane, a.n_seqs - 1);
        const int from = a.start(s), to = a.start(s + 1);
        const float mine = as_global(a.temperature)[s];
        if (const unsigned long long who = __ballot(base + lane < a.n_seqs && from <= row && row < to)) {
            const int l = __builtin_ctzll(who);
            t = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(mine), l));
            return base + l;
        }
    }
    return a.n_seqs;
}

__global__ void __launch_bounds__(ACC_THREADS) ee_accept_stats_kernel(AcceptDev a)
{
    __shared__ float wm[ACC_THREADS / 64];
    __shared__ int wi[ACC_THREADS / 64];
    __shared__ double ws[ACC_THREADS / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, row = blockIdx.y, part = blockIdx.x;
    const int first = part * ACC_PART + tid * ACC_EACH;
    float z[ACC_EACH];
    load_logits(a, row, first, z);
    if (row == 0 && part == 0)
        for (int q = tid; q < a.n_seqs; q += ACC_THREADS) as_global_mut(a.arrived)[q] = 0;
    float t = 0.f;
    if (seq_of(a, row, lane, t) >= a.n_seqs) return;
    const int rule = rule_of(t);
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < ACC_EACH; ++i) m = fmaxf(m, z[i]);
    m = wave_max_f(m);
    if (lane == 0) wm[wave] = m;
    __syncthreads();
    m = fmaxf(fmaxf(wm[0], wm[1]), fmaxf(wm[2], wm[3]));
    double s = 0.0;
    int best = 0x7FFFFFFF;
    if (rule == 0) {
        const Scale scale = scale_of(t, m);
#pragma unroll
        for (int i = 0; i < ACC_EACH; ++i) s += term(scale, z[i]);   // (nothing past the end: -infinity)
        s = wave_sum_d(s);
    } else if (rule == 1) {
#pragma unroll
        for (int i = ACC_EACH - 1; i >= 0; --i)
            if (z[i] == m && first + i < a.V) best = first + i;
        best = wave_min(best);
    }
    if (lane == 0) {
        ws[wave] = s;
        wi[wave] = best;
    }
    __syncthreads();
    if (tid == 0) {
        AcceptRow r;
        r.sum = (ws[0] + ws[1]) + (ws[2] + ws[3]);
        r.m = m;
        r.best = min(min(wi[0], wi[1]), min(wi[2], wi[3]));
        a.rows[(size_t)row * a.parts + part] = r;
    }
}

// A row's parts as one: all lanes of a wave call it and get the same.
__device__ __forceinline__ RowStats join_row(const AcceptDev &a, int row, float t, int lane)
{
    const AcceptRow *r = a.rows + (size_t)row * a.parts;
    RowStats o;
    o.m = -INFINITY;
    for (int p = lane; p < a.parts; p += 64) o.m = fmaxf(o.m, r[p].m);
    o.m = wave_max_f(o.m);
    o.best = 0x7FFFFFFF;
    o.Z = 0.0;
    const Scale scale = scale_of(t, o.m);
    for (int p = lane; p < a.parts; p += 64) {
        const AcceptRow x = r[p];
        if (x.m == o.m) o.best = min(o.best, x.best);
        if (x.sum != 0.0) o.Z += x.sum * term(scale, x.m);
    }
    o.best = wave_min(o.best);
    o.Z = wave_sum_d(o.Z);
    return o;
}

// The ending row's weight of a token (the same expression, bit for bit, wherever it is formed).
__device__ __forceinline__ double weight_of(const Scale &scale, double inv_Z, float z, float p, bool residual)
{
    const double q = term(scale, z) * inv_Z;
    if (!residual) return q;
    return fmax(q - (double)p, 0.0);
}

template <int N>
__device__ __forceinline__ void load_probs(const AcceptDev &a, int row, int first, int draft, float (&p)[N])
{
    if (a.probs) {
        load_some<N>(a.probs + (size_t)row * a.p_stride + first, a.V - first, 0.f, p);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) p[i] = first + i == draft ? 1.f : 0.f;
    }
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

constexpr int ACC_ROWS = 64;            // rows of a sequence whose stats are kept at hand

// (six waves a SIMD cost 12 bytes of spill; four without any: 24 rounds on 100003 tokens 22.0 instead of 20.4 us, one on 32000 12.8 instead of 13.4)
__global__ void __launch_bounds__(ACC_DRAW, 6) ee_accept_draw_kernel(AcceptDev a)
{
    __shared__ double ws[ACC_WAVES];
    __shared__ RowStats stats[ACC_ROWS];
    __shared__ RowStats end_s;
    __shared__ int first_lost, found, positive, part_s, last_s;
    __shared__ double before_s, total_s;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, seq = blockIdx.y, part = blockIdx.x;
    const int r0 = a.start(seq), n = a.start(seq + 1) - r0;
    const float t = as_global(a.temperature)[seq];
    const int rule = rule_of(t);
    auto answer = [&](int kept, int token) {
        if (tid == 0) {
            as_global_mut(a.accept_len)[seq] = kept;
            as_global_mut(a.next_token)[seq] = token;
        }
    };
    if (n <= 0 || rule == 2) {
        if (part == 0) answer(0, n <= 0 ? -1 : 0);
        return;
    }
    if (tid == 0) {
        first_lost = n - 1;
        found = 0x7FFFFFFF;
        positive = -1;
    }
    __syncthreads();
    // keep tests, a row for a wave; the first row that loses its draft ends the round
    for (int i = wave; i < n; i += ACC_WAVES) {
        const int x = i < n - 1 ? as_global(a.drafts)[r0 + i] : -1;
        bool kept = x >= 0 && x < a.V;
        float z = 0.f, p = 1.f, u = 0.f;
        if (kept && rule == 0) {                         // (on their way while the parts are joined)
            const size_t at = (size_t)(r0 + i) * a.z_stride + x;
            z = a.type == EE_FP32   ? as_global(static_cast<const float *>(a.logits))[at]
                : a.type == EE_BF16 ? (float)as_global(static_cast<const __bf16 *>(a.logits))[at]
                                    : (float)as_global(static_cast<const _Float16 *>(a.logits))[at];
            if (a.probs) p = as_global(a.probs)[(size_t)(r0 + i) * a.p_stride + x];
            if (a.u) u = as_global(a.u)[r0 + i];
        }
        const RowStats o = join_row(a, r0 + i, t, lane);
        if (i < ACC_ROWS && lane == 0) stats[i] = o;
        if (i == n - 1) break;
        if (kept && rule == 1) kept = x == o.best;
        if (kept && rule == 0) kept = a.u && (double)u * (double)p < term(scale_of(t, o.m), z) * (1.0 / o.Z);
        if (!kept && lane == 0) atomicMin(&first_lost, i);
    }
    __syncthreads();
    const int i = first_lost, row = r0 + i;
    bool residual = i < n - 1;
    if (i >= ACC_ROWS) {
        if (wave == 0) {
            const RowStats o = join_row(a, row, t, lane);
            if (lane == 0) end_s = o;
        }
        __syncthreads();
    }
    const RowStats e = i < ACC_ROWS ? stats[i] : end_s;
    if (rule == 1 || !(e.Z > 0.0 && e.Z < INFINITY)) {
        if (part == 0) answer(i, rule == 1 && e.best < a.V ? e.best : 0);
        return;
    }
    const double inv_Z = 1.0 / e.Z;
    const Scale scale = scale_of(t, e.m);
    const int draft = as_global(a.drafts)[row];
    float z[ACC_DRAW_EACH], p[ACC_DRAW_EACH];
    {
        const int first = part * ACC_PART + tid * ACC_DRAW_EACH;
        load_logits(a, row, first, z);
        if (residual) load_probs(a, row, first, draft, p);
        double w = 0.0;
#pragma unroll
        for (int k = 0; k < ACC_DRAW_EACH; ++k) w += weight_of(scale, inv_Z, z[k], residual ? p[k] : 0.f, residual);
        w = wave_sum_d(w);
        if (lane == 0) ws[wave] = w;
    }
    __syncthreads();
    unsigned long long *const sums = a.weights + (size_t)seq * a.parts;
    if (tid == 0) {
        __hip_atomic_store(sums + part, (unsigned long long)__double_as_longlong(((ws[0] + ws[1]) + (ws[2] + ws[3])) + ((ws[4] + ws[5]) + (ws[6] + ws[7]))), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        wait_vmem();                                     // the sum is visible device-wide before it is counted
        last_s = __hip_atomic_fetch_add(a.arrived + seq, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == a.parts - 1;
    }
    __syncthreads();
    if (!last_s) return;

    // the part that passes v * total: sums of the parts in order, by wave 0
    const double v = a.v ? (double)as_global(a.v)[row] : 0.0;
    auto sum_of = [&](int q) { return q < a.parts ? __longlong_as_double((long long)__hip_atomic_load(sums + q, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)) : 0.0; };
    if (wave == 0) {
        const double mine = sum_of(lane);                // (64 parts, 262144 tokens, are one load)
        double total = wave_sum_d(mine);
        for (int base = 64; base < a.parts; base += 64) total += wave_sum_d(sum_of(base + lane));
        const bool from_q = residual && !(total > 0.0);  // p covers q everywhere: the row draws from q
        auto weight = [&](int q) {
            if (!from_q) return q < 64 ? mine : sum_of(q);
            if (q >= a.parts) return 0.0;
            const AcceptRow r = a.rows[(size_t)row * a.parts + q];
            return r.sum != 0.0 ? r.sum * term(scale, r.m) * inv_Z : 0.0;
        };
        if (from_q) {
            total = 0.0;
            for (int base = 0; base < a.parts; base += 64) total += wave_sum_d(weight(base + lane));
        }
        const double target = v * total;
        double before = 0.0, last_before = 0.0;
        int at = -1, last_part = 0;
        for (int base = 0; base < a.parts && at < 0; base += 64) {
            const double w = weight(base + lane), incl = before + wave_scan_d(w), excl = incl - w;
            const unsigned long long hit = __ballot(w > 0.0 && incl > target), some = __ballot(w > 0.0);
            if (hit) {
                const int l = __builtin_ctzll(hit);
                at = base + l;
                before = __shfl(excl, l, 64);
            } else {
                if (some) {
                    const int l = 63 - __builtin_clzll(some);
                    last_part = base + l;
                    last_before = __shfl(excl, l, 64);
                }
                before = __shfl(incl, 63, 64);
            }
        }
        if (lane == 0) {                                 // (at < 0: v * total beyond the last sum by rounding)
            part_s = at < 0 ? last_part : at;
            before_s = at < 0 ? last_before : before;
            total_s = from_q ? -total : total;           // (its sign says which weights they are)
        }
    }
    __syncthreads();
    const double total = fabs(total_s), target = v * total;
    if (total_s < 0.0) residual = false;
    const int first = part_s * ACC_PART + tid * ACC_DRAW_EACH;
    if (part_s != part) {
        load_logits(a, row, first, z);
        if (residual) load_probs(a, row, first, draft, p);
    }
    double w[ACC_DRAW_EACH], mine = 0.0;
#pragma unroll
    for (int k = 0; k < ACC_DRAW_EACH; ++k) {
        w[k] = weight_of(scale, inv_Z, z[k], residual ? p[k] : 0.f, residual);
        mine += w[k];
    }
    const double incl = wave_scan_d(mine);
    if (lane == 63) ws[wave] = incl;
    __syncthreads();
    double run = before_s;
    for (int q = 0; q < wave; ++q) run += ws[q];
    run += incl - mine;
    int hit = 0x7FFFFFFF, some = -1;
#pragma unroll
    for (int k = 0; k < ACC_DRAW_EACH; ++k) {
        run += w[k];
        if (w[k] > 0.0) {
            some = first + k;
            if (run > target && hit == 0x7FFFFFFF) hit = first + k;
        }
    }
    if (hit != 0x7FFFFFFF) atomicMin(&found, hit);
    if (some >= 0) atomicMax(&positive, some);
    __syncthreads();
    answer(i, found != 0x7FFFFFFF ? found : max(positive, 0));
}

static size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

struct AcceptSpace {
    size_t weights, arrived, bytes;    // (rows come first)
    int parts;
};
static AcceptSpace accept_space(const ee_accept_args &p)
{
    AcceptSpace s;
    s.parts = (p.vocab + ACC_PART - 1) / ACC_PART;
    s.weights = align256((size_t)p.n_rows * s.parts * sizeof(AcceptRow));
    s.arrived = s.weights + align256((size_t)p.n_seqs * s.parts * sizeof(unsigned long long));
    s.bytes = s.arrived + align256((size_t)p.n_seqs * sizeof(int));
    return s;
}

static int check_accept(const char *call, const ee_accept_args *p)
{
    if (!p) return fail(EE_EINVAL, "%s: null argument", call);
    if (p->device < 0) return fail(EE_EINVAL, "%s: device %d", call, p->device);
    if (p->dtype < EE_BF16 || p->dtype > EE_FP32) return fail(EE_EINVAL, "%s: unknown element type %d", call, p->dtype);
    if (p->vocab < 1 || p->vocab > 1 << 24) return fail(EE_EINVAL, "%s: vocab %d out of range", call, p->vocab);
    if (p->n_seqs < 0 || p->n_seqs > 65535 || p->n_rows < 0 || p->n_rows > 65535)
        return fail(EE_EINVAL, "%s: n_seqs %d or n_rows %d not in [0,65535]", call, p->n_seqs, p->n_rows);
    return EE_OK;
}

}  // namespace ee

using namespace ee;

extern "C" int ee_accept_workspace(const ee_accept_args *p, size_t *bytes)
{
    static const char *const call = "ee_accept_workspace";
    if (!bytes) return fail(EE_EINVAL, "%s: null argument", call);
    *bytes = 0;
    int rc = check_accept(call, p);
    if (rc == EE_OK) *bytes = accept_space(*p).bytes;
    return rc;
}

extern "C" int ee_accept_drafts(const ee_accept_args *p, void *workspace, size_t workspace_bytes, void *stream)
{
    static const char *const call = "ee_accept_drafts";
    int rc = check_accept(call, p);
    if (rc != EE_OK) return rc;
    if (p->n_seqs == 0) return EE_OK;
    if (!p->row_start || !p->temperature || !p->accept_len || !p->next_token) return fail(EE_EINVAL, "%s: null row_start, temperature, accept_len or next_token", call);
    if (p->n_rows && (!p->logits || !p->drafts)) return fail(EE_EINVAL, "%s: null logits or drafts", call);
    if (p->logits_stride < p->vocab || (p->draft_probs && p->probs_stride < p->vocab) || p->logits_stride >= (int64_t)1 << 40 || p->probs_stride >= (int64_t)1 << 40)
        return fail(EE_EINVAL, "%s: a row stride is smaller than vocab", call);
    if ((!p->u) != (!p->v)) return fail(EE_EINVAL, "%s: u and v come together", call);
    if (p->draft_probs && !p->u) return fail(EE_EINVAL, "%s: draft_probs without u and v", call);
    if (!aligned(p->logits, size_of_type(p->dtype))) return fail(EE_EINVAL, "%s: logits are not aligned to their type", call);
    for (const void *x : {(const void *)p->row_start, (const void *)p->drafts, (const void *)p->draft_probs, (const void *)p->u, (const void *)p->v,
                          (const void *)p->temperature, (const void *)p->accept_len, (const void *)p->next_token})
        if (!aligned(x, 4)) return fail(EE_EINVAL, "%s: int32 and fp32 arrays must be 4-byte aligned", call);
    const AcceptSpace sp = accept_space(*p);
    if (!workspace || workspace_bytes < sp.bytes || !aligned(workspace, 256))
        return fail(EE_EINVAL, "%s: the workspace has %zu bytes of %zu, or is not 256-byte aligned", call, workspace_bytes, sp.bytes);
    AcceptDev a;
    a.logits = p->logits;
    a.probs = p->draft_probs;
    a.u = p->u;
    a.v = p->v;
    a.temperature = p->temperature;
    a.row_start = p->row_start;
    a.drafts = p->drafts;
    a.accept_len = p->accept_len;
    a.next_token = p->next_token;
    a.z_stride = p->logits_stride;
    a.p_stride = p->probs_stride;
    unsigned char *ws = static_cast<unsigned char *>(workspace);
    a.rows = reinterpret_cast<AcceptRow *>(ws);
    a.weights = reinterpret_cast<unsigned long long *>(ws + sp.weights);
    a.arrived = reinterpret_cast<int *>(ws + sp.arrived);
    a.type = p->dtype;
    a.n_seqs = p->n_seqs;
    a.n_rows = p->n_rows;
    a.V = p->vocab;
    a.parts = sp.parts;
    DeviceScope scope(p->device);
    HIP_TRY(scope.status);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (p->n_rows) hipLaunchKernelGGL(ee_accept_stats_kernel, dim3(a.parts, p->n_rows), dim3(ACC_THREADS), 0, s, a);
    HIP_TRY(hipGetLastError());
    hipLaunchKernelGGL(ee_accept_draw_kernel, dim3(a.parts, p->n_seqs), dim3(ACC_DRAW), 0, s, a);
    HIP_TRY(hipGetLastError());
    return EE_OK;
}
