// ee_accept_drafts: how many drafted tokens of every sequence its rows' logits keep, and which token follows.
//
// Bound by the logits' bytes (read once) where rows are many, by three dependent launches where they are few.  Probabilities,
// sums and comparisons are in 64 bits: a draw is decided by where v * sum falls among the vocabulary's partial sums, and sums of fp32 terms
// would move those borders by more than rare tokens are wide.  exp in 64 bits is about 40 instructions at half the fp32 rate, which the
// loads cover.  In parts of ACC_PART tokens:
//   1. stats: every row's part: largest logit m (and the lowest token that has it) and sum exp((z - m) / T);
//   2. weights: with a row's parts joined (Z), the keep tests; of the row that ends the round, every part's sum of max(q - p, 0);
//   3. draw: the part in which the sum over the parts passes v * sum, and in it the token.
// Sums are taken in one order whatever the launch: results do not depend on timing.
#include "ee_ops.hpp"

namespace ee {

constexpr int ACC_THREADS = 256, ACC_EACH = 8, ACC_PART = ACC_THREADS * ACC_EACH, ACC_WAVES = ACC_THREADS / 64;

struct AcceptRow {                     // one part of one row
    double sum;                        // sum of exp((z - m) / T)
    float m;
    int best;
};
struct AcceptEnd {                     // the row that ends a sequence's round
    double Z, inv_Z;
    float m;
    int row, accept, last;             // last: all drafts kept
    int best;                          // its largest logit's token
    int rule;                          // 0: sampled, 1: greedy, 2: nothing to draw from
};

struct AcceptDev {
    const void *logits;
    const float *probs, *u, *v, *temperature;
    const int *row_start, *drafts;
    int *accept_len, *next_token;
    long long z_stride, p_stride;
    AcceptRow *rows;                   // [n_rows][parts]
    AcceptEnd *ends;                   // [n_seqs]
    double *weights;                   // [n_seqs][parts]
    int type, n_seqs, n_rows, V, parts;

    __device__ __forceinline__ int start(int s) const { return min(max(as_global(row_start)[s], 0), n_rows); }
};

// Eight neighbouring elements at any alignment of the element type; past the end of the row: `fill`.
template <typename T>
__device__ __forceinline__ void load_eight(const T *p, int n, float fill, float (&x)[ACC_EACH])
{
    if (n >= ACC_EACH) {
        typedef T eight_t __attribute__((ext_vector_type(8), aligned(sizeof(T))));
        const eight_t e = *(const EE_GLOBAL eight_t *)as_global(p);
#pragma unroll
        for (int i = 0; i < ACC_EACH; ++i) x[i] = (float)e[i];
    } else {
#pragma unroll
        for (int i = 0; i < ACC_EACH; ++i) {
            x[i] = fill;
            if (i < n) x[i] = (float)as_global(p)[i];
        }
    }
}
__device__ __forceinline__ void load_logits(const AcceptDev &a, int row, int first, float (&z)[ACC_EACH])
{
    const size_t at = (size_t)row * a.z_stride + first;
    const int n = a.V - first;
    if (a.type == EE_FP32)
        load_eight(static_cast<const float *>(a.logits) + at, n, -INFINITY, z);
    else if (a.type == EE_BF16)
        load_eight(static_cast<const __bf16 *>(a.logits) + at, n, -INFINITY, z);
    else
        load_eight(static_cast<const _Float16 *>(a.logits) + at, n, -INFINITY, z);
}

__device__ __forceinline__ double shfl_xor_d(double x, int d) { return __shfl_xor(x, d, 64); }
__device__ __forceinline__ double wave_sum_d(double x)
{
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) x += shfl_xor_d(x, d);
    return x;
}
__device__ __forceinline__ bool better(float v, int i, float bv, int bi) { return v > bv || (v == bv && i < bi); }

// Rule by a sequence's temperature, as AcceptEnd::rule.
__device__ __forceinline__ int rule_of(float t) { return t == 0.f ? 1 : t > 0.f && t < INFINITY ? 0 : 2; }

// sequence of a row; n_seqs past the last one's rows
__device__ __forceinline__ int seq_of(const AcceptDev &a, int row)
{
    int lo = 0, hi = a.n_seqs;         // the first sequence whose end is behind the row
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (a.start(mid + 1) > row)
            hi = mid;
        else
            lo = mid + 1;
    }
    return lo;
}

__global__ void __launch_bounds__(ACC_THREADS) ee_accept_stats_kernel(AcceptDev a)
{
    __shared__ float wm[ACC_WAVES];
    __shared__ int wi[ACC_WAVES];
    __shared__ double ws[ACC_WAVES];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, row = blockIdx.y, part = blockIdx.x;
    const int first = part * ACC_PART + tid * ACC_EACH;
    float z[ACC_EACH];
    load_logits(a, row, first, z);
    const int seq = seq_of(a, row);
    if (seq >= a.n_seqs || row < a.start(seq)) return;
    const float t = as_global(a.temperature)[seq];
    float m = -INFINITY;
    int best = 0x7FFFFFFF;
#pragma unroll
    for (int i = 0; i < ACC_EACH; ++i)
        if (first + i < a.V && better(z[i], first + i, m, best)) {
            m = z[i];
            best = first + i;
        }
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) {
        const float om = __shfl_xor(m, d, 64);
        const int oi = __shfl_xor(best, d, 64);
        if (better(om, oi, m, best)) {
            m = om;
            best = oi;
        }
    }
    if (lane == 0) {
        wm[wave] = m;
        wi[wave] = best;
    }
    __syncthreads();
    m = wm[0];
    best = wi[0];
#pragma unroll
    for (int w = 1; w < ACC_WAVES; ++w)
        if (better(wm[w], wi[w], m, best)) {
            m = wm[w];
            best = wi[w];
        }
    double s = 0.0;
    if (rule_of(t) == 0) {
        const double inv_t = 1.0 / (double)t, base = m == -INFINITY ? 0.0 : (double)m;
#pragma unroll
        for (int i = 0; i < ACC_EACH; ++i)
            if (first + i < a.V) s += exp(((double)z[i] - base) * inv_t);
        s = wave_sum_d(s);
    }
    if (lane == 0) ws[wave] = s;
    __syncthreads();
    if (tid == 0) {
        AcceptRow r;
        r.sum = ((ws[0] + ws[1]) + (ws[2] + ws[3]));
        r.m = m;
        r.best = best;
        a.rows[(size_t)row * a.parts + part] = r;
    }
}

// A row's parts as one: all lanes of a wave call it and get the same.
__device__ __forceinline__ void join_row(const AcceptDev &a, int row, double inv_t, int lane, float &m, int &best, double &Z)
{
    const AcceptRow *r = a.rows + (size_t)row * a.parts;
    m = -INFINITY;
    best = 0x7FFFFFFF;
    for (int p = lane; p < a.parts; p += 64)
        if (better(r[p].m, r[p].best, m, best)) {
            m = r[p].m;
            best = r[p].best;
        }
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) {
        const float om = __shfl_xor(m, d, 64);
        const int oi = __shfl_xor(best, d, 64);
        if (better(om, oi, m, best)) {
            m = om;
            best = oi;
        }
    }
    Z = 0.0;
    for (int p = lane; p < a.parts; p += 64) {
        const double pm = r[p].m == -INFINITY ? 0.0 : (double)r[p].m;
        if (r[p].sum != 0.0) Z += r[p].sum * exp((pm - (double)m) * inv_t);
    }
    Z = wave_sum_d(Z);
}

// The ending row's weight of a token (the same expression, bit for bit, wherever it is formed).
__device__ __forceinline__ double weight_of(const AcceptEnd &e, double inv_t, float z, float p, bool residual)
{
    const double q = exp(((double)z - (double)e.m) * inv_t) * e.inv_Z;
    if (!residual) return q;
    return fmax(q - (double)p, 0.0);
}

__device__ __forceinline__ void load_probs(const AcceptDev &a, int row, int first, int draft, float (&p)[ACC_EACH])
{
    if (a.probs) {
        load_eight(a.probs + (size_t)row * a.p_stride + first, a.V - first, 0.f, p);
    } else {
#pragma unroll
        for (int i = 0; i < ACC_EACH; ++i) p[i] = first + i == draft ? 1.f : 0.f;
    }
}

__global__ void __launch_bounds__(ACC_THREADS) ee_accept_weights_kernel(AcceptDev a)
{
    __shared__ double ws[ACC_WAVES];
    __shared__ int first_lost;
    __shared__ AcceptEnd end;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, seq = blockIdx.y, part = blockIdx.x;
    const int r0 = a.start(seq), n = a.start(seq + 1) - r0;
    const float t = as_global(a.temperature)[seq];
    const int rule = rule_of(t);
    const double inv_t = rule == 0 ? 1.0 / (double)t : 0.0;
    if (tid == 0) first_lost = max(n - 1, 0);
    __syncthreads();
    if (n > 0) {
        // keep tests: a row for a wave; the first row that loses its draft ends the round
        for (int i = wave; i < n - 1; i += ACC_WAVES) {
            float m;
            int best;
            double Z;
            join_row(a, r0 + i, inv_t, lane, m, best, Z);
            const int x = as_global(a.drafts)[r0 + i];
            bool kept = x >= 0 && x < a.V && rule != 2;
            if (kept && rule == 1) kept = x == best;
            if (kept && rule == 0) {
                const size_t at = (size_t)(r0 + i) * a.z_stride + x;
                const float z = a.type == EE_FP32   ? as_global(static_cast<const float *>(a.logits))[at]
                                : a.type == EE_BF16 ? (float)as_global(static_cast<const __bf16 *>(a.logits))[at]
                                                    : (float)as_global(static_cast<const _Float16 *>(a.logits))[at];
                const double q = exp(((double)z - (double)m) * inv_t) * (1.0 / Z);
                const float p = a.probs ? as_global(a.probs)[(size_t)(r0 + i) * a.p_stride + x] : 1.f;
                kept = a.u && (double)as_global(a.u)[r0 + i] * (double)p < q;
            }
            if (!kept && lane == 0) atomicMin(&first_lost, i);
        }
    }
    __syncthreads();
    const int i = first_lost;
    if (wave == 0) {
        AcceptEnd e = {};
        e.rule = rule;
        e.row = r0 + i;
        e.accept = i;
        e.last = i >= n - 1;
        e.best = -1;
        if (n > 0) {
            join_row(a, r0 + i, inv_t, lane, e.m, e.best, e.Z);
            e.inv_Z = 1.0 / e.Z;
            if (rule == 0 && !(e.Z > 0.0 && e.Z < INFINITY)) e.rule = 2;
        } else {
            e.accept = 0;
            e.row = -1;
        }
        if (lane == 0) {
            end = e;
            if (part == 0) a.ends[seq] = e;
        }
    }
    __syncthreads();
    if (n <= 0 || end.rule != 0) return;
    const int first = part * ACC_PART + tid * ACC_EACH;
    float z[ACC_EACH], p[ACC_EACH];
    load_logits(a, end.row, first, z);
    const bool residual = !end.last;
    double w = 0.0;
    if (residual) {
        load_probs(a, end.row, first, as_global(a.drafts)[end.row], p);
#pragma unroll
        for (int k = 0; k < ACC_EACH; ++k)
            if (first + k < a.V) w += weight_of(end, inv_t, z[k], p[k], true);
    } else {
#pragma unroll
        for (int k = 0; k < ACC_EACH; ++k)
            if (first + k < a.V) w += weight_of(end, inv_t, z[k], 0.f, false);
    }
    w = wave_sum_d(w);
    if (lane == 0) ws[wave] = w;
    __syncthreads();
    if (tid == 0) a.weights[(size_t)seq * a.parts + part] = (ws[0] + ws[1]) + (ws[2] + ws[3]);
}

// inclusive sums over the lanes of a wave
__device__ __forceinline__ double wave_scan_d(double x, int lane)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const double y = __shfl_up(x, d, 64);
        x += lane >= d ? y : 0.0;
    }
    return x;
}

__global__ void __launch_bounds__(ACC_THREADS) ee_accept_draw_kernel(AcceptDev a)
{
    __shared__ double ws[ACC_WAVES];
    __shared__ int found, positive;
    __shared__ int part_s;
    __shared__ double before_s, total_s;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, seq = blockIdx.x;
    const AcceptEnd e = a.ends[seq];
    if (e.row < 0 || e.rule != 0) {
        if (tid == 0) {
            a.accept_len[seq] = e.row < 0 ? 0 : e.accept;
            a.next_token[seq] = e.row < 0 ? -1 : e.rule == 1 ? (e.best < a.V ? e.best : 0) : 0;
        }
        return;
    }
    const double inv_t = 1.0 / (double)as_global(a.temperature)[seq];
    const double v = a.v ? (double)as_global(a.v)[e.row] : 0.0;
    bool residual = !e.last;
    // the part that passes v * total: sums of the parts in order, by wave 0
    const double *pw = a.weights + (size_t)seq * a.parts;
    if (wave == 0) {
        double total = 0.0;
        for (int base = 0; base < a.parts; base += 64) total += wave_sum_d(base + lane < a.parts ? pw[base + lane] : 0.0);
        if (lane == 0) total_s = total;
    }
    __syncthreads();
    double total = total_s;
    const bool from_q = residual && !(total > 0.0);      // p covers q everywhere: the row draws from q
    if (from_q) residual = false;
    auto part_weight = [&](int p) {
        if (p >= a.parts) return 0.0;
        if (!from_q) return pw[p];
        const AcceptRow r = a.rows[(size_t)e.row * a.parts + p];
        const double pm = r.m == -INFINITY ? 0.0 : (double)r.m;
        return r.sum != 0.0 ? r.sum * exp((pm - (double)e.m) * inv_t) * e.inv_Z : 0.0;
    };
    if (wave == 0) {
        if (from_q) {
            total = 0.0;
            for (int base = 0; base < a.parts; base += 64) total += wave_sum_d(part_weight(base + lane));
        }
        const double target = v * total;
        double before = 0.0;
        int part = -1, last_part = 0;
        double last_before = 0.0;
        for (int base = 0; base < a.parts && part < 0; base += 64) {
            const double w = part_weight(base + lane), incl = before + wave_scan_d(w, lane);
            const unsigned long long hit = __ballot(w > 0.0 && incl > target), some = __ballot(w > 0.0);
            const double excl = incl - w;
            if (hit) {
                const int l = __builtin_ctzll(hit);
                part = base + l;
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
        if (part < 0) {                                  // (v * total beyond the last sum by rounding)
            part = last_part;
            before = last_before;
        }
        if (lane == 0) {
            part_s = part;
            before_s = before;
            total_s = total;
            found = 0x7FFFFFFF;
            positive = -1;
        }
    }
    __syncthreads();
    const double target = v * total_s;
    const int first = part_s * ACC_PART + tid * ACC_EACH;
    float z[ACC_EACH], p[ACC_EACH];
    load_logits(a, e.row, first, z);
    if (residual) load_probs(a, e.row, first, as_global(a.drafts)[e.row], p);
    double w[ACC_EACH], mine = 0.0;
#pragma unroll
    for (int k = 0; k < ACC_EACH; ++k) {
        w[k] = first + k < a.V ? weight_of(e, inv_t, z[k], residual ? p[k] : 0.f, residual) : 0.0;
        mine += w[k];
    }
    const double incl = wave_scan_d(mine, lane);
    if (lane == 63) ws[wave] = incl;
    __syncthreads();
    double run = before_s;
    for (int q = 0; q < wave; ++q) run += ws[q];
    run += incl - mine;
    int hit = 0x7FFFFFFF, some = -1;
#pragma unroll
    for (int k = 0; k < ACC_EACH; ++k) {
        run += w[k];
        if (w[k] > 0.0) {
            some = first + k;
            if (run > target && hit == 0x7FFFFFFF) hit = first + k;
        }
    }
    if (hit != 0x7FFFFFFF) atomicMin(&found, hit);
    if (some >= 0) atomicMax(&positive, some);
    __syncthreads();
    if (tid == 0) {
        a.accept_len[seq] = e.accept;
        a.next_token[seq] = found != 0x7FFFFFFF ? found : max(positive, 0);
    }
}

static size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

struct AcceptSpace {
    size_t rows, ends, weights, bytes;
    int parts;
};
static AcceptSpace accept_space(const ee_accept_args &p)
{
    AcceptSpace s;
    s.parts = (p.vocab + ACC_PART - 1) / ACC_PART;
    s.rows = 0;
    s.ends = align256((size_t)p.n_rows * s.parts * sizeof(AcceptRow));
    s.weights = s.ends + align256((size_t)p.n_seqs * sizeof(AcceptEnd));
    s.bytes = s.weights + align256((size_t)p.n_seqs * s.parts * sizeof(double));
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
    a.rows = reinterpret_cast<AcceptRow *>(ws + sp.rows);
    a.ends = reinterpret_cast<AcceptEnd *>(ws + sp.ends);
    a.weights = reinterpret_cast<double *>(ws + sp.weights);
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
    hipLaunchKernelGGL(ee_accept_weights_kernel, dim3(a.parts, p->n_seqs), dim3(ACC_THREADS), 0, s, a);
    HIP_TRY(hipGetLastError());
    hipLaunchKernelGGL(ee_accept_draw_kernel, dim3(p->n_seqs), dim3(ACC_THREADS), 0, s, a);
    HIP_TRY(hipGetLastError());
    return EE_OK;
}
