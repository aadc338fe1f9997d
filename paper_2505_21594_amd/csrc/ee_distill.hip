// ee_distill: the divergence of a student's distribution q = softmax(z / T) from a teacher's most likely tokens, and its gradient.
//
//   rest = 1:  L = sum_j p_j (log p_j - log q_j) + pi (log pi - log rho),  pi = 1 - sum p_j,  rho = the sum of q over the tokens that the list does not name;
//              dL/dz_i = (q_i - p_i) / T for those it names, q_i (1 - pi / rho) / T for the others;
//   rest = 0:  p divided by its sum;  L = sum_j p_j (log p_j - log q_j),  dL/dz_i = (q_i - p_i) / T.
//
// Bound by the logits' bytes, read once, and the gradient's, written once (one MI355X: 4096 rows of 32000, bf16, 111 us, 4.7 TB/s): a workgroup holds its row in
// registers (RowPart) from the sums to the gradient. Rows that are too few to fill the chip, or too long for a workgroup, are taken in parts by two launches, of
// which the second reads the logits again. The tokens that the list names are marked in LDS, one bit each, a thread's bits in one word, and left out of the sums:
// rho is a sum of its own, not a difference.  In powers of two, c = log2(e) / T rounded to fp32 (another temperature by 2^-24 of it, the same one everywhere:
// exponents put right beside sums that are not would take the digits of a small divergence): with r and S' = sum 2^(z c - r) the others' largest exponent and sum, R
// the row's largest and A = 2^(r - R) / S their share's scale, rho = A S' and q_i (1 - pi / rho) = 2^(z_i c - r) (A - pi / S'). Everything that a row has once is in
// 64 bits: the loss is a small difference of large terms.
#include "ee_vocab.hpp"

namespace ee {

struct DistillPart {
    double sum;                        // sum 2^(z c - r) over the tokens that the list does not name
    double r;                          // the largest z c of them: rounded to fp32, or as it is where that is beyond FAR
};

struct DistillDev {
    const void *logits;
    const int *ids;
    const float *logprobs, *d_loss;
    float *loss;
    void *d_logits;
    DistillPart *part;                 // [n_rows][parts]
    float *z;                          // [n_rows][top]  logits of the list's tokens
    long long stride, grad_stride;
    int type, grad_type, V, top, rest, parts, length;
    float c;                           // log2(e) / T
};

// The teacher's list of a row: a lane of a wave for each entry.
struct Entry {
    int id;                            // -1: no entry
    float z;
    double lp;
};
__device__ __forceinline__ Entry entry_of(const DistillDev &a, int row, int lane)
{
    Entry e = {-1, 0.f, 0.0};
    const size_t at = (size_t)row * a.top + min(lane, a.top - 1);      // (no branch before the loads: they go out together with others)
    const int id = as_global(a.ids)[at];
    const float lp = as_global(a.logprobs)[at];
    if (lane < a.top && id >= 0 && id < a.V && lp != -INFINITY) {
        e.id = id;
        e.lp = (double)lp;
    }
    return e;
}

__device__ __forceinline__ double readlane_d(double x, int l)
{
    const unsigned long long b = (unsigned long long)__double_as_longlong(x);
    return join_d((unsigned)__builtin_amdgcn_readlane((int)(unsigned)b, l), (unsigned)__builtin_amdgcn_readlane((int)(unsigned)(b >> 32), l));
}

// What the list alone says; one wave calls it (while its row is on the way).  The log-probability of a token that is named twice becomes that of both; with rest = 0 they become relative
// to the largest, so that a list whose probabilities are all below the numbers of 64 bits has a sum.
struct ListTerms {
    double p, both, share;             // the lane's share of the loss (its probability; its token's where it is the first of several that name it, and 0 of the others), its token's, all entries'
    int distinct;                      // tokens that are named
    bool first;                        // the lane's token is named here for the first time
};
__device__ __forceinline__ ListTerms list_terms(const DistillDev &a, Entry &e)
{
    ListTerms t;
    const int lane = threadIdx.x & 63;
    if (!a.rest) {
        const float most = wave_max_f(e.id >= 0 ? (float)e.lp : -INFINITY);
        if (most != -INFINITY) e.lp -= (double)most;
    }
    t.p = e.id >= 0 ? exp(e.lp) : 0.0;
    // a token that is named twice has both probabilities (few lists do that: the sums only where one does)
    unsigned long long again = 0;                            // lanes behind one that names the same token
#pragma unroll 4
    for (int i = 0; i < a.top; ++i) again |= __ballot(__builtin_amdgcn_readlane(e.id, i) == e.id) & ~0ull << i << 1;
    t.first = e.id >= 0 && !(again >> lane & 1);
    t.both = t.p;
    t.share = wave_sum_d(t.p);
    if (__builtin_expect(__ballot(e.id >= 0 && !t.first) != 0, 0)) {
        int times = 0;
        t.both = 0.0;
        for (int i = 0; i < a.top; ++i) {
            const double other = readlane_d(t.p, i);
            if (__builtin_amdgcn_readlane(e.id, i) == e.id) {
                t.both += other;
                ++times;
            }
        }
        if (e.id >= 0 && times > 1) {
            e.lp = log(t.both);
            t.p = t.first ? t.both : 0.0;
        }
    }
    t.distinct = __popcll(__ballot(t.first));
    return t;
}

// A row's numbers from the others' maximum and sum and from its list; one wave calls it.
struct RowTerms {
    double loss;
    float others;                      // gradient of a token that the list does not name: others * 2^(z c - r)
    float mine;                        // gradient of the lane's token
};
__device__ __forceinline__ RowTerms row_terms(const DistillDev &a, const Entry &e, const ListTerms &t, double r_rest, double s_rest, float d_loss)
{
    constexpr double LN2 = 0.6931471805599453;
    RowTerms r;
    const bool in = e.id >= 0;
    const double c = (double)a.c, p = t.p, share = t.share;
    const double largest = fmax(r_rest, (double)wave_max_f(in ? e.z : -INFINITY) * c), R = largest == -INFINITY ? 0.0 : largest;
    const double z = (double)e.z * c - R, q1 = in ? exp2(z) : 0.0;
    const double down = r_rest == -INFINITY ? 0.0 : r_rest - R, scale_rest = r_rest == -INFINITY ? 0.0 : exp2(down);
    const double S = wave_sum_d(t.first ? q1 : 0.0) + (s_rest != 0.0 ? s_rest * scale_rest : 0.0);
    const bool valid = S > 0.0 && S < INFINITY;
    const double log_S = log2(S), A = scale_rest / S;
    double others, scale = 1.0, shift = 0.0, tail = 0.0;
    if (a.rest) {
        const double pi = share < 1.0 ? 1.0 - share : share >= 1.0 ? 0.0 : share;        // (NaN stays)
        others = A;
        if (pi != 0.0 && t.distinct < a.V) {
            others = s_rest > 0.0 ? A - pi / s_rest : 0.0;
            tail = s_rest > 0.0 ? pi * (log2(pi) - (down + log2(s_rest) - log_S)) * LN2 : (double)INFINITY;
            if (s_rest != s_rest || pi != pi) others = tail = (double)NAN;
        }
    } else {
        scale = share > 0.0 ? 1.0 / share : share == 0.0 ? 0.0 : (double)NAN;
        shift = share > 0.0 ? log(share) : 0.0;
        others = share == 0.0 ? 0.0 : A;
    }
    const double term = in && p != 0.0 && scale != 0.0 ? p * scale * (e.lp - shift - (z - log_S) * LN2) : 0.0;
    r.loss = wave_sum_d(term) + tail;
    double g = share == 0.0 && !a.rest ? 0.0 : q1 / S - t.both * scale;
    if (!valid) r.loss = others = g = (double)NAN;
    const double weight = (double)d_loss * (c * LN2);
    r.others = (float)(others * weight);
    r.mine = (float)(g * weight);
    return r;
}

// The others' largest exponent and sum from the parts of a row, x: of lane l its part l (or any other past the last); one wave calls it.
__device__ __forceinline__ DistillPart first_part(const DistillDev &a, int row, int lane) { return a.part[(size_t)row * a.parts + min(lane, a.parts - 1)]; }
__device__ __forceinline__ double join_parts(const DistillDev &a, int row, int lane, DistillPart x, double &r)
{
    const DistillPart *parts = a.part + (size_t)row * a.parts;
    r = x.r;
    for (int p = lane + 64; p < a.parts; p += 64) r = fmax(r, parts[p].r);
    r = wave_max_d(r);
    double S = 0.0;
    for (int p = lane; p < a.parts;) {
        if (x.sum != 0.0) S += x.sum * (x.r == -INFINITY ? 1.0 : exp2(x.r - r));
        p += 64;
        if (p < a.parts) x = parts[p];
    }
    return wave_sum_d(S);
}

enum DistillMode { WHOLE = 0, STATS = 1, GRAD = 2 };

// (512 threads: six waves a SIMD with 20 to 28 bytes of spill, of wave 0's arithmetic with doubles; five without any: 4096 rows of 32000 130 us for 111, 300 of 200003 86.5 for 85.)
template <int TYPE, int E, int NT, int MODE>
__global__ void __launch_bounds__(NT, NT == 512 ? 6 : 4) ee_distill_kernel(DistillDev a)
{
    typedef RowPart<TYPE, E, NT> Part;
    constexpr int N = Part::N, WAVES = NT / 64;
    __shared__ uint32_t named[MODE == GRAD ? 1 : NT * E / 4];       // a byte for each chunk, a bit for each of its elements
    __shared__ float wr[WAVES];
    __shared__ double ws[WAVES], kept[MODE == WHOLE ? 4 : 1][64];
    __shared__ float kept_z[64];
    __shared__ float others_s, ref_s, taken_s;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int row = a.parts == 1 ? blockIdx.x : blockIdx.x / a.parts, part = a.parts == 1 ? 0 : blockIdx.x - row * a.parts;
    const int first = part * a.length, len = min(a.length, a.V - first);
    const void *logits = row_at(a.logits, TYPE, (size_t)row * a.stride);
    Entry e = {-1, 0.f, 0.0};
    ListTerms list = {0.0, 0.0, 0.0, 0, false};
    if (wave == 0) e = entry_of(a, row, lane);
    Part z;
    z.load(row_at(logits, TYPE, first), len, tid);
    if (wave == 0) {
        if (e.id >= 0) e.z = MODE == GRAD ? as_global(a.z)[(size_t)row * a.top + lane] : logit_at(TYPE, logits, e.id);
        if (MODE == STATS && part == 0 && lane < a.top) as_global_mut(a.z)[(size_t)row * a.top + lane] = e.z;
    }
    const int at = e.id - first;
    const bool here = e.id >= 0 && at >= 0 && at < len;
    double r_rest = 0.0;
    float ref = 0.f;                                         // of the row's exponents, where the gradient is taken
    if constexpr (MODE != GRAD) {
#pragma unroll
        for (int i = 0; i < E / 4; ++i) named[i * NT + tid] = 0;
        __syncthreads();
        if (here) {
            const int q = at / N, byte = (q % NT) * E + q / NT;
            atomicOr(&named[byte / 4], 1u << (byte % 4 * 8 + at % N));
        }
        if (MODE == WHOLE && wave == 0) {
            // (in LDS between the walks over the row: in registers these cost every wave spills)
            list = list_terms(a, e);
            kept[0][lane] = e.lp;
            kept[1][lane] = list.p;
            kept[2][lane] = list.both;
            kept[3][lane] = list.share;
            kept_z[lane] = e.z;
        }
        __syncthreads();
        // (Twice only where the largest logit is beyond FAR: the second time all of them are less by it.)
        float part_r, taken = 0.f;
        for (int pass = 0;; ++pass) {
            // (the named ones become -infinity, which no sum notices)
            float m = -INFINITY;
#pragma unroll
            for (int c = 0; c < E; ++c) {
                const uint32_t marks = named[tid * (E / 4) + c / 4] >> (c % 4 * 8) & 255u;
                if (marks) z.drop(c, marks);
                float x[N];
                z.chunk(c, x);
#pragma unroll
                for (int i = 0; i < N; ++i) m = larger(m, x[i]);
            }
            const float r = m * a.c, ref = reference_of(r);
            float s = 0.f;
            z.again(m);
#pragma unroll
            for (int c = 0; c < E; ++c) {
                float x[N];
                z.chunk(c, x);
#pragma unroll
                for (int i = 0; i < N; ++i) s += __builtin_amdgcn_exp2f(fmaf(x[i], a.c, -ref));
            }
            const float wave_r = wave_max_f(r);
            if (lane == 0) wr[wave] = wave_r;
            __syncthreads();
            part_r = wr[0];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) part_r = fmaxf(part_r, wr[w]);
            const double S1 = wave_sum_d((double)(s * __builtin_amdgcn_exp2f(r < -BELOW ? 0.f : r - part_r)));
            if (lane == 0) ws[wave] = S1;
            __syncthreads();
            if (pass || !(fabsf(part_r) > FAR)) break;
            float most = wave_max_f(m);
            if (lane == 0) wr[wave] = most;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < WAVES; ++w) most = fmaxf(most, wr[w]);
            if (fabsf(most) == INFINITY) break;              // (the sums are 0 or NaN, as they have to be)
            __syncthreads();
            taken = most;
            z.less(taken);
        }
        r_rest = (double)part_r + (double)taken * (double)a.c;
        ref = part_r == -INFINITY ? 0.f : part_r;
        if constexpr (MODE == STATS) {
            if (tid == 0) {
                DistillPart p;
                p.sum = ws[0];
                for (int w = 1; w < WAVES; ++w) p.sum += ws[w];
                p.r = r_rest;
                a.part[(size_t)row * a.parts + part] = p;
            }
            return;
        }
    }
    const float weight = a.d_loss ? as_global(a.d_loss)[row] : 1.f;
    const bool nothing = __builtin_amdgcn_readfirstlane(__float_as_int(weight) << 1) == 0;       // (a weight of 0, whatever the logits are)
    float mine = 0.f;
    bool store_mine = false;
    if (wave == 0) {
        double S;
        if constexpr (MODE == GRAD) {
            list = list_terms(a, e);
            S = join_parts(a, row, lane, first_part(a, row, lane), r_rest);
        } else {
            S = ws[0];
            for (int w = 1; w < WAVES; ++w) S += ws[w];
            e.lp = kept[0][lane];
            list.p = kept[1][lane];
            list.both = kept[2][lane];
            list.share = kept[3][lane];
            e.z = kept_z[lane];
        }
        const RowTerms r = row_terms(a, e, list, r_rest, S, weight);
        if (lane == 0) {
            others_s = r.others;
            if constexpr (MODE == GRAD) {
                const bool far = fabs(r_rest) > (double)FAR && fabs(r_rest) < (double)INFINITY;
                taken_s = far ? (float)(r_rest / (double)a.c) : 0.f;                     // (the logit whose product r is, all 48 bits of it)
                ref_s = far || r_rest == -INFINITY ? 0.f : (float)r_rest;
            }
            if (a.loss && part == 0) as_global_mut(a.loss)[row] = (float)r.loss;
        }
        mine = nothing ? 0.f : r.mine;
        store_mine = list.first && here;
    }
    if (!a.d_logits) return;
    __syncthreads();
    const float others = others_s;
    if constexpr (MODE == GRAD) {
        const float taken = __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(taken_s)));
        ref = ref_s;
        if (taken != 0.f) z.less(taken);
    }
    const size_t out = (size_t)row * a.grad_stride + first;
    auto gradient = [&](const u32x4_t &raw, float (&x)[N]) __attribute__((always_inline)) {
        Part::values(raw, x);
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = __builtin_amdgcn_exp2f(fmaf(x[i], a.c, -ref)) * others;
        if (nothing)
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] = 0.f;
    };
    z.again(others);
#pragma unroll
    for (int c = 0; c < E; ++c) {
        const int from = Part::offset(c, tid);
        if (from + N > len) continue;
        float x[N];
        gradient(z.raw[c], x);
        store_some<N>(a.grad_type, a.d_logits, out + from, x);
    }
    const int last = len / N;                                // the chunk that the part's end is in
    if (len % N != 0 && tid == last % NT) {
        u32x4_t end = z.raw[0];
#pragma unroll
        for (int c = 1; c < E; ++c)
            if (c == last / NT) end = z.raw[c];
        float x[N];
        gradient(end, x);
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (last * N + i < len) store_one(a.grad_type, a.d_logits, out + last * N + i, x[i]);
    }
    wait_vmem();                                             // the workgroup's stores are there: the named tokens' go on top of them
    __syncthreads();
    if (store_mine) store_one(a.grad_type, a.d_logits, out + at, mine);
}

// The loss of rows in parts, where no gradient is wanted: a wave for each row.
__global__ void __launch_bounds__(256) ee_distill_loss_kernel(DistillDev a, int n_rows)
{
    const int lane = threadIdx.x & 63, row = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= n_rows) return;
    const DistillPart part = first_part(a, row, lane);
    const float z = as_global(a.z)[(size_t)row * a.top + min(lane, a.top - 1)];
    Entry e = entry_of(a, row, lane);
    e.z = z;
    double r_rest;
    const double S = join_parts(a, row, lane, part, r_rest);
    const ListTerms list = list_terms(a, e);
    const RowTerms r = row_terms(a, e, list, r_rest, S, 1.f);
    if (lane == 0) as_global_mut(a.loss)[row] = (float)r.loss;
}

struct DistillPlan {
    int shape;                         // threads and chunks a thread: 256 x 4, 512 x 8, 1024 x 8, 1024 x 16
    bool whole;                        // one launch does all of a row; otherwise the sums have one of their own
    RowSplit split;
    size_t part_bytes, bytes;
};
static DistillPlan plan_distill(const ee_distill_args &p, bool grad)
{
    DistillPlan pl;
    const int n = p.dtype == EE_FP32 ? 4 : 8, room[4] = {256 * 4 * n, 512 * 8 * n, 1024 * 8 * n, 1024 * 16 * n};
    // us, one launch for all of a row / two, of which the second reads the logits again.  With a gradient: 600 rows of 100003 85 / 102, 1500 of 70000 139 / 137, fp32 600 of 50003 68 / 83 and 1500 of 60000 154 / 213, so that a row
    // that a workgroup can hold is one part, in the smallest workgroup that can where rows fill the chip and of 1024 threads where they do not (five rows of 32000, fp32, by sixteen
    // chunks a thread 10.6, by eight 8.7).  The loss alone: 4096 rows of 32000 68 / 62, 600 of 100003 61 / 44, 1500 of 70000 88 / 48, five of 32000 6.9 / 7.1: the first launch alone has half the registers.
    const bool many = p.n_rows >= 256;
    pl.whole = grad && p.vocab <= room[3];
    if (pl.whole) {
        pl.shape = p.vocab <= room[0] ? 0 : p.vocab <= room[1] && many ? 1 : p.vocab <= room[2] ? 2 : 3;
        pl.split.parts = 1;
        pl.split.length = p.vocab;
    } else {
        pl.shape = many && p.vocab > room[0] ? 1 : 0;
        pl.split = split_rows(p.n_rows, p.vocab, room[pl.shape], 256 * n, many ? 1 : 512);
    }
    pl.part_bytes = pl.whole ? 0 : align256((size_t)p.n_rows * pl.split.parts * sizeof(DistillPart));
    pl.bytes = pl.part_bytes + (pl.whole ? 0 : align256((size_t)p.n_rows * p.top * sizeof(float)));
    return pl;
}

static int check_distill(const char *call, const ee_distill_args *p)
{
    if (!p) return fail(EE_EINVAL, "%s: null argument", call);
    if (p->device < 0) return fail(EE_EINVAL, "%s: device %d", call, p->device);
    if (p->dtype < EE_BF16 || p->dtype > EE_FP32 || p->grad_dtype < EE_BF16 || p->grad_dtype > EE_FP32)
        return fail(EE_EINVAL, "%s: unknown element type %d or %d", call, p->dtype, p->grad_dtype);
    if (p->vocab < 1 || p->vocab > 1 << 24) return fail(EE_EINVAL, "%s: vocab %d out of range", call, p->vocab);
    if (p->n_rows < 0 || p->n_rows > 1 << 20) return fail(EE_EINVAL, "%s: n_rows %d not in [0,2^20]", call, p->n_rows);
    if (p->top < 1 || p->top > EE_MAX_TOP) return fail(EE_EINVAL, "%s: top %d not in [1,%d]", call, p->top, EE_MAX_TOP);
    if (p->rest != 0 && p->rest != 1) return fail(EE_EINVAL, "%s: rest must be 0 or 1", call);
    if (!(p->temperature > 0.f) || !isfinite(p->temperature) || !isfinite(1.5f / p->temperature)) return fail(EE_EINVAL, "%s: temperature must be positive and finite", call);
    return EE_OK;
}

}  // namespace ee

using namespace ee;

extern "C" int ee_distill_workspace(const ee_distill_args *p, size_t *bytes)
{
    static const char *const call = "ee_distill_workspace";
    if (!bytes) return fail(EE_EINVAL, "%s: null argument", call);
    *bytes = 0;
    int rc = check_distill(call, p);
    if (rc == EE_OK && p->n_rows) *bytes = std::max(plan_distill(*p, false).bytes, plan_distill(*p, true).bytes);   // (whichever results are wanted)
    return rc;
}

typedef void (*distill_kernel_t)(DistillDev);
template <int TYPE>
static distill_kernel_t distill_kernel(int shape, int mode)
{
    if (mode == WHOLE)
        return shape == 0 ? ee_distill_kernel<TYPE, 4, 256, WHOLE> : shape == 1 ? ee_distill_kernel<TYPE, 8, 512, WHOLE> : shape == 2 ? ee_distill_kernel<TYPE, 8, 1024, WHOLE> : ee_distill_kernel<TYPE, 16, 1024, WHOLE>;
    if (mode == STATS) return shape == 0 ? ee_distill_kernel<TYPE, 4, 256, STATS> : ee_distill_kernel<TYPE, 8, 512, STATS>;
    return shape == 0 ? ee_distill_kernel<TYPE, 4, 256, GRAD> : ee_distill_kernel<TYPE, 8, 512, GRAD>;
}

extern "C" int ee_distill(const ee_distill_args *p, void *workspace, size_t workspace_bytes, void *stream)
{
    static const char *const call = "ee_distill";
    int rc = check_distill(call, p);
    if (rc != EE_OK) return rc;
    if (p->n_rows == 0 || (!p->loss && !p->d_logits)) return EE_OK;
    if (!p->logits || !p->ids || !p->logprobs) return fail(EE_EINVAL, "%s: null logits, ids or logprobs", call);
    if (p->n_rows > 1 && (p->logits_stride < p->vocab || p->logits_stride >= (int64_t)1 << 40 || (p->d_logits && (p->d_logits_stride < p->vocab || p->d_logits_stride >= (int64_t)1 << 40))))
        return fail(EE_EINVAL, "%s: a row stride is smaller than vocab", call);
    if (p->d_logits == p->logits && (p->dtype != p->grad_dtype || (p->n_rows > 1 && p->logits_stride != p->d_logits_stride)))
        return fail(EE_EINVAL, "%s: d_logits may be logits only with the same type and stride", call);
    if (!aligned(p->logits, size_of_type(p->dtype)) || !aligned(p->d_logits, size_of_type(p->grad_dtype)))
        return fail(EE_EINVAL, "%s: logits or d_logits are not aligned to their type", call);
    for (const void *x : {(const void *)p->ids, (const void *)p->logprobs, (const void *)p->loss, (const void *)p->d_loss})
        if (!aligned(x, 4)) return fail(EE_EINVAL, "%s: int32 and fp32 arrays must be 4-byte aligned", call);
    const DistillPlan pl = plan_distill(*p, p->d_logits != nullptr);
    if (pl.bytes > workspace_bytes || (pl.bytes && (!workspace || !aligned(workspace, 256))))
        return fail(EE_EINVAL, "%s: the workspace has %zu bytes of %zu, or is not 256-byte aligned", call, workspace_bytes, pl.bytes);
    if ((long long)p->n_rows * pl.split.parts >= 1 << 22) return fail(EE_EINVAL, "%s: too many rows of so many tokens", call);
    if (p->loss && p->loss == p->d_loss) return fail(EE_EINVAL, "%s: loss and d_loss must be arrays of their own", call);    // (a row's parts read d_loss when the first one writes the loss)
    DistillDev a;
    a.logits = p->logits;
    a.ids = p->ids;
    a.logprobs = p->logprobs;
    a.d_loss = p->d_loss;
    a.loss = p->loss;
    a.d_logits = p->d_logits;
    a.part = static_cast<DistillPart *>(workspace);
    a.z = reinterpret_cast<float *>(static_cast<unsigned char *>(workspace) + pl.part_bytes);
    a.stride = p->n_rows > 1 ? p->logits_stride : 0;
    a.grad_stride = p->n_rows > 1 ? p->d_logits_stride : 0;
    a.type = p->dtype;
    a.grad_type = p->grad_dtype;
    a.V = p->vocab;
    a.top = p->top;
    a.rest = p->rest;
    a.parts = pl.split.parts;
    a.length = pl.split.length;
    a.c = (float)(1.4426950408889634 / (double)p->temperature);
    DeviceScope scope(p->device);
    HIP_TRY(scope.status);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const auto kernel = [&](int mode) {
        return p->dtype == EE_BF16 ? distill_kernel<EE_BF16>(pl.shape, mode) : p->dtype == EE_FP16 ? distill_kernel<EE_FP16>(pl.shape, mode) : distill_kernel<EE_FP32>(pl.shape, mode);
    };
    const dim3 grid((unsigned)(p->n_rows * a.parts)), block(pl.shape == 0 ? 256 : pl.shape == 1 ? 512 : 1024);
    hipLaunchKernelGGL(kernel(pl.whole ? WHOLE : STATS), grid, block, 0, s, a);
    HIP_TRY(hipGetLastError());
    if (!pl.whole) {
        if (a.d_logits)
            hipLaunchKernelGGL(kernel(GRAD), grid, block, 0, s, a);
        else
            hipLaunchKernelGGL(ee_distill_loss_kernel, dim3((unsigned)((p->n_rows + 3) / 4)), dim3(256), 0, s, a, p->n_rows);
        HIP_TRY(hipGetLastError());
    }
    return EE_OK;
}
