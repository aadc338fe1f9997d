// ee_score_tokens: log-probabilities of given tokens, a row's entropy and its most likely tokens, in one pass over the logits.
//
//   log p_i = z_i / T - L,  L = log sum exp(z / T);   H = L - sum p z / T;   the `top` largest logits, of equal ones the lower token first.
//
// Bound by the logits' bytes (one MI355X: 2041 rows of 32000, bf16, 26.8 us without lists, 4.9 TB/s; with lists of 20 38.5).  A workgroup holds a row, or a part of
// it, in registers (RowPart): the sums and the search for the largest read memory once.  Sums: every thread takes exponentials relative to its own maximum, so that
// nothing waits for the row's; they meet in 64 bits.  All of it in powers of two: with c = log2(e) / T rounded to fp32 (another temperature by 2^-24 of it; log-
// probabilities are put right to the first order in 64 bits, exponent and sum) an exponential is 2^(z c - r), one multiply-add and one instruction, r a number of
// fp32 itself, so that nothing is lost where the sums are put together. The largest: a wave's bound for n is the n-th largest among the maxima of its 256 groups of
// chunks, which n of its elements reach.  The least of w waves' bounds for top / w is one that `top` elements reach; the chunks with an element above it go to LDS,
// then their elements above it (a few more than `top`), and of those one wave keeps exactly `top`.  (Only waves all of whose lanes have a chunk give a bound: one with a chunk or two
// would let everything through, 2041 rows of 1040 tokens with lists of 64 in 150 us for 20.)  Where this overflows, the row takes as many rounds as tokens are wanted: rows of so many equal
// elements, or of so many that share the 16 bits of the bound's key (fp32 beside a large offset), or one wave's so far below the others' (2041 rows of 32000 all alike, lists of 20: 463 us).
#include "ee_vocab.hpp"

namespace ee {

constexpr int SC_THREADS = 256, SC_WAVES = SC_THREADS / 64;   // of the second launch
constexpr int SC_CHUNKS = 512;         // chunks with a candidate that LDS has room for
constexpr int SC_CAND = 1024;          // candidates

struct ScorePart {
    double sum, dot;                   // sum 2^(z c - r),  sum (z c - r) 2^(z c - r)
    double r;
    int count, unused;                 // candidates that it has
};
// A token in the order of the results: the larger key first, of equal ones the lower token.
struct Cand {
    unsigned key;
    int token;
};

struct ScoreDev {
    const void *logits;
    const int *tokens;
    float *logprob, *entropy, *top_logprobs;
    int *top_ids;
    long long stride;
    ScorePart *part;                   // [n_rows][parts]
    Cand *cand;                        // [n_rows][parts][top]
    int type, n_rows, V, top, parts, length;
    float c;                           // log2(e) / T
    double fix;                        // ... by the c that it is rounded to
};

// floats in the order of unsigned numbers (-0 as +0)
__device__ __forceinline__ unsigned key_of(float x)
{
    const int b = __float_as_int(x + 0.f);
    return (unsigned)(b < 0 ? ~b : b | (int)0x80000000);
}
__device__ __forceinline__ float of_key(unsigned k) { return __int_as_float((int)k < 0 ? (int)(k & 0x7FFFFFFFu) : (int)~k); }
constexpr unsigned KEY_LEAST = 0x00800000u;      // of the lowest finite number

// Largest t whose bits below `low` are zero and that at least k of the wave's 4 x 64 keys (of bits below `bits`) reach; 0 if there are fewer than k.
__device__ __forceinline__ unsigned wave_bound(const unsigned (&u)[4], int k, int bits, int low)
{
    unsigned t = 0;
    for (int b = bits - 1; b >= low; --b) {
        const unsigned x = t | 1u << b;
        int n = 0;
#pragma unroll
        for (int g = 0; g < 4; ++g) n += __popcll(__ballot(u[g] >= x));
        if (n >= k) t = x;
    }
    return t;
}

// Bits of a key that say nothing: of logits of 16 bits.
__host__ __device__ constexpr int idle_bits(int type) { return type == EE_FP32 ? 0 : type == EE_BF16 ? 16 : 13; }

__device__ __forceinline__ int lanes_before(unsigned long long who) { return __builtin_amdgcn_mbcnt_hi((unsigned)(who >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)who, 0)); }

// Of the wave's 4 x 64 candidates (key 0: none) the k best to list[0 ..], in no order; their number.
__device__ __forceinline__ int wave_best(const unsigned (&key)[4], const int (&token)[4], int k, int idle, Cand *list)
{
    unsigned u[4];
#pragma unroll
    for (int g = 0; g < 4; ++g) u[g] = key[g] >> idle;
    const unsigned t = max(wave_bound(u, k, 32 - idle, 0), 1u);
    int above = 0, equal = 0;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        above += __popcll(__ballot(u[g] > t));
        equal += __popcll(__ballot(u[g] == t));
    }
    // of those equal to the bound the lowest tokens: the largest bound on their complements that enough of them reach
    unsigned v = 0;
    if (above + equal > k) {
        unsigned w[4];
#pragma unroll
        for (int g = 0; g < 4; ++g) w[g] = u[g] == t ? 0x1FFFFFFu - (unsigned)token[g] : 0u;
        v = wave_bound(w, k - above, 25, 0);
    }
    int n = 0;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const bool in = u[g] > t || (u[g] == t && 0x1FFFFFFu - (unsigned)token[g] >= v);
        const unsigned long long who = __ballot(in);
        if (in) list[n + lanes_before(who)] = Cand{key[g], token[g]};
        n += __popcll(who);
    }
    return n;
}
// ... of n candidates in LDS; list has room for 64.
__device__ __forceinline__ int wave_best_of(const Cand *cands, int n, int k, int idle, int lane, Cand *list)
{
    unsigned key[4];
    int token[4], kept = 0;
    for (int base = 0; base < n; base += base ? 192 : 256) {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int i = base + g * 64 + lane;
            const bool old = g == 3 && base, in = old ? lane < kept : i < n;
            const Cand x = in ? (old ? list[lane] : cands[i]) : Cand{0, 0};
            key[g] = x.key;
            token[g] = x.token;
        }
        wave_lds_order();
        kept = wave_best(key, token, k, idle, list);
        wave_lds_order();
    }
    return kept;
}

// What one wave writes for a row: its n (at most 64) best in order, and the row's numbers.
__device__ __forceinline__ void write_row(const ScoreDev &a, int row, int lane, double S, double D, double r, const Cand *list, int n)
{
    constexpr double LN2 = 0.6931471805599453;
    const bool valid = S > 0.0 && S < INFINITY;               // (NaN, +infinity or nothing but -infinity: no softmax)
    const double c = (double)a.c, mean = D / S, log_S = valid ? log2(S) : (double)NAN, log_q = log_S + mean * (a.fix - 1.0);   // (d log2 sum 2^(f y) / df = sum q y)
    if (lane == 0) {
        if (a.logprob) {
            const int t = as_global(a.tokens)[row];
            float lp = valid ? -INFINITY : NAN;
            if (valid && t >= 0 && t < a.V) lp = (float)((((double)logit_at(a.type, row_at(a.logits, a.type, (size_t)row * a.stride), t) * c - r) * a.fix - log_q) * LN2);
            as_global_mut(a.logprob)[row] = lp;
        }
        if (a.entropy) as_global_mut(a.entropy)[row] = (float)fmax((log_S - mean) * LN2, valid ? 0.0 : (double)NAN);
    }
    if (a.top == 0) return;
    if (!valid) n = 0;
    const Cand mine = lane < n ? list[lane] : Cand{0, -1};
    int rank = 0;
    for (int i = 0; i < n; ++i) {
        const unsigned k = (unsigned)__builtin_amdgcn_readlane((int)mine.key, i);
        const int t = __builtin_amdgcn_readlane(mine.token, i);
        rank += k > mine.key || (k == mine.key && t < mine.token);
    }
    if (lane < a.top) {
        const size_t at = (size_t)row * a.top + (lane < n ? rank : lane);
        as_global_mut(a.top_ids)[at] = mine.token;
        as_global_mut(a.top_logprobs)[at] = lane < n ? (float)((((double)of_key(mine.key) * c - r) * a.fix - log_q) * LN2) : valid ? -INFINITY : NAN;
    }
}

// The waves' sums from their threads' (relative to the r of each; nothing where that is below -BELOW), relative to the part's r, which comes back.
template <int WAVES>
__device__ __forceinline__ float wave_sums(float r, float s, float d, int lane, int wave, float *wr, double *ws, double *wd)
{
    const float wave_r = wave_max_f(r);
    if (lane == 0) wr[wave] = wave_r;
    __syncthreads();
    float all = wr[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) all = fmaxf(all, wr[w]);
    const float down = r < -BELOW ? 0.f : r - all;            // (such a thread has sums of 0, or of NaN)
    const float scale = __builtin_amdgcn_exp2f(down);
    const double S1 = (double)(s * scale), D1 = (double)(d * scale) + (s != 0.f ? (double)down * S1 : 0.0);
    const double S2 = wave_sum_d(S1), D2 = wave_sum_d(D1);
    if (lane == 0) {
        ws[wave] = S2;
        wd[wave] = D2;
    }
    return all;
}

template <int TYPE, int E, int NT>
__global__ void __launch_bounds__(NT, NT == 512 ? 6 : 4) ee_score_kernel(ScoreDev a)
{
    typedef RowPart<TYPE, E, NT> Part;
    constexpr int N = Part::N, WAVES = NT / 64;
    __shared__ float wr[WAVES];
    __shared__ double ws[WAVES], wd[WAVES];
    __shared__ unsigned bound[WAVES];
    __shared__ u32x4_t chunks[SC_CHUNKS];
    __shared__ int chunk_at[SC_CHUNKS];
    __shared__ Cand cands[SC_CAND], best[64];
    __shared__ int n_chunks, n_cands;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int row = a.parts == 1 ? blockIdx.x : blockIdx.x / a.parts, part = a.parts == 1 ? 0 : blockIdx.x - row * a.parts;
    const int first = part * a.length, len = min(a.length, a.V - first);
    Part z;
    z.load(row_at(a.logits, TYPE, (size_t)row * a.stride + first), len, tid);
    if (tid == 0) n_chunks = n_cands = 0;
    float cm[E], m = -INFINITY;
#pragma unroll
    for (int c = 0; c < E; ++c) {
        float x[N];
        z.chunk(c, x);
        cm[c] = x[0];
#pragma unroll
        for (int i = 1; i < N; ++i) cm[c] = larger(cm[c], x[i]);
        m = larger(m, cm[c]);
    }
    const float r = m * a.c, ref = reference_of(r);
    float s = 0.f, d = 0.f;
    z.again(m);
#pragma unroll
    for (int c = 0; c < E; ++c) {
        float x[N];
        z.chunk(c, x);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float y = fmaf(x[i], a.c, -ref), e = __builtin_amdgcn_exp2f(y);
            s += e;
            d += fmaxf(y, -3e38f) * e;                       // (-infinity times 0 is nothing)
        }
    }
    z.again(s, d);
    const int k = min(a.top, len), holding = max(min(len / (64 * N), WAVES), 1);             // (waves all of whose lanes have a chunk: as many groups as a list is long)
    if (k > 0) {
        unsigned u[4];
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            float x = -INFINITY;
#pragma unroll
            for (int c = g; c < E; c += 4) x = larger(x, cm[c]);
            u[g] = key_of(x);
        }
        const unsigned t = wave < holding ? wave_bound(u, (k + holding - 1) / holding, 32, 16) : ~0u;
        if (lane == 0) bound[wave] = t;
    }
    const float part_r = wave_sums<WAVES>(r, s, d, lane, wave, wr, ws, wd);
    __syncthreads();
    int count = 0;
    if (k > 0) {
        unsigned least = bound[0];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) least = min(least, bound[w]);
        const float t = of_key(max(least, KEY_LEAST));
        int mine = 0;
#pragma unroll
        for (int c = 0; c < E; ++c) mine += __popcll(__ballot(cm[c] >= t));
        int at = 0;
        if (lane == 0 && mine) at = atomicAdd(&n_chunks, mine);
        at = __builtin_amdgcn_readfirstlane(at);
        if (mine)
#pragma unroll
            for (int c = 0; c < E; ++c) {
                const bool in = cm[c] >= t;
                const unsigned long long who = __ballot(in);
                const int place = at + lanes_before(who);
                if (in && place < SC_CHUNKS) {
                    chunks[place] = z.raw[c];
                    chunk_at[place] = Part::offset(c, tid);
                }
                at += __popcll(who);
            }
        __syncthreads();
        const int n = min(n_chunks, SC_CHUNKS);
        for (int base = wave * 64; base < n * N; base += NT) {
            const int i = base + lane;
            float x = -INFINITY;
            if (i < n * N) {
                if constexpr (TYPE == EE_FP32)
                    x = reinterpret_cast<const float *>(chunks)[i];
                else if constexpr (TYPE == EE_BF16)
                    x = bf16_to_f32(reinterpret_cast<const uint16_t *>(chunks)[i]);
                else
                    x = (float)reinterpret_cast<const _Float16 *>(chunks)[i];
            }
            const bool in = x >= t;
            const unsigned long long who = __ballot(in);
            int place = 0;
            if (lane == 0 && who) place = atomicAdd(&n_cands, __popcll(who));
            place = __builtin_amdgcn_readfirstlane(place) + lanes_before(who);
            if (in && place < SC_CAND) cands[place] = Cand{key_of(x), first + chunk_at[i / N] + i % N};
        }
        __syncthreads();
        if (n_chunks <= SC_CHUNKS && n_cands <= SC_CAND) {
            if (wave == 0) count = wave_best_of(cands, n_cands, k, idle_bits(TYPE), lane, best);
        } else {
            // many equal ones: a round for each token, the best behind the last one in order, by reading the part again (registers that live through this cost
            // every row of a call).  (Of finite logits; -infinity is none.)
            __shared__ unsigned long long round_best[WAVES];
            unsigned long long last = ~0ull;
            const void *part_at = row_at(a.logits, TYPE, (size_t)row * a.stride + first);
            for (int r = 0; r < k; ++r) {
                unsigned long long mine_best = 0;
#pragma unroll 1
                for (int at = 0; at < len; at += Part::ROOM / E) {
                    RowPart<TYPE, 1, NT> some;
                    some.load(row_at(part_at, TYPE, at), len - at, tid);
                    float x[N];
                    some.chunk(0, x);
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        const unsigned long long o = (unsigned long long)key_of(x[i]) << 32 | (0x7FFFFFFFu - (unsigned)(first + at + tid * N + i));
                        if (x[i] >= -3.4028235e38f && o < last && o > mine_best) mine_best = o;
                    }
                }
                for (int o = 32; o > 0; o >>= 1) {
                    const unsigned long long other = __shfl_xor(mine_best, o, 64);
                    mine_best = other > mine_best ? other : mine_best;
                }
                if (lane == 0) round_best[wave] = mine_best;
                __syncthreads();
                last = 0;
#pragma unroll
                for (int w = 0; w < WAVES; ++w) last = max(last, round_best[w]);
                __syncthreads();
                if (last == 0) break;
                if (tid == 0) best[r] = Cand{(unsigned)(last >> 32), (int)(0x7FFFFFFFu - (unsigned)last)};
                count = r + 1;
            }
            __syncthreads();
        }
    }
    double R = (double)part_r;
    if (fabsf(part_r) > FAR) {
        // (by reading the part again, as above: few rows do)
        const void *part_at = row_at(a.logits, TYPE, (size_t)row * a.stride + first);
        float most = -INFINITY;
#pragma unroll 1
        for (int at = 0; at < len; at += Part::ROOM / E) {
            RowPart<TYPE, 1, NT> some;
            some.load(row_at(part_at, TYPE, at), len - at, tid);
            float x[N];
            some.chunk(0, x);
#pragma unroll
            for (int i = 0; i < N; ++i) most = fmaxf(most, x[i]);
        }
        most = wave_max_f(most);
        if (lane == 0) wr[wave] = most;                      // (everybody has read it: two barriers since)
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WAVES; ++w) most = fmaxf(most, wr[w]);
        if (fabsf(most) != INFINITY) {                       // (otherwise the sums are 0 or NaN, as they have to be)
            float s = 0.f, d = 0.f;
#pragma unroll 1
            for (int at = 0; at < len; at += Part::ROOM / E) {
                RowPart<TYPE, 1, NT> some;
                some.load(row_at(part_at, TYPE, at), len - at, tid);
                float x[N];
                some.chunk(0, x);
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const float y = (x[i] - most) * a.c, e = __builtin_amdgcn_exp2f(y);
                    s += e;
                    d += fmaxf(y, -3e38f) * e;
                }
            }
            const double S = wave_sum_d((double)s), D = wave_sum_d((double)d);
            if (lane == 0) {
                ws[wave] = S;
                wd[wave] = D;
            }
            R = (double)most * (double)a.c;
            __syncthreads();
        }
    }
    if (wave != 0) return;
    wave_lds_order();
    double S = ws[0], D = wd[0];
    for (int w = 1; w < WAVES; ++w) {
        S += ws[w];
        D += wd[w];
    }
    if (a.parts == 1) {
        write_row(a, row, lane, S, D, R, best, count);
        return;
    }
    const size_t at = (size_t)row * a.parts + part;
    if (lane == 0) {
        ScorePart p;
        p.sum = S;
        p.dot = D;
        p.r = R;
        p.count = count;
        p.unused = 0;
        a.part[at] = p;
    }
    if (lane < count) a.cand[at * a.top + lane] = best[lane];
}

// A row's parts as one.
__global__ void __launch_bounds__(SC_THREADS) ee_score_join_kernel(ScoreDev a)
{
    __shared__ Cand lists[SC_WAVES][64], best[64];
    __shared__ int counts[SC_WAVES];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, row = blockIdx.x;
    const ScorePart *parts = a.part + (size_t)row * a.parts;
    const Cand *cand = a.cand + (size_t)row * a.parts * a.top;
    if (a.top > 0) {
        // a quarter of the parts' lists for each wave, 192 candidates at a time beside the best so far
        const int per = (a.parts + SC_WAVES - 1) / SC_WAVES, from = min(wave * per, a.parts) * a.top, to = min((wave + 1) * per, a.parts) * a.top;
        const int idle = idle_bits(a.type);
        int n = 0;
        for (int base = from; base < to; base += 192) {
            unsigned u[4];
            int token[4];
#pragma unroll
            for (int g = 0; g < 3; ++g) {
                const int i = base + g * 64 + lane;
                bool in = i < to;
                if (in) {
                    const int p = i / a.top;
                    in = i - p * a.top < parts[p].count;
                }
                const Cand x = in ? cand[i] : Cand{0, 0};
                u[g] = x.key;
                token[g] = x.token;
            }
            const Cand x = lane < n ? lists[wave][lane] : Cand{0, 0};
            u[3] = x.key;
            token[3] = x.token;
            wave_lds_order();
            n = wave_best(u, token, a.top, idle, lists[wave]);
            wave_lds_order();
        }
        if (lane == 0) counts[wave] = n;
    }
    __syncthreads();
    if (wave != 0) return;
    int n = 0;
    if (a.top > 0) {
        unsigned u[4];
        int token[4];
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const Cand x = lane < counts[g] ? lists[g][lane] : Cand{0, 0};
            u[g] = x.key;
            token[g] = x.token;
        }
        n = wave_best(u, token, a.top, idle_bits(a.type), best);
        wave_lds_order();
    }
    double r = -INFINITY;
    for (int p = lane; p < a.parts; p += 64) r = fmax(r, parts[p].r);
    r = wave_max_d(r);
    double S = 0.0, D = 0.0;
    for (int p = lane; p < a.parts; p += 64) {
        const ScorePart x = parts[p];
        const double down = x.r == -INFINITY ? 0.0 : x.r - r, e = exp2(down);
        S += x.sum * e;
        if (x.sum != 0.0) D += (x.dot + down * x.sum) * e;
    }
    S = wave_sum_d(S);
    D = wave_sum_d(D);
    write_row(a, row, lane, S, D, r, best, n);
}

typedef void (*score_kernel_t)(ScoreDev);
struct ScorePlan {
    int shape;                         // threads and chunks a thread: 256 x 4, 512 x 8, 1024 x 8
    RowSplit split;
    size_t part_bytes, bytes;
};
// A row that a workgroup can hold is one part: a second launch costs more than what more workgroups save (five rows of 32000 in 32 parts each 13.7 us).
static ScorePlan plan_score(const ee_score_args &p)
{
    ScorePlan pl;
    const int n = p.dtype == EE_FP32 ? 4 : 8, room[3] = {256 * 4 * n, 512 * 8 * n, 1024 * 8 * n};
    const bool many = (long long)p.n_rows * ((p.vocab + room[1] - 1) / room[1]) >= 512;
    pl.shape = p.vocab <= room[0] ? 0 : p.vocab <= room[1] && p.n_rows >= 256 ? 1 : p.vocab <= room[2] && !many ? 2 : many ? 1 : 0;
    pl.split = split_rows(p.n_rows, p.vocab, room[pl.shape], 256 * n, p.vocab <= room[pl.shape] || many ? 1 : 512);
    pl.part_bytes = pl.split.parts > 1 ? align256((size_t)p.n_rows * pl.split.parts * sizeof(ScorePart)) : 0;
    pl.bytes = pl.part_bytes + (pl.split.parts > 1 ? align256((size_t)p.n_rows * pl.split.parts * p.top * sizeof(Cand)) : 0);
    return pl;
}

static int check_score(const char *call, const ee_score_args *p)
{
    if (!p) return fail(EE_EINVAL, "%s: null argument", call);
    if (p->device < 0) return fail(EE_EINVAL, "%s: device %d", call, p->device);
    if (p->dtype < EE_BF16 || p->dtype > EE_FP32) return fail(EE_EINVAL, "%s: unknown element type %d", call, p->dtype);
    if (p->vocab < 1 || p->vocab > 1 << 24) return fail(EE_EINVAL, "%s: vocab %d out of range", call, p->vocab);
    if (p->n_rows < 0 || p->n_rows > 1 << 20) return fail(EE_EINVAL, "%s: n_rows %d not in [0,2^20]", call, p->n_rows);
    if (p->top < 0 || p->top > EE_MAX_TOP) return fail(EE_EINVAL, "%s: top %d not in [0,%d]", call, p->top, EE_MAX_TOP);
    if (!(p->temperature > 0.f) || !isfinite(p->temperature) || !isfinite(1.5f / p->temperature)) return fail(EE_EINVAL, "%s: temperature must be positive and finite", call);
    return EE_OK;
}

}  // namespace ee

using namespace ee;

extern "C" int ee_score_workspace(const ee_score_args *p, size_t *bytes)
{
    static const char *const call = "ee_score_workspace";
    if (!bytes) return fail(EE_EINVAL, "%s: null argument", call);
    *bytes = 0;
    int rc = check_score(call, p);
    if (rc == EE_OK && p->n_rows) *bytes = plan_score(*p).bytes;
    return rc;
}

extern "C" int ee_score_tokens(const ee_score_args *p, void *workspace, size_t workspace_bytes, void *stream)
{
    static const char *const call = "ee_score_tokens";
    int rc = check_score(call, p);
    if (rc != EE_OK) return rc;
    if (p->n_rows == 0) return EE_OK;
    if (!p->logits) return fail(EE_EINVAL, "%s: null logits", call);
    if (p->logprob && !p->tokens) return fail(EE_EINVAL, "%s: logprob without tokens", call);
    if (p->top && (!p->top_ids || !p->top_logprobs)) return fail(EE_EINVAL, "%s: null top_ids or top_logprobs", call);
    if (p->n_rows > 1 && (p->logits_stride < p->vocab || p->logits_stride >= (int64_t)1 << 40)) return fail(EE_EINVAL, "%s: the row stride is smaller than vocab", call);
    if (!aligned(p->logits, size_of_type(p->dtype))) return fail(EE_EINVAL, "%s: logits are not aligned to their type", call);
    for (const void *x : {(const void *)p->tokens, (const void *)p->logprob, (const void *)p->entropy, (const void *)p->top_ids, (const void *)p->top_logprobs})
        if (!aligned(x, 4)) return fail(EE_EINVAL, "%s: int32 and fp32 arrays must be 4-byte aligned", call);
    const ScorePlan pl = plan_score(*p);
    if (pl.bytes > workspace_bytes || (pl.bytes && (!workspace || !aligned(workspace, 256))))
        return fail(EE_EINVAL, "%s: the workspace has %zu bytes of %zu, or is not 256-byte aligned", call, workspace_bytes, pl.bytes);
    if ((long long)p->n_rows * pl.split.parts >= 1 << 22) return fail(EE_EINVAL, "%s: too many rows of so many tokens", call);
    ScoreDev a;
    a.logits = p->logits;
    a.tokens = p->tokens;
    a.logprob = p->logprob;
    a.entropy = p->entropy;
    a.top_ids = p->top_ids;
    a.top_logprobs = p->top_logprobs;
    a.stride = p->n_rows > 1 ? p->logits_stride : 0;
    a.part = static_cast<ScorePart *>(workspace);
    a.cand = reinterpret_cast<Cand *>(static_cast<unsigned char *>(workspace) + pl.part_bytes);
    a.type = p->dtype;
    a.n_rows = p->n_rows;
    a.V = p->vocab;
    a.top = p->top;
    a.parts = pl.split.parts;
    a.length = pl.split.length;
    a.c = (float)(1.4426950408889634 / (double)p->temperature);
    a.fix = 1.4426950408889634 / (double)p->temperature / (double)a.c;
    DeviceScope scope(p->device);
    HIP_TRY(scope.status);
    static const score_kernel_t kernels[3][3] = {{ee_score_kernel<EE_BF16, 4, 256>, ee_score_kernel<EE_BF16, 8, 512>, ee_score_kernel<EE_BF16, 8, 1024>},
                                                 {ee_score_kernel<EE_FP16, 4, 256>, ee_score_kernel<EE_FP16, 8, 512>, ee_score_kernel<EE_FP16, 8, 1024>},
                                                 {ee_score_kernel<EE_FP32, 4, 256>, ee_score_kernel<EE_FP32, 8, 512>, ee_score_kernel<EE_FP32, 8, 1024>}};
    const hipStream_t s = static_cast<hipStream_t>(stream);
    hipLaunchKernelGGL(kernels[p->dtype][pl.shape], dim3((unsigned)(p->n_rows * pl.split.parts)), dim3(256 << pl.shape), 0, s, a);
    HIP_TRY(hipGetLastError());
    if (a.parts > 1) {
        hipLaunchKernelGGL(ee_score_join_kernel, dim3((unsigned)p->n_rows), dim3(SC_THREADS), 0, s, a);
        HIP_TRY(hipGetLastError());
    }
    return EE_OK;
}
