// Products by tiles through LDS: bound by the matrix cores and by how they are fed where rows are many, by the weights' bytes where they are few (ee_gemm16_thin_kernel).
// One MI355X, bf16, us and TFLOP/s (a library's product of the same matrices in the same run): 2041 x 4096 x 11008 forward 179, 1030 (159, 1158), dx 163, 1127, dW 174, 1055;
// 8192 x 8192 x 8192 930, 1183 (661, 1664), 960, 880 (dW 1250 TFLOP/s); 4096 x 4096 x 4096 128 (87), 126, 116.  Five rows of 4096 through 32000 columns 52.8 us, 5.0 TB/s.
//
// What the tile's loads cost decides: with the sum's index contiguous and lane l at row l & 15 (the operands' own order) 2041 x 4096 x 11008 forward took 267 us, with four lanes a
// row 206, and 179 with whole lines of 128 bytes (KS = 2; half lines are fetched twice, as the cache of a compute unit does not hold them from one step to the next).
// 256 x 128 tiles of 64 of the sum leave a compute unit one workgroup: 244 us.
#include "ee_linear.hpp"

#include <atomic>

namespace ee {

// Eight neighbouring elements of row r at column c of an array of R rows and C columns; 0 outside it.  Rows start at multiples of 16 bytes.
__device__ __forceinline__ u32x4_t load_piece(const uint16_t *p, long long ld, int R, int C, int r, int c)
{
    u32x4_t v = {0, 0, 0, 0};
    if (r >= R || c >= C) return v;
    const uint16_t *q = p + (size_t)r * ld + c;
    if (c + 8 <= C) return *as_global(reinterpret_cast<const u32x4_t *>(q));
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (c + i < C) v[i / 2] |= (uint32_t)as_global(q)[i] << (i % 2 * 16);
    return v;
}

// A tile of TI x TJ results by four waves, each a quarter of it.  32 KS of the sum at a time (a step) go from memory straight to LDS (NS steps, NS - 1 of them on their
// way), without a register, in an order that suits the waves' reads:
//   sum's index contiguous in memory: rows of 64 KS bytes, by four (KS = 2: eight) neighbouring lanes each (neighbouring lanes that read neighbouring lines cost four times the
//                               look-ups); a row's pieces are swapped by its number, so that eight lanes of a read meet every bank once;
//   result's index contiguous: rows of the step, pieces of 32 bytes swapped by the row's number, so that the transposing reads (ds_read_b64_tr_b16: four rows x 16
//   columns for 16 lanes) of a wave meet no bank twice.
// The weights' side is the first operand: a lane has four neighbouring results of a row.
template <int TI_, int TJ_, int KS_, int NS_>
struct Tile {
    static constexpr int TI = TI_, TJ = TJ_, KS = KS_, NS = NS_;
    static constexpr size_t LDS = (size_t)NS * (TI + TJ) * KS * 64;
};
typedef Tile<256, 128, 1, 3> LargeTile;      // where the result's index is contiguous on both sides
typedef Tile<192, 128, 2, 2> WideTile;       // ... and where it is not: whole lines of 128 bytes
typedef Tile<128, 128, 2, 2> MediumTile;
typedef Tile<64, 64, 2, 3> SmallTile;

// Operand of T rows (of results): its units of a kilobyte in a step.
template <bool ALONG, int T, int KS>
struct Operand {
    static constexpr int UNITS = T * KS / 16, EACH = UNITS / 4;      // ... and of a wave
    static constexpr int PIECES = T / 8;                             // pieces of a row of the step, where the result's index is contiguous

    // which of the pieces (pairs of them) of row k of the step are swapped
    static __device__ __forceinline__ int swap(int k) { return T >= 128 ? (k & 3) | (k >> 3 & 1) << 2 : k & 3; }
    // what lane l of unit u holds: results r .. of the tile, sum's index k .. of the step
    static __device__ __forceinline__ void place(int u, int l, int &r, int &k)
    {
        if (ALONG && KS == 1) {
            r = u * 16 + (l >> 2);
            k = ((l & 3) ^ (l >> 3 & 3)) * 8;
        } else if (ALONG) {
            r = u * 8 + (l >> 3);
            k = ((l & 7) ^ (l >> 3)) * 8;
        } else {
            k = u * (512 / T) + l / PIECES;
            const int c = l % PIECES;
            r = ((((c >> 1) ^ swap(k)) << 1) | (c & 1)) * 8;
        }
    }
    // byte offset of a lane's piece from the step's first element of the tile; results beyond the array's `n` are read from its first
    static __device__ __forceinline__ int offset(int u, int l, int n, long long ld)
    {
        int r, k;
        place(u, l, r, k);
        if (ALONG) return (int)(min(r, n - 1) * ld + k) * 2;
        return (int)(k * ld + (r < n ? r : 0)) * 2;
    }
    // lane's part of the operand for results 16 f .. 16 f + 15 of the tile and the h-th 32 of the step
    static __device__ __forceinline__ u32x4_t read(const char *at, int f, int h, int lane)
    {
        const int s = lane & 15, quad = lane >> 4;
        if (ALONG && KS == 1) return *reinterpret_cast<const u32x4_t *>(at + f * 1024 + s * 64 + (quad ^ (s >> 1 & 3)) * 16);
        if (ALONG) return *reinterpret_cast<const u32x4_t *>(at + f * 2048 + s * 128 + ((h * 4 + quad) ^ (s & 7)) * 16);
        typedef __attribute__((ext_vector_type(4))) short s16x4_v;
        const int k = h * 32 + quad * 8 + (s >> 2);
        const char *p = at + k * (T * 2) + ((f ^ swap(k)) * 32 + (s & 3) * 8);
        EE_LDS s16x4_v *q = (EE_LDS s16x4_v *)(p);
        const s16x4_v a = __builtin_amdgcn_ds_read_tr16_b64_v4i16(q), b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((EE_LDS s16x4_v *)(p + 4 * T * 2));
        const u32x2_t x = __builtin_bit_cast(u32x2_t, a), y = __builtin_bit_cast(u32x2_t, b);
        return (u32x4_t){x[0], x[1], y[0], y[1]};
    }
};

// What a second term of fp16 is multiplied by.  It is 2^-11 of the first at most: as it is, a subnormal number for a first term under 2^-3, with digits lost.  For the largest first term, 65504, it
// is 16 at most, and the product still a number of the type.  The two are off by 2^-22 of what they stand for, or by 2^-36 (half the smallest fp16, 2^-25, by 2^11) where that is more.
constexpr float TERM_FP16 = 2048.f;

template <int TYPE, bool A_ALONG, bool B_ALONG, typename TILE>
__global__ void __launch_bounds__(256, 2) ee_gemm16_kernel(GemmDev g)
{
    constexpr int TI = TILE::TI, TJ = TILE::TJ, KS = TILE::KS, NS = TILE::NS, STEP = 32 * KS;
    typedef Operand<A_ALONG, TI, KS> OpA;
    typedef Operand<B_ALONG, TJ, KS> OpB;
    constexpr int PER = OpA::EACH + OpB::EACH, FI = TI / 32, FJ = TJ / 32;
    constexpr unsigned STAGE = (TI + TJ) * KS * 64, B_AT = TI * KS * 64;
    extern __shared__ __align__(16) char lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wi = wave & 1, wj = wave >> 1;
    // Workgroups go to the XCDs in turn; each XCD has a contiguous run of the tiles, which walk groups of eight blocks of rows over all blocks of columns: what
    // runs together on an XCD shares operands in its L2.
    const int T = g.ni * g.nj * g.splits;
    int t, part, i0, j0;
    {
        const int x = blockIdx.x % NUM_XCD, n = blockIdx.x / NUM_XCD, base = T / NUM_XCD, extra = T % NUM_XCD;
        t = x * base + min(x, extra) + n;
        part = t / (g.ni * g.nj);
        t -= part * g.ni * g.nj;
        const int group = t / (8 * g.nj), rem = t - group * 8 * g.nj, width = min(8, g.ni - group * 8);
        j0 = rem / width;
        i0 = (group * 8 + rem - j0 * width) * TI;
        j0 *= TJ;
    }
    const int lo = part * g.per, hi = min(lo + g.per, g.K);
    // The last step is loaded with a look at every piece where it is not whole, or where a piece at the end of its rows is not.
    const bool ragged = !A_ALONG && (g.I & 7), ragged_b = !B_ALONG && (g.J & 7);
    // (Rows too far apart for 32-bit offsets: all steps are.)
    const int full = g.far ? 0 : max((hi - lo) / STEP - (hi == g.K && (hi - lo) % STEP == 0 && (ragged || ragged_b)), 0);
    const unsigned lds0 = lds_offset(lds);
    int off_a[OpA::EACH], off_b[OpB::EACH];
#pragma unroll
    for (int i = 0; i < OpA::EACH; ++i) off_a[i] = OpA::offset(wave * OpA::EACH + i, lane, g.I - i0, g.lda);
#pragma unroll
    for (int i = 0; i < OpB::EACH; ++i) off_b[i] = OpB::offset(wave * OpB::EACH + i, lane, g.J - j0, g.ldb);
    const char *const b0 = reinterpret_cast<const char *>(g.B + (B_ALONG ? (size_t)j0 * g.ldb + lo : (size_t)lo * g.ldb + j0));
    const size_t step_a = A_ALONG ? STEP * 2 : (size_t)g.lda * (STEP * 2), step_b = B_ALONG ? STEP * 2 : (size_t)g.ldb * (STEP * 2);

    f32x4_t acc[FJ][FI];
#pragma unroll
    for (int j = 0; j < FJ; ++j)
#pragma unroll
        for (int i = 0; i < FI; ++i) acc[j][i] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
    auto compute = [&](const char *st) __attribute__((always_inline)) {
#pragma unroll
        for (int h = 0; h < KS; ++h) {
            u32x4_t a[FI], b[FJ];
#pragma unroll
            for (int j = 0; j < FJ; ++j) b[j] = OpB::read(st + B_AT, wj * FJ + j, h, lane);
#pragma unroll
            for (int i = 0; i < FI; ++i) a[i] = OpA::read(st, wi * FI + i, h, lane);
#pragma unroll
            for (int i = 0; i < FI; ++i)
#pragma unroll
                for (int j = 0; j < FJ; ++j) acc[j][i] = mfma16<TYPE>(b[j], a[i], acc[j][i]);
        }
    };
    for (int term = 0; term < g.terms; ++term) {
        const uint16_t *const A = g.A + term * g.plane;
        const char *const a0 = reinterpret_cast<const char *>(A + (A_ALONG ? (size_t)i0 * g.lda + lo : (size_t)lo * g.lda + i0));
        auto request = [&](int s, int buf) __attribute__((always_inline)) {
            const unsigned dst = lds0 + buf * STAGE;
            const void *pa = uniform_ptr(a0 + s * step_a), *pb = uniform_ptr(b0 + s * step_b);
#pragma unroll
            for (int i = 0; i < OpA::EACH; ++i) load_lds_kb(pa, off_a[i], dst + (wave * OpA::EACH + i) * 1024);
#pragma unroll
            for (int i = 0; i < OpB::EACH; ++i) load_lds_kb(pb, off_b[i], dst + B_AT + (wave * OpB::EACH + i) * 1024);
        };
#pragma unroll
        for (int s = 0; s < NS - 1; ++s)
            if (s < full) request(s, s);
        int buf = 0;
        for (int s = 0; s < full; ++s) {
            // this wave's loads of stage s have landed; after the barrier everybody's have, and nobody reads the buffer of stage s - 1 any more
            if (s + NS - 2 < full)
                wait_pending<PER *(NS - 2)>();
            else
                wait_pending<0>();
            lds_barrier();
            if (s + NS - 1 < full) request(s + NS - 1, buf == 0 ? NS - 1 : buf - 1);
            compute(lds + buf * STAGE);
            buf = buf + 1 == NS ? 0 : buf + 1;
        }
        for (int k0 = lo + full * STEP; k0 < hi; k0 += STEP) {
            lds_barrier();
#pragma unroll
            for (int i = 0; i < OpA::EACH; ++i) {
                int r, k;
                OpA::place(wave * OpA::EACH + i, lane, r, k);
                *reinterpret_cast<u32x4_t *>(lds + (wave * OpA::EACH + i) * 1024 + lane * 16) = A_ALONG ? load_piece(A, g.lda, g.I, hi, i0 + r, k0 + k) : load_piece(A, g.lda, hi, g.I, k0 + k, i0 + r);
            }
#pragma unroll
            for (int i = 0; i < OpB::EACH; ++i) {
                int r, k;
                OpB::place(wave * OpB::EACH + i, lane, r, k);
                *reinterpret_cast<u32x4_t *>(lds + B_AT + (wave * OpB::EACH + i) * 1024 + lane * 16) = B_ALONG ? load_piece(g.B, g.ldb, g.J, hi, j0 + r, k0 + k) : load_piece(g.B, g.ldb, hi, g.J, k0 + k, j0 + r);
            }
            lds_barrier();
            compute(lds);
        }
        if (term + 1 < g.terms) {
            lds_barrier();
            if constexpr (TYPE == EE_FP16)
#pragma unroll
                for (int j = 0; j < FJ; ++j)
#pragma unroll
                    for (int i = 0; i < FI; ++i) acc[j][i] *= 1.f / TERM_FP16;
        }
    }
    // Results turn in LDS (some rows of a wave at a time), so that stores are whole lines and the code behind the sums is there once, not for every register.
    constexpr int COLS = FJ * 16, LD = COLS + 4, LANES = COLS / 4, ROOM = (int)(TILE::LDS / (4 * 16 * LD * 4)), HALF = FI % 4 == 0 && ROOM >= 4 ? 4 : FI % 3 == 0 && ROOM >= 3 ? 3 : 2;
    static_assert(FI % HALF == 0 && HALF <= ROOM, "a turn fits the steps' room");
    float *const turn = reinterpret_cast<float *>(lds) + wave * (HALF * 16 * LD);
    const int col = j0 + wj * COLS + lane % LANES * 4;
    const f32x4_t bias = bias_at(g, col);
#pragma unroll
    for (int h = 0; h < FI; h += HALF) {
        if (h == 0) lds_barrier();                           // (every wave has read the last stage)
#pragma unroll
        for (int i = 0; i < HALF; ++i)
#pragma unroll
            for (int j = 0; j < FJ; ++j) *reinterpret_cast<f32x4_t *>(turn + (i * 16 + (lane & 15)) * LD + j * 16 + (lane >> 4) * 4) = acc[j][h + i];
        wave_lds_order();
        constexpr int APART = 64 / LANES, AT_ONCE = HALF * 16 / APART < 4 ? HALF * 16 / APART : 4;
        if (col < g.J)
#pragma unroll 1
            for (int r = lane / LANES; r < HALF * 16; r += APART * AT_ONCE) {
                const int row = i0 + (wi * FI + h) * 16 + r;
                f32x4_t v[AT_ONCE];
#pragma unroll
                for (int e = 0; e < AT_ONCE; ++e) v[e] = *reinterpret_cast<const f32x4_t *>(turn + (r + e * APART) * LD + lane % LANES * 4);
                if (g.splits == 1) {
                    finish<AT_ONCE>(g, row, APART, col, bias, v);
                } else {
#pragma unroll
                    for (int e = 0; e < AT_ONCE; ++e)
                        if (row + e * APART < g.I) *as_global_mut(reinterpret_cast<f32x4_t *>(g.part + ((size_t)part * g.I + row + e * APART) * g.part_ld + col)) = v[e];
                }
            }
        wave_lds_order();
    }
}

// Few rows: bound by the weights' bytes.  A workgroup has 16 TN columns of results, its four waves take steps of 32 of the sum in turn, each through
// a ring of its own in LDS (no barrier but the last): 10 KB on their way for a wave, 80 for a compute unit.  The rows are MT tiles of 16; the waves' sums meet in LDS.
// (Five rows of 4096 through 32000 columns: 52.8 us, 5.0 TB/s; by tiles whose waves share a ring 73.7.)
constexpr int THIN_STAGES = 3;
template <int TN, int MT>
constexpr size_t thin_lds() { return (size_t)4 * THIN_STAGES * (TN + MT) * 1024; }

template <int TYPE, int TN, int MT>
__global__ void __launch_bounds__(256, 2) ee_gemm16_thin_kernel(GemmDev g)
{
    typedef Operand<true, 16 * TN * 4, 1> Op;      // (only its placing of rows: kilobytes of 16 rows x 32)
    constexpr int NS = THIN_STAGES, PER = TN + MT, STAGE = PER * 1024;
    static_assert(4 * TN * MT * 1024 <= thin_lds<TN, MT>(), "the sums fit the rings' room");
    extern __shared__ __align__(16) char lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n0 = blockIdx.x * 16 * TN, part = blockIdx.y, lo = part * g.per, hi = min(lo + g.per, g.K);
    const int full = g.far ? 0 : (hi - lo) / 32, steps = (hi - lo + 31) / 32;
    char *const ring = lds + wave * NS * STAGE;
    const unsigned lds0 = lds_offset(ring);
    const char *const w0 = reinterpret_cast<const char *>(g.B + (size_t)n0 * g.ldb + lo), *const x0 = reinterpret_cast<const char *>(g.A + lo);
    int off[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) off[i] = i < TN ? Op::offset(i, lane, g.J - n0, g.ldb) : Op::offset(i - TN, lane, g.I, g.lda);
    auto request = [&](int s, int buf) __attribute__((always_inline)) {
        const void *pw = uniform_ptr(w0 + (size_t)s * 64), *px = uniform_ptr(x0 + (size_t)s * 64);
#pragma unroll
        for (int i = 0; i < PER; ++i) load_lds_kb(i < TN ? pw : px, off[i], lds0 + buf * STAGE + i * 1024);
    };
    f32x4_t acc[TN][MT];
#pragma unroll
    for (int n = 0; n < TN; ++n)
#pragma unroll
        for (int m = 0; m < MT; ++m) acc[n][m] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
    auto compute = [&](const char *st) __attribute__((always_inline)) {
        u32x4_t w[TN], x[MT];
#pragma unroll
        for (int i = 0; i < TN; ++i) w[i] = Op::read(st, i, 0, lane);
#pragma unroll
        for (int i = 0; i < MT; ++i) x[i] = Op::read(st, TN + i, 0, lane);
#pragma unroll
        for (int n = 0; n < TN; ++n)
#pragma unroll
            for (int m = 0; m < MT; ++m) acc[n][m] = mfma16<TYPE>(w[n], x[m], acc[n][m]);
    };
#pragma unroll
    for (int i = 0; i < NS - 1; ++i)
        if (wave + 4 * i < full) request(wave + 4 * i, i);
    int buf = 0;
    for (int s = wave; s < full; s += 4) {
        if (s + 4 * (NS - 2) < full)
            wait_pending<PER *(NS - 2)>();
        else
            wait_pending<0>();
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // (the last step's reads are done before its place is written again)
        if (s + 4 * (NS - 1) < full) request(s + 4 * (NS - 1), buf == 0 ? NS - 1 : buf - 1);
        compute(ring + buf * STAGE);
        buf = buf + 1 == NS ? 0 : buf + 1;
    }
    // steps that are not whole
    for (int s = full + (wave - full % 4 + 4) % 4; s < steps; s += 4) {
        wave_lds_order();
        int r, k;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            Op::place(i < TN ? i : i - TN, lane, r, k);
            k += lo + s * 32;
            *reinterpret_cast<u32x4_t *>(ring + i * 1024 + lane * 16) = i < TN ? load_piece(g.B, g.ldb, g.J, hi, n0 + r, k) : load_piece(g.A, g.lda, g.I, hi, r, k);
        }
        wave_lds_order();
        compute(ring);
    }
    lds_barrier();
#pragma unroll
    for (int n = 0; n < TN; ++n)
#pragma unroll
        for (int m = 0; m < MT; ++m) *reinterpret_cast<f32x4_t *>(lds + (((wave * TN + n) * MT + m) * 64 + lane) * 16) = acc[n][m];
    lds_barrier();
    for (int i = wave; i < TN * MT; i += 4) {
        f32x4_t v = *reinterpret_cast<const f32x4_t *>(lds + (i * 64 + lane) * 16);
#pragma unroll
        for (int w = 1; w < 4; ++w) v += *reinterpret_cast<const f32x4_t *>(lds + ((w * TN * MT + i) * 64 + lane) * 16);
        const int row = i % MT * 16 + (lane & 15), col = n0 + i / MT * 16 + (lane >> 4) * 4;
        if (row >= g.I || col >= g.J) continue;
        if (g.splits == 1) {
            f32x4_t one[1] = {v};
            finish<1>(g, row, 1, col, bias_at(g, col), one);
        } else {
            *as_global_mut(reinterpret_cast<f32x4_t *>(g.part + ((size_t)part * g.I + row) * g.part_ld + col)) = v;
        }
    }
}

// The parts of a sum, in their order.
__global__ void __launch_bounds__(256) ee_gemm16_join_kernel(GemmDev g)
{
    const int per_row = (int)(g.part_ld / 4);
    const size_t at = (size_t)blockIdx.x * 256 + threadIdx.x;
    const int row = (int)(at / per_row), col = (int)(at - (size_t)row * per_row) * 4;
    if (row >= g.I || col >= g.J) return;
    const float *p = g.part + (size_t)row * g.part_ld + col;
    f32x4_t v = *as_global(reinterpret_cast<const f32x4_t *>(p));
#pragma unroll 4
    for (int s = 1; s < g.splits; ++s) v += *as_global(reinterpret_cast<const f32x4_t *>(p + (size_t)s * g.I * g.part_ld));
    f32x4_t one[1] = {v};
    finish<1>(g, row, 1, col, bias_at(g, col), one);
}

// dz = dy act'(z) as 16-bit terms, and sums of its columns over a part of the rows: a thread has eight columns.  Bound by bytes (2041 x 11008 bf16, the sums alone: 16.3 us, 45 MB, 2.8 TB/s).
struct SlopeDev {
    const uint16_t *dy, *pre;
    long long dy_stride, pre_stride, ldz, plane;
    uint16_t *dz;                      // [terms][rows][ldz], or null
    float *part;                       // [parts][n], or null
    int type, act, terms, rows, n, per;   // per: rows of a part
};
constexpr int SL_COLS = 32, SL_SUBS = 8;    // 256 columns of a workgroup, eight rows at a time
__global__ void __launch_bounds__(SL_COLS *SL_SUBS) ee_slope_kernel(SlopeDev a)
{
    __shared__ float sums[SL_SUBS][SL_COLS * 8];
    const int c = threadIdx.x % SL_COLS, sub = threadIdx.x / SL_COLS, col = (blockIdx.x * SL_COLS + c) * 8;
    const int from = blockIdx.y * a.per, to = min(from + a.per, a.rows);
    float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (col < a.n)
        for (int row = from + sub; row < to; row += SL_SUBS) {
            const u32x4_t v = load_piece(a.dy, a.dy_stride, a.rows, a.n, row, col);
            u32x4_t z = {0, 0, 0, 0};
            if (a.act != EE_ACT_NONE) z = load_piece(a.pre, a.pre_stride, a.rows, a.n, row, col);
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint16_t vb = (uint16_t)(v[i / 2] >> (i % 2 * 16)), zb = (uint16_t)(z[i / 2] >> (i % 2 * 16));
                x[i] = a.type == EE_BF16 ? bf16_to_f32(vb) : (float)__builtin_bit_cast(_Float16, vb);
                if (a.act != EE_ACT_NONE) x[i] *= act_slope(a.act, a.type == EE_BF16 ? bf16_to_f32(zb) : (float)__builtin_bit_cast(_Float16, zb));
                s[i] += x[i];
            }
            for (int t = 0; t < a.terms; ++t) {
                u32x4_t w;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    w[i] = a.type == EE_BF16 ? pack_bf16(x[2 * i], x[2 * i + 1]) : pack_fp16(x[2 * i], x[2 * i + 1]);
                    const float lo = a.type == EE_BF16 ? __uint_as_float(w[i] << 16) : (float)__builtin_bit_cast(_Float16, (uint16_t)w[i]);
                    const float hi = a.type == EE_BF16 ? __uint_as_float(w[i] & 0xFFFF0000u) : (float)__builtin_bit_cast(_Float16, (uint16_t)(w[i] >> 16));
                    const float up = a.type == EE_BF16 ? 1.f : TERM_FP16;
                    x[2 * i] = fabsf(lo) == INFINITY ? 0.f : (x[2 * i] - lo) * up;       // (an infinity is one term, not one and its negative)
                    x[2 * i + 1] = fabsf(hi) == INFINITY ? 0.f : (x[2 * i + 1] - hi) * up;
                }
                *as_global_mut(reinterpret_cast<u32x4_t *>(a.dz + t * a.plane + (size_t)row * a.ldz + col)) = w;
            }
        }
    if (!a.part) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) sums[sub][c * 8 + i] = s[i];
    __syncthreads();
    const int mine = blockIdx.x * SL_COLS * 8 + threadIdx.x;
    if (mine < a.n) {
        float all = 0.f;
#pragma unroll
        for (int i = 0; i < SL_SUBS; ++i) all += sums[i][threadIdx.x];
        as_global_mut(a.part)[(size_t)blockIdx.y * a.n + mine] = all;
    }
}

typedef void (*gemm16_kernel_t)(GemmDev);
template <int TYPE, typename TILE>
static gemm16_kernel_t gemm16_kernel(bool a_along, bool b_along)
{
    // (a kernel that no plan takes is not built)
    if constexpr (TILE::TI == 256) {
        return ee_gemm16_kernel<TYPE, false, false, TILE>;
    } else if constexpr (TILE::TI == 192) {
        return b_along ? ee_gemm16_kernel<TYPE, true, true, TILE> : ee_gemm16_kernel<TYPE, true, false, TILE>;
    } else {
        return a_along ? (b_along ? ee_gemm16_kernel<TYPE, true, true, TILE> : ee_gemm16_kernel<TYPE, true, false, TILE>) : ee_gemm16_kernel<TYPE, false, false, TILE>;
    }
}
template <typename TILE>
static gemm16_kernel_t gemm16_kernel(bool bf16, bool a_along, bool b_along)
{
    return bf16 ? gemm16_kernel<EE_BF16, TILE>(a_along, b_along) : gemm16_kernel<EE_FP16, TILE>(a_along, b_along);
}

template <int TYPE, int MT>
static gemm16_kernel_t thin_kernel(int tn)
{
    static_assert(thin_lds<4, 1>() <= 64 << 10 && thin_lds<2, 2>() <= 64 << 10, "what a launch gets unasked");
    if constexpr (MT == 1)
        if (tn == 4) return ee_gemm16_thin_kernel<TYPE, 4, 1>;
    return tn == 1 ? ee_gemm16_thin_kernel<TYPE, 1, MT> : ee_gemm16_thin_kernel<TYPE, 2, MT>;
}

enum GemmForm { LARGE, MEDIUM, SMALL, THIN };
// How a product is split: in tiles (or few rows at a time), and parts of the sum, by an estimate of its time in us: the tiles of the busiest compute unit at 4.7e-7 us for each
// element of a tile and of the sum (times what a tile's shape costs, and what workgroups with few beside them on their compute unit do), a start and an end, and the
// parts' way through memory.  Measured, us, the chosen way first, then the best of the others (L, M, S: the tile, parts behind it): 2041 x 4096 x 11008 forward L1 181,
// M1 186; dx M1 176, L2 205; dW L1 184, M1 205; 4096 columns M1 69, L1 82; 384 columns S1 19.6, S2 18.4 (which the estimate misses), M6 20.8; 128 rows of 4096 x 4096 S4 13.7, S2 15.2; 300 x 1000 x
// 1000 S1 8.0, M4 11.5; dW of 512 x 512 from 8000 rows S4 16.3, S6 15.8, M12 20.1.
static double gemm_time(int form, bool a_along, double tiles, int area, int K, int splits, double results)
{
    const double shape = form == LARGE ? (a_along ? 1.04 : 1.15) : form == MEDIUM ? 1.0 : 0.68;
    const double each = tiles * splits / 256, busiest = each <= 1 ? 1 : (ceil(each) + each) / 2;
    const double alone = 0.45 + 0.55 * std::min(1.0, each / (form == SMALL ? 3 : 2));
    return busiest * area * (double)K / splits * 4.7e-7 / (shape * alone) + 4 + (splits > 1 ? 5 + splits * results * 8 / 4e6 : 0);
}
struct GemmPlan16 {
    int form, tn;                     // tn: of few rows, tiles of 16 columns for a workgroup
    int ni, nj, splits, per;
    long long part_ld;
    size_t bytes;
};
static GemmPlan16 plan_gemm16(int I, int J, int K, bool a_along, bool b_along)
{
    GemmPlan16 pl = {};
    const auto count = [](int n, int t) { return std::max((n + t - 1) / t, 1); };
    pl.tn = 1;
    if (a_along && b_along && I <= 32) {
        pl.form = THIN;
        while (pl.tn < (I > 16 ? 2 : 4) && J >= 16 * 2 * pl.tn * 400) pl.tn *= 2;
        pl.ni = 1;
        pl.nj = count(J, 16 * pl.tn);
        pl.splits = std::min(std::max(1, K / 512), std::max(1, 512 / pl.nj));
    } else {
        double best = 0;
        for (int form = LARGE; form <= SMALL; ++form) {
            const int ti = form == LARGE ? (a_along ? 192 : 256) : form == MEDIUM ? 128 : 64, tj = form == SMALL ? 64 : 128;
            const long long n = (long long)count(I, ti) * count(J, tj);
            for (int splits = 1; splits <= 16 && (splits == 1 || (K / splits >= 256 && n * splits <= 1024)); ++splits) {
                const double t = gemm_time(form, a_along, (double)n, ti * tj, K, splits, (double)I * J);
                if (best == 0 || t < best) {
                    best = t;
                    pl.form = form;
                    pl.ni = count(I, ti);
                    pl.nj = count(J, tj);
                    pl.splits = splits;
                }
            }
        }
    }
    pl.per = std::max(((K + pl.splits - 1) / pl.splits + 63) / 64 * 64, 64);
    pl.splits = std::max(1, (K + pl.per - 1) / pl.per);
    pl.part_ld = ((long long)J + 3) / 4 * 4;
    pl.bytes = pl.splits > 1 ? align256((size_t)pl.splits * I * pl.part_ld * sizeof(float)) : 0;
    return pl;
}
constexpr long long GEMM_FAR = 1 << 21;            // elements from row to row that 32-bit offsets within a tile allow
static int launch_gemm16(GemmDev g, bool a_along, bool b_along, void *space, hipStream_t s)
{
    const GemmPlan16 pl = plan_gemm16(g.I, g.J, g.K, a_along, b_along);
    g.ni = pl.ni;
    g.nj = pl.nj;
    g.splits = pl.splits;
    g.per = pl.per;
    g.part = static_cast<float *>(space);
    g.part_ld = pl.part_ld;
    g.far = g.lda > GEMM_FAR || g.ldb > GEMM_FAR;
    const bool bf16 = g.type == EE_BF16;
    if (pl.form == THIN) {
        const bool two = g.I > 16;
        const gemm16_kernel_t k = bf16 ? (two ? thin_kernel<EE_BF16, 2>(pl.tn) : thin_kernel<EE_BF16, 1>(pl.tn)) : (two ? thin_kernel<EE_FP16, 2>(pl.tn) : thin_kernel<EE_FP16, 1>(pl.tn));
        hipLaunchKernelGGL(k, dim3((unsigned)pl.nj, (unsigned)pl.splits), dim3(256), (size_t)4 * THIN_STAGES * (pl.tn + (two ? 2 : 1)) * 1024, s, g);
    } else if (pl.form != LARGE) {
        const bool small = pl.form == SMALL;
        static_assert(SmallTile::LDS <= 64 << 10 && MediumTile::LDS <= 64 << 10, "what a launch gets unasked");
        hipLaunchKernelGGL(small ? gemm16_kernel<SmallTile>(bf16, a_along, b_along) : gemm16_kernel<MediumTile>(bf16, a_along, b_along), dim3((unsigned)(pl.ni * pl.nj * pl.splits)), dim3(256),
                           small ? SmallTile::LDS : MediumTile::LDS, s, g);
    } else {
        const gemm16_kernel_t k = a_along ? gemm16_kernel<WideTile>(bf16, true, b_along) : gemm16_kernel<LargeTile>(bf16, false, false);
        const size_t lds = a_along ? WideTile::LDS : LargeTile::LDS;      // (more than a launch gets unasked: said once for a kernel on a device)
        static std::atomic<uint64_t> said[2][2][2];
        std::atomic<uint64_t> &mine = said[bf16][a_along][b_along];
        int device = 0;
        HIP_TRY(hipGetDevice(&device));
        const uint64_t bit = 1ull << (device & 63);
        if (device >= 64 || !(mine.load(std::memory_order_relaxed) & bit)) {
            HIP_TRY(hipFuncSetAttribute(reinterpret_cast<const void *>(k), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
            if (device < 64) mine.fetch_or(bit, std::memory_order_relaxed);
        }
        hipLaunchKernelGGL(k, dim3((unsigned)(pl.ni * pl.nj * pl.splits)), dim3(256), lds, s, g);
    }
    HIP_TRY(hipGetLastError());
    if (pl.splits > 1) {
        const size_t n = (size_t)g.I * (pl.part_ld / 4);
        hipLaunchKernelGGL(ee_gemm16_join_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, g);
        HIP_TRY(hipGetLastError());
    }
    return EE_OK;
}

static int check_sizes(const char *call, int device, int dtype, int act, int n_rows, int n_in, int n_out)
{
    if (device < 0) return fail(EE_EINVAL, "%s: device %d", call, device);
    if (dtype != EE_BF16 && dtype != EE_FP16) return fail(EE_EINVAL, "%s: operands must be bf16 or fp16 (type %d)", call, dtype);
    if (act < EE_ACT_NONE || act > EE_ACT_GELU) return fail(EE_EINVAL, "%s: unknown activation %d", call, act);
    if (n_rows < 0 || n_rows > EE_LINEAR_MAX) return fail(EE_EINVAL, "%s: n_rows %d not in [0,2^22]", call, n_rows);
    if (n_in < 1 || n_in > EE_LINEAR_MAX || n_out < 1 || n_out > EE_LINEAR_MAX) return fail(EE_EINVAL, "%s: n_in %d or n_out %d not in [1,2^22]", call, n_in, n_out);
    const auto tiles = [](int a, int b) { return (((long long)a + 63) / 64) * (((long long)b + 63) / 64); };
    if (std::max(tiles(n_rows, n_in), std::max(tiles(n_rows, n_out), tiles(n_in, n_out))) >= 1 << 23) return fail(EE_EINVAL, "%s: n_rows %d, n_in %d, n_out %d are too many at once", call, n_rows, n_in, n_out);
    return EE_OK;
}
// rows of an array: 16-byte aligned, `width` elements at least from one to the next
static int check_matrix(const char *call, const char *what, const void *p, int type, int64_t stride, int n_rows, int width)
{
    if (!p) return EE_OK;
    if (type < EE_BF16 || type > EE_FP32) return fail(EE_EINVAL, "%s: unknown element type %d of %s", call, type, what);
    if (!aligned(p, 16)) return fail(EE_EINVAL, "%s: %s must be 16-byte aligned", call, what);
    if (!stride_ok(stride, type, n_rows)) return fail(EE_EINVAL, "%s: the row stride of %s keeps no 16-byte alignment", call, what);
    if (n_rows > 1 && stride < width) return fail(EE_EINVAL, "%s: the row stride of %s is smaller than its row", call, what);
    return EE_OK;
}

static int check_linear(const char *call, const ee_linear_args *p)
{
    if (!p) return fail(EE_EINVAL, "%s: null argument", call);
    return check_sizes(call, p->device, p->dtype, p->act, p->n_rows, p->n_in, p->n_out);
}

struct GradPlan {
    int terms_dx, terms_dw, terms;     // of dz, where it is formed
    int parts, per;                    // of the rows, for the bias's gradient and dz
    long long ldz;
    size_t dz_bytes, part_bytes, gemm_bytes;
    size_t bytes() const { return dz_bytes + part_bytes + gemm_bytes; }
};
static GradPlan plan_grad(const ee_linear_grad_args &p)
{
    GradPlan pl = {};
    // dz in three terms of bf16 (2^-24 of it) or two of fp16 (2^-22 of it, or 2^-36) for fp32 results.  In one for 16-bit results, which are rounded as coarsely themselves: a second one would bring their
    // error against 64 bits from 0.0023 to 0.0017 of their size, by a second product (bf16 with SiLU, one term / two: 2041 x 4096 x 384 36.2 us / 57, 2041 x 4096 x 11008 420 / 725).
    const int exact = p.dtype == EE_BF16 ? 3 : 2;
    pl.terms_dx = p.act != EE_ACT_NONE && p.dx_dtype == EE_FP32 ? exact : 1;
    pl.terms_dw = p.act != EE_ACT_NONE && p.dw_dtype == EE_FP32 ? exact : 1;
    pl.terms = p.act == EE_ACT_NONE ? 0 : std::max(pl.terms_dx, pl.terms_dw);
    pl.ldz = ((long long)p.n_out + 7) / 8 * 8;
    const int columns = (p.n_out + SL_COLS * 8 - 1) / (SL_COLS * 8);
    pl.per = std::max(SL_SUBS, (int)(((long long)p.n_rows * columns + 1023) / 1024 + SL_SUBS - 1) / SL_SUBS * SL_SUBS);
    pl.parts = (p.n_rows + pl.per - 1) / pl.per;
    pl.dz_bytes = align256((size_t)pl.terms * p.n_rows * pl.ldz * 2);
    pl.part_bytes = align256((size_t)pl.parts * p.n_out * sizeof(float));
    pl.gemm_bytes = std::max(plan_gemm16(p.n_rows, p.n_in, p.n_out, true, false).bytes, plan_gemm16(p.n_out, p.n_in, p.n_rows, false, false).bytes);
    return pl;
}
static int check_linear_grad(const char *call, const ee_linear_grad_args *p)
{
    if (!p) return fail(EE_EINVAL, "%s: null argument", call);
    if (p->dx_dtype < EE_BF16 || p->dx_dtype > EE_FP32 || p->dw_dtype < EE_BF16 || p->dw_dtype > EE_FP32)
        return fail(EE_EINVAL, "%s: unknown element type %d or %d", call, p->dx_dtype, p->dw_dtype);
    return check_sizes(call, p->device, p->dtype, p->act, p->n_rows, p->n_in, p->n_out);
}

}  // namespace ee

using namespace ee;

extern "C" int ee_debug_linear_plan(int32_t n_rows, int32_t n_in, int32_t n_out, int32_t product, int32_t plan[4])
{
    static const char *const call = "ee_debug_linear_plan";
    if (!plan) return fail(EE_EINVAL, "%s: null argument", call);
    if (product < 0 || product > 2) return fail(EE_EINVAL, "%s: product %d not in [0,2]", call, product);
    int rc = check_sizes(call, 0, EE_BF16, EE_ACT_NONE, n_rows, n_in, n_out);
    if (rc != EE_OK) return rc;
    const bool a_along = product != 2, b_along = product == 0;
    const int I = product == 2 ? n_out : n_rows;
    const GemmPlan16 pl = product == 0 ? plan_gemm16(I, n_out, n_in, true, true) : plan_gemm16(I, n_in, product == 1 ? n_out : n_rows, a_along, b_along);
    plan[0] = pl.form == THIN ? (I > 16 ? 32 : 16) : pl.form == LARGE ? (a_along ? 192 : 256) : pl.form == MEDIUM ? 128 : 64;
    plan[1] = pl.form == THIN ? 16 * pl.tn : pl.form == SMALL ? 64 : 128;
    plan[2] = pl.splits;
    plan[3] = pl.per;
    return EE_OK;
}

extern "C" int ee_linear_workspace(const ee_linear_args *p, size_t *bytes)
{
    static const char *const call = "ee_linear_workspace";
    if (!bytes) return fail(EE_EINVAL, "%s: null argument", call);
    *bytes = 0;
    int rc = check_linear(call, p);
    if (rc == EE_OK) *bytes = plan_gemm16(p->n_rows, p->n_out, p->n_in, true, true).bytes;
    return rc;
}

extern "C" int ee_linear(const ee_linear_args *p, void *workspace, size_t workspace_bytes, void *stream)
{
    static const char *const call = "ee_linear";
    int rc = check_linear(call, p);
    if (rc == EE_OK) rc = check_matrix(call, "x", p->x, p->dtype, p->x_stride, p->n_rows, p->n_in);
    if (rc == EE_OK) rc = check_matrix(call, "weight", p->weight, p->dtype, p->weight_stride, p->n_out, p->n_in);
    if (rc == EE_OK) rc = check_matrix(call, "y", p->y, p->out_dtype, p->y_stride, p->n_rows, p->n_out);
    if (rc == EE_OK) rc = check_matrix(call, "residual", p->residual, p->residual_dtype, p->residual_stride, p->n_rows, p->n_out);
    if (rc == EE_OK) rc = check_matrix(call, "pre", p->pre, p->dtype, p->pre_stride, p->n_rows, p->n_out);
    if (rc != EE_OK) return rc;
    if (p->n_rows == 0) return EE_OK;
    if (!p->x || !p->weight || !p->y) return fail(EE_EINVAL, "%s: null x, weight or y", call);
    if (p->y == p->x || p->y == p->weight || (p->pre && (p->pre == p->x || p->pre == p->weight || p->pre == p->y || p->pre == p->residual))) return fail(EE_EINVAL, "%s: y and pre must be arrays of their own", call);
    if (p->residual == p->y && (p->residual_dtype != p->out_dtype || (p->n_rows > 1 && p->residual_stride != p->y_stride)))
        return fail(EE_EINVAL, "%s: y may be residual only with the same type and stride", call);
    if (!aligned(p->bias, 4)) return fail(EE_EINVAL, "%s: fp32 arrays must be 4-byte aligned", call);
    const size_t need = plan_gemm16(p->n_rows, p->n_out, p->n_in, true, true).bytes;
    if (need > workspace_bytes || (need && (!workspace || !aligned(workspace, 256))))
        return fail(EE_EINVAL, "%s: the workspace has %zu bytes of %zu, or is not 256-byte aligned", call, workspace_bytes, need);
    GemmDev g = {};
    g.A = static_cast<const uint16_t *>(p->x);
    g.B = static_cast<const uint16_t *>(p->weight);
    g.lda = p->n_rows > 1 ? p->x_stride : 0;
    g.ldb = p->n_out > 1 ? p->weight_stride : 0;
    g.terms = 1;
    g.I = p->n_rows;
    g.J = p->n_out;
    g.K = p->n_in;
    g.bias = p->bias;
    g.residual = p->residual;
    g.y = p->y;
    g.pre = p->pre;
    g.res_stride = p->n_rows > 1 ? p->residual_stride : 0;
    g.y_stride = p->n_rows > 1 ? p->y_stride : 0;
    g.pre_stride = p->n_rows > 1 ? p->pre_stride : 0;
    g.res_type = p->residual_dtype;
    g.y_type = p->out_dtype;
    g.type = p->dtype;
    g.act = p->act;
    DeviceScope scope(p->device);
    HIP_TRY(scope.status);
    return launch_gemm16(g, true, true, workspace, static_cast<hipStream_t>(stream));
}

extern "C" int ee_linear_grad_workspace(const ee_linear_grad_args *p, size_t *bytes)
{
    static const char *const call = "ee_linear_grad_workspace";
    if (!bytes) return fail(EE_EINVAL, "%s: null argument", call);
    *bytes = 0;
    int rc = check_linear_grad(call, p);
    if (rc == EE_OK) *bytes = plan_grad(*p).bytes();
    return rc;
}

extern "C" int ee_linear_grad(const ee_linear_grad_args *p, void *workspace, size_t workspace_bytes, void *stream)
{
    static const char *const call = "ee_linear_grad";
    int rc = check_linear_grad(call, p);
    if (rc == EE_OK) rc = check_matrix(call, "x", p->x, p->dtype, p->x_stride, p->n_rows, p->n_in);
    if (rc == EE_OK) rc = check_matrix(call, "weight", p->weight, p->dtype, p->weight_stride, p->n_out, p->n_in);
    if (rc == EE_OK) rc = check_matrix(call, "dy", p->dy, p->dtype, p->dy_stride, p->n_rows, p->n_out);
    if (rc == EE_OK) rc = check_matrix(call, "pre", p->pre, p->dtype, p->pre_stride, p->n_rows, p->n_out);
    if (rc == EE_OK) rc = check_matrix(call, "dx", p->dx, p->dx_dtype, p->dx_stride, p->n_rows, p->n_in);
    if (rc == EE_OK) rc = check_matrix(call, "d_weight", p->d_weight, p->dw_dtype, p->dw_stride, p->n_out, p->n_in);
    if (rc != EE_OK) return rc;
    if (!p->dx && !p->d_weight && !p->d_bias) return EE_OK;
    if (p->n_rows) {
        if (!p->dy) return fail(EE_EINVAL, "%s: null dy", call);
        if (p->act != EE_ACT_NONE && !p->pre) return fail(EE_EINVAL, "%s: an activation's gradient needs pre", call);
        if ((p->dx && !p->weight) || (p->d_weight && !p->x)) return fail(EE_EINVAL, "%s: dx needs weight, d_weight needs x", call);
    }
    for (const void *out : {(const void *)p->dx, (const void *)p->d_weight})
        if (out && (out == p->x || out == p->weight || out == p->dy || out == p->pre || (out == p->dx && out == p->d_weight)))
            return fail(EE_EINVAL, "%s: dx and d_weight must be arrays of their own", call);
    if (!aligned(p->d_bias, 4)) return fail(EE_EINVAL, "%s: fp32 arrays must be 4-byte aligned", call);
    const GradPlan pl = plan_grad(*p);
    if (pl.bytes() > workspace_bytes || (pl.bytes() && (!workspace || !aligned(workspace, 256))))
        return fail(EE_EINVAL, "%s: the workspace has %zu bytes of %zu, or is not 256-byte aligned", call, workspace_bytes, pl.bytes());
    DeviceScope scope(p->device);
    HIP_TRY(scope.status);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    uint16_t *const dz = static_cast<uint16_t *>(workspace);
    float *const part = reinterpret_cast<float *>(static_cast<unsigned char *>(workspace) + pl.dz_bytes);
    void *const space = static_cast<unsigned char *>(workspace) + pl.dz_bytes + pl.part_bytes;
    const long long plane = (long long)p->n_rows * pl.ldz;
    if (pl.parts && (p->d_bias || p->act != EE_ACT_NONE)) {
        SlopeDev a = {};
        a.dy = static_cast<const uint16_t *>(p->dy);
        a.pre = static_cast<const uint16_t *>(p->pre);
        a.dy_stride = p->n_rows > 1 ? p->dy_stride : 0;
        a.pre_stride = p->n_rows > 1 ? p->pre_stride : 0;
        a.ldz = pl.ldz;
        a.plane = plane;
        a.dz = dz;
        a.part = p->d_bias ? part : nullptr;
        a.type = p->dtype;
        a.act = p->act;
        a.terms = p->dx || p->d_weight ? pl.terms : 0;
        a.rows = p->n_rows;
        a.n = p->n_out;
        a.per = pl.per;
        hipLaunchKernelGGL(ee_slope_kernel, dim3((unsigned)((p->n_out + SL_COLS * 8 - 1) / (SL_COLS * 8)), (unsigned)pl.parts), dim3(SL_COLS * SL_SUBS), 0, s, a);
        HIP_TRY(hipGetLastError());
    }
    launch_column_sums(part, pl.parts, p->n_out, p->d_bias, nullptr, nullptr, s);
    HIP_TRY(hipGetLastError());
    GemmDev g = {};
    g.type = p->dtype;
    g.act = EE_ACT_NONE;
    g.plane = -plane;
    const uint16_t *const first_term = p->act == EE_ACT_NONE ? static_cast<const uint16_t *>(p->dy) : dz;
    g.lda = p->act != EE_ACT_NONE ? pl.ldz : p->n_rows > 1 ? p->dy_stride : 0;
    if (p->dx && p->n_rows) {
        g.B = static_cast<const uint16_t *>(p->weight);
        g.ldb = p->n_out > 1 ? p->weight_stride : 0;
        g.terms = pl.terms_dx;
        g.A = first_term + (pl.terms_dx - 1) * plane;
        g.I = p->n_rows;
        g.J = p->n_in;
        g.K = p->n_out;
        g.y = p->dx;
        g.y_type = p->dx_dtype;
        g.y_stride = p->n_rows > 1 ? p->dx_stride : 0;
        if ((rc = launch_gemm16(g, true, false, space, s)) != EE_OK) return rc;
    }
    if (p->d_weight) {
        g.B = static_cast<const uint16_t *>(p->x);
        g.ldb = p->n_rows > 1 ? p->x_stride : 0;
        g.terms = pl.terms_dw;
        g.A = first_term + (pl.terms_dw - 1) * plane;
        g.I = p->n_out;
        g.J = p->n_in;
        g.K = p->n_rows;
        g.y = p->d_weight;
        g.y_type = p->dw_dtype;
        g.y_stride = p->n_out > 1 ? p->dw_stride : 0;
        if ((rc = launch_gemm16(g, false, false, space, s)) != EE_OK) return rc;
    }
    return EE_OK;
}
