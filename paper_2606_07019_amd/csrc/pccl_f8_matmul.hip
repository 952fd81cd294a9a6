// Products of 8-bit operands with a scale for 128 values of k, out[m][n] = sum
// over k of A[m][k] B[n][k]; the experts' products over rows in expert order;
// and their weights' gradient.
//
// 16-bit results come from the matrix units' 8-bit form: 32 rows of each
// operand over 64 values of k with a scale byte for every row and block of 32,
// so that a block's scale costs nothing.  That instruction drops, of every eight
// products it adds, what is below 2^-13 of the largest (measured: 2^16 + 2^3 is
// kept, 2^16 + 2^2 is not; sums of such eights are kept to 24 bits).  On normal
// values the results' error is 1.4e-5 of their norm, 4.4e-5 with a value twenty
// times the others in every row: a hundredth of what rounding to bf16 costs, a
// tenth of f16.  Results of 32 bits are summed in 32 bits: codes become bf16,
// scaled, which is exact between 2^-126 and 2^128, for the 16-bit form (32 rows
// over 16 values of k); blocks beyond 2^128 are summed unscaled.
//
// Either form has lane l of a wave give row l % 32 of an operand, and sixteen
// sums, four neighbours in rows 8 q + 4 (l / 32) of the first operand, row l %
// 32 of the second.  B goes first, so a lane's sums are neighbours in out.
// Which lane holds which values of a block does not matter, as long as it is the
// same for both operands: all of a block have one scale.
#include "pccl_ops.h"

namespace pccl {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef const __attribute__((address_space(1))) void *gptr;
typedef __attribute__((address_space(3))) void *lptr;

// 32 codes of a row.
struct Piece {
    u32x4 lo, hi;
};

// Eight codes as bf16 values, scaled.
__device__ inline bf16x8 wide(uint32_t w0, uint32_t w1, float scale)
{
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, true);
    return bf16x8{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}

// The lowest scale byte with which a block's largest codes pass bf16's numbers: 256 * 2^120 does.
// A wave that meets one makes its sums anew (with that and without, in us, where none
// does: 8192^3 783 and 784, 2040 x 2080 x 1500 22.0 and 21.7, 64 x 4096 x 4096 11.6 and
// 11.5; made anew behind the stores, so that the loop's registers stay as they were:
// 788, 22.1 and 11.6).
constexpr uint32_t BEYOND = 247;

// A sum of products of codes with both scales; ldexp takes them to where the sum lies, whatever each of them is.
__device__ inline float with_scales(float sum, uint32_t xs, uint32_t ys)
{
    return xs == 255u || ys == 255u ? __uint_as_float(0x7FC00000u) : ldexpf(sum, (int)(xs + ys) - 254);
}

// c += y x over a block of 128 values, its scales applied to its sum, as blocks
// beyond what bf16 holds need it.  Lane l has 64 codes of row l % 32 of either.
__device__ inline void add_unscaled(f32x16 &c, const uint8_t *x, uint32_t xs, const uint8_t *y, uint32_t ys)
{
    f32x16 sum = {};
#pragma unroll
    for (int q = 0; q < 4; q++) {
        const u32x4 v = reinterpret_cast<const u32x4 *>(y)[q], w = reinterpret_cast<const u32x4 *>(x)[q];
        sum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wide(v.x, v.y, 1.f), wide(w.x, w.y, 1.f), sum, 0, 0, 0);
        sum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wide(v.z, v.w, 1.f), wide(w.z, w.w, 1.f), sum, 0, 0, 0);
    }
#pragma unroll
    for (int q = 0; q < 16; q++) {
        const int row = q / 4 * 8 + q % 4;   // of y: 4 more in the upper half of the lanes
        c[q] += with_scales(sum[q], xs, (uint32_t)__shfl((int)ys, row + (int)(threadIdx.x & 32u) / 8));
    }
}

// c[i][j] += y[j] x[i] over 64 values of k, for products FROM up to TO in the
// order of c; a scale is the lowest byte of its word.
template <bool EXACT, int FROM, int TO, int TM, int TN>
__device__ inline void products(f32x16 (&c)[TM][TN], const Piece (&x)[TM], const uint32_t (&xs)[TM], const Piece (&y)[TN], const uint32_t (&ys)[TN])
{
    if constexpr (EXACT) {
        float fx[TM], fy[TN];
#pragma unroll
        for (int i = 0; i < TM; i++) fx[i] = mx_scale(xs[i] & 0xFFu);
#pragma unroll
        for (int j = 0; j < TN; j++) fy[j] = mx_scale(ys[j] & 0xFFu);
#pragma unroll
        for (int q = 0; q < 4; q++) {
            bf16x8 wx[TM], wy[TN];
#pragma unroll
            for (int j = 0; j < TN; j++) {
                const u32x4 &v = q < 2 ? y[j].lo : y[j].hi;
                wy[j] = wide(v[q % 2 * 2], v[q % 2 * 2 + 1], fy[j]);
            }
#pragma unroll
            for (int i = 0; i < TM; i++) {
                const u32x4 &v = q < 2 ? x[i].lo : x[i].hi;
                wx[i] = wide(v[q % 2 * 2], v[q % 2 * 2 + 1], fx[i]);
            }
#pragma unroll
            for (int p = FROM; p < TO; p++) c[p / TN][p % TN] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wy[p % TN], wx[p / TN], c[p / TN][p % TN], 0, 0, 0);
        }
    } else {
        auto whole = [](const Piece &p) { return i32x8{(int)p.lo.x, (int)p.lo.y, (int)p.lo.z, (int)p.lo.w, (int)p.hi.x, (int)p.hi.y, (int)p.hi.z, (int)p.hi.w}; };
#pragma unroll
        for (int p = FROM; p < TO; p++) {
            const int i = p / TN, j = p % TN;
            c[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(whole(y[j]), whole(x[i]), c[i][j], 0, 0, 0, (int)ys[j], 0, (int)xs[i]);
        }
    }
    // keeps them in front of what follows: nothing else would
#pragma unroll
    for (int p = FROM; p < TO; p++) asm volatile("" : "+a"(c[p / TN][p % TN]));
}

// The order of N products with READS reads from LDS and COPIES copies evenly between them.
template <int N, int READS, int COPIES, int I = 0>
__device__ inline void mixed()
{
    if constexpr (I < N) {
        constexpr int r = (I + 1) * READS / N - I * READS / N, c = (I + 1) * COPIES / N - I * COPIES / N;
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        if constexpr (r > 0) __builtin_amdgcn_sched_group_barrier(0x100, r, 0);
        if constexpr (c > 0) __builtin_amdgcn_sched_group_barrier(0x020, c, 0);
        mixed<N, READS, COPIES, I + 1>();
    }
}

// Four neighbouring sums of row `row`, from column `col` on, to any address.
template <class T>
__device__ inline void store4(T *out, uint64_t ld, uint64_t row, uint64_t col, uint64_t n, f32x4 v)
{
    T t[4];
#pragma unroll
    for (int i = 0; i < 4; i++) t[i] = Elem<T>::put(v[i]);
    T *p = out + row * ld + col;
    if (col + 4 <= n) {
        __builtin_memcpy(p, t, sizeof t);
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; i++)
        if (col + i < n) p[i] = t[i];
}

template <int N>
struct Number {
    static constexpr int value = N;
};

// f(Number<0>{}), ... f(Number<N - 1>{})
template <int N>
struct Each {
    template <class F>
    static __device__ inline void run(F &&f)
    {
        Each<N - 1>::run(f);
        f(Number<N - 1>{});
    }
};
template <>
struct Each<0> {
    template <class F>
    static __device__ inline void run(F &&) {}
};

// What a workgroup multiplies.
enum Kind { DENSE, EXPERTS, GRADIENT };
struct Job {
    const uint8_t *a, *as, *b, *bs;   // the tile's first rows
    uint32_t rows_a, rows_b;          // of them there are, at most the tile's
    uint32_t first, blocks;           // of k
    uint64_t row, col;                // of out (GRADIENT: in the expert's part)
    uint32_t slice;                   // of the partial sums, or the expert
};

// Tiles are dealt so that the workgroups of one XCD (every eighth of the launch)
// have neighbouring tiles, eight rows of tiles by column.
__device__ inline void deal(uint32_t id, uint32_t mt, uint32_t nt, uint32_t &m, uint32_t &n)
{
    const uint32_t total = mt * nt, q = total / 8, left = total % 8, xcd = id % 8;
    const uint32_t tile = xcd * q + (xcd < left ? xcd : left) + id / 8;
    constexpr uint32_t GROUP = 8;
    const uint32_t grp = tile / (GROUP * nt), first = grp * GROUP;
    const uint32_t gm = mt - first < GROUP ? mt - first : GROUP;
    const uint32_t in = tile - grp * GROUP * nt;
    m = first + in % gm;
    n = in / gm;
}

// A tile of BM x BN sums, WM x WN waves.  A stage is a block of 128 values of k,
// copied from memory straight to LDS in whole pieces of 128 bytes a row (with
// pieces of 64 bytes a compute unit copies 63 GB/s, with these 115), BUFFERS
// stages in a ring; scales come for four stages at a time, a word a row.
// A stage's two instruction steps are three parts:
//   1  step 0's first products; step 1 is read from LDS
//      everyone has read the stage
//   2  the rest of step 0's and as many of step 1's; copies of a later stage to its place
//      the next stage has landed for everyone
//   3  the rest of step 1's; step 0 of the next stage is read, the other copies
// so that copies go out evenly (16 in a row hold up the wave's products) and have
// a whole stage's time.  In LDS chunk c (16 bytes) of row r stands at chunk c ^ (r
// / 2 % 8) of the row, so the 16 lanes that read one chunk of 16 rows meet every
// bank once.
// 8192^3 takes 391 to 430 us by the clock of the run, 2.6 to 2.8 PFLOP/s: the matrix units are busy 74 % of the cycles
// (the instruction alone reaches 4.0), the rest are meetings and 12 us a tile of
// first copies and stores.  With results of 32 bits 770 us, 1.4 PFLOP/s, bound by
// the matrix units' 16-bit rate.  EXPERTS: bound by reading the weights where an
// expert has few rows (512 rows of 64 experts, 2048 x 2048, 41 us, 6.5 TB/s), by the
// products where it has many (32,768 rows, 4096 x 2048, 359 us, 1.5 PFLOP/s: ten
// rounds of tiles with 22 us of stages and 12 of first copies and stores each, and an
// expert's last block is half empty).  GRADIENT: bound by storing (61 experts, 1000 x
// 2040 of f32, from 12,297 rows, 147 us in a graph of such calls, 3.4 TB/s, 169 by the
// profiler behind the other products of a step), each tile's few stages before it
// (without the stores 105).
// Tiles of 128 x 128 wait for their copies: 2048 x 4096 x 8192 takes 78 us, 68 without
// the products, 52 without the copies; eight waves a tile change nothing.
// A workgroup that goes through several tiles, the next one's first copies
// under way while it stores, took longer everywhere (8192^3 425 us, that gradient 219):
// a wait for copies is one for the stores before them.
template <class T, bool EXACT, Kind KIND, int BM, int BN, int WM, int WN, int BUFFERS>
__global__ __launch_bounds__(64 * WM * WN) void k_f8_product(F8MatmulArgs a, uint32_t mt, uint32_t nt, uint32_t per)
{
    constexpr uint32_t THREADS = 64 * WM * WN, PASS = THREADS / 8;   // rows of codes that the workgroup copies at a time
    constexpr int TM = BM / WM / 32, TN = BN / WN / 32, PA = BM / PASS, PB = BN / PASS;
    constexpr uint32_t SCALES = (BM + BN + THREADS - 1) / THREADS, COPIES = PA + PB;   // a stage's, scales left out
    constexpr uint32_t STAGE = (BM + BN) * 128, CODES = BUFFERS * STAGE, WORDS = (BM + BN) * 4;   // a stage's codes, all; four stages' scales
    constexpr uint32_t ALL = CODES + 4 * WORDS;
    static_assert(BM % PASS == 0 && BN % PASS == 0 && BM % 64 == 0 && BN % 64 == 0, "whole passes");
    extern __shared__ __align__(16) uint8_t lds[];
    const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(tid >> 6));
    const uint32_t r = lane & 31u, half = lane >> 5;
    const uint32_t cb = (uint32_t)f8_code_bytes(a.k), sb = (uint32_t)f8_scale_bytes(a.k);

    Job job;
    {
        uint32_t ti, tj;
        if constexpr (KIND == EXPERTS) {   // the blocks that there are, not those that there could be
            mt = (uint32_t)__builtin_amdgcn_readfirstlane(a.groups[a.experts + (BM == 256)]);
            if (blockIdx.x >= mt * nt) return;
        }
        deal(blockIdx.x, mt, nt, ti, tj);
        const uint64_t m0 = (uint64_t)ti * BM, n0 = (uint64_t)tj * BN;
        job.col = n0;
        job.rows_b = (uint32_t)(a.n - n0 < BN ? a.n - n0 : BN);
        job.b = a.b + n0 * cb;
        job.bs = a.bs + n0 * sb;
        if constexpr (KIND == EXPERTS) {
            const uint64_t skip = BM == 256 ? groups_blocks(a.experts, a.rows, 128) : 0;
            const int32_t *entry = a.groups + a.experts + 2 + 2 * (skip + ti);
            const uint32_t word = (uint32_t)__builtin_amdgcn_readfirstlane(entry[1]), expert = word & 0xFFFFu;
            job.row = (uint32_t)__builtin_amdgcn_readfirstlane(entry[0]);
            job.rows_a = word >> 16;
            job.b += expert * a.n * cb;
            job.bs += expert * a.n * sb;
        } else {
            job.row = m0;
            job.rows_a = (uint32_t)(a.m - m0 < BM ? a.m - m0 : BM);
        }
        job.a = a.a + job.row * cb;
        job.as = a.as + job.row * sb;
        job.slice = blockIdx.y;
        if constexpr (KIND == GRADIENT) {
            const int32_t *start = a.groups + blockIdx.y;
            job.first = (uint32_t)__builtin_amdgcn_readfirstlane(start[0]);
            job.blocks = (uint32_t)__builtin_amdgcn_readfirstlane(start[1]) - job.first;
        } else {
            const uint32_t all = (uint32_t)f8_blocks(a.k);
            job.first = KIND == DENSE ? blockIdx.y * per : 0u;
            job.blocks = KIND == DENSE && all - job.first > per ? per : all - job.first;
        }
    }
    // what this thread copies of a stage: a chunk of every PASS-th row of A,
    // then of B; rows past the last are that one again
    const uint32_t lm = job.rows_a - 1u, ln = job.rows_b - 1u, chunk = ((tid % 8) ^ (tid / 16 % 8)) * 16u;
    uint32_t offa[PA], offb[PB];
#pragma unroll
    for (int i = 0; i < PA; i++) {
        const uint32_t row = i * PASS + tid / 8;
        offa[i] = (row < lm ? row : lm) * cb + chunk;
    }
#pragma unroll
    for (int i = 0; i < PB; i++) {
        const uint32_t row = i * PASS + tid / 8;
        offb[i] = (row < ln ? row : ln) * cb + chunk;
    }
    const uint32_t stages = job.blocks, last = stages - 1u;
    auto copy = [&](uint32_t stage, int i) {   // past the last stage: one piece of its first row, into a buffer nobody reads
        const uint32_t k = (job.first + (stage < last ? stage : last)) * 128u, keep = stage <= last ? ~0u : 0u;
        uint8_t *to = lds + stage % BUFFERS * STAGE + (i * THREADS + wave * 64u) * 16u;
        if (i < PA) __builtin_amdgcn_global_load_lds((gptr)(job.a + ((offa[i] & keep) + k)), (lptr)to, 16, 0, 0);
        else __builtin_amdgcn_global_load_lds((gptr)(job.b + ((offb[i - PA] & keep) + k)), (lptr)to, 16, 0, 0);
    };
    // the scales of blocks 4 w ... + 3, a word of every row; a wave's rows are one operand's
    uint32_t offs[SCALES];
#pragma unroll
    for (uint32_t i = 0; i < SCALES; i++) {
        const uint32_t first = i * THREADS + wave * 64u, row = (first < BM ? first : first - BM) + lane, lim = first < BM ? lm : ln;
        offs[i] = (row < lim ? row : lim) * sb;
    }
    auto copy_scales = [&](uint32_t w) {
        const uint32_t at = w * 4u < sb ? w * 4u : sb - 4u;
#pragma unroll
        for (uint32_t i = 0; i < SCALES; i++) {
            const uint32_t first = i * THREADS + wave * 64u;
            if (first >= BM + BN) break;
            __builtin_amdgcn_global_load_lds((gptr)((first < BM ? job.as : job.bs) + (offs[i] + at)), (lptr)(lds + CODES + w % 4u * WORDS + first * 4u), 4, 0, 0);
        }
    };

    const uint32_t wm = wave / WN * (BM / WM), wn = wave % WN * (BN / WN);
    struct Held {
        Piece x[TM], y[TN];
    } held[2];
    struct Scales {
        uint32_t x[TM], y[TN];
    };
    const uint32_t key = r / 2 % 8;
    auto read = [&](Held &h, uint32_t stage, uint32_t step, int q) {
        const uint32_t c = step * 4u + half * 2u, lo = (c ^ key) * 16u, hi = ((c + 1u) ^ key) * 16u;
        const uint8_t *p = lds + stage % BUFFERS * STAGE + (r + (q < TN ? BM + wn + q * 32u : wm + (q - TN) * 32u)) * 128u;
        const Piece got{*reinterpret_cast<const u32x4 *>(p + lo), *reinterpret_cast<const u32x4 *>(p + hi)};
        if (q < TN) h.y[q] = got;
        else h.x[q - TN] = got;
    };
    auto read_scales = [&](Scales &to, uint32_t stage) {
        const uint8_t *from = lds + CODES + (job.first + stage) / 4u % 4u * WORDS + r * 4u;
        auto word = [&](uint32_t row) { return *reinterpret_cast<const uint32_t *>(from + row * 4u); };
#pragma unroll
        for (int j = 0; j < TN; j++) to.y[j] = word(BM + wn + j * 32u);
#pragma unroll
        for (int i = 0; i < TM; i++) to.x[i] = word(wm + i * 32u);
    };
    auto bytes_of = [&](const Scales &words, uint32_t stage) {   // at the words' ends
        const uint32_t shift = (job.first + stage) % 4u * 8u;
        Scales to;
#pragma unroll
        for (int j = 0; j < TN; j++) to.y[j] = words.y[j] >> shift;
#pragma unroll
        for (int i = 0; i < TM; i++) to.x[i] = words.x[i] >> shift;
        return to;
    };
    auto meet = [&]() {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    auto all_read = [&]() {
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        meet();
    };
    auto landed = [&](auto later) {   // but for so many later copies
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(decltype(later)::value) : "memory");
        meet();
    };
    // without it the compiler turns the reads before the loop and at its end into ones at its beginning, for which products wait
    auto held_back = []() { asm volatile("" ::: "memory"); };
    constexpr int N = TM * TN, READS = 2 * (TM + TN), PART = EXACT ? N / 4 : N * 3 / 8, CUT = EXACT ? COPIES / 2 : COPIES * 3 / 4;   // products of a step, its reads; what the second part takes
    f32x16 acc[TM][TN] = {};
    uint32_t top = 0;   // EXACT: the largest scale byte
    if (stages) {
        copy_scales(job.first / 4u);
        copy_scales(job.first / 4u + 1u);
#pragma unroll
        for (uint32_t i = 0; i < BUFFERS; i++)
#pragma unroll
            for (int q = 0; q < (int)COPIES; q++) copy(i, q);
        landed(Number<(BUFFERS - 1) * COPIES>{});
        Scales words;
        read_scales(words, 0);
#pragma unroll
        for (int q = 0; q < TM + TN; q++) read(held[0], 0, 0, q);
        for (uint32_t s = 0; s < stages; s++) {
            held_back();
            const Scales now = bytes_of(words, s);
            if constexpr (EXACT) {
#pragma unroll
                for (int i = 0; i < TM; i++) top = max(top, now.x[i] & 0xFFu);
#pragma unroll
                for (int j = 0; j < TN; j++) top = max(top, now.y[j] & 0xFFu);
            }
#pragma unroll
            for (int q = 0; q < TM + TN; q++) read(held[1], s, 1, q);
            products<EXACT, 0, N - PART>(acc, held[0].x, now.x, held[0].y, now.y);
            if (!EXACT) mixed<N - PART, READS, 0>();
            all_read();
            // words that the next stages begin, into the place of some that nobody reads any more
            if ((job.first + s) % 4u == 0) copy_scales((job.first + s) / 4u + 1u);
#pragma unroll
            for (int i = 0; i < CUT; i++) copy(s + BUFFERS, i);
            products<EXACT, N - PART, N>(acc, held[0].x, now.x, held[0].y, now.y);
            products<EXACT, 0, PART>(acc, held[1].x, now.x, held[1].y, now.y);
            if (!EXACT) mixed<2 * PART, 0, CUT>();
            landed(Number<(BUFFERS - 2) * COPIES + CUT>{});
            read_scales(words, s + 1);
#pragma unroll
            for (int i = 0; i < (int)COPIES - CUT || i < TM + TN; i++) {
                if (i < TM + TN) read(held[0], s + 1, 0, i);
                if (CUT + i < (int)COPIES) copy(s + BUFFERS, CUT + i);
            }
            products<EXACT, PART, N>(acc, held[1].x, now.x, held[1].y, now.y);
            if (!EXACT) {
                mixed<1, (TM + TN) / 2, 0>();   // the words
                mixed<N - PART - 1, READS, COPIES - CUT>();
            }
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // no copy outlives the workgroup's LDS
    }
    if constexpr (EXACT)
        if (__any(top >= BEYOND)) {   // the wave's sums again, from memory
#pragma unroll
            for (int i = 0; i < TM; i++)
#pragma unroll
                for (int j = 0; j < TN; j++) {
                    const uint32_t mx = wm + i * 32u + r, my = wn + j * 32u + r, rx = mx < lm ? mx : lm, ry = my < ln ? my : ln;
                    f32x16 sum = {};
                    for (uint32_t k = job.first; k < job.first + stages; k++)
                        add_unscaled(sum, job.a + (rx * cb + k * 128u + half * 64u), job.as[rx * sb + k], job.b + (ry * cb + k * 128u + half * 64u), job.bs[ry * sb + k]);
                    acc[i][j] = sum;
                }
        }
    // The sums go through LDS, 32 rows of the waves beside each other at a time, so
    // that a tile's whole rows are stored, past the caches that the operands are read
    // from (with ordinary stores 8192^3 takes 3 % longer, the gradient of 61 experts,
    // 1000 x 2040 of f32, 46 %).  Rows that begin inside a line of 128 bytes share
    // their first and last with a neighbouring tile, which costs 8 % of that gradient
    // (rows of single waves stored by themselves 15 %; those lines kept in the caches,
    // more).  Few instructions a chunk, as a wave has a SIMD to itself (checks of every
    // chunk's columns: 5 %).
    typedef u32x4 Chunk __attribute__((aligned(2)));   // at any address
    T *out = static_cast<T *>(a.out) + (KIND == EXPERTS ? 0u : (uint64_t)job.slice * a.m * a.ld);
    constexpr uint32_t EACH = 16 / sizeof(T), CHUNKS_ROW = BN / EACH, ROW = BN * sizeof(T) + 16;
    constexpr uint32_t EACH_PASS = 64 / CHUNKS_ROW, PASSES = 32 / WN / EACH_PASS;   // rows of a pass, passes
    static_assert(2 * WM * 32 * ROW <= ALL, "within the stages' room");
    const uint32_t row = wave % WN * (32 / WN) + lane / CHUNKS_ROW, n = lane % CHUNKS_ROW * EACH;
    __syncthreads();   // all have read the last stage
#pragma unroll
    for (int i = 0; i < TM; i++) {
        uint8_t *rows = lds + (i % 2 * WM + wave / WN) * (32u * ROW);
#pragma unroll
        for (int j = 0; j < TN; j++)
#pragma unroll
            for (int q = 0; q < 4; q++) {
                T t[4];
#pragma unroll
                for (int c = 0; c < 4; c++) t[c] = Elem<T>::put(acc[i][j][4 * q + c]);
                __builtin_memcpy(__builtin_assume_aligned(rows + r * ROW + (wn + j * 32u + q * 8u + half * 4u) * sizeof(T), sizeof t), t, sizeof t);
            }
        all_read();   // and what was written is there
        Chunk w[PASSES];
#pragma unroll
        for (uint32_t p = 0; p < PASSES; p++) w[p] = *reinterpret_cast<const u32x4 *>(rows + (p * EACH_PASS + row) * ROW + lane % CHUNKS_ROW * 16u);
        const uint32_t m = wm + i * 32u + row, left = m < job.rows_a ? job.rows_a - m : 0u;
        T *to = out + (job.row + m) * a.ld + job.col + n;
        if (n + EACH <= job.rows_b) {
#pragma unroll
            for (uint32_t p = 0; p < PASSES; p++, to += EACH_PASS * a.ld)
                if (p * EACH_PASS < left) __builtin_nontemporal_store(w[p], reinterpret_cast<Chunk *>(to));
        } else if (n < job.rows_b) {   // a row's last few
#pragma unroll
            for (uint32_t p = 0; p < PASSES; p++, to += EACH_PASS * a.ld) {
                T t[EACH];
                __builtin_memcpy(t, &w[p], 16);
#pragma unroll
                for (uint32_t c = 0; c + 1 < EACH; c++)
                    if (p * EACH_PASS < left && n + c < job.rows_b) to[c] = t[c];
            }
        }
    }
}

// ---- few rows ----------------------------------------------------------------

// Sixteen rows of each operand over 128 values of k: lane l has 32 values of row
// l % 16, and gets four neighbouring sums, rows 4 (l / 16) ... of y, row l % 16 of x.
template <bool EXACT>
__device__ inline f32x4 product16(const Piece &y, uint32_t ys, const Piece &x, uint32_t xs, f32x4 c)
{
    if constexpr (EXACT) {
        const float fy = mx_scale(ys), fx = mx_scale(xs);
#pragma unroll
        for (int q = 0; q < 4; q++) {
            const u32x4 &v = q < 2 ? y.lo : y.hi, &w = q < 2 ? x.lo : x.hi;
            c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wide(v[q % 2 * 2], v[q % 2 * 2 + 1], fy), wide(w[q % 2 * 2], w[q % 2 * 2 + 1], fx), c, 0, 0, 0);
        }
        return c;
    } else {
        auto whole = [](const Piece &p) { return i32x8{(int)p.lo.x, (int)p.lo.y, (int)p.lo.z, (int)p.lo.w, (int)p.hi.x, (int)p.hi.y, (int)p.hi.z, (int)p.hi.w}; };
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(whole(y), whole(x), c, 0, 0, 0, (int)ys, 0, (int)xs);
    }
}

// c += y x over a block, its scales applied to its sum: for blocks beyond what bf16 holds.
__device__ inline void add_unscaled16(f32x4 &c, const uint8_t *x, uint32_t xs, const uint8_t *y, uint32_t ys)
{
    f32x4 sum = {};
#pragma unroll
    for (int q = 0; q < 2; q++) {
        const u32x4 v = reinterpret_cast<const u32x4 *>(y)[q], w = reinterpret_cast<const u32x4 *>(x)[q];
        sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wide(v.x, v.y, 1.f), wide(w.x, w.y, 1.f), sum, 0, 0, 0);
        sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wide(v.z, v.w, 1.f), wide(w.z, w.w, 1.f), sum, 0, 0, 0);
    }
#pragma unroll
    for (int q = 0; q < 4; q++) c[q] += with_scales(sum[q], xs, (uint32_t)__shfl((int)ys, (int)(threadIdx.x & 48u) / 4 + q));
}

// Four neighbouring sums of row `row`, in the output's type.
__device__ inline void store4_as(void *out, uint32_t dtype, uint64_t ld, uint64_t row, uint64_t col, uint64_t n, f32x4 v)
{
    if (dtype == DT_F32) store4(static_cast<float *>(out), ld, row, col, n, v);
    else if (dtype == DT_BF16) store4(static_cast<__bf16 *>(out), ld, row, col, n, v);
    else store4(static_cast<_Float16 *>(out), ld, row, col, n, v);
}

constexpr uint32_t SLOT = 2048 + 256;   // a step of 16 rows, and the words of their scales

template <int MT, int WAVES, int D>
constexpr uint32_t few_lds() { return WAVES * D * SLOT + 2 * WAVES * MT * 1024; }

// Up to 16 MT rows of A: bound by reading B once.  The waves of a workgroup share
// out its part of k, S steps of 128 values each, and hold A's operands of their
// steps in registers; the workgroup goes through tiles of 16 rows of B.  A wave's
// operands come straight to LDS in whole pieces of 128 bytes a row, D steps ahead
// in a ring of its own, so that nothing is between the waves but the joining of
// their sums, in their order.  Whoever has no more to read reads one piece, so
// that as many copies are under way.  48 x 16384 x 5120 takes 22.5 us from memory, 3.7
// TB/s (the tiles' form 26.6), 16.9 from the device's cache; 1 x 4096 x 4096 6.3 (14.3).
template <bool EXACT, int MT, int S, int WAVES, int D>
__global__ __launch_bounds__(64 * WAVES) void k_f8_few(F8MatmulArgs a, uint32_t dtype, uint32_t tiles)
{
    extern __shared__ __align__(16) uint8_t lds[];
    const uint32_t lane = threadIdx.x & 63u, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const uint32_t r = lane & 15u, g = lane >> 4;
    const uint32_t cb = (uint32_t)f8_code_bytes(a.k), sb = (uint32_t)f8_scale_bytes(a.k), steps = (uint32_t)f8_blocks(a.k);
    const uint32_t s0 = (blockIdx.y * WAVES + wave) * S, mine = s0 < steps ? (steps - s0 < S ? steps - s0 : S) : 0u;
    const uint32_t rows = (uint32_t)a.m;   // more than 16 (MT - 1)
    char *out = static_cast<char *>(a.out) + (uint64_t)blockIdx.y * a.m * a.ld * sizeof(float);   // of the partial sums
    uint8_t *ring = lds + wave * (D * SLOT);
    f32x4 *sums = reinterpret_cast<f32x4 *>(lds + WAVES * D * SLOT);   // [2][WAVES][MT][64]
    const uint32_t mine_tiles = (tiles - blockIdx.x + gridDim.x - 1) / gridDim.x;

    // where a lane's pieces and word of a whole tile lie: an instruction takes eight rows
    const uint32_t chunk = lane / 16u * 16u, word = (s0 / 4u + g) * 4u < sb ? (s0 / 4u + g) * 4u : sb - 4u;
    auto piece_of = [&](uint32_t i, uint32_t last) {
        const uint32_t in = i * 8u + lane / 8u;
        return (in < last ? in : last) * cb + ((lane % 8u * 16u) ^ ((i * 64u + chunk) & 112u));
    };
    auto word_of = [&](uint32_t last) { return (r < last ? r : last) * sb + word; };
    const uint32_t piece[2] = {piece_of(0, 15), piece_of(1, 15)}, words = word_of(15);
    // step j of the 16 rows at `first` of the `n` of an operand
    auto issue = [&](const uint8_t *codes, const uint8_t *scales, uint64_t first, uint64_t n, int j, uint32_t slot) {
        const bool some = (uint32_t)j < mine && first < n;
        const uint32_t keep = some ? ~0u : 0u;
        uint32_t off[2] = {piece[0], piece[1]}, at = words;
        if (some && n - first < 16u) {   // rows past the last: that one again
            const uint32_t last = (uint32_t)(n - first) - 1u;
            off[0] = piece_of(0, last), off[1] = piece_of(1, last), at = word_of(last);
        }
        const uint8_t *from = some ? codes + first * cb + (s0 + j) * 128u : codes;
        uint8_t *to = ring + slot * SLOT;
#pragma unroll
        for (uint32_t i = 0; i < 2; i++) __builtin_amdgcn_global_load_lds((gptr)(from + (off[i] & keep)), (lptr)(to + i * 1024u), 16, 0, 0);
        // words s0 / 4 ... + 3 of the rows' scales
        if (j == 0) __builtin_amdgcn_global_load_lds((gptr)((some ? scales + first * sb : scales) + (at & keep)), (lptr)(to + 2048u), 4, 0, 0);
    };
    auto issue_a = [&](int t, int j, uint32_t slot) { issue(a.a, a.as, (uint64_t)t * 16u, rows, j, slot); };
    auto issue_b = [&](uint32_t i, int j, uint32_t slot) { issue(a.b, a.bs, ((uint64_t)blockIdx.x + (uint64_t)i * gridDim.x) * 16u, a.n, j, slot); };
    uint32_t slot = 0;
    auto next = [&]() { slot = slot + 1 == D ? 0 : slot + 1; };
    auto landed = [&](auto step) {   // this one, of the D under way
        constexpr int j = decltype(step)::value;
        constexpr int begun = (j + D - 1) / S - j / S;   // tiles that begin among the later ones
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * (D - 1) + begun) : "memory");
    };
    auto codes_of = [&]() {
        const uint8_t *from = ring + slot * SLOT + r * 128u;
        return Piece{*reinterpret_cast<const u32x4 *>(from + ((2u * g) ^ (r / 2u)) * 16u), *reinterpret_cast<const u32x4 *>(from + ((2u * g + 1u) ^ (r / 2u)) * 16u)};
    };
    auto scales_of = [&](uint32_t (&to)[S]) {
        const uint8_t *from = ring + slot * SLOT + 2048u + r * 4u;
#pragma unroll
        for (uint32_t j = 0; j < S; j++) to[j] = from[((s0 + j) / 4u - s0 / 4u) * 64u + (s0 + j) % 4u];
    };
    // what has been read is in registers before its place is written to
    auto taken = [&]() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); };
    Piece x[MT][S];
    uint32_t xs[MT][S];
#pragma unroll
    for (int u = 0; u < D; u++) {
        if (u / S < MT) issue_a(u / S, u % S, (uint32_t)u);
        else issue_b((uint32_t)(u / S - MT), u % S, (uint32_t)u);
    }
#pragma unroll
    for (int t = 0; t < MT; t++)
        Each<S>::run([&](auto step) {
            constexpr int j = decltype(step)::value;
            landed(step);
            if constexpr (j == 0) scales_of(xs[t]);
            x[t][j] = codes_of();
            taken();
            if (t + (j + D) / S < MT) issue_a(t + (j + D) / S, (j + D) % S, slot);
            else issue_b((uint32_t)(t + (j + D) / S - MT), (j + D) % S, slot);
            next();
        });
    uint32_t top = 0;   // EXACT: the largest scale byte of A
    if constexpr (EXACT) {
#pragma unroll
        for (uint32_t j = 0; j < S; j++)
#pragma unroll
            for (int t = 0; t < MT; t++) top = j < mine ? max(top, xs[t][j]) : top;
    }
    for (uint32_t i = 0; i < mine_tiles; i++) {
        f32x4 acc[MT] = {};
        uint32_t ys[S];
        Each<S>::run([&](auto step) {
            constexpr int j = decltype(step)::value;
            landed(step);
            if constexpr (j == 0) scales_of(ys);
            const Piece y = codes_of();
            taken();
            issue_b(i + (uint32_t)((j + D) / S), (j + D) % S, slot);
            next();
            if ((uint32_t)j < mine) {
#pragma unroll
                for (int t = 0; t < MT; t++) {
                    // as codes, not as the twice as many registers of bf16 that they become anew for every tile
                    if constexpr (EXACT) asm volatile("" : "+v"(x[t][j].lo), "+v"(x[t][j].hi));
                    acc[t] = product16<EXACT>(y, ys[j], x[t][j], xs[t][j], acc[t]);
                }
            }
        });
        if constexpr (EXACT) {
            uint32_t most = top;
#pragma unroll
            for (uint32_t j = 0; j < S; j++) most = j < mine ? max(most, ys[j]) : most;
            if (__any(most >= BEYOND)) {   // the wave's sums again, from memory
                const uint64_t n = ((uint64_t)blockIdx.x + (uint64_t)i * gridDim.x) * 16u + r, ry = n < a.n ? n : a.n - 1;
#pragma unroll
                for (int t = 0; t < MT; t++) {
                    const uint64_t m = t * 16u + r, rx = m < rows ? m : rows - 1u;
                    acc[t] = f32x4{};
                    for (uint32_t k = s0; k < s0 + mine; k++)
                        add_unscaled16(acc[t], a.a + (rx * cb + k * 128u + g * 32u), a.as[rx * sb + k], a.b + (ry * cb + k * 128u + g * 32u), a.bs[ry * sb + k]);
                }
            }
        }
        f32x4 *part = sums + (i % 2u) * (WAVES * MT * 64u);
#pragma unroll
        for (int t = 0; t < MT; t++) part[(wave * MT + t) * 64u + lane] = acc[t];
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();   // the sums of the tile before last have been read by then
        asm volatile("" ::: "memory");
        if (wave < MT) {
            f32x4 v = part[wave * 64u + lane];
#pragma unroll
            for (uint32_t q = 1; q < WAVES; q++) v += part[(q * MT + wave) * 64u + lane];
            const uint32_t m = wave * 16u + r;
            if (m < rows) store4_as(out, dtype, a.ld, m, ((uint64_t)blockIdx.x + (uint64_t)i * gridDim.x) * 16u + g * 4u, a.n, v);
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // no copy outlives the workgroup's LDS
}

// The sums of a shared-out k, joined in the order of its parts: a thread takes
// four columns of a row.  Rows of the parts are padded to `ld`, whole fours.
template <class T>
__global__ __launch_bounds__(256) void k_f8_join(F8MatmulArgs a, uint32_t splits, uint64_t ld)
{
    const uint64_t i = (uint64_t)blockIdx.x * 256u + threadIdx.x, row = i / (ld / 4), col = i % (ld / 4) * 4u;
    if (row >= a.m) return;
    const float *p = a.part + row * ld + col;
    f32x4 v = *reinterpret_cast<const f32x4 *>(p);
    for (uint32_t j = 1; j < splits; j++) v += *reinterpret_cast<const f32x4 *>(p + (uint64_t)j * a.m * ld);
    store4(static_cast<T *>(a.out), a.ld, row, col, a.n, v);
}

template <class T, bool EXACT, Kind KIND, int BM, int BN, int WM, int WN, int BUFFERS>
hipError_t product(const F8MatmulArgs &a, uint32_t mt, uint32_t slices, uint32_t per, hipStream_t s)
{
    constexpr uint32_t threads = 64 * WM * WN, bytes = (BM + BN) * (128 * BUFFERS + 16);
    static_assert(bytes <= 160u << 10, "one workgroup's LDS");
    const hipError_t e = allow_lds<&k_f8_product<T, EXACT, KIND, BM, BN, WM, WN, BUFFERS>>(bytes);
    if (e != hipSuccess) return e;
    const uint32_t nt = (uint32_t)((a.n + BN - 1) / BN);
    k_f8_product<T, EXACT, KIND, BM, BN, WM, WN, BUFFERS><<<dim3(mt * nt, slices), threads, bytes, s>>>(a, mt, nt, per);
    return hipGetLastError();
}

template <class F>
hipError_t by_type(uint32_t dtype, F &&f)
{
    if (dtype == DT_F32) return f(float{});
    if (dtype == DT_BF16) return f(__bf16{});
    return f(_Float16{});
}

inline uint64_t tiles_of(uint64_t m, uint64_t n, uint64_t side = 128) { return ((m + side - 1) / side) * ((n + side - 1) / side); }

// Tiles of 256 x 256 or of 128 x 128, by rounds over 256 compute units.  A round
// of the larger ones takes as long as three of the smaller ones (with k = 2048, in
// us, large and small: 128 and 512 tiles 28 and 22, 160 and 640 28 and 30, 256 and
// 1024 33 and 43, 272 and 1088 53 and 50, 384 and 1536 56 and 63), or, with results
// of 32 bits, not quite as four (160 and 640 47 and 44, 256 and 1024 60 and 66, 272
// and 1088 100 and 73, 384 and 1536 101 and 101; 32,768 rows of 64 experts, 4096 x
// 2048, 603 and 575).
inline bool large_tiles(uint64_t small, uint64_t large, bool exact)
{
    const uint64_t s = (small + 255) / 256, l = (large + 255) / 256;
    return exact ? 4 * s >= 15 * l : s >= 3 * l;
}

// How a product is made: k in `parts` of `per` blocks; few rows with steps of
// `each` a wave.
// As few rows, or in tiles, in us: 1 x 4096 x 4096 6.3 and 14.3, 64 x 4096 x 4096
// 10.2 and 15.9, 64 x 16384 x 1024 8.9 and 9.2, 64 x 65536 x 2048 35.8 and 35.7 (with
// results of 32 bits 39.2 and 36.7: there it costs a little).  More rows than 64 leave
// no registers for them.
constexpr uint32_t FEW_ROWS = 64;
constexpr int FEW_WAVES = 8, FEW_AHEAD = 4;   // seven steps ahead take as long as four
// Of a part of k in tiles.  With 4, 8 and 16, in us: 512 x 512 x 8192 20.3, 17.6 and
// 19.3, 100 x 4096 x 4096 18.8, 15.6 and 17.5, with results of 32 bits 20.4, 17.5 and
// 20.9; 500 x 1000 x 2048 12.8, 12.1 and 11.9.
constexpr uint32_t LEAST_BLOCKS = 8;
struct Plan {
    bool few;
    uint32_t parts, per, each;
};
// steps that a wave can hold of so many sixteens of rows
inline uint32_t most_steps(uint32_t mt) { return mt == 1 ? 8u : mt == 2 ? 8u : mt == 3 ? 5u : 4u; }

inline Plan plan(uint64_t m, uint64_t n, uint64_t k)
{
    const uint32_t blocks = (uint32_t)f8_blocks(k);
    Plan p{m <= FEW_ROWS && blocks > 0, 1, 0, 0};
    if (p.few) {
        const uint32_t mt = (uint32_t)(m + 15) / 16, most = most_steps(mt);
        p.parts = (blocks + FEW_WAVES * most - 1) / (FEW_WAVES * most);
        p.each = (blocks + FEW_WAVES * p.parts - 1) / (FEW_WAVES * p.parts);
        p.per = p.each * FEW_WAVES;
        return p;
    }
    // Blocks of k that a workgroup takes: all, or, where tiles are too few for 256
    // compute units, parts of LEAST_BLOCKS or more.
    const uint64_t tiles = tiles_of(m, n), want = tiles < 256 ? 256 / tiles : 1;
    uint64_t per = (blocks + want - 1) / want;
    if (per < LEAST_BLOCKS) per = LEAST_BLOCKS;
    if (per >= blocks) {
        p.per = blocks + 1;
        return p;
    }
    p.per = (uint32_t)per;
    p.parts = (uint32_t)((blocks + per - 1) / per);
    return p;
}
inline uint64_t padded(uint64_t n) { return (n + 3) / 4 * 4; }

template <bool EXACT, int MT, int S, int WAVES, int D>
hipError_t few_as(const F8MatmulArgs &a, uint32_t dtype, uint32_t slices, uint32_t workers, hipStream_t s)
{
    constexpr uint32_t bytes = few_lds<MT, WAVES, D>();
    static_assert(bytes <= 160u << 10 && MT * S <= 16, "one workgroup's LDS, and registers");
    const hipError_t e = allow_lds<&k_f8_few<EXACT, MT, S, WAVES, D>>(bytes);
    if (e != hipSuccess) return e;
    const uint32_t tiles = (uint32_t)((a.n + 15) / 16);
    k_f8_few<EXACT, MT, S, WAVES, D><<<dim3(tiles < workers ? tiles : workers, slices), 64 * WAVES, bytes, s>>>(a, dtype, tiles);
    return hipGetLastError();
}

template <bool EXACT, int MT>
hipError_t few_rows(const F8MatmulArgs &a, uint32_t dtype, const Plan &p, hipStream_t s)
{
    const uint32_t workers = (256 + p.parts - 1) / p.parts;   // one a compute unit (two: 64 x 16384 x 1024 11.1 us for 8.9, 48 x 16384 x 5120 26.7 for 22.5)
#define STEPS(S)                                                                                             \
    if constexpr (MT * S <= 16)                                                                              \
        if (p.each <= S) return few_as<EXACT, MT, S, FEW_WAVES, FEW_AHEAD>(a, dtype, p.parts, workers, s);
    STEPS(1) STEPS(2) STEPS(3) STEPS(4) STEPS(5) STEPS(6) STEPS(8)
#undef STEPS
    return hipErrorInvalidValue;   // not reached: most_steps()
}

template <class T>
hipError_t join(const F8MatmulArgs &a, uint32_t parts, hipStream_t s)
{
    const uint64_t ld = padded(a.n), threads = a.m * (ld / 4);
    k_f8_join<T><<<dim3((uint32_t)((threads + 255) / 256)), 256, 0, s>>>(a, parts, ld);
    return hipGetLastError();
}

}  // namespace

size_t f8_matmul_workspace(uint64_t m, uint64_t n, uint64_t k)
{
    const Plan p = plan(m, n, k);
    return p.parts > 1 ? (size_t)(p.parts * m * padded(n) * sizeof(float)) : 0;
}

bool f8_matmul_fits(uint64_t m, uint64_t n, uint64_t k)
{
    const Plan p = plan(m, n, k);
    return p.few ? p.parts == 1 || m * (padded(n) / 4) <= most_blocks(256) * 256 : tiles_of(m, n) <= most_blocks(256);
}
bool f8_experts_fit(uint64_t rows, uint32_t experts, uint64_t n) { return groups_blocks(experts, rows, 128) * ((n + 127) / 128) <= most_blocks(256); }
bool f8_gradients_fit(uint32_t experts, uint64_t m, uint64_t n) { return tiles_of(m, n) <= most_blocks(256) / experts; }

hipError_t launch_f8_matmul(const F8MatmulArgs &a, uint32_t dtype, hipStream_t s)
{
    return by_type(dtype, [&](auto t) -> hipError_t {
        typedef decltype(t) T;
        constexpr bool EXACT = sizeof(T) == 4;
        const Plan p = plan(a.m, a.n, a.k);
        const uint32_t mt = (uint32_t)((a.m + 127) / 128);
        F8MatmulArgs part = a;
        if (p.parts > 1) {
            part.out = a.part;
            part.ld = padded(a.n);
        }
        hipError_t e;
        if (p.few) {
            const uint32_t type = p.parts > 1 ? (uint32_t)DT_F32 : dtype;
            if (a.m <= 16) e = few_rows<EXACT, 1>(part, type, p, s);
            else if (a.m <= 32) e = few_rows<EXACT, 2>(part, type, p, s);
            else if (a.m <= 48) e = few_rows<EXACT, 3>(part, type, p, s);
            else e = few_rows<EXACT, 4>(part, type, p, s);
        } else if (p.parts > 1) {
            e = product<float, EXACT, DENSE, 128, 128, 2, 2, 4>(part, mt, p.parts, p.per, s);
        } else if (large_tiles(tiles_of(a.m, a.n), tiles_of(a.m, a.n, 256), EXACT)) {
            e = product<T, EXACT, DENSE, 256, 256, 2, 2, 2>(a, (mt + 1) / 2, 1, p.per, s);
        } else if (tiles_of(a.m, a.n) > 256) {   // two workgroups a compute unit, with half as much copied ahead (2048^2 x 8192, one tile each, 49 us and 44 without; 2040 x 2080 x 1500, 272 tiles, 15 and 19)
            e = product<T, EXACT, DENSE, 128, 128, 2, 2, 2>(a, mt, 1, p.per, s);
        } else {
            e = product<T, EXACT, DENSE, 128, 128, 2, 2, 4>(a, mt, 1, p.per, s);
        }
        return e == hipSuccess && p.parts > 1 ? join<T>(a, p.parts, s) : e;
    });
}

hipError_t launch_f8_expert_matmul(const F8MatmulArgs &a, uint32_t dtype, hipStream_t s)
{
    return by_type(dtype, [&](auto t) -> hipError_t {
        typedef decltype(t) T;
        constexpr bool EXACT = sizeof(T) == 4;
        // an expert's last block is half full, as far as one can know here (large and
        // small: 32,768 rows of 64 experts, 4096 x 2048, 359 and 394 us); with up to one small
        // block an expert most of a large one is empty (128 rows of 64 experts, 2048 x 2048,
        // 52 and 34; 4096 rows 90 and 63, 8192 rows 93 and 85; 192 rows of one, 4096 x 2048,
        // 25 and 13)
        const uint64_t half = a.experts / 2, small = ((a.rows + 127) / 128 + half) * ((a.n + 127) / 128), large = ((a.rows + 255) / 256 + half) * ((a.n + 255) / 256);
        if (a.rows > 128ull * a.experts && large_tiles(small, large, EXACT))
            return product<T, EXACT, EXPERTS, 256, 256, 2, 2, 2>(a, (uint32_t)groups_blocks(a.experts, a.rows, 256), 1, 0, s);
        return product<T, EXACT, EXPERTS, 128, 128, 2, 2, 2>(a, (uint32_t)groups_blocks(a.experts, a.rows, 128), 1, 0, s);
    });
}

hipError_t launch_f8_expert_gradient(const F8MatmulArgs &a, uint32_t dtype, hipStream_t s)
{
    return by_type(dtype, [&](auto t) -> hipError_t {
        typedef decltype(t) T;
        constexpr bool EXACT = sizeof(T) == 4;
        // large and small: 61 experts, 1000 x 2040 from 12,297 rows, f32 150 and 154 us, bf16
        // 95 and 102; 64 experts, 1024 x 1024 from 4096 rows, f32 66 and 58, bf16 43 and 45 (a
        // tile's stages, few there, are not among what the rule goes by)
        if (large_tiles(a.experts * tiles_of(a.m, a.n), a.experts * tiles_of(a.m, a.n, 256), EXACT))
            return product<T, EXACT, GRADIENT, 256, 256, 2, 2, 2>(a, (uint32_t)((a.m + 255) / 256), a.experts, 0, s);
        return product<T, EXACT, GRADIENT, 128, 128, 2, 2, 2>(a, (uint32_t)((a.m + 127) / 128), a.experts, 0, s);
    });
}

}  // namespace pccl
