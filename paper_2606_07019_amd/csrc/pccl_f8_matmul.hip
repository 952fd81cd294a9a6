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
// scaled, which is exact, for the 16-bit form (32 rows over 16 values of k).
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

// 32 bytes of a row, and the byte of its scale.
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

// Four neighbouring sums of row `row`, from column `col` on.
template <class T>
__device__ inline void store4(T *out, uint64_t ld, uint64_t row, uint64_t col, uint64_t n, f32x4 v, bool vec)
{
    T t[4];
#pragma unroll
    for (int i = 0; i < 4; i++) t[i] = Elem<T>::put(v[i]);
    T *p = out + row * ld + col;
    if (vec && col + 4 <= n) {
        __builtin_memcpy(__builtin_assume_aligned(p, sizeof t), t, sizeof t);
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
    auto copy = [&](uint32_t stage, int i) {   // past the last stage: that one again, into a buffer nobody reads
        const uint32_t k = (job.first + (stage < last ? stage : last)) * 128u;
        uint8_t *to = lds + stage % BUFFERS * STAGE + (i * THREADS + wave * 64u) * 16u;
        if (i < PA) __builtin_amdgcn_global_load_lds((gptr)(job.a + (offa[i] + k)), (lptr)to, 16, 0, 0);
        else __builtin_amdgcn_global_load_lds((gptr)(job.b + (offb[i - PA] + k)), (lptr)to, 16, 0, 0);
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
    // The sums go through LDS, 32 rows of the wave's at a time, so that whole rows of them are stored.
    T *out = static_cast<T *>(a.out) + (KIND == EXPERTS ? 0u : (uint64_t)job.slice * a.m * a.ld);
    constexpr uint32_t COLS = BN / WN, EACH = 16 / sizeof(T), CHUNKS_ROW = COLS / EACH, ROW = COLS * sizeof(T) + 16;
    static_assert(WM * WN * 32 * ROW <= ALL, "within the stages' room");
    __syncthreads();   // all have read the last stage
    uint8_t *own = lds + wave * (32u * ROW);
#pragma unroll
    for (int i = 0; i < TM; i++) {
#pragma unroll
        for (int j = 0; j < TN; j++)
#pragma unroll
            for (int q = 0; q < 4; q++) {
                T t[4];
#pragma unroll
                for (int c = 0; c < 4; c++) t[c] = Elem<T>::put(acc[i][j][4 * q + c]);
                __builtin_memcpy(__builtin_assume_aligned(own + r * ROW + (j * 32u + q * 8u + half * 4u) * sizeof(T), sizeof t), t, sizeof t);
            }
#pragma unroll
        for (uint32_t p = 0; p < CHUNKS_ROW / 2; p++) {
            const uint32_t row = p * (64u / CHUNKS_ROW) + lane / CHUNKS_ROW, col = lane % CHUNKS_ROW * EACH;
            const uint32_t m = wm + i * 32u + row, n = wn + col;
            if (m >= job.rows_a || n >= job.rows_b) continue;
            T t[EACH];
            __builtin_memcpy(t, __builtin_assume_aligned(own + row * ROW + col * sizeof(T), 16), 16);
            T *to = out + (job.row + m) * a.ld + job.col + n;
            if (n + EACH <= job.rows_b) {
                __builtin_memcpy(to, t, 16);   // at any address
                continue;
            }
#pragma unroll
            for (uint32_t c = 0; c < EACH; c++)
                if (n + c < job.rows_b) to[c] = t[c];
        }
    }
}

// The sums of a shared-out k, joined in the order of its parts: a thread takes
// four columns of a row.  Rows of the parts are padded to `ld`, whole fours.
template <class T>
__global__ __launch_bounds__(256) void k_f8_join(F8MatmulArgs a, uint32_t splits, uint64_t ld, bool vec)
{
    const uint64_t i = (uint64_t)blockIdx.x * 256u + threadIdx.x, row = i / (ld / 4), col = i % (ld / 4) * 4u;
    if (row >= a.m) return;
    const float *p = a.part + row * ld + col;
    f32x4 v = *reinterpret_cast<const f32x4 *>(p);
    for (uint32_t j = 1; j < splits; j++) v += *reinterpret_cast<const f32x4 *>(p + (uint64_t)j * a.m * ld);
    store4(static_cast<T *>(a.out), a.ld, row, col, a.n, v, vec);
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

inline uint64_t tiles_of(uint64_t m, uint64_t n) { return ((m + 127) / 128) * ((n + 127) / 128); }

// Blocks of k that a workgroup takes: all, or, where tiles are too few for 256
// compute units, parts of sixteen blocks (2048 values) or more.
constexpr uint32_t LEAST_BLOCKS = 16;
inline uint32_t blocks_each(uint64_t m, uint64_t n, uint64_t k)
{
    const uint64_t blocks = f8_blocks(k), tiles = tiles_of(m, n), want = tiles < 256 ? 256 / tiles : 1;
    uint64_t per = (blocks + want - 1) / want;
    if (per < LEAST_BLOCKS) per = LEAST_BLOCKS;
    return (uint32_t)(per < blocks ? per : blocks + (blocks == 0));
}
inline uint64_t padded(uint64_t n) { return (n + 3) / 4 * 4; }

}  // namespace

size_t f8_matmul_workspace(uint64_t m, uint64_t n, uint64_t k)
{
    const uint64_t blocks = f8_blocks(k), per = blocks_each(m, n, k);
    if (per >= blocks) return 0;
    return (size_t)((blocks + per - 1) / per * m * padded(n) * sizeof(float));
}

bool f8_matmul_fits(uint64_t m, uint64_t n, uint64_t) { return tiles_of(m, n) <= most_blocks(256); }
bool f8_experts_fit(uint64_t rows, uint32_t experts, uint64_t n) { return groups_blocks(experts, rows, 128) * ((n + 127) / 128) <= most_blocks(256); }
bool f8_gradients_fit(uint32_t experts, uint64_t m, uint64_t n) { return tiles_of(m, n) <= most_blocks(256) / experts; }

hipError_t launch_f8_matmul(const F8MatmulArgs &a, uint32_t dtype, hipStream_t s)
{
    return by_type(dtype, [&](auto t) -> hipError_t {
        typedef decltype(t) T;
        constexpr bool EXACT = sizeof(T) == 4;
        const uint32_t mt = (uint32_t)((a.m + 127) / 128), blocks = (uint32_t)f8_blocks(a.k), per = blocks_each(a.m, a.n, a.k);
        if (tiles_of(a.m, a.n) >= 512) return product<T, EXACT, DENSE, 256, 256, 2, 2, 2>(a, (mt + 1) / 2, 1, blocks + 1, s);
        if (per >= blocks) return product<T, EXACT, DENSE, 128, 128, 2, 2, 4>(a, mt, 1, per, s);
        F8MatmulArgs part = a;
        part.out = a.part;
        part.ld = padded(a.n);
        const uint32_t splits = (blocks + per - 1) / per;
        const hipError_t e = product<float, EXACT, DENSE, 128, 128, 2, 2, 4>(part, mt, splits, per, s);
        if (e != hipSuccess) return e;
        const uint64_t threads = a.m * (part.ld / 4);
        const bool vec = (reinterpret_cast<uintptr_t>(a.out) | (a.ld * sizeof(T))) % (4 * sizeof(T)) == 0;
        k_f8_join<T><<<dim3((uint32_t)((threads + 255) / 256)), 256, 0, s>>>(a, splits, part.ld, vec);
        return hipGetLastError();
    });
}

hipError_t launch_f8_expert_matmul(const F8MatmulArgs &a, uint32_t dtype, hipStream_t s)
{
    return by_type(dtype, [&](auto t) -> hipError_t {
        typedef decltype(t) T;
        if (a.rows / a.experts >= 256) return product<T, sizeof(T) == 4, EXPERTS, 256, 256, 2, 2, 2>(a, (uint32_t)groups_blocks(a.experts, a.rows, 256), 1, 0, s);
        return product<T, sizeof(T) == 4, EXPERTS, 128, 128, 2, 2, 4>(a, (uint32_t)groups_blocks(a.experts, a.rows, 128), 1, 0, s);
    });
}

hipError_t launch_f8_expert_gradient(const F8MatmulArgs &a, uint32_t dtype, hipStream_t s)
{
    return by_type(dtype, [&](auto t) -> hipError_t {
        typedef decltype(t) T;
        return product<T, sizeof(T) == 4, GRADIENT, 128, 128, 2, 2, 4>(a, (uint32_t)((a.m + 127) / 128), a.experts, 0, s);
    });
}

}  // namespace pccl
