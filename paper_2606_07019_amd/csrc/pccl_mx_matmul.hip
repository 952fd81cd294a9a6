// The product of two microscaled operands, out[m][n] = sum over k of
// A[m][k] B[n][k], on the matrix units' 4-bit form: one instruction takes
// 16 rows of each operand over 128 values of k with a scale byte for every
// row and block of 32, and sums in 32 bits.  Lane l of a wave gives row
// l % 16 of an operand, block l / 16 of the step (16 bytes of codes), and gets
// four sums: rows 4 (l / 16) ... + 3 of the first operand, row l % 16 of the
// second.  B goes first, so a lane's sums are neighbours in out.
//
// The form with 32 rows of each operand over 64 values of k is the faster one
// (6.6 PFLOP/s from registers with random values, 4.6 for 16 rows) and serves
// many rows: lane l gives row l % 32, one block, and gets sixteen sums, four
// neighbours in rows 8 q + 4 (l / 32) of the first operand.
#include "pccl_ops.h"

namespace pccl {
namespace {

__device__ inline f32x4 mfma_mx(u32x4 a, uint32_t as, u32x4 b, uint32_t bs, f32x4 c)
{
    const i32x8 x = {(int)a.x, (int)a.y, (int)a.z, (int)a.w, 0, 0, 0, 0};
    const i32x8 y = {(int)b.x, (int)b.y, (int)b.z, (int)b.w, 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, c, 4, 4, 0, (int)as, 0, (int)bs);
}

typedef float f32x16 __attribute__((ext_vector_type(16)));

// SEL: which byte of the words holds the scale.
template <int SEL>
__device__ inline f32x16 mfma_mx32(u32x4 a, uint32_t as, u32x4 b, uint32_t bs, f32x16 c)
{
    const i32x8 x = {(int)a.x, (int)a.y, (int)a.z, (int)a.w, 0, 0, 0, 0};
    const i32x8 y = {(int)b.x, (int)b.y, (int)b.z, (int)b.w, 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, y, c, 4, 4, SEL, (int)as, SEL, (int)bs);
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
        if constexpr (sizeof(T) == 4) {
            u32x4 w;
            __builtin_memcpy(&w, t, 16);
            *reinterpret_cast<u32x4 *>(p) = w;
        } else {
            u32x2 w;
            __builtin_memcpy(&w, t, 8);
            *reinterpret_cast<u32x2 *>(p) = w;
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; i++)
        if (col + i < n) p[i] = t[i];
}

// ---- few rows ----------------------------------------------------------------

// Four neighbouring sums of row `row`, in the output's type.
__device__ inline void store4_as(const MxMatmulArgs &a, uint32_t dtype, uint64_t row, uint64_t col, f32x4 v, bool vec)
{
    if (dtype == DT_F32) store4(static_cast<float *>(a.out), a.ld, row, col, a.n, v, vec);
    else if (dtype == DT_BF16) store4(static_cast<__bf16 *>(a.out), a.ld, row, col, a.n, v, vec);
    else store4(static_cast<_Float16 *>(a.out), a.ld, row, col, a.n, v, vec);
}

constexpr int SKINNY_WAVES = 8;
constexpr uint32_t SKINNY_MAX_STEPS = 8;   // steps of k a wave holds A's operands of

// Up to 16 MT rows of A: bound by reading B once.  The eight waves of a
// workgroup share out k, S steps each, and hold A's operands of their steps in
// registers; the workgroup goes through tiles of 16 rows of B.  A wave reads
// its part of a tile along the rows (neighbouring lanes in one 64-byte piece;
// read in the operands' order every lane's 16 bytes cost a cycle of the compute
// unit's port, and 48 x 16384 x 5120 took 38 us), AHEAD tiles ahead, turns it
// round through LDS, and the waves' sums are joined there in their order.  48 x
// 16384 x 5120 takes 15 us with B from memory (3.0 TB/s), 14 from the device's
// cache; 1 x 4096 x 4096 5.0 and 4.6.
template <int MT, int S, int AHEAD>
__global__ __launch_bounds__(64 * SKINNY_WAVES) void k_mx_skinny(MxMatmulArgs a, uint32_t dtype, bool vec, uint32_t tiles)
{
    constexpr int WORDS = (S + 3) / 4;   // a lane reads the scales of a row for every fourth step
    __shared__ __align__(16) uint8_t turned[SKINNY_WAVES][S * 1024 + WORDS * 256];
    __shared__ f32x4 sums[SKINNY_WAVES][MT][64];
    const uint32_t lane = threadIdx.x & 63u, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const uint32_t r = lane & 15u, g = lane >> 4;
    const uint32_t steps = (uint32_t)mx_steps(a.k), s0 = wave * S;
    const uint32_t mine = s0 < steps ? (steps - s0 < S ? steps - s0 : S) : 0u;   // of them there are
    const uint64_t cb = mx_code_bytes(a.k), sb = mx_scale_bytes(a.k);

    auto step = [&](uint32_t j) { return s0 + j < steps ? s0 + j : steps - 1; };
    struct Tile {
        u32x4 v[S];
        uint32_t s[WORDS];
    } w[AHEAD];
    // 16 rows from `first` on along their rows (past the last: that one again)
    auto read = [&](Tile &to, const uint8_t *codes, const uint8_t *scales, uint64_t first, uint64_t rows) {
        const uint64_t row = first + lane / 4 < rows ? first + lane / 4 : rows - 1, srow = first + r < rows ? first + r : rows - 1;
        const uint8_t *p = codes + row * cb + lane % 4 * 16u, *q = scales + srow * sb;
#pragma unroll
        for (int j = 0; j < S; j++) to.v[j] = *reinterpret_cast<const u32x4 *>(p + (uint64_t)step(j) * 64u);
#pragma unroll
        for (int j = 0; j < WORDS; j++) to.s[j] = *reinterpret_cast<const uint32_t *>(q + (uint64_t)step(j * 4 + g) * 4u);
    };
    // past the last tile: that one again, so that no branch is about a read
    auto read_b = [&](Tile &to, uint32_t tile) { read(to, a.b, a.bs, (uint64_t)(tile < tiles ? tile : tiles - 1) * 16u, a.n); };
    uint8_t *lds = turned[wave];
    auto turn = [&](const Tile &from) {
#pragma unroll
        for (int j = 0; j < S; j++)
            *reinterpret_cast<u32x4 *>(lds + j * 1024u + lane / 4 * 64u + ((lane % 4) ^ (lane / 16)) * 16u) = from.v[j];
#pragma unroll
        for (int j = 0; j < WORDS; j++) *reinterpret_cast<uint32_t *>(lds + S * 1024u + j * 256u + (g * 16u + r) * 4u) = from.s[j];
    };
    auto codes_of = [&](int j) { return *reinterpret_cast<const u32x4 *>(lds + j * 1024u + r * 64u + ((g ^ (r / 4)) * 16u)); };
    auto scale_of = [&](int j) { return (uint32_t)lds[S * 1024u + j / 4 * 256u + (j % 4 * 16u + r) * 4u + g]; };
    u32x4 x[MT][S];
    uint32_t xs[MT][S];
    if (steps) {
        Tile first[MT];
#pragma unroll
        for (int t = 0; t < MT; t++) read(first[t], a.a, a.as, (uint64_t)t * 16u, a.m);
#pragma unroll
        for (int d = 0; d < AHEAD; d++) read_b(w[d], blockIdx.x + d * gridDim.x);
#pragma unroll
        for (int t = 0; t < MT; t++) {
            turn(first[t]);
#pragma unroll
            for (int j = 0; j < S; j++) {
                x[t][j] = codes_of(j);
                xs[t][j] = scale_of(j);
            }
        }
    }
    auto tile_of = [&](Tile &b, uint32_t tile) {
        f32x4 acc[MT] = {};
        if (steps) {
            turn(b);
            read_b(b, tile + AHEAD * gridDim.x);
#pragma unroll
            for (int j = 0; j < S; j++) {
                if ((uint32_t)j >= mine) break;
                const u32x4 y = codes_of(j);
                const uint32_t ys = scale_of(j);
#pragma unroll
                for (int t = 0; t < MT; t++) acc[t] = mfma_mx(y, ys, x[t][j], xs[t][j], acc[t]);
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();   // the sums before have been read; reads under way stay so
        asm volatile("" ::: "memory");
#pragma unroll
        for (int t = 0; t < MT; t++) sums[wave][t][lane] = acc[t];
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (wave < MT) {
            f32x4 v = sums[0][wave][lane];
#pragma unroll
            for (int q = 1; q < SKINNY_WAVES; q++) v += sums[q][wave][lane];
            const uint64_t m = (uint64_t)wave * 16u + r;
            if (m < a.m) store4_as(a, dtype, m, (uint64_t)tile * 16u + g * 4u, v, vec);
        }
    };
    for (uint32_t tile = blockIdx.x; tile < tiles;) {
#pragma unroll
        for (int d = 0; d < AHEAD; d++) {
            if (d && tile >= tiles) break;
            tile_of(w[d], tile);
            tile += gridDim.x;
        }
    }
}

// ---- many rows ---------------------------------------------------------------

typedef const __attribute__((address_space(1))) void *gptr;
typedef __attribute__((address_space(3))) void *lptr;

template <int I>
struct Index {
    static constexpr int value = I;
};

// A tile of BM x BN sums, 2 x WN waves of (BM / 2) x (BN / WN).  A stage is 256
// values of k (128 bytes of codes a row), copied from memory straight to LDS,
// BUFFERS stages in a ring.  A compute unit's port takes one 64-byte piece a
// cycle, and a row's scales are a piece of their own: they are copied for four
// stages at a time (32 bytes a row), a quarter of the rows with every stage
// (a word a row and stage cost more than the codes did: 8192^3 in 345 us).
// A stage has four
// instruction steps; lanes of half h of a wave take its blocks 4 h ... + 3 in
// turn, so that their scales are one word.  While a step is multiplied from
// registers the next one is read from LDS, and a stage's last step is
// multiplied after the next one's first is on its way.  In LDS chunk c (16
// bytes) of row r stands at chunk c ^ (r / 2 % 8) of the row, so the 16 lanes
// that read one chunk of 16 rows meet every bank once.  8192^3 takes 306 us by
// itself (3.6 PFLOP/s): the matrix units are busy 45 % of its cycles, LDS reads 23
// %, and waves wait 30 % of their time, since every stage's barrier brings the two
// waves of a SIMD to the same point.
// Two chunks of scales go with two stages of codes (LDS holds no more), three
// with up to four.
constexpr int scale_chunks(int buffers) { return buffers == 2 ? 2 : 3; }

template <class T, int BM, int BN, int WN, int BUFFERS>
__global__ __launch_bounds__(128 * WN) void k_mx_tile(MxMatmulArgs a, uint32_t mt, uint32_t nt, uint32_t per)
{
    constexpr uint32_t THREADS = 128 * WN, PASS = THREADS / 8;   // rows of codes that the workgroup copies at a time
    constexpr int TM = BM / 64, TN = BN / WN / 32, PA = BM / PASS, PB = BN / PASS, WORDS = 2 * (BM + BN) / THREADS, COPIES = PA + PB + WORDS;
    constexpr uint32_t STAGE = (BM + BN) * 128, CHUNK = (BM + BN) * 32, CODES = BUFFERS * STAGE;   // codes of a stage, scales of four; all codes
    constexpr uint32_t CHUNKS = scale_chunks(BUFFERS);
    static_assert(BM == BN && BM % PASS == 0 && 2 * (BM + BN) % THREADS == 0, "whole passes, and quarters of one operand's rows");
    extern __shared__ __align__(16) uint8_t lds[];
    const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(tid >> 6));
    const uint32_t r = lane & 31u, half = lane >> 5;
    // tiles are dealt so that the workgroups of one XCD (every eighth of the
    // launch) have neighbouring tiles, eight rows of tiles by column
    const uint32_t total = mt * nt, id = blockIdx.x;
    const uint32_t q = total / 8, left = total % 8, xcd = id % 8;
    const uint32_t tile = xcd * q + (xcd < left ? xcd : left) + id / 8;
    constexpr uint32_t GROUP = 8;
    const uint32_t grp = tile / (GROUP * nt), first = grp * GROUP;
    const uint32_t gm = mt - first < GROUP ? mt - first : GROUP;
    const uint32_t in = tile - grp * GROUP * nt;
    const uint64_t m0 = (uint64_t)(first + in % gm) * BM, n0 = (uint64_t)(in / gm) * BN;

    const uint32_t cb = (uint32_t)mx_code_bytes(a.k), sb = (uint32_t)mx_scale_bytes(a.k), steps = (uint32_t)mx_steps(a.k);
    // this workgroup's stages: `stages` of them from s0 on, a multiple of four
    const uint32_t s0 = blockIdx.y * per, all = (steps + 1) / 2, stages = all - s0 < per ? all - s0 : per;
    // what this thread copies of a stage: a chunk of every PASS-th row of A,
    // then of B, and words of scales; rows past the last are that one again
    const uint8_t *ca = a.a + m0 * cb, *cn = a.b + n0 * cb, *sa = a.as + m0 * sb, *sn = a.bs + n0 * sb;
    const uint32_t lm = (uint32_t)(a.m - m0 < BM ? a.m - m0 : BM) - 1u, ln = (uint32_t)(a.n - n0 < BN ? a.n - n0 : BN) - 1u;
    const uint32_t chunk = ((tid % 8) ^ (tid / 16 % 8)) * 16u;
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
    // a quarter of the scales of stages 4 c ... + 3; word w of a row stands at w ^ (row / 8 % 8)
    auto copy_scales = [&](uint32_t c, uint32_t quarter) {
        const uint8_t *from = quarter < 2 ? sa : sn;
        const uint32_t lim = quarter < 2 ? lm : ln;
#pragma unroll
        for (int i = 0; i < WORDS; i++) {
            const uint32_t row = quarter % 2 * (BM / 2) + (i * THREADS + tid) / 8, at = (s0 / 4 + c) * 32u + ((tid % 8) ^ (row / 8 % 8)) * 4u;
            const uint32_t off = (row < lim ? row : lim) * sb + (at < sb ? at : sb - 4u);
            __builtin_amdgcn_global_load_lds((gptr)(from + off), (lptr)(lds + CODES + c % CHUNKS * CHUNK + (quarter * (WORDS * THREADS) + i * THREADS + wave * 64u) * 4u), 4, 0, 0);
        }
    };
    auto copy = [&](uint32_t stage) {   // past the last stage: that one again, into a buffer nobody reads
        uint8_t *to = lds + stage % BUFFERS * STAGE;
        const uint32_t k = s0 + (stage < stages ? stage : stages - 1);
        // a row may end after a stage's first half: that is copied twice, the second with scales of nothing
        const uint32_t over = k * 128u + chunk >= cb ? 64u : 0u;
#pragma unroll
        for (int i = 0; i < PA; i++)
            __builtin_amdgcn_global_load_lds((gptr)(ca + (offa[i] + k * 128u - over)), (lptr)(to + (i * THREADS + wave * 64u) * 16u), 16, 0, 0);
#pragma unroll
        for (int i = 0; i < PB; i++)
            __builtin_amdgcn_global_load_lds((gptr)(cn + (offb[i] + k * 128u - over)), (lptr)(to + BM * 128u + (i * THREADS + wave * 64u) * 16u), 16, 0, 0);
        // the next chunk of scales, into the place of one that nobody reads any
        // more: with two places that is so from the stage on that is multiplied now
        if (CHUNKS == 3) copy_scales(stage / 4 + 1, stage % 4);
        else if (stage) copy_scales((stage - 1) / 4 + 1, (stage - 1) % 4);
    };

    const uint32_t wm = wave / WN * (BM / 2), wn = wave % WN * (BN / WN);
    struct Held {
        u32x4 x[TM], y[TN];
    } held[2];
    struct Scales {
        uint32_t x[TM], y[TN];   // of this stage; of the one before, whose last step is still to be multiplied
    } now, before;
    const uint32_t key = r / 2 % 8;
    auto read = [&](Held &h, uint32_t stage, uint32_t step) {
        const uint8_t *from = lds + stage % BUFFERS * STAGE + r * 128u + (((half * 4u + step) ^ key) * 16u);
#pragma unroll
        for (int i = 0; i < TN; i++) h.y[i] = *reinterpret_cast<const u32x4 *>(from + (BM + wn + i * 32u) * 128u);
#pragma unroll
        for (int i = 0; i < TM; i++) h.x[i] = *reinterpret_cast<const u32x4 *>(from + (wm + i * 32u) * 128u);
    };
    auto read_scales = [&](Scales &to, uint32_t stage) {
        const uint8_t *from = lds + CODES + stage / 4 % CHUNKS * CHUNK;
        const bool none = half && (s0 + stage) * 2 + 1 >= steps;   // both scales 2^-127: products vanish
        auto word = [&](uint32_t row) {
            return none ? 0u : *reinterpret_cast<const uint32_t *>(from + row * 32u + (((stage % 4 * 2u + half) ^ (row / 8 % 8)) * 4u));
        };
#pragma unroll
        for (int i = 0; i < TN; i++) to.y[i] = word(BM + wn + i * 32u + r);
#pragma unroll
        for (int i = 0; i < TM; i++) to.x[i] = word(wm + i * 32u + r);
    };
    T *out = static_cast<T *>(a.out) + (uint64_t)blockIdx.y * a.m * a.ld;
    f32x16 acc[TM][TN] = {};
    auto products = [&](auto sel, const Held &h, const Scales &s) {
        constexpr int SEL = decltype(sel)::value;
#pragma unroll
        for (int i = 0; i < TM; i++)
#pragma unroll
            for (int j = 0; j < TN; j++) acc[i][j] = mfma_mx32<SEL>(h.y[j], s.y[j], h.x[i], s.x[i], acc[i][j]);
    };
    // LDS reads and products take turns
    auto mix = [&]() {
#pragma unroll
        for (int i = 0; i < TM + TN; i++) {
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        }
    };
    // the stage has landed for everyone, and nobody reads the buffer that the next copy goes to
    auto ready = [&]() {
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((BUFFERS - 2) * COPIES) : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    if (stages) {
#pragma unroll
        for (uint32_t i = 0; i < 4; i++) copy_scales(0, i);
#pragma unroll
        for (uint32_t i = 0; i < BUFFERS - 1; i++) copy(i);
        held[1] = Held{};   // nothing is left over before the first stage
        before = Scales{};
        for (uint32_t s = 0; s < stages; s++) {
            ready();
            copy(s + BUFFERS - 1);
            read_scales(now, s);
            read(held[0], s, 0);
            products(Index<3>{}, held[1], before);
            read(held[1], s, 1);
            products(Index<0>{}, held[0], now);
            mix();
            read(held[0], s, 2);
            products(Index<1>{}, held[1], now);
            mix();
            read(held[1], s, 3);
            products(Index<2>{}, held[0], now);
            mix();
            before = now;
        }
        products(Index<3>{}, held[1], before);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // no copy outlives the workgroup's LDS
    }
    // The sums go through LDS, 32 rows of the wave's at a time, so that whole
    // rows of them are stored: as they lie in registers a store has 16 bytes in
    // each of 32 rows, and 8192^3 wrote 1.8 times its result to memory (337 us; 326 so).
    constexpr uint32_t COLS = BN / WN, EACH = 16 / sizeof(T), CHUNKS_ROW = COLS / EACH, ROW = COLS * sizeof(T) + 16;
    static_assert(2 * WN * 32 * ROW <= CODES, "within the stages' room");
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
            const uint64_t m = m0 + wm + i * 32u + row, n = n0 + wn + col;
            if (m >= a.m) continue;
            T t[EACH];
            __builtin_memcpy(t, __builtin_assume_aligned(own + row * ROW + col * sizeof(T), 16), 16);
            if (n + EACH <= a.n) {
                __builtin_memcpy(out + m * a.ld + n, t, 16);   // at any address
                continue;
            }
#pragma unroll
            for (uint32_t c = 0; c < EACH; c++)
                if (n + c < a.n) out[m * a.ld + n + c] = t[c];
        }
    }
}

// The sums of a shared-out k, joined in the order of its parts: a thread takes
// four columns of a row.  Rows of the parts are padded to `ld`, whole fours.
template <class T>
__global__ __launch_bounds__(256) void k_mx_join(const float *parts, uint32_t splits, uint64_t m, uint64_t n, uint64_t ld, T *out, uint64_t ld_out, bool vec)
{
    const uint64_t i = (uint64_t)blockIdx.x * 256u + threadIdx.x, row = i / (ld / 4), col = i % (ld / 4) * 4u;
    if (row >= m) return;
    const float *p = parts + row * ld + col;
    f32x4 v = *reinterpret_cast<const f32x4 *>(p);
    for (uint32_t j = 1; j < splits; j++) v += *reinterpret_cast<const f32x4 *>(p + (uint64_t)j * m * ld);
    store4(out, ld_out, row, col, n, v, vec);
}

template <int MT, int S>
hipError_t skinny_as(const MxMatmulArgs &a, uint32_t dtype, bool vec, hipStream_t s)
{
    const uint32_t tiles = (uint32_t)((a.n + 15) / 16);
    // Two workgroups a compute unit where a wave holds one or two steps, one
    // beyond (B from memory, with 256 and with 512 workgroups: 1 x 65536 x 1024
    // 19.9 and 13.0 us, 64 x 65536 x 2048 27.4 and 22.7, 64 x 16384 x 2048 9.5 and
    // 10.5, 1 x 16384 x 5120 12.3 and 13.9, 64 x 16384 x 4096 13.1 and 16.5; three
    // and four steps of one row over the longest n alone gain with 512, 33.0 and 30.0)
    constexpr uint32_t most = S <= 2 ? 512u : 256u;
    constexpr int ahead = MT * S <= 16 ? 2 : 1;
    k_mx_skinny<MT, S, ahead><<<dim3(tiles < most ? tiles : most), 64 * SKINNY_WAVES, 0, s>>>(a, dtype, vec, tiles);
    return hipGetLastError();
}

template <int MT>
hipError_t skinny_rows(const MxMatmulArgs &a, uint32_t dtype, bool vec, hipStream_t s)
{
    const uint32_t each = ((uint32_t)mx_steps(a.k) + SKINNY_WAVES - 1) / SKINNY_WAVES;
    if (each <= 1) return skinny_as<MT, 1>(a, dtype, vec, s);
    if (each <= 2) return skinny_as<MT, 2>(a, dtype, vec, s);
    if (each <= 3) return skinny_as<MT, 3>(a, dtype, vec, s);
    if (each <= 4) return skinny_as<MT, 4>(a, dtype, vec, s);
    if (each <= 5) return skinny_as<MT, 5>(a, dtype, vec, s);
    if (each <= 6) return skinny_as<MT, 6>(a, dtype, vec, s);
    return skinny_as<MT, 8>(a, dtype, vec, s);
}

template <class T, int BM, int BN, int WN, int BUFFERS>
hipError_t tiled(const MxMatmulArgs &a, uint32_t per, hipStream_t s)
{
    constexpr uint32_t threads = 128 * WN, bytes = (BUFFERS * 128 + scale_chunks(BUFFERS) * 32) * (BM + BN);
    static_assert(bytes <= 160u << 10, "one workgroup's LDS");
    const hipError_t e = allow_lds<&k_mx_tile<T, BM, BN, WN, BUFFERS>>(bytes);
    if (e != hipSuccess) return e;
    const uint32_t mt = (uint32_t)((a.m + BM - 1) / BM), nt = (uint32_t)((a.n + BN - 1) / BN);
    const uint32_t stages = (uint32_t)(mx_steps(a.k) + 1) / 2, parts = stages ? (stages + per - 1) / per : 1;
    k_mx_tile<T, BM, BN, WN, BUFFERS><<<dim3(mt * nt, parts), threads, bytes, s>>>(a, mt, nt, per);
    return hipGetLastError();
}

// Few rows, and k short enough for eight waves to hold their operands.  Against
// the form for many rows, B from memory: 1 x 4096 x 4096 5.0 and 11.3 us, 64 x
// 4096 x 4096 7.1 and 13.4, 64 x 1024 x 8192 9.3 and 12.7, 64 x 65536 x 2048 23.5
// and 25.8; nothing is left at 64 rows with the shortest k (64 x 16384 x 1024 8.1
// and 7.6).
inline bool few_rows(uint64_t m, uint64_t k) { return m <= 64 && mx_steps(k) <= SKINNY_WAVES * SKINNY_MAX_STEPS; }

// Stages of k that a workgroup of 128 x 128 sums takes: all, or, where such
// tiles are too few for 256 compute units, parts of eight stages (2048 values)
// or more, whole chunks of scales each.  16 x 4096 x 28672 takes 83 us whole and
// 22 us in eight parts, 256 x 1024 x 8192 28 and 15; with parts of 16 stages the
// latter takes 19, and 1000 x 1000 x 4096, where two parts gain least, 16 either way.
constexpr uint32_t LEAST_STAGES = 8;
inline uint64_t small_tiles(uint64_t m, uint64_t n) { return ((m + 127) / 128) * ((n + 127) / 128); }
inline uint32_t stages_each(uint64_t m, uint64_t n, uint64_t k)
{
    const uint64_t stages = (mx_steps(k) + 1) / 2, tiles = small_tiles(m, n), want = tiles < 256 ? 256 / tiles : 1;
    uint64_t per = (stages + want - 1) / want;
    if (per < LEAST_STAGES) per = LEAST_STAGES;
    per = (per + 3) / 4 * 4;
    return (uint32_t)(per < stages ? per : stages + (stages == 0));
}
inline uint64_t padded(uint64_t n) { return (n + 3) / 4 * 4; }
inline uint64_t big_tiles(uint64_t m, uint64_t n) { return ((m + 255) / 256) * ((n + 255) / 256); }

// 256 x 256 sums a workgroup, four products for two operands read from LDS, where
// such tiles occupy half of the compute units and smaller ones would not be done
// in one round (256 and 128 either way, k of 8192: 64 tiles of 256, 2048 x 2048,
// 58 and 32 us; 81, 2300 x 2300, 61 and 56; 128, 2048 x 4096, 60 and 61; 144, 3000 x
// 3000, 61 and 87; 1024, 8192 x 8192, 303 and 458; but 128 x 32768, 256 of the
// smaller ones, 62 and 42).  128 x 128 otherwise, eight waves all the same: two to a
// SIMD (2040 x 1500 x 8192 29.1 us, with four waves 30.7).
template <class T>
hipError_t tiles_of(const MxMatmulArgs &a, bool vec, hipStream_t s)
{
    const uint32_t stages = (uint32_t)(mx_steps(a.k) + 1) / 2;
    if (big_tiles(a.m, a.n) >= 128 && small_tiles(a.m, a.n) > 256) return tiled<T, 256, 256, 4, 2>(a, stages + 1, s);
    const uint32_t per = stages_each(a.m, a.n, a.k);
    if (per >= stages) return tiled<T, 128, 128, 4, 4>(a, per, s);
    MxMatmulArgs part = a;
    part.out = a.part;
    part.ld = padded(a.n);
    const hipError_t e = tiled<float, 128, 128, 4, 4>(part, per, s);
    if (e != hipSuccess) return e;
    const uint64_t threads = a.m * (part.ld / 4);
    k_mx_join<T><<<dim3((uint32_t)((threads + 255) / 256)), 256, 0, s>>>(a.part, (stages + per - 1) / per, a.m, a.n, part.ld, static_cast<T *>(a.out), a.ld, vec);
    return hipGetLastError();
}

}  // namespace

size_t mx_matmul_workspace(uint64_t m, uint64_t n, uint64_t k)
{
    const uint64_t stages = (mx_steps(k) + 1) / 2, per = stages_each(m, n, k);
    if (few_rows(m, k) || per >= stages) return 0;
    return (size_t)((stages + per - 1) / per * m * padded(n) * sizeof(float));
}

// Few rows take 512 workgroups at most, smaller tiles a few hundred.
bool mx_matmul_fits(uint64_t m, uint64_t n, uint64_t k) { return few_rows(m, k) || big_tiles(m, n) <= most_blocks(512); }

hipError_t launch_mx_matmul(const MxMatmulArgs &a, uint32_t dtype, hipStream_t s)
{
    const size_t elem = dtype == DT_F32 ? 4 : 2;
    const bool vec = (reinterpret_cast<uintptr_t>(a.out) | (a.ld * elem)) % (4 * elem) == 0;
    if (few_rows(a.m, a.k)) {
        if (a.m <= 16) return skinny_rows<1>(a, dtype, vec, s);
        if (a.m <= 32) return skinny_rows<2>(a, dtype, vec, s);
        if (a.m <= 48) return skinny_rows<3>(a, dtype, vec, s);
        return skinny_rows<4>(a, dtype, vec, s);
    }
    if (dtype == DT_F32) return tiles_of<float>(a, vec, s);
    if (dtype == DT_BF16) return tiles_of<__bf16>(a, vec, s);
    return tiles_of<_Float16>(a, vec, s);
}

}  // namespace pccl
