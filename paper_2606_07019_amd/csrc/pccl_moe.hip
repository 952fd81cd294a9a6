// A mixture-of-experts layer for a few tokens:
//
//   l = x Wr^T;  w, ids = top k of softmax(l)
//   y_t = sum_j w_tj Wd[e] (silu(Wg[e] x_t) * (Wu[e] x_t)),  e = ids_tj
//
// With few tokens the experts' weights are read once and used for a handful of
// columns, so the layer is bound by that reading; the matrix units are used
// because they take 16 tokens at the price of one.  Weight rows are the first
// operand of the 16x16x32 products (lane l: row l % 16, eight values of k per
// product), the expert's tokens the second.  Neighbouring lanes thus need
// neighbouring rows, while memory wants them along a row (a compute unit's
// port takes one 64-byte piece a cycle: read in the operands' order, 1 KiB
// took 64 cycles and that bounded the kernels).  So a wave reads weights along
// their rows into registers and turns a block round through 4 KiB of LDS of its
// own when it multiplies it.  It is the other waves of a SIMD that read in the
// meantime: a wave that read one to four blocks ahead of its products held
// registers that cost more waves than that gave (16 tokens and 128 experts in
// 4 bits: the two products 177 us with none ahead, 201 with one).
#include "pccl_topk.h"

namespace pccl {
namespace {

constexpr uint32_t STEP = 128;      // rows of inner values are padded to whole steps of 128
constexpr int WAVES = 4;            // waves of a workgroup that share out k
constexpr int PICK_WAVES = 16;
constexpr uint32_t NO_PLACE = 0xFFFFFFFFu;
constexpr uint32_t PARTS = 3;       // bf16 parts of an inner value
constexpr uint32_t MAX_SPLITS = 8;  // parts of the router's product over hidden, summed up by the picking lanes

// What the kernels of one call hand on, carved from the workspace.
struct MoeSpace {
    float *part_logits;   // [splits][tokens][experts padded to 16]
    uint32_t *active;     // [0]: experts in use; then the experts
    uint32_t *first;      // [experts in use + 1]: where each one's places start
    uint32_t *slots;      // [places]: token of each place, in expert order
    float *shares;        // [places]: its weight
    uint32_t *place;      // [tokens][topk]: the slot's place, NO_PLACE for an empty pick
    uint16_t *parts;      // the inner values, in three parts: [tiles of 16 places][products][PARTS][lane][8],
                          // as the products' second operands have them
    float *outs;          // [places][hidden]: the experts' outputs, weighted
    uint64_t inner;       // padded inner size
    uint32_t splits, row; // parts of the logits, and the length of their rows
};

// Workgroups that share the router's product over hidden, so that about 128
// take part.
__host__ inline uint32_t logit_splits(uint32_t tokens, uint32_t experts, uint32_t hidden)
{
    const uint32_t tiles = (experts + 15) / 16 * ((tokens + 15) / 16), most = (hidden + STEP - 1) / STEP;
    uint32_t want = (128 + tiles - 1) / tiles;
    if (want > MAX_SPLITS) want = MAX_SPLITS;
    return want < most ? want : most;
}

__host__ inline size_t carve(MoeSpace &m, char *base, uint32_t tokens, uint32_t experts, uint32_t topk, uint32_t hidden, uint32_t inter)
{
    size_t off = 0;
    auto take = [&](size_t bytes) {
        char *p = base ? base + off : nullptr;
        off += (bytes + 255) & ~size_t(255);
        return p;
    };
    const uint64_t places = (uint64_t)tokens * topk;
    m.splits = logit_splits(tokens, experts, hidden);
    m.inner = (inter + STEP - 1) / STEP * (uint64_t)STEP;
    m.row = (experts + 15) / 16 * 16;
    m.part_logits = (float *)take((size_t)m.splits * tokens * m.row * 4);
    m.active = (uint32_t *)take((experts + 1ull) * 4);
    m.first = (uint32_t *)take((experts + 1ull) * 4);
    m.slots = (uint32_t *)take(places * 4);
    m.shares = (float *)take(places * 4);
    m.place = (uint32_t *)take(places * 4);
    const uint64_t tiles = places / 16 + (places < experts ? places : experts) + 1;
    m.parts = (uint16_t *)take(tiles * 16 * m.inner * PARTS * 2);
    m.outs = (float *)take(places * hidden * 4);
    return off;
}

// ---- the products' operands ---------------------------------------------------

template <class C>
struct Frag;
template <>
struct Frag<__bf16> {
    typedef bf16x8 V;
    static __device__ f32x4 mul(u32x4 a, u32x4 b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(V, a), __builtin_bit_cast(V, b), c, 0, 0, 0);
    }
};
template <>
struct Frag<_Float16> {
    typedef f16x8 V;
    static __device__ f32x4 mul(u32x4 a, u32x4 b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(V, a), __builtin_bit_cast(V, b), c, 0, 0, 0);
    }
};

// Eight values from k on of a row that ends at `end`; zeros beyond it.  VEC: the
// row starts on 16 bytes and has whole groups of eight.  Otherwise they are read
// at any address too, and one by one at the row's end alone (16 tokens, 32
// experts of 2044 x 500: up and down 149 us with values one by one, 50 us so).
template <bool VEC>
__device__ inline u32x4 row8(const uint16_t *row, uint32_t k, uint32_t end)
{
    if (VEC) return k < end ? *reinterpret_cast<const u32x4 *>(row + k) : u32x4{0, 0, 0, 0};
    u32x4 v;
    if (k + 8 <= end) {   // 16 bytes at any address
        __builtin_memcpy(&v, row + k, 16);
        return v;
    }
    uint16_t t[8];
#pragma unroll
    for (int i = 0; i < 8; i++) t[i] = k + i < end ? row[k + i] : (uint16_t)0;
    __builtin_memcpy(&v, t, 16);
    return v;
}

// Weight rows as a wave reads them: blocks of M tiles of 16 rows by VALUES of
// k.  begin() takes a tile's rows, read() starts a block's reads (a lane takes
// chunks of 16 bytes, neighbours along a row), turn() writes them to LDS, and
// operand() gives the lane's eight values of a product there: chunk c of row r
// stands where the 16 lanes that read one chunk of 16 rows meet every bank
// once.
//
// 16-bit rows: 128 bytes and two products a block; product i takes values 32 i
// + 8 (l / 16) ... + 7.  Microscaled rows: 128 bytes, two steps of four products;
// a lane's chunk of a step is one group of 32 values with its scale, and product
// j takes its values 8 j ... + 7 (both operands count k alike, so the order is
// free).  Whole 128-byte lines either way: with half lines a compute unit's
// first-level cache had as many misses under way for half the bytes.

// A matrix of one expert: rows of `len` bytes, 32-bit offsets from `base`.
struct Rows {
    const char *base;
    const uint8_t *scales;
    uint32_t rows, len, slen;
};

template <class T, int M, bool VEC>
struct Plain {
    typedef T C;                         // the products' type
    static constexpr uint32_t PRODUCTS = 2, VALUES = 64, LDS = M * 2048;
    struct Block {
        u32x4 v[2 * M];
    };
    uint32_t off[2 * M], chunk, len;
    __device__ void begin(const Rows &w, const uint32_t (&row)[M])
    {
        const uint32_t lane = threadIdx.x & 63u;
        chunk = lane % 8 * 16u;
        len = w.len;
#pragma unroll
        for (int j = 0; j < 2 * M; j++) {
            const uint32_t r = row[j / 2] + j % 2 * 8u + lane / 8;
            off[j] = (r < w.rows ? r : w.rows - 1) * w.len;
        }
    }
    __device__ void read(Block &b, const Rows &w, uint32_t block, bool there) const
    {
        const uint32_t at = block * 128u + chunk, in = at < len ? at : 0u;   // past the row's end its start is read and not used
        if constexpr (VEC) {
#pragma unroll
            for (int j = 0; j < 2 * M; j++) b.v[j] = *reinterpret_cast<const u32x4 *>(w.base + (there ? off[j] + in : 0u));
        } else if (there) {   // rows that start or end anywhere
#pragma unroll
            for (int j = 0; j < 2 * M; j++) b.v[j] = row8<false>(reinterpret_cast<const uint16_t *>(w.base + off[j]), in / 2, len / 2);
        }
    }
    __device__ void turn(const Block &b, uint8_t *lds, uint32_t block) const
    {
        const uint32_t lane = threadIdx.x & 63u;
#pragma unroll
        for (int j = 0; j < 2 * M; j++) {
            const uint32_t r = j % 2 * 8u + lane / 8;
            u32x4 v = b.v[j];
            if (block * 128u + chunk >= len) v = u32x4{0, 0, 0, 0};
            *reinterpret_cast<u32x4 *>(lds + j / 2 * 2048u + r * 128u + ((lane % 8) ^ (r / 2)) * 16u) = v;
        }
    }
    __device__ void operands(const uint8_t *lds, int i, uint32_t r, uint32_t g, u32x4 (&v)[PRODUCTS]) const
    {
#pragma unroll
        for (uint32_t p = 0; p < PRODUCTS; p++)
            v[p] = *reinterpret_cast<const u32x4 *>(lds + i * 2048u + r * 128u + (((p * 4u + g) ^ (r / 2)) * 16u));
    }
    static __device__ uint32_t at(uint32_t block, uint32_t g, uint32_t p) { return block * VALUES + p * 32u + g * 8u; }
    // the product and lane group that take value k, for its place among the second operands
    static __device__ void place(uint32_t k, uint32_t &product, uint32_t &g)
    {
        product = k / 32;
        g = k % 32 / 8;
    }
};

template <int M>
struct Micro {
    typedef __bf16 C;                    // holds every microscaled value exactly
    static constexpr uint32_t PRODUCTS = 8, VALUES = 256, WORDS = (M + 1) / 2, LDS = M * 2048 + WORDS * 256;
    struct Block {
        u32x4 v[2 * M];
        uint32_t s[WORDS];
    };
    uint32_t off[2 * M], soff[WORDS], chunk, word, len, slen;
    __device__ void begin(const Rows &w, const uint32_t (&row)[M])
    {
        const uint32_t lane = threadIdx.x & 63u;
        chunk = lane % 8 * 16u;
        word = lane % 2 * 4u;
        len = w.len;
        slen = w.slen;
#pragma unroll
        for (int j = 0; j < 2 * M; j++) {
            const uint32_t r = row[j / 2] + j % 2 * 8u + lane / 8;
            off[j] = (r < w.rows ? r : w.rows - 1) * w.len;
        }
#pragma unroll
        for (uint32_t j = 0; j < WORDS; j++) {   // a lane's word of scales: of sub-tile 2 j or 2 j + 1
            const uint32_t first = lane < 32 || 2 * j + 1 >= M ? row[2 * j] : row[2 * j + 1 < M ? 2 * j + 1 : 2 * j];
            const uint32_t r = first + lane % 32 / 2;
            soff[j] = (r < w.rows ? r : w.rows - 1) * w.slen;
        }
    }
    __device__ void read(Block &b, const Rows &w, uint32_t block, bool there) const
    {
        // a row may end after a block's first step: its start is read instead and not used
        const uint32_t at = block * 128u + chunk, in = at < len ? at : 0u, sat = block * 8u + word, sin = sat < slen ? sat : 0u;
#pragma unroll
        for (int j = 0; j < 2 * M; j++) b.v[j] = *reinterpret_cast<const u32x4 *>(w.base + (there ? off[j] + in : 0u));
#pragma unroll
        for (uint32_t j = 0; j < WORDS; j++) b.s[j] = *reinterpret_cast<const uint32_t *>(w.scales + (there ? soff[j] + sin : 0u));
    }
    __device__ void turn(const Block &b, uint8_t *lds, uint32_t block) const
    {
        const uint32_t lane = threadIdx.x & 63u;
#pragma unroll
        for (int j = 0; j < 2 * M; j++) {
            const uint32_t r = j % 2 * 8u + lane / 8;
            u32x4 v = b.v[j];
            if (block * 128u + chunk >= len) v = u32x4{0, 0, 0, 0};
            *reinterpret_cast<u32x4 *>(lds + j / 2 * 2048u + r * 128u + ((lane % 8) ^ (r / 2)) * 16u) = v;
        }
#pragma unroll
        for (uint32_t j = 0; j < WORDS; j++) reinterpret_cast<uint32_t *>(lds + M * 2048u)[j * 64u + lane] = b.s[j];
    }
    __device__ void operands(const uint8_t *lds, int i, uint32_t r, uint32_t g, u32x4 (&v)[PRODUCTS]) const
    {
#pragma unroll
        for (uint32_t u = 0; u < 2; u++) {
            const u32x4 c = *reinterpret_cast<const u32x4 *>(lds + i * 2048u + r * 128u + (((u * 4u + g) ^ (r / 2)) * 16u));
            const float f = mx_scale(lds[M * 2048u + (i * 16u + r) * 8u + u * 4u + g]);
#pragma unroll
            for (uint32_t j = 0; j < 4; j++) {
                u32x4 &o = v[u * 4 + j];
                o.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[j], f, 0));
                o.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[j], f, 1));
                o.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[j], f, 2));
                o.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[j], f, 3));
            }
        }
    }
    static __device__ uint32_t at(uint32_t block, uint32_t g, uint32_t p) { return block * VALUES + p / 4 * 128u + g * 32u + p % 4 * 8u; }
    static __device__ void place(uint32_t k, uint32_t &product, uint32_t &g)
    {
        product = k / 128 * 4 + k % 32 / 8;
        g = k % 128 / 32;
    }
};

// A 32-bit value in three parts of bf16, eight digits each: v = hi + mid + lo,
// exactly, over the whole range (digits below 2^-133 aside).  The parts are cut
// off and not rounded, so that each has v's sign and a finite value never gives
// an infinity; of an infinity the first part holds all (the difference would
// be a NaN).  An f16 value's eleven digits end within the second part.
__device__ inline void split(float v, uint16_t &hi, uint16_t &mid, uint16_t &lo)
{
    const uint32_t h = __float_as_uint(v) & 0xFFFF0000u;
    const float rest = __builtin_isinf(v) ? 0.f : v - __uint_as_float(h);
    const uint32_t m = __float_as_uint(rest) & 0xFFFF0000u;
    hi = (uint16_t)(h >> 16);
    mid = (uint16_t)(m >> 16);
    lo = (uint16_t)(__float_as_uint(rest - __uint_as_float(m)) >> 16);
}

// Eight f16 values in two operands of bf16.
__device__ inline void split8(u32x4 v, u32x4 &hi, u32x4 &lo)
{
    uint16_t h[8], l[8], none;
    _Float16 f[8];
    __builtin_memcpy(f, &v, 16);
#pragma unroll
    for (int j = 0; j < 8; j++) split((float)f[j], h[j], l[j], none);
    __builtin_memcpy(&hi, h, 16);
    __builtin_memcpy(&lo, l, 16);
}

// A value that all lanes of a wave have alike, kept as one.
__device__ inline uint32_t uniform(uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); }

// ---- the router's product -------------------------------------------------------

// Sums of products `first`, `first` + `by`, ... of 32 values of k: 16 experts
// from e0 on (rows) by 16 tokens from t0 on.
template <class T, bool VEC>
__device__ inline f32x4 logit_tile(const MoeArgs &a, uint32_t e0, uint32_t t0, uint32_t first, uint32_t by, uint32_t r, uint32_t g)
{
    const uint32_t e = e0 + r < a.experts ? e0 + r : a.experts - 1;
    const uint32_t t = t0 + r < a.tokens ? t0 + r : a.tokens - 1;
    const uint16_t *wrow = static_cast<const uint16_t *>(a.router) + (uint64_t)e * a.hidden;
    const uint16_t *xrow = static_cast<const uint16_t *>(a.x) + (uint64_t)t * a.ld_x;
    const uint32_t products = (a.hidden + 31) / 32;
    f32x4 acc = {};
    uint32_t p = first;
    constexpr int U = VEC ? 8 : 2;   // so many at a time: their reads are under way together
    for (; p + (U - 1) * by < products; p += U * by) {
        u32x4 w[U], x[U];
#pragma unroll
        for (int u = 0; u < U; u++) {
            w[u] = row8<VEC>(wrow, (p + u * by) * 32u + g * 8u, a.hidden);
            x[u] = row8<VEC>(xrow, (p + u * by) * 32u + g * 8u, a.hidden);
        }
#pragma unroll
        for (int u = 0; u < U; u++) acc = Frag<T>::mul(w[u], x[u], acc);
    }
    for (; p < products; p += by) {
        const uint32_t k = p * 32u + g * 8u;
        acc = Frag<T>::mul(row8<VEC>(wrow, k, a.hidden), row8<VEC>(xrow, k, a.hidden), acc);
    }
    return acc;
}

// A workgroup: 16 experts, 16 tokens, one part of hidden, shared out over its waves.
template <class T, bool VEC>
__global__ __launch_bounds__(64 * WAVES) void k_moe_logits(MoeArgs a, MoeSpace m)
{
    __shared__ f32x4 sums[WAVES][64];
    const uint32_t lane = threadIdx.x & 63u, wave = uniform(threadIdx.x >> 6), r = lane & 15u, g = lane >> 4;
    const uint32_t e0 = blockIdx.x * 16u, t0 = blockIdx.z * 16u;
    sums[wave][lane] = logit_tile<T, VEC>(a, e0, t0, blockIdx.y * WAVES + wave, m.splits * WAVES, r, g);
    __syncthreads();
    if (wave) return;
    f32x4 v = sums[0][lane];
#pragma unroll
    for (int w = 1; w < WAVES; w++) v += sums[w][lane];
    if (t0 + r < a.tokens)
        *reinterpret_cast<f32x4 *>(m.part_logits + ((uint64_t)blockIdx.y * a.tokens + t0 + r) * m.row + e0 + g * 4u) = v;
}

// ---- the picks --------------------------------------------------------------------

// One workgroup: every token's picks (16 or 64 lanes a row, as in the router),
// then the experts in use with their tokens, by one bit for every (expert,
// token).  All of it stays in LDS; bound by the latency of its few steps
// (6 us for one token, 9 for 64).
template <int LANES, int V>
__global__ __launch_bounds__(64 * PICK_WAVES) void k_moe_pick(MoeArgs a, MoeSpace m)
{
    constexpr int HELD = picks_held<LANES>(), PER = 64 / LANES;
    extern __shared__ __align__(16) unsigned long long rows[];   // [sets of 64 tokens][experts], then the rest
    __shared__ uint32_t sums[PICK_WAVES];
    const uint32_t sets = (a.tokens + 63) / 64, slots = a.tokens * a.topk;
    uint32_t *base = reinterpret_cast<uint32_t *>(rows + sets * a.experts);
    int32_t *ids = reinterpret_cast<int32_t *>(base + a.experts);
    float *weights = reinterpret_cast<float *>(ids + slots);
    const uint32_t lane = threadIdx.x & 63u, wave = uniform(threadIdx.x >> 6), sub = lane % LANES;
    for (uint32_t i = threadIdx.x; i < sets * a.experts; i += 64 * PICK_WAVES) rows[i] = 0;
    __syncthreads();
    for (uint32_t t0 = wave * PER; t0 < a.tokens; t0 += PICK_WAVES * PER) {
        const uint32_t t = t0 + lane / LANES, row = t < a.tokens ? t : a.tokens - 1;
        f32x4 v[V / 4] = {};
        if (sub * V < m.row) {
            const float *q = m.part_logits + (uint64_t)row * m.row + sub * V;
            const uint64_t by = (uint64_t)a.tokens * m.row;
#pragma unroll
            for (uint32_t s = 0; s < MAX_SPLITS; s++)
                if (s < m.splits) {
#pragma unroll
                    for (int i = 0; i < V / 4; i++)
                        if (sub * V + i * 4 < m.row) v[i] += *reinterpret_cast<const f32x4 *>(q + s * by + i * 4);
                }
        }
        const bool there = !a.mask || a.mask[row];
        uint32_t key[V];
#pragma unroll
        for (int i = 0; i < V; i++) key[i] = there && sub * V + i < a.experts ? Key<float>::of(v[i / 4][i % 4], 0) : 0u;
        int32_t id[HELD];
        float w[HELD];
        topk_row<float, LANES, V>(key, a.topk, a.normalize, sub, id, w);
#pragma unroll
        for (int h = 0; h < HELD; h++) {
            const uint32_t j = sub + 16u * h;
            if (t >= a.tokens || j >= a.topk) continue;
            ids[t * a.topk + j] = id[h];
            weights[t * a.topk + j] = w[h];
            if (id[h] >= 0) atomicOr(&rows[t / 64 * a.experts + id[h]], 1ull << (t % 64));   // LDS; bits of a set
        }
    }
    __syncthreads();
    // threads take experts in order (all of them at most 1,024 = the workgroup);
    // both scans at once: experts in use above bit 16, their places below
    const uint32_t e = threadIdx.x;
    uint32_t c = 0;
    if (e < a.experts)
        for (uint32_t q = 0; q < sets; q++) c += (uint32_t)__popcll(rows[q * a.experts + e]);
    uint32_t all;
    const uint32_t at = block_scan<PICK_WAVES>(c | (c ? 1u << 16 : 0u), sums, all);
    if (e < a.experts) base[e] = at & 0xFFFFu;
    if (c) {
        m.active[1 + (at >> 16)] = e;
        m.first[at >> 16] = at & 0xFFFFu;
    }
    if (threadIdx.x == 0) {
        m.active[0] = all >> 16;
        m.first[all >> 16] = all & 0xFFFFu;
    }
    __syncthreads();
    for (uint32_t s = threadIdx.x; s < slots; s += 64 * PICK_WAVES) {
        const int32_t id = ids[s];
        if (id < 0) {
            m.place[s] = NO_PLACE;
            continue;
        }
        const uint32_t t = s / a.topk;
        uint32_t place = base[id];
        for (uint32_t q = 0; q < t / 64; q++) place += (uint32_t)__popcll(rows[q * a.experts + id]);
        place += (uint32_t)__popcll(rows[t / 64 * a.experts + id] & ((1ull << (t % 64)) - 1ull));
        m.slots[place] = t;
        m.shares[place] = weights[s];
        m.place[s] = place;
    }
}
static_assert(MOE_MAX_TOKENS * ROUTE_MAX_TOPK < 1u << 16, "places fit 16 bits of the scan");

// ---- gate and up ---------------------------------------------------------------------

// Both kernels below: tiles of M x 16 rows of one expert in use, for all its
// tokens, NT tiles of 16 at a time.  The four waves of a workgroup SHARE a
// tile's k and join their sums in LDS in their order, or each has tiles of its
// own.
struct Walk {
    uint32_t tile, tiles, by;   // this wave's tiles
    uint32_t b0, b1;            // this wave's blocks of k
    uint32_t p0, p1;            // the expert's places, taken 16 NT at a time
};
struct At {
    uint32_t tile, b, p;
};

template <bool SHARE>
__device__ inline Walk share_out(const MoeSpace &m, uint32_t wave, uint32_t tiles, uint32_t blocks)
{
    Walk w;
    const uint32_t per = SHARE ? (blocks + WAVES - 1) / WAVES : blocks;
    w.tile = SHARE ? blockIdx.x : blockIdx.x * WAVES + wave;
    w.tiles = tiles;
    w.by = SHARE ? gridDim.x : gridDim.x * WAVES;
    w.b0 = SHARE ? wave * per : 0u;
    w.b1 = w.b0 + per < blocks ? w.b0 + per : blocks;
    w.p0 = m.first[blockIdx.y];
    w.p1 = m.first[blockIdx.y + 1];
    return w;
}

// Runs a wave through its tiles, tokens and blocks: rows(at, there) starts the
// reads of a block's rows, tokens(at) of what its products take of the tokens,
// turn(at) brings the rows in order, multiply(at, n) makes the products,
// join(at, n) ends a tile.  Past the end (not `there`) as many reads are made of
// nothing in particular: their number must not depend on a branch, or the
// compiler has to wait for all of them where some are used.
template <int NT, class Rows, class Tokens, class Turn, class Multiply, class Join>
__device__ inline void walk(const Walk &w, Rows rows, Tokens tokens, Turn turn, Multiply multiply, Join join)
{
    auto next = [&](At at) {
        if (++at.b < w.b1) return at;
        at.b = w.b0;
        at.p += 16 * NT;
        if (at.p < w.p1) return at;
        at.p = w.p0;
        at.tile += w.by;
        return at;
    };
    auto count = [&](const At &at) { return w.p1 - at.p < 16 * NT ? w.p1 - at.p : 16 * NT; };
    At at{w.tile, w.b0, w.p0};
    if (w.b0 >= w.b1) {   // no blocks for this wave: it only joins
        for (; at.tile < w.tiles; at = next(at)) join(at, count(at));
        return;
    }
    rows(at, at.tile < w.tiles);
    tokens(at);
    while (at.tile < w.tiles) {
        const At then = next(at);
        turn(at);
        multiply(at, count(at));
        if (at.b + 1 == w.b1) join(at, count(at));
        rows(then, then.tile < w.tiles);
        tokens(then);
        at = then;
    }
}

// A barrier for LDS alone: reads under way stay under way.
__device__ inline void lds_barrier()
{
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// What a block's products take of one token: its second operands.  Whole
// groups of eight are read from the row's start where they lie past its end
// (no branch about a read), and cleared before they are used.
template <class W, bool VEC>
__device__ inline void load_tokens(u32x4 (&b)[W::PRODUCTS], const uint16_t *row, uint32_t block, uint32_t g, uint32_t len)
{
#pragma unroll
    for (uint32_t i = 0; i < W::PRODUCTS; i++) {
        const uint32_t at = W::at(block, g, i);
        b[i] = VEC ? *reinterpret_cast<const u32x4 *>(row + (at < len ? at : 0u)) : row8<false>(row, at, len);
    }
}
template <class W, bool VEC>
__device__ inline void clear_tokens(u32x4 (&b)[W::PRODUCTS], uint32_t block, uint32_t g, uint32_t len)
{
    if (!VEC || (block + 1) * W::VALUES <= len) return;
#pragma unroll
    for (uint32_t i = 0; i < W::PRODUCTS; i++)
        if (W::at(block, g, i) >= len) b[i] = u32x4{0, 0, 0, 0};
}

template <class T, class C, uint32_t N>
__device__ inline f32x4 up_products(const u32x4 (&p)[N], const u32x4 (&b)[N], f32x4 sum)
{
#pragma unroll
    for (uint32_t i = 0; i < N; i++) {
        if constexpr (__is_same(T, C)) {
            sum = Frag<C>::mul(p[i], b[i], sum);
        } else {   // f16 tokens against microscaled weights
            u32x4 bh, bl;
            split8(b[i], bh, bl);
            sum = Frag<C>::mul(p[i], bh, sum);
            sum = Frag<C>::mul(p[i], bl, sum);
        }
    }
    return sum;
}

// Gate and up rows: sub-tiles 2 i and 2 i + 1 of a wave's tile.  Bound by reading
// them: 64 tokens, 64 experts of 2048 x 1400 in 16 bits 136 us (5.4 TB/s), 16
// tokens, 128 experts of 4096 x 1536 in 4 bits 95 us (4.8 TB/s).
template <class T, class W, bool VEC, int M, int NT, bool SHARE>
__global__ __launch_bounds__(64 * WAVES) void k_moe_up(MoeArgs a, MoeSpace m, uint32_t len, uint32_t slen)
{
    __shared__ __align__(16) uint8_t lds[WAVES][W::LDS];
    __shared__ f32x4 sums[SHARE ? WAVES : 1][M][64];
    __shared__ uint32_t who[MOE_MAX_TOKENS];   // the expert's tokens
    typedef typename W::C C;
    const uint32_t lane = threadIdx.x & 63u, wave = uniform(threadIdx.x >> 6), r = lane & 15u, g = lane >> 4;
    constexpr uint32_t SPAN = M / 2 * 16;   // inner values of a tile
    const Walk k = share_out<SHARE>(m, wave, (uint32_t)((m.inner + SPAN - 1) / SPAN), (a.hidden + W::VALUES - 1) / W::VALUES);
    const uint32_t used = m.active[0], e = m.active[1 + blockIdx.y];
    if (blockIdx.y >= used) return;
    const uint64_t first = (uint64_t)e * 2u * a.inter;
    const Rows up{static_cast<const char *>(a.up) + first * len, a.up_scales + first * slen, 2u * a.inter, len, slen};
    W rows;
    typename W::Block block;
    u32x4 v[W::PRODUCTS];
    for (uint32_t i = threadIdx.x; i < k.p1 - k.p0; i += 64 * WAVES) who[i] = m.slots[k.p0 + i];
    __syncthreads();
    // lanes without a token read the last one's values (their sums are not used)
    auto token = [&](uint32_t place) {
        return static_cast<const uint16_t *>(a.x) + (uint64_t)who[(place < k.p1 ? place : k.p1 - 1) - k.p0] * a.ld_x;
    };
    const uint16_t *x = token(k.p0 + r);
    uint32_t held = k.p0, tile = NO_PLACE;   // whose rows x points to; the tile whose rows are read
    auto read_rows = [&](const At &at, bool there) {
        if (there && at.tile != tile) {
            tile = at.tile;
            uint32_t row[M];
#pragma unroll
            for (int i = 0; i < M; i++) {   // inner values past the last are padding: a row is read, zeros are stored
                const uint32_t in = tile * SPAN + i / 2 * 16u;
                row[i] = (in < a.inter ? in : 0u) + (i % 2 ? a.inter : 0u);
            }
            rows.begin(up, row);
        }
        rows.read(block, up, at.b, there);
    };
    auto read_tokens = [&](const At &at) {
        if (at.p != held) {
            held = at.p;
            x = token(at.p + r);
        }
        load_tokens<W, VEC>(v, x, at.b, g, a.hidden);
    };
    auto turn = [&](const At &at) { rows.turn(block, lds[wave], at.b); };
    f32x4 acc[M][NT] = {};
    auto multiply = [&](const At &at, uint32_t n) {
        clear_tokens<W, VEC>(v, at.b, g, a.hidden);
        u32x4 p[M][W::PRODUCTS];
#pragma unroll
        for (int i = 0; i < M; i++) {
            rows.operands(lds[wave], i, r, g, p[i]);
            acc[i][0] = up_products<T, C>(p[i], v, acc[i][0]);
        }
#pragma unroll
        for (int t = 1; t < NT; t++) {
            if (t * 16u >= n) break;
            u32x4 y[W::PRODUCTS];
            load_tokens<W, VEC>(y, token(at.p + t * 16u + r), at.b, g, a.hidden);
            clear_tokens<W, VEC>(y, at.b, g, a.hidden);
#pragma unroll
            for (int i = 0; i < M; i++) acc[i][t] = up_products<T, C>(p[i], y, acc[i][t]);
        }
    };
    auto join = [&](const At &at, uint32_t n) {
#pragma unroll
        for (int t = 0; t < NT; t++) {
            if (t * 16u >= n) break;
            f32x4 s[M];
#pragma unroll
            for (int i = 0; i < M; i++) {
                s[i] = acc[i][t];
                acc[i][t] = f32x4{0, 0, 0, 0};
            }
            if constexpr (SHARE) {
                lds_barrier();   // the sums before have been read
#pragma unroll
                for (int i = 0; i < M; i++) sums[wave][i][lane] = s[i];
                lds_barrier();
                if (wave != 0) continue;
#pragma unroll
                for (int i = 0; i < M; i++)
#pragma unroll
                    for (int w = 1; w < WAVES; w++) s[i] += sums[w][i][lane];
            }
            if (t * 16u + r >= n) continue;
#pragma unroll
            for (int i = 0; i < M / 2; i++) {
                const uint32_t i0 = at.tile * SPAN + i * 16u + g * 4u;
                if (i0 >= m.inner) continue;
                const f32x4 gate = s[2 * i], lift = s[2 * i + 1];
                uint16_t part[PARTS][4];
#pragma unroll
                for (int q = 0; q < 4; q++) {
                    const float h = i0 + q < a.inter ? gate[q] / (1.f + expf(-gate[q])) * lift[q] : 0.f;
                    split(h, part[0][q], part[1][q], part[2][q]);
                }
                uint32_t product, group;
                W::place(i0, product, group);
                const uint64_t to =
                    (((uint64_t)(k.p0 / 16 + blockIdx.y + (at.p - k.p0) / 16 + t) * (m.inner / 32) + product) * (PARTS * 64u) + group * 16u + r) * 8u + i0 % 8;
#pragma unroll
                for (uint32_t q = 0; q < PARTS; q++) __builtin_memcpy(__builtin_assume_aligned(m.parts + to + q * 512u, 8), part[q], 8);
            }
        }
    };
    walk<NT>(k, read_rows, read_tokens, turn, multiply, join);
}

// Down rows, against the parts of the inner values: the first part's products
// are summed up by themselves, the others' (2^-7 of them and less) beside them.
// An f16 weight is taken in two parts of bf16, since a 32-bit inner value passes
// the range of f16 on either side.  The same layers: 95 us (3.9 TB/s) and 76 us
// (3.0 TB/s); rows are shorter here, and the parts are read beside them.  Two
// parts took 89 and 64 us and left 2^-17 of a value; three waves a SIMD, where
// the compiler by itself settles for two, took the latter from 84 to 76.
template <class W, int M, int NT, bool SHARE>
__global__ __launch_bounds__(64 * WAVES, NT == 1 ? 3 : 1) void k_moe_down(MoeArgs a, MoeSpace m, uint32_t len, uint32_t slen)
{
    __shared__ __align__(16) uint8_t lds[WAVES][W::LDS];
    __shared__ f32x4 sums[SHARE ? WAVES : 1][M][64];
    typedef Frag<__bf16> F;
    constexpr bool TWO = !__is_same(typename W::C, __bf16);
    constexpr uint32_t N = W::PRODUCTS, SPAN = M * 16;
    const uint32_t lane = threadIdx.x & 63u, wave = uniform(threadIdx.x >> 6), r = lane & 15u, g = lane >> 4;
    const Walk k = share_out<SHARE>(m, wave, (a.hidden + SPAN - 1) / SPAN, (uint32_t)((m.inner + W::VALUES - 1) / W::VALUES));
    const uint32_t used = m.active[0], e = m.active[1 + blockIdx.y];
    if (blockIdx.y >= used) return;
    const uint64_t first = (uint64_t)e * a.hidden;
    const Rows down{static_cast<const char *>(a.down) + first * len, a.down_scales + first * slen, a.hidden, len, slen};
    W rows;
    typename W::Block block;
    u32x4 v[N][PARTS];
    uint32_t tile = NO_PLACE;   // the tile whose rows are read
    const uint32_t products = (uint32_t)(m.inner / 32);
    // lanes without a token read the last one's values (their sums are not used)
    auto inner = [&](u32x4 (&x)[N][PARTS], const At &at, uint32_t t) {
        const uint32_t n = k.p1 - at.p - t * 16u, who = r < n ? r : n - 1;
        const uint64_t from = ((uint64_t)(k.p0 / 16 + blockIdx.y + (at.p - k.p0) / 16 + t) * products + at.b * N) * (PARTS * 64u) + g * 16u + who;
#pragma unroll
        for (uint32_t i = 0; i < N; i++) {
            // a block's second step may be missing: its first is read again, and cleared
            const uint64_t q = from + (at.b * N + i < products ? i * (PARTS * 64u) : 0u);
#pragma unroll
            for (uint32_t c = 0; c < PARTS; c++) x[i][c] = reinterpret_cast<const u32x4 *>(m.parts)[q + c * 64u];
        }
    };
    auto read_rows = [&](const At &at, bool there) {
        if (there && at.tile != tile) {
            tile = at.tile;
            uint32_t row[M];
#pragma unroll
            for (int i = 0; i < M; i++) row[i] = tile * SPAN + i * 16u;
            rows.begin(down, row);
        }
        rows.read(block, down, at.b, there);
    };
    auto read_tokens = [&](const At &at) { inner(v, at, 0); };
    auto turn = [&](const At &at) { rows.turn(block, lds[wave], at.b); };
    auto clear = [&](u32x4 (&x)[N][PARTS], const At &at) {
        if ((at.b + 1) * N <= products) return;
#pragma unroll
        for (uint32_t i = 0; i < N; i++)
            if (at.b * N + i >= products)
#pragma unroll
                for (uint32_t c = 0; c < PARTS; c++) x[i][c] = u32x4{0, 0, 0, 0};
    };
    f32x4 acc[M][NT] = {}, rest[M][NT] = {};
    u32x4 p[M][N], low[TWO ? M : 1][N];   // the weights, or their two parts
    auto multiply_by = [&](const u32x4 (&x)[N][PARTS], int i, int t) {
#pragma unroll
        for (uint32_t j = 0; j < N; j++) {
            acc[i][t] = F::mul(p[i][j], x[j][0], acc[i][t]);
#pragma unroll
            for (uint32_t c = 1; c < PARTS; c++) rest[i][t] = F::mul(p[i][j], x[j][c], rest[i][t]);
            if constexpr (TWO) {
#pragma unroll
                for (uint32_t c = 0; c < PARTS; c++) rest[i][t] = F::mul(low[i][j], x[j][c], rest[i][t]);
            }
        }
    };
    auto multiply = [&](const At &at, uint32_t n) {
        clear(v, at);
#pragma unroll
        for (int i = 0; i < M; i++) {
            rows.operands(lds[wave], i, r, g, p[i]);
            if constexpr (TWO) {
#pragma unroll
                for (uint32_t j = 0; j < N; j++) split8(p[i][j], p[i][j], low[i][j]);
            }
            multiply_by(v, i, 0);
        }
#pragma unroll
        for (int t = 1; t < NT; t++) {
            if (t * 16u >= n) break;
            u32x4 x[N][PARTS];
            inner(x, at, t);
            clear(x, at);
#pragma unroll
            for (int i = 0; i < M; i++) multiply_by(x, i, t);
        }
    };
    auto join = [&](const At &at, uint32_t n) {
#pragma unroll
        for (int t = 0; t < NT; t++) {
            if (t * 16u >= n) break;
            f32x4 s[M];
#pragma unroll
            for (int i = 0; i < M; i++) {
                s[i] = acc[i][t] + rest[i][t];
                acc[i][t] = rest[i][t] = f32x4{0, 0, 0, 0};
            }
            if constexpr (SHARE) {
                lds_barrier();   // the sums before have been read
#pragma unroll
                for (int i = 0; i < M; i++) sums[wave][i][lane] = s[i];
                lds_barrier();
                if (wave != 0) continue;
#pragma unroll
                for (int i = 0; i < M; i++)
#pragma unroll
                    for (int q = 1; q < WAVES; q++) s[i] += sums[q][i][lane];
            }
            if (t * 16u + r >= n) continue;
            const uint32_t place = at.p + t * 16u + r;
            const float share = m.shares[place];
#pragma unroll
            for (int i = 0; i < M; i++) {
                const uint32_t h = at.tile * SPAN + i * 16u + g * 4u;
                float *to = m.outs + (uint64_t)place * a.hidden + h;
                const f32x4 o = s[i] * share;
                if (a.hidden % 4 == 0) {
                    if (h < a.hidden) *reinterpret_cast<f32x4 *>(to) = o;
                    continue;
                }
#pragma unroll
                for (int q = 0; q < 4; q++)
                    if (h + q < a.hidden) to[q] = o[q];
            }
        }
    };
    walk<NT>(k, read_rows, read_tokens, turn, multiply, join);
}

// Each token's sum over its picks, in their order; zeros without any.
template <class T>
__global__ __launch_bounds__(256) void k_moe_sum(MoeArgs a, MoeSpace m)
{
    const uint32_t t = blockIdx.y, h = blockIdx.x * 256u + threadIdx.x;
    if (h >= a.hidden) return;
    float v = 0.f;
#pragma unroll 4
    for (uint32_t j = 0; j < a.topk; j++) {
        const uint32_t p = m.place[t * a.topk + j];
        if (p != NO_PLACE) v += m.outs[(uint64_t)p * a.hidden + h];
    }
    static_cast<T *>(a.y)[(uint64_t)t * a.ld_y + h] = Elem<T>::put(v);
}

// Whether each wave has tiles of its own rather than a part of the blocks of a
// workgroup's: where sharing leaves less than two blocks a wave, so that
// rounding up leaves waves without work, and the tiles of the experts in use (at
// most `most`) are enough to keep every compute unit's waves busy all the same.
// Whole layers, shared and this way, 16 tokens, 8 of 128 experts in 4 bits: 1024
// x 256 values (one block) 37 and 32 us, 1024 x 512 47 and 44, 4096 x 1536 (six)
// 226 and 216, 1024 x 2048 (eight) 100 and 103, 1024 x 3840 171 and 179; fewer
// tiles, 1024 x 1024: 2048 of them 59 and 58, 1024 38 and 39, 512 25 and 28.
inline bool own_tiles(uint64_t blocks, uint64_t tiles, uint64_t most) { return blocks < 2 * WAVES && tiles * most >= 2048; }

template <class T, class W, bool VEC, int NT>
hipError_t experts_as(const MoeArgs &a, const MoeSpace &m, hipStream_t s)
{
    constexpr int M = 2;
    const uint64_t places = (uint64_t)a.tokens * a.topk;
    const uint32_t most = places < a.experts ? (uint32_t)places : a.experts;
    const bool mx = a.up_scales != nullptr;
    const uint32_t ul = mx ? (uint32_t)mx_code_bytes(a.hidden) : a.hidden * 2u, us = mx ? (uint32_t)mx_scale_bytes(a.hidden) : 0u;
    const uint32_t dl = mx ? (uint32_t)mx_code_bytes(a.inter) : a.inter * 2u, ds = mx ? (uint32_t)mx_scale_bytes(a.inter) : 0u;
    const uint32_t up = (uint32_t)((m.inner + M * 8 - 1) / (M * 8)), down = (a.hidden + M * 16 - 1) / (M * 16);
    auto groups = [&](uint32_t tiles, bool own) { return dim3(own ? (tiles + WAVES - 1) / WAVES : tiles, most); };
    if (own_tiles((a.hidden + W::VALUES - 1) / W::VALUES, up, most)) k_moe_up<T, W, VEC, M, NT, false><<<groups(up, true), 64 * WAVES, 0, s>>>(a, m, ul, us);
    else k_moe_up<T, W, VEC, M, NT, true><<<groups(up, false), 64 * WAVES, 0, s>>>(a, m, ul, us);
    if (own_tiles((m.inner + W::VALUES - 1) / W::VALUES, down, most)) k_moe_down<W, M, NT, false><<<groups(down, true), 64 * WAVES, 0, s>>>(a, m, dl, ds);
    else k_moe_down<W, M, NT, true><<<groups(down, false), 64 * WAVES, 0, s>>>(a, m, dl, ds);
    k_moe_sum<T><<<dim3((a.hidden + 255) / 256, a.tokens), 256, 0, s>>>(a, m);
    return hipGetLastError();
}

// Tiles of 16 tokens that share one reading of the weights: one where experts
// have a few tokens on average (few have more than 16, and theirs are read
// again, from the caches), four beyond, at the price of registers.  Weights in 4
// bits cost less to read again and more registers to unpack.  64 experts of 2048
// x 1400, 8 picks, one and four: in 16 bits 64 tokens 249 and 254 us, 96 269 and
// 268, 128 320 and 292, 256 497 and 357; in 4 bits 128 tokens 186 and 188, 192 222
// and 216, 256 288 and 256.
template <class T, class W, bool VEC>
hipError_t experts_of(const MoeArgs &a, const MoeSpace &m, hipStream_t s)
{
    const uint64_t few = a.up_scales ? 24 : 12;   // tokens of an expert
    if (a.tokens <= 16 || (uint64_t)a.tokens * a.topk <= few * a.experts) return experts_as<T, W, VEC, 1>(a, m, s);
    return experts_as<T, W, VEC, 4>(a, m, s);
}

template <int LANES, int V>
hipError_t pick_as(const MoeArgs &a, const MoeSpace &m, hipStream_t s)
{
    auto room = [](uint32_t tokens, uint32_t experts, uint32_t topk) { return (tokens + 63) / 64 * experts * 8u + experts * 4u + tokens * topk * 8u; };
    const hipError_t e = allow_lds<&k_moe_pick<LANES, V>>(room(MOE_MAX_TOKENS, ROUTE_MAX_EXPERTS, ROUTE_MAX_TOPK));
    if (e != hipSuccess) return e;
    k_moe_pick<LANES, V><<<1, 64 * PICK_WAVES, room(a.tokens, a.experts, a.topk), s>>>(a, m);
    return hipGetLastError();
}

template <class T>
hipError_t picks(const MoeArgs &a, const MoeSpace &m, bool vec, hipStream_t s)
{
    const dim3 grid((a.experts + 15) / 16, m.splits, (a.tokens + 15) / 16);
    if (vec) k_moe_logits<T, true><<<grid, 64 * WAVES, 0, s>>>(a, m);
    else k_moe_logits<T, false><<<grid, 64 * WAVES, 0, s>>>(a, m);
    if (a.experts <= 64) return pick_as<16, 4>(a, m, s);
    if (a.experts <= 128) return pick_as<16, 8>(a, m, s);
    if (a.experts <= NARROW_EXPERTS) return pick_as<16, 16>(a, m, s);
    if (a.experts <= 512) return pick_as<64, 8>(a, m, s);
    return pick_as<64, 16>(a, m, s);
}

template <class T>
hipError_t moe_as(const MoeArgs &a, hipStream_t s)
{
    MoeSpace m;
    carve(m, a.ws, a.tokens, a.experts, a.topk, a.hidden, a.inter);
    auto aligned = [](const void *p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; };
    // whole groups of eight values: rows are read 16 bytes at a time
    const bool vx = aligned(a.x) && a.ld_x % 8 == 0 && a.hidden % 8 == 0;
    const hipError_t e = picks<T>(a, m, vx && aligned(a.router), s);
    if (e != hipSuccess) return e;
    if (a.up_scales) return vx ? experts_of<T, Micro<2>, true>(a, m, s) : experts_of<T, Micro<2>, false>(a, m, s);
    if (vx && aligned(a.up) && aligned(a.down) && a.inter % 8 == 0) return experts_of<T, Plain<T, 2, true>, true>(a, m, s);
    return experts_of<T, Plain<T, 2, false>, false>(a, m, s);
}

}  // namespace

size_t moe_workspace(uint32_t tokens, uint32_t experts, uint32_t topk, uint32_t hidden, uint32_t inter)
{
    MoeSpace m;
    return carve(m, nullptr, tokens, experts, topk, hidden, inter);
}

hipError_t launch_moe(const MoeArgs &a, uint32_t dtype, hipStream_t s)
{
    return dtype == DT_BF16 ? moe_as<__bf16>(a, s) : moe_as<_Float16>(a, s);
}

}  // namespace pccl
