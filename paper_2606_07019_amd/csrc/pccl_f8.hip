// 8-bit floating point (E4M3) with one power-of-two scale for 128 values: the
// blocks of rows that belong to one expert, packing and unpacking.
//
// For a block with largest magnitude a the scale is the smallest 2^e, e >=
// -127, with a <= 448 * 2^e, so that nothing is clipped; the scale byte is e +
// 127, and each value becomes the E4M3 value nearest to x / 2^e, ties to the
// even code.  A block of zeros has the byte 0, one that holds a NaN or an
// infinity the byte 255 (NaN).  Dividing by a power of two and rounding once is
// exact arithmetic, so the codes do not depend on how the work is split.
#include "pccl_topk.h"

namespace pccl {
namespace {

// ---- the experts' blocks of rows ---------------------------------------------

constexpr uint32_t GROUP_THREADS = 1024;   // at least ROUTE_MAX_EXPERTS

// Exclusive sums of the threads' values.
__device__ inline uint64_t scan64(uint64_t v, uint64_t *sums)
{
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    uint64_t x = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint64_t y = __shfl_up((unsigned long long)x, o);
        if (lane >= (uint32_t)o) x += y;
    }
    __syncthreads();
    if (lane == 63u) sums[wave] = x;
    __syncthreads();
    uint64_t before = 0;
    for (uint32_t w = 0; w < wave; w++) before += sums[w];
    return before + x - v;
}

// Every workgroup sums up the counts (a negative one is none, rows past `rows`
// are no one's) and fills its share of the two lists, a block a thread.  Bound by
// its launch and two scans: 64 experts, 512 rows, 4.6 us; 32,768 rows 6.0.
__global__ __launch_bounds__(GROUP_THREADS) void k_groups(GroupsArgs a)
{
    __shared__ uint32_t first[ROUTE_MAX_EXPERTS + 1], start[2][ROUTE_MAX_EXPERTS + 1];
    __shared__ uint64_t sums[GROUP_THREADS / 64];
    const uint32_t e = threadIdx.x;
    const int32_t given = e < a.experts ? a.counts[e] : 0;
    const uint64_t c = given > 0 ? (uint64_t)given : 0u;
    const uint64_t at = scan64(c, sums), end = at + c;
    const uint32_t from = (uint32_t)(at < a.rows ? at : a.rows), to = (uint32_t)(end < a.rows ? end : a.rows);
    const uint32_t n = to - from, n1 = (n + 127) / 128, n2 = (n + 255) / 256;
    const uint64_t s = scan64((uint64_t)n1 << 32 | n2, sums);
    if (e < a.experts) {
        first[e] = from;
        start[0][e] = (uint32_t)(s >> 32);
        start[1][e] = (uint32_t)s;
        if (e + 1 == a.experts) {
            first[e + 1] = to;
            start[0][e + 1] = (uint32_t)(s >> 32) + n1;
            start[1][e + 1] = (uint32_t)s + n2;
        }
    }
    __syncthreads();
    if (blockIdx.x == 0)
        for (uint32_t i = e; i <= a.experts + 1; i += GROUP_THREADS) a.table[i] = (int32_t)(i <= a.experts ? start[0][i] : start[1][a.experts]);
    const uint64_t all = a.blocks + a.blocks2;
    for (uint64_t j = (uint64_t)blockIdx.x * GROUP_THREADS + e; j < all; j += (uint64_t)gridDim.x * GROUP_THREADS) {
        const uint32_t l = j >= a.blocks, size = 128u << l;
        const uint32_t b = (uint32_t)(l ? j - a.blocks : j);
        int32_t *out = a.table + a.experts + 2 + 2 * j;
        if (b >= start[l][a.experts]) {
            out[0] = out[1] = 0;
            continue;
        }
        uint32_t lo = 0, hi = a.experts;   // the last expert that starts at or before the block (those of no blocks start where the next does)
        while (hi - lo > 1) {
            const uint32_t mid = (lo + hi) / 2;
            if (start[l][mid] <= b) lo = mid;
            else hi = mid;
        }
        const uint32_t row = first[lo] + (b - start[l][lo]) * size, left = first[lo + 1] - row;
        out[0] = (int32_t)row;
        out[1] = (int32_t)(lo | (left < size ? left : size) << 16);
    }
}

// ---- packing -------------------------------------------------------------------

// The scale byte of a block, from the bits of its largest magnitude.
template <class T>
struct F8In;
template <>
struct F8In<float> {
    static __device__ uint32_t byte(uint32_t top)
    {
        if (top >= 0x7F800000u) return 255u;
        const uint32_t f = (top >> 23) + ((top & 0x7FFFFFu) > 0x600000u);   // 448 = 1.75 * 2^8
        return f > 8u ? f - 8u : 0u;
    }
};
template <>
struct F8In<__bf16> {
    static __device__ uint32_t byte(uint32_t top) { return F8In<float>::byte(top << 16); }
};
template <>
struct F8In<_Float16> {
    static __device__ uint32_t byte(uint32_t top)
    {
        if (top >= 0x7C00u) return 255u;
        return F8In<float>::byte(__float_as_uint((float)__builtin_bit_cast(_Float16, (uint16_t)top)));
    }
};

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef short s16x2 __attribute__((ext_vector_type(2)));

// Eight values of one lane: 16-bit types hold two to a word.
template <class T>
struct Eight {
    static constexpr int W = sizeof(T) * 2;   // words
    uint32_t w[W];
};

// From any address; only a row's last values are read one by one.
template <class T>
__device__ inline Eight<T> load8(const T *p, uint64_t left)
{
    Eight<T> o;
    if (left >= 8) {
        __builtin_memcpy(o.w, p, sizeof o.w);
        return o;
    }
    T t[8];
#pragma unroll
    for (int i = 0; i < 8; i++) t[i] = (uint64_t)i < left ? p[i] : (T)0.f;
    __builtin_memcpy(o.w, t, sizeof t);
    return o;
}

template <class T>
__device__ inline Eight<T> nothing()
{
    Eight<T> o;
#pragma unroll
    for (int i = 0; i < Eight<T>::W; i++) o.w[i] = 0;
    return o;
}

// Largest magnitude of the eight, as ordered bits.
template <class T>
__device__ inline uint32_t top_of(const Eight<T> &o)
{
    if constexpr (sizeof(T) == 4) {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const uint32_t a = o.w[i] & 0x7FFFFFFFu;
            m = a > m ? a : m;
        }
        return m;
    } else {
        u16x2 m = {0, 0};
#pragma unroll
        for (int i = 0; i < 4; i++) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, o.w[i] & 0x7FFF7FFFu));
        return m.x > m.y ? m.x : m.y;
    }
}

// Two values to the low (HI false) or high half of a word.
template <bool HI>
__device__ inline s16x2 pair(s16x2 old, float a, float b, float scale) { return __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(old, a, b, scale, HI); }
template <class T, bool HI>
__device__ inline s16x2 pair(s16x2 old, uint32_t two, float scale)
{
    if constexpr (__is_same(T, __bf16)) return __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(old, __builtin_bit_cast(bf16x2, two), scale, HI);
    else return __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(old, __builtin_bit_cast(f16x2, two), scale, HI);
}
// Four values (two words of two, or four floats) to a word of codes.
template <class T>
__device__ inline uint32_t codes4(const uint32_t *w, float scale)
{
    s16x2 r = {0, 0};
    if constexpr (sizeof(T) == 4) {
        r = pair<false>(r, __uint_as_float(w[0]), __uint_as_float(w[1]), scale);
        r = pair<true>(r, __uint_as_float(w[2]), __uint_as_float(w[3]), scale);
    } else {
        r = pair<T, false>(r, w[0], scale);
        r = pair<T, true>(r, w[1], scale);
    }
    return __builtin_bit_cast(uint32_t, r);
}
template <class T>
__device__ inline u32x2 codes8(const Eight<T> &o, uint32_t byte)
{
    if (byte == 255u) return u32x2{0u, 0u};
    const float s = mx_scale(byte);
    return u32x2{codes4<T>(o.w, s), codes4<T>(o.w + Eight<T>::W / 2, s)};
}

constexpr int ROWS = 2;   // of a wave

// The rows alone: a wave packs 512 values of two rows, so that what it reads,
// its codes and its scales are contiguous (1 KiB of 16-bit values, 512 and 4
// bytes a row).  Bound by memory: 8192 x 8192 of bf16 32 us, 6.3 TB/s from and to the
// device's cache.
template <class T>
__global__ __launch_bounds__(256) void k_f8_rows(F8QuantizeArgs a, uint32_t chunks)
{
    const T *x = static_cast<const T *>(a.x);
    const uint32_t lane = threadIdx.x & 63u;
    const uint64_t item = (uint64_t)blockIdx.x * 4u + (threadIdx.x >> 6);
    const uint64_t row0 = item / chunks * ROWS, col0 = item % chunks * 512u, col = col0 + lane * 8u;
    const uint64_t cb = f8_code_bytes(a.cols), sb = f8_scale_bytes(a.cols);
    if (row0 >= a.rows) return;
    Eight<T> o[ROWS];
#pragma unroll
    for (int p = 0; p < ROWS; p++) o[p] = row0 + p < a.rows && col < a.cols ? load8<T>(x + (row0 + p) * a.ld + col, a.cols - col) : nothing<T>();
#pragma unroll
    for (int p = 0; p < ROWS; p++) {
        const uint64_t r = row0 + p;
        const uint32_t byte = F8In<T>::byte(row_max<16>(top_of(o[p])));
        const u32x2 code = codes8(o[p], byte);
        uint32_t word = (uint32_t)__builtin_amdgcn_readlane((int)byte, 0);
        word |= (uint32_t)__builtin_amdgcn_readlane((int)byte, 16) << 8;
        word |= (uint32_t)__builtin_amdgcn_readlane((int)byte, 32) << 16;
        word |= (uint32_t)__builtin_amdgcn_readlane((int)byte, 48) << 24;
        if (r < a.rows) {
            if (col < cb) *reinterpret_cast<u32x2 *>(a.codes + r * cb + col) = code;
            if (lane == 0) *reinterpret_cast<uint32_t *>(a.scales + r * sb + col0 / F8_BLOCK) = word;
        }
    }
}

constexpr uint32_t TILE = 128;   // rows and columns of a workgroup's tile: one block either way

// One workgroup packs a tile of 128 x 128 values.  A lane holds eight values of HELD
// neighbouring rows; sixteen lanes share a row's block, and the largest of the
// columns meet in LDS.  A column's codes are made in the lanes that hold its rows,
// HELD bytes at a time, and put together in LDS, from where whole columns are
// stored: piece u (8 bytes) of column c stands at u ^ 2 (c / 8 % 8).
// Bound by memory: every value is read once for both directions (16384 x 4096 of
// bf16 both ways 46 us, 5.8 TB/s; 61 matrices of 1000 x 2040 in tiles 99 us, 5 TB/s).
//   BOTH: the rows' packing too.  TILES: one scale for the whole tile.
// With `groups` the tile's rows are a block of one expert's.
// A short last block of an expert takes a tile's time all the same (12,288 x 2040 of
// bf16, 96 whole blocks, 27.2 us, as without groups; 12,297 rows of 61 experts, 131
// blocks, 28.9): 4 TB/s, as the tiles of one matrix of that size.
// Eight waves a tile (2040 x 1500 of bf16 both ways 8.7 us; four, of eight rows a lane, 11.8).
constexpr int HELD = 4, TILE_THREADS = 2048 / HELD, TILE_WAVES = TILE_THREADS / 64;

template <class T, bool BOTH, bool TILES>
__global__ __launch_bounds__(TILE_THREADS) void k_f8_tile(F8QuantizeArgs a, uint32_t col_tiles, uint32_t row_tiles, uint32_t stored)
{
    __shared__ __align__(16) uint8_t turned[TILE * TILE];
    __shared__ __align__(16) uint32_t tops[TILE_WAVES][TILE];
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    const uint32_t tc = blockIdx.x % col_tiles, rest = blockIdx.x / col_tiles, tr = rest % row_tiles, matrix = rest / row_tiles;
    uint64_t first = (uint64_t)matrix * a.rows + (uint64_t)tr * TILE;
    uint32_t n = (uint32_t)(a.rows - (uint64_t)tr * TILE < TILE ? a.rows - (uint64_t)tr * TILE : TILE);
    if (a.groups) {
        const int32_t *entry = a.groups + a.experts + 2 + 2 * (uint64_t)tr;
        first = (uint32_t)entry[0];
        n = (uint32_t)entry[1] >> 16;
        if (n == 0) return;
    }
    const uint32_t cg = lane & 15u, r0 = (wave * 4u + (lane >> 4)) * HELD;
    const uint64_t col = (uint64_t)tc * TILE + cg * 8u;
    const T *x = static_cast<const T *>(a.x);
    Eight<T> o[HELD];
#pragma unroll
    for (int p = 0; p < HELD; p++) o[p] = r0 + p < n && col < a.cols ? load8<T>(x + (first + r0 + p) * a.ld + col, a.cols - col) : nothing<T>();

    uint32_t rowtop[HELD];
#pragma unroll
    for (int p = 0; p < HELD; p++) rowtop[p] = BOTH || TILES ? top_of(o[p]) : 0u;
    uint32_t tile_byte = 0;
    if constexpr (TILES) {
        uint32_t t = 0;
#pragma unroll
        for (int p = 0; p < HELD; p++) t = rowtop[p] > t ? rowtop[p] : t;
        t = row_max<64>(t);
        if (lane == 0) tops[wave][0] = t;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < TILE_WAVES; w++) t = tops[w][0] > t ? tops[w][0] : t;
        tile_byte = F8In<T>::byte(t);
    }
    if constexpr (BOTH) {
        const uint64_t cb = f8_code_bytes(a.cols), sb = f8_scale_bytes(a.cols);
#pragma unroll
        for (int p = 0; p < HELD; p++) {
            const uint32_t byte = TILES ? tile_byte : F8In<T>::byte(row_max<16>(rowtop[p]));
            const u32x2 code = codes8(o[p], byte);
            if (r0 + p < n) {
                const uint64_t r = first + r0 + p;
                *reinterpret_cast<u32x2 *>(a.codes + r * cb + col) = code;
                if (cg == 0) {
                    a.scales[r * sb + tc] = (uint8_t)byte;
                    if (tc + 1 == col_tiles)
                        for (uint64_t i = tc + 1; i < sb; i++) a.scales[r * sb + i] = 0;
                }
            }
        }
    }
    if (!a.codes_t) return;
    uint32_t bytes[8];
    if constexpr (TILES) {
#pragma unroll
        for (int i = 0; i < 8; i++) bytes[i] = tile_byte;
    } else {
        uint32_t top[8];
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < 8; i++) {
                top[i] = 0;
#pragma unroll
                for (int p = 0; p < HELD; p++) {
                    const uint32_t v = o[p].w[i] & 0x7FFFFFFFu;
                    top[i] = v > top[i] ? v : top[i];
                }
#pragma unroll
                for (int x = 16; x < 64; x <<= 1) {
                    const uint32_t v = (uint32_t)__shfl_xor((int)top[i], x);
                    top[i] = v > top[i] ? v : top[i];
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; i++) {
                u16x2 t = {0, 0};
#pragma unroll
                for (int p = 0; p < HELD; p++) t = __builtin_elementwise_max(t, __builtin_bit_cast(u16x2, o[p].w[i] & 0x7FFF7FFFu));
#pragma unroll
                for (int x = 16; x < 64; x <<= 1)
                    t = __builtin_elementwise_max(t, __builtin_bit_cast(u16x2, __shfl_xor(__builtin_bit_cast(int, t), x)));
                top[2 * i] = t.x;
                top[2 * i + 1] = t.y;
            }
        }
        if (lane < 16) {
            *reinterpret_cast<u32x4 *>(&tops[wave][cg * 8]) = u32x4{top[0], top[1], top[2], top[3]};
            *reinterpret_cast<u32x4 *>(&tops[wave][cg * 8 + 4]) = u32x4{top[4], top[5], top[6], top[7]};
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; i++) top[i] = 0;
#pragma unroll
        for (int w = 0; w < TILE_WAVES; w++)
#pragma unroll
            for (int h = 0; h < 2; h++) {
                const u32x4 t = *reinterpret_cast<const u32x4 *>(&tops[w][cg * 8 + h * 4]);
#pragma unroll
                for (int i = 0; i < 4; i++) top[h * 4 + i] = t[i] > top[h * 4 + i] ? t[i] : top[h * 4 + i];
            }
#pragma unroll
        for (int i = 0; i < 8; i++) bytes[i] = F8In<T>::byte(top[i]);
    }
    const uint32_t unit = ((r0 / 8u) ^ ((cg & 7u) * 2u)) * 8u + r0 % 8u;
#pragma unroll
    for (int i = 0; i < 8; i++) {
        uint32_t v[HELD * sizeof(T) / 4];   // the column's rows
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int p = 0; p < HELD; p++) v[p] = o[p].w[i];
        } else {
#pragma unroll
            for (int p = 0; p < HELD / 2; p++) v[p] = __builtin_amdgcn_perm(o[2 * p + 1].w[i / 2], o[2 * p].w[i / 2], i % 2 ? 0x07060302u : 0x05040100u);
        }
        const float scale = mx_scale(bytes[i]);
#pragma unroll
        for (int p = 0; p < HELD / 4; p++)
            *reinterpret_cast<uint32_t *>(turned + (cg * 8u + i) * TILE + unit + 4 * p) = bytes[i] == 255u ? 0u : codes4<T>(v + p * sizeof(T), scale);
    }
    // `stored`: blocks of a column that there is room for
    const uint64_t cbt = (uint64_t)stored * TILE, sbt = (stored + 3u) / 4u * 4u;
    const uint64_t column0 = (uint64_t)matrix * a.cols;
    if (wave == 0 && lane < 16) {
#pragma unroll
        for (int i = 0; i < 8; i++)
            if (col + i < a.cols) {
                a.scales_t[(column0 + col + i) * sbt + tr] = (uint8_t)bytes[i];
                if (tr + 1 == stored)
                    for (uint64_t j = tr + 1; j < sbt; j++) a.scales_t[(column0 + col + i) * sbt + j] = 0;
            }
    }
    __syncthreads();
#pragma unroll
    for (uint32_t i = 0; i < 1024 / TILE_THREADS; i++) {
        const uint32_t c = i * (TILE_THREADS / 8) + threadIdx.x / 8, q = threadIdx.x % 8;   // 16 bytes of a column
        const uint64_t cc = (uint64_t)tc * TILE + c;
        if (cc < a.cols)
            *reinterpret_cast<u32x4 *>(a.codes_t + (column0 + cc) * cbt + (uint64_t)tr * TILE + q * 16u) =
                *reinterpret_cast<const u32x4 *>(turned + c * TILE + ((2u * q) ^ (c / 8 % 8 * 2u)) * 8u);
    }
}

template <class T>
hipError_t quantize_as(const F8QuantizeArgs &a, hipStream_t s)
{
    if (!a.codes_t && !a.tiles) {   // one matrix
        const uint32_t chunks = (uint32_t)((a.cols + 511) / 512);
        const uint64_t most = most_blocks(256) * 4 / chunks * ROWS;   // rows of a launch
        for (uint64_t r = 0; r < a.rows; r += most) {
            F8QuantizeArgs part = a;
            part.x = static_cast<const T *>(a.x) + r * a.ld;
            part.rows = a.rows - r < most ? a.rows - r : most;
            part.codes += r * f8_code_bytes(a.cols);
            part.scales += r * f8_scale_bytes(a.cols);
            const uint64_t items = (part.rows + ROWS - 1) / ROWS * chunks;
            k_f8_rows<T><<<dim3((uint32_t)((items + 3) / 4)), 256, 0, s>>>(part, chunks);
        }
        return hipGetLastError();
    }
    const uint32_t ct = (uint32_t)f8_blocks(a.cols);
    const uint32_t rt = (uint32_t)(a.groups ? groups_blocks(a.experts, a.rows, 128) : f8_blocks(a.rows));
    const dim3 grid((uint32_t)(ct * (uint64_t)rt * a.batch));
    if (a.tiles) k_f8_tile<T, true, true><<<grid, TILE_THREADS, 0, s>>>(a, ct, rt, rt);
    else if (a.codes) k_f8_tile<T, true, false><<<grid, TILE_THREADS, 0, s>>>(a, ct, rt, rt);
    else k_f8_tile<T, false, false><<<grid, TILE_THREADS, 0, s>>>(a, ct, rt, rt);
    return hipGetLastError();
}

// ---- unpacking -------------------------------------------------------------------

typedef u32x4 Chunk __attribute__((aligned(2)));   // at any address

// A wave unpacks 512 values of a row, a store of 16 bytes a lane at a time, so that
// each store writes whole lines.  Bound by writing them: 16384 x 4096 of bf16 31 us,
// 6.4 TB/s read and written (stored through the caches a pass of packing both ways
// and unpacking both took 137 us, so 113); of f32 53 us, 6.3 TB/s (with 32 bytes of a
// lane beside each other 104).  Rows of 4091 take 38 us, in single values 93.
template <class T>
__global__ __launch_bounds__(256) void k_f8_unpack(F8DequantizeArgs a, uint32_t chunks)
{
    constexpr uint32_t V = 16 / sizeof(T);
    const uint64_t item = (uint64_t)blockIdx.x * 4u + (threadIdx.x >> 6), row = item / chunks;
    if (row >= a.rows) return;
    const uint8_t *codes = a.codes + row * f8_code_bytes(a.cols), *scales = a.scales + row * f8_scale_bytes(a.cols);
    T *out = static_cast<T *>(a.out) + row * a.ld;
#pragma unroll
    for (uint32_t i = 0; i < 8 / V; i++) {
        const uint64_t col = item % chunks * 512u + i * (64u * V) + (threadIdx.x & 63u) * V;
        if (col >= a.cols) return;
        uint32_t code[V / 4];
        __builtin_memcpy(code, __builtin_assume_aligned(codes + col, V), V);
        const float s = mx_scale(scales[col / F8_BLOCK]);
        T t[V];
#pragma unroll
        for (uint32_t w = 0; w < V / 4; w++) {
            const f32x2 p = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(code[w], s, false), q = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(code[w], s, true);
            t[4 * w] = Elem<T>::put(p.x);
            t[4 * w + 1] = Elem<T>::put(p.y);
            t[4 * w + 2] = Elem<T>::put(q.x);
            t[4 * w + 3] = Elem<T>::put(q.y);
        }
        if (a.cols - col >= V) {
            Chunk c;
            __builtin_memcpy(&c, t, 16);
            __builtin_nontemporal_store(c, reinterpret_cast<Chunk *>(out + col));
            continue;
        }
#pragma unroll
        for (uint32_t c = 0; c + 1 < V; c++)   // a row's last few
            if (col + c < a.cols) out[col + c] = t[c];
    }
}

template <class T>
hipError_t dequantize_as(const F8DequantizeArgs &a, hipStream_t s)
{
    const uint32_t chunks = (uint32_t)((a.cols + 511) / 512);
    const uint64_t most = most_blocks(256) * 4 / chunks;   // rows of a launch
    for (uint64_t r = 0; r < a.rows; r += most) {
        F8DequantizeArgs part = a;
        part.codes += r * f8_code_bytes(a.cols);
        part.scales += r * f8_scale_bytes(a.cols);
        part.rows = a.rows - r < most ? a.rows - r : most;
        part.out = static_cast<T *>(a.out) + r * a.ld;
        k_f8_unpack<T><<<dim3((uint32_t)((part.rows * chunks + 3) / 4)), 256, 0, s>>>(part, chunks);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_groups(const GroupsArgs &a, hipStream_t s)
{
    const uint64_t want = (a.blocks + a.blocks2 + GROUP_THREADS - 1) / GROUP_THREADS;
    k_groups<<<dim3((uint32_t)(want < 1 ? 1 : want < 256 ? want : 256)), GROUP_THREADS, 0, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_f8_quantize(const F8QuantizeArgs &a, uint32_t dtype, hipStream_t s)
{
    if (dtype == DT_F32) return quantize_as<float>(a, s);
    if (dtype == DT_BF16) return quantize_as<__bf16>(a, s);
    return quantize_as<_Float16>(a, s);
}

hipError_t launch_f8_dequantize(const F8DequantizeArgs &a, uint32_t dtype, hipStream_t s)
{
    if (dtype == DT_F32) return dequantize_as<float>(a, s);
    if (dtype == DT_BF16) return dequantize_as<__bf16>(a, s);
    return dequantize_as<_Float16>(a, s);
}

}  // namespace pccl
