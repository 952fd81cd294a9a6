// Microscaled 4-bit floating point (OCP Microscaling Formats, version 1.0:
// blocks of 32 E2M1 values with one E8M0 scale): packing and unpacking.
//
// For a block with largest magnitude a: e = max(floor(log2 a) - 2, -127), the
// scale byte is e + 127, and each value becomes the E2M1 value nearest to
// x / 2^e (ties to the even code, 6 at most).  A block of zeros has the byte
// 0, a block holding a NaN or an infinity the byte 255 (NaN).  Dividing by a
// power of two and rounding once is exact arithmetic, so the codes do not
// depend on how the work is split.
#include "pccl_ops.h"

namespace pccl {
namespace {

// ---- packing ---------------------------------------------------------------

template <class T>
struct MxIn;
// bits of the magnitude that order like the magnitude, and the scale byte
template <>
struct MxIn<float> {
    static __device__ uint32_t byte(uint32_t top)
    {
        if (top >= 0x7F800000u) return 255u;
        const uint32_t f = top >> 23;
        return f > 2u ? f - 2u : 0u;
    }
};
template <>
struct MxIn<__bf16> {
    static __device__ uint32_t byte(uint32_t top) { return MxIn<float>::byte(top << 16); }
};
template <>
struct MxIn<_Float16> {
    static __device__ uint32_t byte(uint32_t top)
    {
        if (top >= 0x7C00u) return 255u;
        const float v = (float)__builtin_bit_cast(_Float16, (uint16_t)top);
        return MxIn<float>::byte(__float_as_uint(v));
    }
};

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

// Eight values of one lane: 16-bit types hold two to a word.
template <class T>
struct Oct {
    static constexpr int W = sizeof(T) * 2;   // words
    uint32_t w[W];
};

// Global memory is read 16 bytes at a time from any address, so rows need not
// start on 16 bytes (2040 x 1500 of bf16, both directions: 13.5 us with values
// read one by one, 10.9 us this way); only a row's last ones are read one by one.
template <class T>
__device__ inline Oct<T> load8(const T *p, uint64_t left)
{
    Oct<T> o;
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

// Largest magnitude of the eight, as ordered bits.
template <class T>
__device__ inline uint32_t top_of(const Oct<T> &o)
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

// Two values to a byte (the first in the low half) at byte B of `old`.
template <class T, int B>
__device__ inline uint32_t cvt2(uint32_t old, uint32_t pair, float scale)
{
    if constexpr (__is_same(T, __bf16))
        return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(old, __builtin_bit_cast(bf16x2, pair), scale, B);
    else
        return __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(old, __builtin_bit_cast(f16x2, pair), scale, B);
}
template <int B>
__device__ inline uint32_t cvt2(uint32_t old, float a, float b, float scale)
{
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(old, a, b, scale, B);
}

template <class T>
__device__ inline uint32_t codes8(const Oct<T> &o, uint32_t byte)
{
    if (byte == 255u) return 0u;
    const float s = mx_scale(byte);
    uint32_t r = 0;
    if constexpr (sizeof(T) == 4) {
        r = cvt2<0>(r, __uint_as_float(o.w[0]), __uint_as_float(o.w[1]), s);
        r = cvt2<1>(r, __uint_as_float(o.w[2]), __uint_as_float(o.w[3]), s);
        r = cvt2<2>(r, __uint_as_float(o.w[4]), __uint_as_float(o.w[5]), s);
        r = cvt2<3>(r, __uint_as_float(o.w[6]), __uint_as_float(o.w[7]), s);
    } else {
        r = cvt2<T, 0>(r, o.w[0], s);
        r = cvt2<T, 1>(r, o.w[1], s);
        r = cvt2<T, 2>(r, o.w[2], s);
        r = cvt2<T, 3>(r, o.w[3], s);
    }
    return r;
}

constexpr uint32_t TILE = 128;   // rows and columns of a workgroup's tile: one stored step either way

// One workgroup packs a tile of 128 x 128 values; each of its four waves has
// 32 rows, one block of the columns' packing.  A lane holds eight values of a
// row; four lanes share a block of the rows' packing.  For the columns the
// wave's part goes through LDS, where a lane then reads two columns of 32
// rows.  Memory-bound: every value is read once for both directions (16384 x
// 8192 of bf16 both ways: 112 us, 3.7 TB/s).
template <class T, bool ROWS>
__global__ __launch_bounds__(256) void k_mx_quantize(MxQuantizeArgs a, uint32_t col_tiles)
{
    __shared__ __align__(16) uint32_t part[4][32 * TILE * sizeof(T) / 4];
    __shared__ __align__(16) uint8_t tsc[TILE][4];
    const T *x = static_cast<const T *>(a.x);
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    const uint32_t tr = blockIdx.x / col_tiles, tc = blockIdx.x % col_tiles;
    const uint64_t row0 = (uint64_t)tr * TILE + wave * 32u;
    const uint32_t c0 = (lane & 15u) * 8u;
    const uint64_t col = (uint64_t)tc * TILE + c0;
    const uint64_t cb = mx_code_bytes(a.cols), sb = mx_scale_bytes(a.cols);
    Oct<T> o[8];
#pragma unroll
    for (int p = 0; p < 8; p++) {
        const uint64_t r = row0 + p * 4 + (lane >> 4);
        if (r < a.rows && col < a.cols) {
            o[p] = load8<T>(x + r * a.ld + col, a.cols - col);
        } else {
#pragma unroll
            for (int i = 0; i < Oct<T>::W; i++) o[p].w[i] = 0;
        }
    }
#pragma unroll
    for (int p = 0; p < 8; p++) {
        u32x4 *q = reinterpret_cast<u32x4 *>(&part[wave][((p * 4 + (lane >> 4)) * TILE + c0) * sizeof(T) / 4]);
#pragma unroll
        for (int i = 0; i < Oct<T>::W / 4; i++)
            q[i] = u32x4{o[p].w[4 * i], o[p].w[4 * i + 1], o[p].w[4 * i + 2], o[p].w[4 * i + 3]};
    }
    if (ROWS) {
#pragma unroll
        for (int p = 0; p < 8; p++) {
            const uint64_t r = row0 + p * 4 + (lane >> 4);
            uint32_t t = top_of(o[p]);
            uint32_t u = (uint32_t)__shfl_xor((int)t, 1);
            t = u > t ? u : t;
            u = (uint32_t)__shfl_xor((int)t, 2);
            t = u > t ? u : t;
            const uint32_t byte = MxIn<T>::byte(t);
            const uint32_t code = codes8(o[p], byte);
            if (r < a.rows) {
                *reinterpret_cast<uint32_t *>(a.codes + r * cb + col / 2) = code;
                if ((lane & 3u) == 0) a.scales[r * sb + col / MX_BLOCK] = (uint8_t)byte;
            }
        }
    }
    __syncthreads();
    const uint64_t cbt = mx_code_bytes(a.rows), sbt = mx_scale_bytes(a.rows);
    const uint32_t c = lane * 2;
    u32x4 out[2];
    uint32_t byte[2];
    if constexpr (sizeof(T) == 4) {
        float v[2][32];
        uint32_t top[2] = {0, 0};
#pragma unroll
        for (int r = 0; r < 32; r++) {
            const u32x2 w = *reinterpret_cast<const u32x2 *>(&part[wave][r * TILE + c]);
            v[0][r] = __uint_as_float(w.x);
            v[1][r] = __uint_as_float(w.y);
            const uint32_t p = w.x & 0x7FFFFFFFu, q = w.y & 0x7FFFFFFFu;
            top[0] = p > top[0] ? p : top[0];
            top[1] = q > top[1] ? q : top[1];
        }
#pragma unroll
        for (int h = 0; h < 2; h++) {
            byte[h] = MxIn<T>::byte(top[h]);
            const float s = mx_scale(byte[h]);
#pragma unroll
            for (int q = 0; q < 4; q++) {
                uint32_t t = 0;
                t = cvt2<0>(t, v[h][8 * q], v[h][8 * q + 1], s);
                t = cvt2<1>(t, v[h][8 * q + 2], v[h][8 * q + 3], s);
                t = cvt2<2>(t, v[h][8 * q + 4], v[h][8 * q + 5], s);
                t = cvt2<3>(t, v[h][8 * q + 6], v[h][8 * q + 7], s);
                out[h][q] = byte[h] == 255u ? 0u : t;
            }
        }
    } else {
        uint32_t w[32];
        u16x2 top = {0, 0};
#pragma unroll
        for (int r = 0; r < 32; r++) {
            w[r] = part[wave][r * (TILE / 2) + lane];
            top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, w[r] & 0x7FFF7FFFu));
        }
#pragma unroll
        for (int h = 0; h < 2; h++) {
            byte[h] = MxIn<T>::byte(h ? top.y : top.x);
            const float s = mx_scale(byte[h]);
            const uint32_t sel = h ? 0x07060302u : 0x05040100u;   // the column's halves of two rows
#pragma unroll
            for (int q = 0; q < 4; q++) {
                uint32_t t = 0;
                t = cvt2<T, 0>(t, __builtin_amdgcn_perm(w[8 * q + 1], w[8 * q], sel), s);
                t = cvt2<T, 1>(t, __builtin_amdgcn_perm(w[8 * q + 3], w[8 * q + 2], sel), s);
                t = cvt2<T, 2>(t, __builtin_amdgcn_perm(w[8 * q + 5], w[8 * q + 4], sel), s);
                t = cvt2<T, 3>(t, __builtin_amdgcn_perm(w[8 * q + 7], w[8 * q + 6], sel), s);
                out[h][q] = byte[h] == 255u ? 0u : t;
            }
        }
    }
    // the columns' codes go out by way of LDS, 64 bytes of a column at a
    // time; piece w of column c stands at (w + c / 2) % 4 of the column
    __syncthreads();
    u32x4 *out_lds = reinterpret_cast<u32x4 *>(part);
#pragma unroll
    for (int h = 0; h < 2; h++) {
        tsc[c + h][wave] = (uint8_t)byte[h];
        out_lds[(c + h) * 4u + ((wave + lane) & 3u)] = out[h];
    }
    __syncthreads();
#pragma unroll
    for (uint32_t i = 0; i < 2; i++) {
        const uint32_t at = i * 64u + threadIdx.x / 4, w = threadIdx.x % 4;
        const uint64_t cc = (uint64_t)tc * TILE + at;
        if (cc < a.cols)
            *reinterpret_cast<u32x4 *>(a.codes_t + cc * cbt + (uint64_t)tr * (TILE / 2) + w * 16u) = out_lds[at * 4u + ((w + at / 2) & 3u)];
    }
    const uint64_t cc = (uint64_t)tc * TILE + threadIdx.x;
    if (threadIdx.x < TILE && cc < a.cols)
        *reinterpret_cast<uint32_t *>(a.scales_t + cc * sbt + (uint64_t)tr * 4u) =
            *reinterpret_cast<const uint32_t *>(tsc[threadIdx.x]);
}

// The rows alone: a wave packs 512 values of eight rows at a time, so that what
// it reads, its codes and its scales are contiguous (1 KiB, 256 and 16 bytes;
// 8192 x 8192 of bf16: 36.5 us, 4.7 TB/s).
template <class T>
__global__ __launch_bounds__(256) void k_mx_rows(MxQuantizeArgs a, uint32_t chunks)
{
    const T *x = static_cast<const T *>(a.x);
    const uint32_t lane = threadIdx.x & 63u;
    const uint64_t item = (uint64_t)blockIdx.x * 4u + (threadIdx.x >> 6);
    const uint64_t row0 = item / chunks * 8u, col = item % chunks * 512u + lane * 8u;
    const uint64_t cb = mx_code_bytes(a.cols), sb = mx_scale_bytes(a.cols);
    if (row0 >= a.rows) return;
    Oct<T> o[8];
#pragma unroll
    for (int p = 0; p < 8; p++) {
        const uint64_t r = row0 + p;
        if (r < a.rows && col < a.cols) {
            o[p] = load8<T>(x + r * a.ld + col, a.cols - col);
        } else {
#pragma unroll
            for (int i = 0; i < Oct<T>::W; i++) o[p].w[i] = 0;
        }
    }
#pragma unroll
    for (int p = 0; p < 8; p++) {
        const uint64_t r = row0 + p;
        uint32_t t = top_of(o[p]);
        uint32_t u = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)t, 0xB1, 0xF, 0xF, false);   // lanes 1 0 3 2 of four
        t = u > t ? u : t;
        u = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)t, 0x4E, 0xF, 0xF, false);            // lanes 2 3 0 1
        t = u > t ? u : t;
        const uint32_t byte = MxIn<T>::byte(t);
        const uint32_t code = codes8(o[p], byte);
        // four blocks' scales to a word, at the first of their sixteen lanes
        uint32_t word = byte;
        word |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)byte, 0x104, 0xF, 0xF, false) << 8;
        word |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)byte, 0x108, 0xF, 0xF, false) << 16;
        word |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)byte, 0x10C, 0xF, 0xF, false) << 24;
        if (r < a.rows && col / 2 < cb) {
            *reinterpret_cast<uint32_t *>(a.codes + r * cb + col / 2) = code;
            if (lane % 16 == 0) *reinterpret_cast<uint32_t *>(a.scales + r * sb + col / MX_BLOCK) = word;
        }
    }
}

template <class T>
hipError_t quantize_as(const MxQuantizeArgs &a, hipStream_t s)
{
    if (!a.codes_t) {
        const uint32_t chunks = (uint32_t)((a.cols + 511) / 512);
        const uint64_t most = most_blocks(256) * 4 / chunks * 8;   // rows of a launch
        for (uint64_t r = 0; r < a.rows; r += most) {
            MxQuantizeArgs part = a;
            part.x = static_cast<const T *>(a.x) + r * a.ld;
            part.rows = a.rows - r < most ? a.rows - r : most;
            part.codes += r * mx_code_bytes(a.cols);
            part.scales += r * mx_scale_bytes(a.cols);
            const uint64_t items = (part.rows + 7) / 8 * chunks;
            k_mx_rows<T><<<dim3((uint32_t)((items + 3) / 4)), 256, 0, s>>>(part, chunks);
        }
        return hipGetLastError();
    }
    const uint32_t ct = (uint32_t)((a.cols + TILE - 1) / TILE), rt = (uint32_t)((a.rows + TILE - 1) / TILE);
    const dim3 grid(ct * rt);
    if (a.codes) {
        k_mx_quantize<T, true><<<grid, 256, 0, s>>>(a, ct);
    } else {
        k_mx_quantize<T, false><<<grid, 256, 0, s>>>(a, ct);
    }
    return hipGetLastError();
}

// ---- unpacking -------------------------------------------------------------

template <class T>
__device__ inline void put8(T *p, const float v[8], bool vec, uint64_t left)
{
    T t[8];
#pragma unroll
    for (int i = 0; i < 8; i++) t[i] = Elem<T>::put(v[i]);
    if (vec && left >= 8) {
        u32x4 w[sizeof t / 16];
        __builtin_memcpy(w, t, sizeof t);
#pragma unroll
        for (unsigned i = 0; i < sizeof t / 16; i++) reinterpret_cast<u32x4 *>(p)[i] = w[i];
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; i++)
        if ((uint64_t)i < left) p[i] = t[i];
}

// A wave unpacks 512 values of a row, eight a lane.  Bound by writing them
// (16384 x 8192 to bf16: 71 us, 4.8 TB/s).
template <class T>
__global__ __launch_bounds__(256) void k_mx_dequantize(MxDequantizeArgs a, uint32_t chunks, bool vec)
{
    const uint64_t item = (uint64_t)blockIdx.x * 4u + (threadIdx.x >> 6);
    const uint64_t row = item / chunks;
    const uint64_t col = (item % chunks) * 512u + (threadIdx.x & 63u) * 8u;
    if (row >= a.rows || col >= a.cols) return;
    const uint32_t code = *reinterpret_cast<const uint32_t *>(a.codes + row * mx_code_bytes(a.cols) + col / 2);
    const float s = mx_scale(a.scales[row * mx_scale_bytes(a.cols) + col / MX_BLOCK]);
    float v[8];
#define PAIR(i)                                                                  \
    {                                                                            \
        const f32x2 q = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, s, i);    \
        v[2 * i] = q.x;                                                          \
        v[2 * i + 1] = q.y;                                                      \
    }
    PAIR(0) PAIR(1) PAIR(2) PAIR(3)
#undef PAIR
    put8(static_cast<T *>(a.out) + row * a.ld + col, v, vec, a.cols - col);
}

template <class T>
hipError_t dequantize_as(const MxDequantizeArgs &a, hipStream_t s)
{
    const bool vec = (reinterpret_cast<uintptr_t>(a.out) | (a.ld * sizeof(T))) % 16 == 0;
    const uint32_t chunks = (uint32_t)((a.cols + 511) / 512);
    const uint64_t most = most_blocks(256) * 4 / chunks;   // rows of a launch
    for (uint64_t r = 0; r < a.rows; r += most) {
        MxDequantizeArgs part = a;
        part.codes += r * mx_code_bytes(a.cols);
        part.scales += r * mx_scale_bytes(a.cols);
        part.rows = a.rows - r < most ? a.rows - r : most;
        part.out = static_cast<T *>(a.out) + r * a.ld;
        k_mx_dequantize<T><<<dim3((uint32_t)((part.rows * chunks + 3) / 4)), 256, 0, s>>>(part, chunks, vec);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_mx_quantize(const MxQuantizeArgs &a, uint32_t dtype, hipStream_t s)
{
    if (dtype == DT_F32) return quantize_as<float>(a, s);
    if (dtype == DT_BF16) return quantize_as<__bf16>(a, s);
    return quantize_as<_Float16>(a, s);
}

hipError_t launch_mx_dequantize(const MxDequantizeArgs &a, uint32_t dtype, hipStream_t s)
{
    if (dtype == DT_F32) return dequantize_as<float>(a, s);
    if (dtype == DT_BF16) return dequantize_as<__bf16>(a, s);
    return dequantize_as<_Float16>(a, s);
}

}  // namespace pccl
