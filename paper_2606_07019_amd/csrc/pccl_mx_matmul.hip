// The product of two microscaled operands, out[m][n] = sum over k of
// A[m][k] B[n][k], on the matrix units' 4-bit form: one instruction takes
// 16 rows of each operand over 128 values of k with a scale byte for every
// row and block of 32, and sums in 32 bits.  Lane l of a wave gives row
// l % 16 of an operand, block l / 16 of the step (16 bytes of codes), and gets
// four sums: rows 4 (l / 16) ... + 3 of the first operand, row l % 16 of the
// second.  B goes first, so a lane's sums are neighbours in out.
#include "pccl_ops.h"

namespace pccl {
namespace {

__device__ inline f32x4 mfma_mx(u32x4 a, uint32_t as, u32x4 b, uint32_t bs, f32x4 c)
{
    const i32x8 x = {(int)a.x, (int)a.y, (int)a.z, (int)a.w, 0, 0, 0, 0};
    const i32x8 y = {(int)b.x, (int)b.y, (int)b.z, (int)b.w, 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, c, 4, 4, 0, (int)as, 0, (int)bs);
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

constexpr int SKINNY_WAVES = 8;

// Up to 16 MT rows of A: bound by reading B once.  A workgroup has 16 rows of
// B; its waves share out k, read both operands straight into registers (no
// row of B is used twice, A's come from L2) and join their sums in LDS, in the
// waves' order.
template <class T, int MT>
__global__ __launch_bounds__(64 * SKINNY_WAVES) void k_mx_skinny(MxMatmulArgs a, bool vec)
{
    __shared__ f32x4 sums[SKINNY_WAVES][MT][64];
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    const uint32_t r = lane & 15u, g = lane >> 4;
    const uint32_t steps = (uint32_t)mx_steps(a.k);
    const uint64_t cb = mx_code_bytes(a.k), sb = mx_scale_bytes(a.k);
    const uint64_t n0 = (uint64_t)blockIdx.x * 16u;
    const uint64_t row = n0 + r < a.n ? n0 + r : a.n - 1;
    const uint8_t *bp = a.b + row * cb + g * 16u, *bsp = a.bs + row * sb;
    const uint8_t *ap[MT], *asp[MT];
#pragma unroll
    for (int t = 0; t < MT; t++) {
        const uint64_t m = (uint64_t)t * 16u + r < a.m ? (uint64_t)t * 16u + r : a.m - 1;
        ap[t] = a.a + m * cb + g * 16u;
        asp[t] = a.as + m * sb;
    }
    const uint32_t per = (steps + SKINNY_WAVES - 1) / SKINNY_WAVES;
    const uint32_t s0 = wave * per, s1 = s0 + per < steps ? s0 + per : steps;
    f32x4 acc[MT] = {};
    const uint32_t sh = g * 8u;
    for (uint32_t s = s0; s < s1; s++) {
        const u32x4 b = *reinterpret_cast<const u32x4 *>(bp + (uint64_t)s * 64u);
        const uint32_t bs = *reinterpret_cast<const uint32_t *>(bsp + (uint64_t)s * 4u) >> sh;
#pragma unroll
        for (int t = 0; t < MT; t++) {
            const u32x4 x = *reinterpret_cast<const u32x4 *>(ap[t] + (uint64_t)s * 64u);
            const uint32_t xs = *reinterpret_cast<const uint32_t *>(asp[t] + (uint64_t)s * 4u) >> sh;
            acc[t] = mfma_mx(b, bs, x, xs, acc[t]);
        }
    }
#pragma unroll
    for (int t = 0; t < MT; t++) sums[wave][t][lane] = acc[t];
    __syncthreads();
    if (threadIdx.x < 64 * MT) {
        const uint32_t t = threadIdx.x >> 6;
        f32x4 v = sums[0][t][lane];
#pragma unroll
        for (int w = 1; w < SKINNY_WAVES; w++) v += sums[w][t][lane];
        const uint64_t m = (uint64_t)t * 16u + r;
        if (m < a.m) store4(static_cast<T *>(a.out), a.ld, m, n0 + g * 4u, a.n, v, vec);
    }
}

// ---- many rows ---------------------------------------------------------------

typedef const __attribute__((address_space(1))) void *gptr;
typedef __attribute__((address_space(3))) void *lptr;

// A tile of BM x BN sums; WM x WN waves.  A stage is 256 values of k (128
// bytes of codes a row, whole lines), copied from memory straight to LDS, two
// stages in turn: the next one's copies run while this one is multiplied.
// In LDS chunk c (16 bytes) of row r stands at chunk c ^ (r / 2 % 8) of the
// row, so the 16 lanes that read one chunk of 16 rows meet every bank once.
template <class T, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void k_mx_tile(MxMatmulArgs a, uint32_t mt, uint32_t nt, bool vec)
{
    constexpr int THREADS = 64 * WM * WN, TM = BM / WM / 16, TN = BN / WN / 16;
    constexpr int CODES = (BM + BN) * 128, SCALES = (BM + BN) * 8;
    extern __shared__ __align__(16) uint8_t lds[];
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t r = lane & 15u, g = lane >> 4;
    // tiles are dealt so that the workgroups of one XCD (every eighth of the
    // launch) have neighbouring tiles, eight rows of tiles by column
    const uint32_t total = mt * nt, id = blockIdx.x;
    const uint32_t q = total / 8, rest = total % 8, xcd = id % 8;
    const uint32_t tile = xcd * q + (xcd < rest ? xcd : rest) + id / 8;
    constexpr uint32_t GROUP = 8;
    const uint32_t grp = tile / (GROUP * nt), first = grp * GROUP;
    const uint32_t gm = mt - first < GROUP ? mt - first : GROUP;
    const uint32_t in = tile - grp * GROUP * nt;
    const uint64_t m0 = (uint64_t)(first + in % gm) * BM, n0 = (uint64_t)(in / gm) * BN;

    const uint64_t cb = mx_code_bytes(a.k), sb = mx_scale_bytes(a.k);
    const uint32_t steps = (uint32_t)mx_steps(a.k), stages = (steps + 1) / 2;

    // what this thread copies: row and chunk of each of its 16-byte pieces
    // (A's rows first, then B's), row and word of its scales
    constexpr int PIECES = CODES / 16 / THREADS, WORDS = (SCALES / 4 + THREADS - 1) / THREADS;
    static_assert(CODES / 16 % THREADS == 0 && BM * 8 % THREADS == 0, "whole pieces a thread");
    const uint8_t *src[PIECES];
    uint32_t off[PIECES];
#pragma unroll
    for (int i = 0; i < PIECES; i++) {
        const uint32_t piece = i * THREADS + threadIdx.x, row = piece / 8, c = (piece % 8) ^ (row / 2 % 8);
        off[i] = c * 16u;
        if (row < BM) {
            const uint64_t m = m0 + row < a.m ? m0 + row : a.m - 1;
            src[i] = a.a + m * cb;
        } else {
            const uint64_t n = n0 + row - BM < a.n ? n0 + row - BM : a.n - 1;
            src[i] = a.b + n * cb;
        }
    }
    const uint8_t *ssrc[WORDS];
    uint32_t soff[WORDS];
#pragma unroll
    for (int i = 0; i < WORDS; i++) {
        const uint32_t w = i * THREADS + threadIdx.x, row = w / 2;
        soff[i] = (w % 2) * 4u;
        if (row < BM) {
            const uint64_t m = m0 + row < a.m ? m0 + row : a.m - 1;
            ssrc[i] = a.as + m * sb;
        } else {
            const uint64_t n = n0 + row - BM < a.n ? n0 + row - BM : a.n - 1;
            ssrc[i] = a.bs + n * sb;
        }
    }
    auto copy = [&](uint32_t stage) {
        uint8_t *base = lds + (stage & 1u) * (CODES + SCALES);
        const uint32_t kb = stage * 128u, ks = stage * 8u;
#pragma unroll
        for (int i = 0; i < PIECES; i++) {
            // a row may end inside the last stage: its first half is read instead (and not multiplied)
            const uint32_t at = kb + off[i] < cb ? kb + off[i] : kb + off[i] - 64u;
            __builtin_amdgcn_global_load_lds((gptr)(src[i] + at), (lptr)(base + (i * THREADS + wave * 64u) * 16u), 16, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < WORDS; i++) {
            const uint32_t at = ks + soff[i] < sb ? ks + soff[i] : ks + soff[i] - 4u;
            if (i * THREADS + wave * 64u < SCALES / 4)
                __builtin_amdgcn_global_load_lds((gptr)(ssrc[i] + at), (lptr)(base + CODES + (i * THREADS + wave * 64u) * 4u), 4, 0, 0);
        }
    };

    const uint32_t wm = wave / WN, wn = wave % WN;
    const uint32_t arow = wm * (BM / WM) + r, brow = BM + wn * (BN / WN) + r;
    f32x4 acc[TM][TN] = {};
    if (stages) copy(0);
    for (uint32_t st = 0; st < stages; st++) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // this wave's copies of the stage have landed
        __builtin_amdgcn_s_barrier();                      // everyone's have, and nobody reads the other buffer
        asm volatile("" ::: "memory");
        if (st + 1 < stages) copy(st + 1);
        const uint8_t *base = lds + (st & 1u) * (CODES + SCALES);
        const uint32_t subs = steps - st * 2 < 2 ? 1u : 2u;
        for (uint32_t u = 0; u < subs; u++) {
            u32x4 x[TM], y[TN];
            uint32_t xs[TM], ys[TN];
#pragma unroll
            for (int i = 0; i < TM; i++) {
                const uint32_t row = arow + i * 16u;
                x[i] = *reinterpret_cast<const u32x4 *>(base + row * 128u + (((u * 4u + g) ^ (row / 2 % 8)) * 16u));
                xs[i] = base[CODES + row * 8u + u * 4u + g];
            }
#pragma unroll
            for (int i = 0; i < TN; i++) {
                const uint32_t row = brow + i * 16u;
                y[i] = *reinterpret_cast<const u32x4 *>(base + row * 128u + (((u * 4u + g) ^ (row / 2 % 8)) * 16u));
                ys[i] = base[CODES + row * 8u + u * 4u + g];
            }
#pragma unroll
            for (int i = 0; i < TM; i++)
#pragma unroll
                for (int j = 0; j < TN; j++) acc[i][j] = mfma_mx(y[j], ys[j], x[i], xs[i], acc[i][j]);
        }
    }
#pragma unroll
    for (int i = 0; i < TM; i++) {
        const uint64_t m = m0 + arow + i * 16u;
        if (m >= a.m) continue;
#pragma unroll
        for (int j = 0; j < TN; j++)
            store4(static_cast<T *>(a.out), a.ld, m, n0 + (brow - r - BM) + j * 16u + g * 4u, a.n, acc[i][j], vec);
    }
}

template <class T, int MT>
hipError_t skinny(const MxMatmulArgs &a, bool vec, hipStream_t s)
{
    k_mx_skinny<T, MT><<<dim3((uint32_t)((a.n + 15) / 16)), 64 * SKINNY_WAVES, 0, s>>>(a, vec);
    return hipGetLastError();
}

template <class T, int BM, int BN, int WM, int WN>
hipError_t tiled(const MxMatmulArgs &a, bool vec, hipStream_t s)
{
    constexpr uint32_t bytes = 2 * ((BM + BN) * 128 + (BM + BN) * 8);
    static const hipError_t once = hipFuncSetAttribute(reinterpret_cast<const void *>(&k_mx_tile<T, BM, BN, WM, WN>),
                                                       hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (once != hipSuccess) return once;
    const uint32_t mt = (uint32_t)((a.m + BM - 1) / BM), nt = (uint32_t)((a.n + BN - 1) / BN);
    k_mx_tile<T, BM, BN, WM, WN><<<dim3(mt * nt), 64 * WM * WN, bytes, s>>>(a, mt, nt, vec);
    return hipGetLastError();
}

template <class T>
hipError_t matmul_as(const MxMatmulArgs &a, hipStream_t s)
{
    const bool vec = (reinterpret_cast<uintptr_t>(a.out) | (a.ld * sizeof(T))) % (4 * sizeof(T)) == 0;
    if (a.m <= 16) return skinny<T, 1>(a, vec, s);
    if (a.m <= 32) return skinny<T, 2>(a, vec, s);
    if (a.m <= 48) return skinny<T, 3>(a, vec, s);
    if (a.m <= 64) return skinny<T, 4>(a, vec, s);
    const uint64_t big = ((a.m + 255) / 256) * ((a.n + 255) / 256);
    if (big >= 256) return tiled<T, 256, 256, 2, 4>(a, vec, s);
    return tiled<T, 128, 128, 2, 2>(a, vec, s);
}

}  // namespace

size_t mx_matmul_workspace(uint64_t, uint64_t, uint64_t) { return 0; }

hipError_t launch_mx_matmul(const MxMatmulArgs &a, uint32_t dtype, hipStream_t s)
{
    if (dtype == DT_F32) return matmul_as<float>(a, s);
    if (dtype == DT_BF16) return matmul_as<__bf16>(a, s);
    return matmul_as<_Float16>(a, s);
}

}  // namespace pccl
