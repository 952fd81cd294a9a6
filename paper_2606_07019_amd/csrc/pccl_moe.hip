// A mixture-of-experts layer for a few tokens:
//
//   l = x Wr^T;  w, ids = top k of softmax(l)
//   y_t = sum_j w_tj Wd[e] (silu(Wg[e] x_t) * (Wu[e] x_t)),  e = ids_tj
//
// With few tokens the experts' weights are read once and used for a handful of
// columns, so the layer is bound by that reading; the matrix units are used
// because they take 16 tokens at the price of one.  Weight rows are the first
// operand of the 16x16x32 products (lane l: row l % 16, eight values of k per
// product), the expert's tokens the second.  Weights go from memory to
// registers, each used once there.
#include "pccl_topk.h"

namespace pccl {
namespace {

constexpr uint32_t STEP = 128;      // values of k a wave takes at a time: four products
constexpr int WAVES = 4;
constexpr int TILES = 4;            // tiles of 16 tokens that share one reading of the weights

// What the kernels of one call hand on, carved from the workspace.
struct MoeSpace {
    float *part_logits;   // [splits][tokens][experts]
    int32_t *ids;         // [tokens][topk]
    float *weights;       // [tokens][topk]
    int32_t *place;       // [tokens][topk]: the slot's place in expert order, -1 for none
    uint32_t *active;     // [0]: experts in use; then the experts
    uint32_t *first;      // [experts in use + 1]: where each one's places start
    uint32_t *slots;      // [places]: token of each place
    uint16_t *hi, *lo;    // [places][inner size padded to a step]: the inner values, in two parts
    float *outs;          // [places][hidden]
    uint64_t inner;       // padded inner size
    uint32_t splits;
};

// Workgroups that share the router's product over hidden: enough for the
// chip's compute units to have one each.
__host__ inline uint32_t logit_splits(uint32_t experts, uint32_t hidden)
{
    const uint32_t tiles = (experts + 15) / 16, steps = (hidden + STEP - 1) / STEP;
    const uint32_t want = (128 + tiles - 1) / tiles;
    return want < steps ? want : steps;
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
    m.splits = logit_splits(experts, hidden);
    m.inner = (inter + STEP - 1) / STEP * (uint64_t)STEP;
    m.part_logits = (float *)take((size_t)m.splits * tokens * experts * 4);
    m.ids = (int32_t *)take(places * 4);
    m.weights = (float *)take(places * 4);
    m.place = (int32_t *)take(places * 4);
    m.active = (uint32_t *)take((experts + 1ull) * 4);
    m.first = (uint32_t *)take((experts + 1ull) * 4);
    m.slots = (uint32_t *)take(places * 4);
    m.hi = (uint16_t *)take(places * m.inner * 2);
    m.lo = (uint16_t *)take(places * m.inner * 2);
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

// Eight values from k on of a row that ends at `end`; zeros beyond it.
template <bool VEC>
__device__ inline u32x4 row8(const uint16_t *row, uint32_t k, uint32_t end)
{
    if (VEC) return k < end ? *reinterpret_cast<const u32x4 *>(row + k) : u32x4{0, 0, 0, 0};
    uint16_t t[8];
#pragma unroll
    for (int i = 0; i < 8; i++) t[i] = k + i < end ? row[k + i] : (uint16_t)0;
    u32x4 v;
    __builtin_memcpy(&v, t, 16);
    return v;
}

// One step of weights: what a lane holds of a row, and its four first
// operands.  16-bit rows: product i takes values 32 i + 8 (l / 16) ... + 7 of
// the step; microscaled rows: a lane's 16 bytes are one block, product i takes
// its values 8 i ... + 7 (both operands count k alike, so the order is free).
template <class T, bool VEC>
struct Plain {
    typedef T C;                         // the products' type
    static constexpr bool MX = false;
    u32x4 v[4];
    __device__ void load(const uint16_t *row, const uint8_t *, uint32_t step, uint32_t g, uint32_t end)
    {
#pragma unroll
        for (int i = 0; i < 4; i++) v[i] = row8<VEC>(row, step * STEP + i * 32u + g * 8u, end);
    }
    __device__ u32x4 operand(int i) const { return v[i]; }
    static __device__ uint32_t at(uint32_t step, uint32_t g, int i) { return step * STEP + i * 32u + g * 8u; }
};
struct Micro {
    typedef __bf16 C;                    // holds every microscaled value exactly
    static constexpr bool MX = true;
    u32x4 v;
    uint32_t byte;
    __device__ void load(const uint16_t *row, const uint8_t *scales, uint32_t step, uint32_t g, uint32_t)
    {
        v = *reinterpret_cast<const u32x4 *>(reinterpret_cast<const uint8_t *>(row) + step * 64u + g * 16u);
        byte = scales[step * 4u + g];
    }
    __device__ u32x4 operand(int i) const
    {
        const float s = mx_scale(byte);
        const uint32_t c = v[i];
        u32x4 r;
        r.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 0));
        r.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 1));
        r.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 2));
        r.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 3));
        return r;
    }
    static __device__ uint32_t at(uint32_t step, uint32_t g, int i) { return step * STEP + g * 32u + i * 8u; }
};

// A 32-bit value in two parts of the products' type: v = hi HI + lo LO.  The
// second holds what the first rounds away, which leaves 2^-17 of the value at
// most with bf16.  f16 has few exponents: its first part is kept 2^8 smaller,
// so that values up to 2^24 fit, and its second 2^11 larger than the rest is,
// so that small values keep their digits (2^-28 is left at most).
template <class C>
struct Parts;
template <>
struct Parts<__bf16> {
    static constexpr float HI = 1.f, LO = 1.f;
};
template <>
struct Parts<_Float16> {
    static constexpr float HI = 256.f, LO = 0.125f;
};
template <class C>
__device__ inline void split(float v, uint16_t &hi, uint16_t &lo)
{
    const C h = (C)(v * (1.f / Parts<C>::HI));
    const C l = (C)((v - (float)h * Parts<C>::HI) * (1.f / Parts<C>::LO));
    hi = __builtin_bit_cast(uint16_t, h);
    lo = __builtin_bit_cast(uint16_t, l);
}

// ---- the router's product -------------------------------------------------------

// A workgroup: 16 experts, 16 tokens, one part of hidden, shared out over its waves.
template <class T, bool VEC>
__global__ __launch_bounds__(64 * WAVES) void k_moe_logits(MoeArgs a, MoeSpace m)
{
    __shared__ f32x4 sums[WAVES][64];
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, r = lane & 15u, g = lane >> 4;
    const uint32_t e0 = blockIdx.x * 16u, t0 = blockIdx.z * 16u;
    const uint32_t e = e0 + r < a.experts ? e0 + r : a.experts - 1;
    const uint32_t t = t0 + r < a.tokens ? t0 + r : a.tokens - 1;
    const uint16_t *wrow = static_cast<const uint16_t *>(a.router) + (uint64_t)e * a.hidden;
    const uint16_t *xrow = static_cast<const uint16_t *>(a.x) + (uint64_t)t * a.ld_x;
    const uint32_t products = (a.hidden + 31) / 32;
    const uint32_t parts = m.splits * WAVES, mine = blockIdx.y * WAVES + wave;
    f32x4 acc = {};
    for (uint32_t p = mine; p < products; p += parts) {
        const uint32_t k = p * 32u + g * 8u;
        acc = Frag<T>::mul(row8<VEC>(wrow, k, a.hidden), row8<VEC>(xrow, k, a.hidden), acc);
    }
    sums[wave][lane] = acc;
    __syncthreads();
    if (wave) return;
    f32x4 v = sums[0][lane];
#pragma unroll
    for (int w = 1; w < WAVES; w++) v += sums[w][lane];
    if (t0 + r < a.tokens) {
        float *out = m.part_logits + ((uint64_t)blockIdx.y * a.tokens + t0 + r) * a.experts;
#pragma unroll
        for (int i = 0; i < 4; i++)
            if (e0 + g * 4 + i < a.experts) out[e0 + g * 4 + i] = v[i];
    }
}

// ---- the picks --------------------------------------------------------------------

constexpr int PICK_WAVES = 16;

// One workgroup: every token's picks, then the experts in use with their
// tokens.  One bit for every (expert, token) as in the router.
template <int VPL>
__global__ __launch_bounds__(64 * PICK_WAVES) void k_moe_pick(MoeArgs a, MoeSpace m)
{
    constexpr int SETS = MOE_MAX_TOKENS / 64;
    __shared__ uint64_t rows[SETS][64 * VPL];
    __shared__ uint32_t base[64 * VPL], sums[PICK_WAVES];
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    for (uint32_t i = threadIdx.x; i < SETS * 64 * VPL; i += 64 * PICK_WAVES) (&rows[0][0])[i] = 0;
    __syncthreads();
    for (uint32_t t = wave; t < a.tokens; t += PICK_WAVES) {
        const bool there = !a.mask || a.mask[t];
        uint32_t key[VPL];
#pragma unroll
        for (int i = 0; i < VPL; i++) {
            const uint32_t e = lane * VPL + i;
            key[i] = 0;
            if (there && e < a.experts) {
                float v = 0.f;
                for (uint32_t s = 0; s < m.splits; s++) v += m.part_logits[((uint64_t)s * a.tokens + t) * a.experts + e];
                key[i] = key_of(v);
            }
        }
        int32_t id;
        float w;
        topk_row<VPL>(key, a.topk, a.normalize, lane, id, w);
        if (lane < a.topk) {
            m.ids[t * a.topk + lane] = id;
            m.weights[t * a.topk + lane] = w;
            if (id >= 0) atomicOr((unsigned long long *)&rows[t / 64][id], 1ull << (t % 64));   // LDS; bits of a set
        }
    }
    __threadfence_block();
    __syncthreads();
    // threads take experts in order (all of them at most 1,024 = the workgroup)
    const uint32_t e = threadIdx.x;
    uint32_t c = 0;
    if (e < a.experts) {
#pragma unroll
        for (int q = 0; q < SETS; q++) c += (uint32_t)__popcll(rows[q][e]);
    }
    uint32_t places, used;
    const uint32_t at = block_scan<PICK_WAVES>(c, sums, places);
    const uint32_t nth = block_scan<PICK_WAVES>(c ? 1u : 0u, sums, used);
    if (e < a.experts) base[e] = at;
    if (c) {
        m.active[1 + nth] = e;
        m.first[nth] = at;
    }
    if (threadIdx.x == 0) {
        m.active[0] = used;
        m.first[used] = places;
    }
    __syncthreads();
    for (uint32_t s = threadIdx.x; s < a.tokens * a.topk; s += 64 * PICK_WAVES) {
        const int32_t id = m.ids[s];
        const uint32_t t = s / a.topk;
        int32_t p = -1;
        if (id >= 0) {
            uint32_t below = 0;
            for (uint32_t q = 0; q < t / 64; q++) below += (uint32_t)__popcll(rows[q][id]);
            below += (uint32_t)__popcll(rows[t / 64][id] & ((1ull << (t % 64)) - 1ull));
            p = (int32_t)(base[id] + below);
            m.slots[p] = t;
        }
        m.place[s] = p;
    }
}

// ---- gate and up ---------------------------------------------------------------------

// Sums of one step's four products for the rows of `w` and NT tiles of tokens.
template <class T, class W, bool VEC, int NT>
__device__ inline void step_x(const W &w, const uint16_t *const (&x)[NT], uint32_t step, uint32_t g, uint32_t end, f32x4 (&acc)[NT])
{
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const u32x4 a = w.operand(i);
#pragma unroll
        for (int t = 0; t < NT; t++) {
            const u32x4 b = row8<VEC>(x[t], W::at(step, g, i), end);
            if constexpr (__is_same(T, typename W::C)) {
                acc[t] = Frag<T>::mul(a, b, acc[t]);
            } else {   // f16 tokens against microscaled weights: two bf16 parts hold an f16 value exactly
                uint16_t h[8], l[8];
                _Float16 v[8];
                __builtin_memcpy(v, &b, 16);
#pragma unroll
                for (int q = 0; q < 8; q++) split<__bf16>((float)v[q], h[q], l[q]);
                u32x4 bh, bl;
                __builtin_memcpy(&bh, h, 16);
                __builtin_memcpy(&bl, l, 16);
                acc[t] = Frag<__bf16>::mul(a, bh, acc[t]);
                acc[t] = Frag<__bf16>::mul(a, bl, acc[t]);
            }
        }
    }
}

template <class T, class W, bool VEC, int NT>
__device__ inline void up_tile(const MoeArgs &a, const MoeSpace &m, const uint16_t *gate, const uint16_t *lift, const uint8_t *gs,
                               const uint8_t *ls, uint32_t p0, uint32_t n, uint32_t i0, f32x4 *sums)
{
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, r = lane & 15u, g = lane >> 4;
    const uint16_t *x[NT];
#pragma unroll
    for (int t = 0; t < NT; t++) {
        const uint32_t at = t * 16u + r < n ? t * 16u + r : n - 1;
        x[t] = static_cast<const uint16_t *>(a.x) + (uint64_t)m.slots[p0 + at] * a.ld_x;
    }
    const uint32_t steps = (a.hidden + STEP - 1) / STEP;
    const uint32_t per = (steps + WAVES - 1) / WAVES;
    const uint32_t s0 = wave * per, s1 = s0 + per < steps ? s0 + per : steps;
    f32x4 ga[NT] = {}, ua[NT] = {};
    for (uint32_t s = s0; s < s1; s++) {
        W gw, uw;
        gw.load(gate, gs, s, g, a.hidden);
        uw.load(lift, ls, s, g, a.hidden);
        step_x<T, W, VEC, NT>(gw, x, s, g, a.hidden, ga);
        step_x<T, W, VEC, NT>(uw, x, s, g, a.hidden, ua);
    }
    __syncthreads();   // the sums of the tokens before have been read
#pragma unroll
    for (int t = 0; t < NT; t++) {
        sums[(wave * 2 * NT + t) * 64 + lane] = ga[t];
        sums[(wave * 2 * NT + NT + t) * 64 + lane] = ua[t];
    }
    __syncthreads();
    if (threadIdx.x < NT * 64) {
        const uint32_t t = threadIdx.x >> 6;
        f32x4 gv = {}, uv = {};
#pragma unroll
        for (int w = 0; w < WAVES; w++) {
            gv += sums[(w * 2 * NT + t) * 64 + lane];
            uv += sums[(w * 2 * NT + NT + t) * 64 + lane];
        }
        if (t * 16u + r < n) {
            const uint64_t at = (uint64_t)(p0 + t * 16u + r) * m.inner + i0 + g * 4u;
            uint16_t hi[4], lo[4];
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const float v = i0 + g * 4 + i < a.inter ? gv[i] / (1.f + expf(-gv[i])) * uv[i] : 0.f;
                split<typename W::C>(v, hi[i], lo[i]);
            }
            __builtin_memcpy(__builtin_assume_aligned(m.hi + at, 8), hi, 8);
            __builtin_memcpy(__builtin_assume_aligned(m.lo + at, 8), lo, 8);
        }
    }
}

// A workgroup: 16 inner values of one expert in use, for all its tokens.
template <class T, class W, bool VEC>
__global__ __launch_bounds__(64 * WAVES) void k_moe_up(MoeArgs a, MoeSpace m)
{
    __shared__ f32x4 sums[WAVES * 2 * TILES * 64];
    if (blockIdx.y >= m.active[0]) return;
    const uint32_t e = m.active[1 + blockIdx.y], r = threadIdx.x & 15u;
    const uint32_t p0 = m.first[blockIdx.y], p1 = m.first[blockIdx.y + 1];
    const uint32_t i0 = blockIdx.x * 16u;   // inner values past the last are padding: rows clamped, zeros stored
    const uint32_t row = i0 + r < a.inter ? i0 + r : a.inter - 1;
    const uint64_t bytes = W::MX ? mx_code_bytes(a.hidden) : a.hidden * 2ull, sb = mx_scale_bytes(a.hidden);
    const uint64_t gr = (uint64_t)e * 2u * a.inter + row, ur = gr + a.inter;
    const uint16_t *gate = reinterpret_cast<const uint16_t *>(static_cast<const char *>(a.up) + gr * bytes);
    const uint16_t *lift = reinterpret_cast<const uint16_t *>(static_cast<const char *>(a.up) + ur * bytes);
    const uint8_t *gs = W::MX ? a.up_scales + gr * sb : nullptr, *ls = W::MX ? a.up_scales + ur * sb : nullptr;
    for (uint32_t p = p0; p < p1; p += 16 * TILES) {
        const uint32_t n = p1 - p < 16 * TILES ? p1 - p : 16 * TILES;
        if (n <= 16) up_tile<T, W, VEC, 1>(a, m, gate, lift, gs, ls, p, n, i0, sums);
        else if (n <= 32) up_tile<T, W, VEC, 2>(a, m, gate, lift, gs, ls, p, n, i0, sums);
        else up_tile<T, W, VEC, 4>(a, m, gate, lift, gs, ls, p, n, i0, sums);
    }
}

// ---- down ---------------------------------------------------------------------------

template <class T, class W, int NT>
__device__ inline void down_tile(const MoeArgs &a, const MoeSpace &m, const uint16_t *row, const uint8_t *sc, uint32_t p0, uint32_t n,
                                 uint32_t h0, f32x4 *sums)
{
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, r = lane & 15u, g = lane >> 4;
    const uint16_t *hi[NT], *lo[NT];
#pragma unroll
    for (int t = 0; t < NT; t++) {
        const uint64_t at = (uint64_t)(p0 + (t * 16u + r < n ? t * 16u + r : n - 1)) * m.inner;
        hi[t] = m.hi + at;
        lo[t] = m.lo + at;
    }
    const uint32_t steps = (a.inter + STEP - 1) / STEP;
    const uint32_t per = (steps + WAVES - 1) / WAVES;
    const uint32_t s0 = wave * per, s1 = s0 + per < steps ? s0 + per : steps;
    f32x4 acc[NT] = {}, rest[NT] = {};
    for (uint32_t s = s0; s < s1; s++) {
        W w;
        w.load(row, sc, s, g, a.inter);
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const u32x4 x = w.operand(i);
            const uint32_t k = W::at(s, g, i);
#pragma unroll
            for (int t = 0; t < NT; t++) {
                acc[t] = Frag<typename W::C>::mul(x, *reinterpret_cast<const u32x4 *>(hi[t] + k), acc[t]);
                rest[t] = Frag<typename W::C>::mul(x, *reinterpret_cast<const u32x4 *>(lo[t] + k), rest[t]);
            }
        }
    }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < NT; t++) sums[(wave * NT + t) * 64 + lane] = acc[t] * Parts<typename W::C>::HI + rest[t] * Parts<typename W::C>::LO;
    __syncthreads();
    if (threadIdx.x < NT * 64) {
        const uint32_t t = threadIdx.x >> 6;
        f32x4 v = {};
#pragma unroll
        for (int w = 0; w < WAVES; w++) v += sums[(w * NT + t) * 64 + lane];
        if (t * 16u + r < n) {
            float *out = m.outs + (uint64_t)(p0 + t * 16u + r) * a.hidden + h0 + g * 4u;
#pragma unroll
            for (int i = 0; i < 4; i++)
                if (h0 + g * 4 + i < a.hidden) out[i] = v[i];
        }
    }
}

// A workgroup: 16 outputs of one expert in use, for all its tokens.
template <class T, class W>
__global__ __launch_bounds__(64 * WAVES) void k_moe_down(MoeArgs a, MoeSpace m)
{
    __shared__ f32x4 sums[WAVES * TILES * 64];
    if (blockIdx.y >= m.active[0]) return;
    const uint32_t e = m.active[1 + blockIdx.y], r = threadIdx.x & 15u;
    const uint32_t p0 = m.first[blockIdx.y], p1 = m.first[blockIdx.y + 1];
    const uint32_t h0 = blockIdx.x * 16u;
    const uint64_t bytes = W::MX ? mx_code_bytes(a.inter) : a.inter * 2ull;
    const uint64_t row = (uint64_t)e * a.hidden + (h0 + r < a.hidden ? h0 + r : a.hidden - 1);
    const uint16_t *w = reinterpret_cast<const uint16_t *>(static_cast<const char *>(a.down) + row * bytes);
    const uint8_t *sc = W::MX ? a.down_scales + row * mx_scale_bytes(a.inter) : nullptr;
    for (uint32_t p = p0; p < p1; p += 16 * TILES) {
        const uint32_t n = p1 - p < 16 * TILES ? p1 - p : 16 * TILES;
        if (n <= 16) down_tile<T, W, 1>(a, m, w, sc, p, n, h0, sums);
        else if (n <= 32) down_tile<T, W, 2>(a, m, w, sc, p, n, h0, sums);
        else down_tile<T, W, 4>(a, m, w, sc, p, n, h0, sums);
    }
}

// Each token's weighted sum over its picks, in their order; zeros without any.
template <class T>
__global__ __launch_bounds__(256) void k_moe_join(MoeArgs a, MoeSpace m)
{
    const uint32_t t = blockIdx.y, h = blockIdx.x * 256u + threadIdx.x;
    if (h >= a.hidden) return;
    float v = 0.f;
    for (uint32_t j = 0; j < a.topk; j++) {
        const int32_t p = m.place[t * a.topk + j];
        if (p >= 0) v += m.weights[t * a.topk + j] * m.outs[(uint64_t)p * a.hidden + h];
    }
    static_cast<T *>(a.y)[(uint64_t)t * a.ld_y + h] = Elem<T>::put(v);
}

template <class T, class WU, class WD, bool VEC>
hipError_t experts_as(const MoeArgs &a, const MoeSpace &m, hipStream_t s)
{
    const uint64_t places = (uint64_t)a.tokens * a.topk;
    const uint32_t most = places < a.experts ? (uint32_t)places : a.experts;
    k_moe_up<T, WU, VEC><<<dim3((uint32_t)(m.inner / 16), most), 64 * WAVES, 0, s>>>(a, m);
    k_moe_down<T, WD><<<dim3((a.hidden + 15) / 16, most), 64 * WAVES, 0, s>>>(a, m);
    k_moe_join<T><<<dim3((a.hidden + 255) / 256, a.tokens), 256, 0, s>>>(a, m);
    return hipGetLastError();
}

template <class T>
hipError_t moe_as(const MoeArgs &a, hipStream_t s)
{
    MoeSpace m;
    carve(m, a.ws, a.tokens, a.experts, a.topk, a.hidden, a.inter);
    auto aligned = [](const void *p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; };
    // whole groups of eight values: the router's and the tokens' rows are read 16 bytes at a time
    const bool vx = aligned(a.x) && a.ld_x % 8 == 0 && a.hidden % 8 == 0;
    const bool vr = vx && aligned(a.router);
    const dim3 grid((a.experts + 15) / 16, m.splits, (a.tokens + 15) / 16);
    if (vr) k_moe_logits<T, true><<<grid, 64 * WAVES, 0, s>>>(a, m);
    else k_moe_logits<T, false><<<grid, 64 * WAVES, 0, s>>>(a, m);
    if (a.experts <= 64) k_moe_pick<1><<<1, 64 * PICK_WAVES, 0, s>>>(a, m);
    else if (a.experts <= 128) k_moe_pick<2><<<1, 64 * PICK_WAVES, 0, s>>>(a, m);
    else if (a.experts <= 256) k_moe_pick<4><<<1, 64 * PICK_WAVES, 0, s>>>(a, m);
    else if (a.experts <= 512) k_moe_pick<8><<<1, 64 * PICK_WAVES, 0, s>>>(a, m);
    else k_moe_pick<16><<<1, 64 * PICK_WAVES, 0, s>>>(a, m);
    if (a.up_scales) return vx ? experts_as<T, Micro, Micro, true>(a, m, s) : experts_as<T, Micro, Micro, false>(a, m, s);
    const bool vu = vx && aligned(a.up), vd = aligned(a.down) && a.inter % 8 == 0;
    if (vu && vd) return experts_as<T, Plain<T, true>, Plain<T, true>, true>(a, m, s);
    return experts_as<T, Plain<T, false>, Plain<T, false>, false>(a, m, s);
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
