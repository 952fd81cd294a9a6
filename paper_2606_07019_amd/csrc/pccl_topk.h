// The router's row step, shared by the router and the mixture-of-experts
// layer: the lanes of a row of logits (16 up to 256 experts, four rows a wave;
// a whole wave beyond) hold V neighbouring ones each as whole numbers that
// order like them, and draw the largest k.
#pragma once

#include "pccl_ops.h"

namespace pccl {

// Logits as keys that order like them, a NaN above everything, both zeros
// alike; nothing at or below EMPTY (minus infinity) is drawn.  A 16-bit logit
// leaves room for its index, lowest first: such keys differ, so the largest
// one says where it stands.
template <class T>
struct Key;
template <>
struct Key<float> {
    static constexpr uint32_t EMPTY = 0x007FFFFFu;
    static constexpr bool INDEXED = false;
    static __device__ uint32_t of(float v, uint32_t)
    {
        if (v != v) return 0xFFFFFFFFu;
        const uint32_t b = __float_as_uint(v + 0.f);
        return b & 0x80000000u ? ~b : b | 0x80000000u;
    }
    static __device__ float value(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }
    static __device__ uint32_t index(uint32_t) { return 0; }
};
template <class T>
struct Key16 {
    static constexpr bool INDEXED = true;
    static __device__ uint32_t of(T v, uint32_t e)
    {
        uint32_t b = __builtin_bit_cast(uint16_t, v);
        b = b & 0x8000u ? 0x10000u - b : b + 0x8000u;   // minus zero lands on plus zero
        if (v != v) b = 0xFFFFu;
        return b << 16 | (0xFFFFu - e);
    }
    static __device__ float value(uint32_t k)
    {
        k >>= 16;
        const uint16_t b = (uint16_t)(k & 0x8000u ? k - 0x8000u : 0x10000u - k);
        return (float)__builtin_bit_cast(T, b);
    }
    static __device__ uint32_t index(uint32_t k) { return 0xFFFFu - (k & 0xFFFFu); }
};
template <>
struct Key<__bf16> : Key16<__bf16> {
    static constexpr uint32_t EMPTY = 0x0080FFFFu;   // minus infinity, any index
};
template <>
struct Key<_Float16> : Key16<_Float16> {
    static constexpr uint32_t EMPTY = 0x0400FFFFu;
};

template <int CTRL, int ROWS>
__device__ inline uint32_t dpp(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xF, false);
}

// Reductions over the LANES lanes of a row, on the lanes' own paths; every
// lane of the row gets the result.
template <int LANES, class Op>
__device__ inline uint32_t reduce(uint32_t v, Op op)
{
    if constexpr (LANES == 16) {   // rotations within 16 lanes
        v = op(v, dpp<0x128, 0xF>(v));
        v = op(v, dpp<0x124, 0xF>(v));
        v = op(v, dpp<0x122, 0xF>(v));
        return op(v, dpp<0x121, 0xF>(v));
    } else {                       // shifts (zeros come in), a row's last lane into the next, the lower half's into the upper
        v = op(v, dpp<0x111, 0xF>(v));
        v = op(v, dpp<0x112, 0xF>(v));
        v = op(v, dpp<0x114, 0xF>(v));
        v = op(v, dpp<0x118, 0xF>(v));
        v = op(v, dpp<0x142, 0xA>(v));
        v = op(v, dpp<0x143, 0xC>(v));
        return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
    }
}
template <int LANES>
__device__ inline uint32_t row_max(uint32_t v)
{
    return reduce<LANES>(v, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}
template <int LANES>
__device__ inline float row_sum(float v)
{
    return __uint_as_float(reduce<LANES>(__float_as_uint(v), [](uint32_t a, uint32_t b) {
        return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
    }));
}

// Lanes of a row for so many experts, and the picks a lane may have to hold.
constexpr uint32_t NARROW_EXPERTS = 256;
template <int LANES>
constexpr int picks_held() { return LANES == 16 ? (int)ROUTE_MAX_TOPK / 16 : 1; }

// Draws the k largest of the row's keys, ties to the lowest index; lane `sub`
// of the row gets pick sub (and 16 + sub where a row has 16 lanes): its index
// (-1: none left) and weight, the softmax over the whole row or, normalised,
// over the picks, with its statistics in 32 bits.  A row with nothing above
// minus infinity has no picks.
template <class T, int LANES, int V>
__device__ inline void topk_row(uint32_t (&key)[V], uint32_t k, bool normalize, uint32_t sub, int32_t (&id)[picks_held<LANES>()],
                                float (&weight)[picks_held<LANES>()])
{
    typedef Key<T> K;
    constexpr int HELD = picks_held<LANES>();
    auto local_max = [&]() {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < V; i++) m = key[i] > m ? key[i] : m;
        return m;
    };
    uint32_t best = row_max<LANES>(local_max());
    const float top = K::value(best);
    float total = 0.f;
    if (!normalize) {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < V; i++) sum += key[i] > K::EMPTY ? expf(K::value(key[i]) - top) : 0.f;
        total = row_sum<LANES>(sum);
    }
    uint32_t got[HELD];
#pragma unroll
    for (int h = 0; h < HELD; h++) {
        id[h] = -1;
        got[h] = 0;
    }
    for (uint32_t j = 0; j < k; j++) {
        if (LANES == 64 && best <= K::EMPTY) break;
        uint32_t at;
        if constexpr (K::INDEXED) {
            at = K::index(best);
#pragma unroll
            for (int i = 0; i < V; i++) key[i] = key[i] == best ? 0u : key[i];
        } else {
            uint32_t mine = 0;   // the lowest index is the largest of the negated ones
#pragma unroll
            for (int i = V - 1; i >= 0; i--) mine = key[i] == best ? ~(sub * V + i) : mine;
            at = ~row_max<LANES>(mine);
#pragma unroll
            for (int i = 0; i < V; i++) key[i] = at == sub * V + i ? 0u : key[i];
        }
#pragma unroll
        for (int h = 0; h < HELD; h++)
            if (sub + 16u * h == j) {
                got[h] = best;
                id[h] = best > K::EMPTY ? (int32_t)at : -1;
            }
        best = row_max<LANES>(local_max());
    }
    float e[HELD], sum = 0.f;
#pragma unroll
    for (int h = 0; h < HELD; h++) {
        e[h] = id[h] >= 0 ? expf(K::value(got[h]) - top) : 0.f;
        sum += e[h];
    }
    if (normalize) total = row_sum<LANES>(sum);
#pragma unroll
    for (int h = 0; h < HELD; h++) weight[h] = id[h] >= 0 ? e[h] / total : 0.f;
}

// Exclusive scan over the threads of a workgroup of WAVES waves; `sums` is
// LDS of WAVES words.  Returns the sum of the threads before, `all` the total.
template <int WAVES>
__device__ inline uint32_t block_scan(uint32_t v, uint32_t *sums, uint32_t &all)
{
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    uint32_t x = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t y = (uint32_t)__shfl_up((int)x, o);
        if (lane >= (uint32_t)o) x += y;
    }
    __syncthreads();
    if (lane == 63u) sums[wave] = x;
    __syncthreads();
    uint32_t before = 0;
    all = 0;
#pragma unroll
    for (int w = 0; w < WAVES; w++) {
        if ((uint32_t)w < wave) before += sums[w];
        all += sums[w];
    }
    return before + x - v;
}

}  // namespace pccl
