// The router's row step, shared by the router and the mixture-of-experts
// layer: a wave holds a row of logits, VPL neighbouring ones a lane, as
// 32-bit keys that order like the logits, and draws the largest k.
#pragma once

#include "pccl_ops.h"

namespace pccl {

constexpr uint32_t KEY_EMPTY = 0x007FFFFFu;   // minus infinity; nothing at or below it is drawn

// A float as a whole number that orders like it: a NaN above everything,
// both zeros alike.
__device__ inline uint32_t key_of(float v)
{
    if (v != v) return 0xFFFFFFFFu;
    const uint32_t b = __float_as_uint(v + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ inline float of_key(uint32_t k)
{
    return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}

// Reductions over a wave on the lanes' own paths (rows of 16, then across);
// the result is uniform.
template <int CTRL, int ROWS>
__device__ inline uint32_t dpp(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xF, false);
}
__device__ inline uint32_t dpp_max(uint32_t v)
{
    auto up = [&](uint32_t w) { v = w > v ? w : v; };
    up(dpp<0x111, 0xF>(v));   // one, two, four and eight lanes along a row of 16
    up(dpp<0x112, 0xF>(v));
    up(dpp<0x114, 0xF>(v));
    up(dpp<0x118, 0xF>(v));
    up(dpp<0x142, 0xA>(v));   // a row's last lane into the next row
    up(dpp<0x143, 0xC>(v));   // the lower half's last lane into the upper half
    return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}
__device__ inline float dpp_sum(float v)
{
    auto up = [&](uint32_t w) { v += __uint_as_float(w); };
    up(dpp<0x111, 0xF>(__float_as_uint(v)));
    up(dpp<0x112, 0xF>(__float_as_uint(v)));
    up(dpp<0x114, 0xF>(__float_as_uint(v)));
    up(dpp<0x118, 0xF>(__float_as_uint(v)));
    up(dpp<0x142, 0xA>(__float_as_uint(v)));
    up(dpp<0x143, 0xC>(__float_as_uint(v)));
    return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), 63));
}

// Draws the k largest of the row's keys, ties to the lowest index, and gives
// lane j the j-th pick's index (-1: none left) and weight: the softmax over
// the whole row or, normalised, over the picks.  One pass of the statistics in
// 32 bits; a row with nothing above minus infinity has no picks.
template <int VPL>
__device__ inline void topk_row(uint32_t (&key)[VPL], uint32_t k, bool normalize, uint32_t lane, int32_t &id, float &weight)
{
    uint32_t local = 0;
#pragma unroll
    for (int i = 0; i < VPL; i++) local = key[i] > local ? key[i] : local;
    uint32_t best = dpp_max(local);
    const float top = of_key(best);
    float total = 0.f;
    if (!normalize && best > KEY_EMPTY) {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < VPL; i++)
            if (key[i] > KEY_EMPTY) sum += expf(of_key(key[i]) - top);
        total = dpp_sum(sum);
    }
    id = -1;
    uint32_t got = KEY_EMPTY;
    for (uint32_t j = 0; j < k && best > KEY_EMPTY; j++) {
        int at = VPL;
#pragma unroll
        for (int i = VPL - 1; i >= 0; i--)
            if (key[i] == best) at = i;
        const uint64_t have = __ballot(at < VPL);
        const int first = __ffsll((unsigned long long)have) - 1;
        const int pick = __builtin_amdgcn_readlane(at, first);
        if (lane == j) {
            id = first * VPL + pick;
            got = best;
        }
        local = 0;
#pragma unroll
        for (int i = 0; i < VPL; i++) {
            if ((int)lane == first && i == pick) key[i] = 0;
            local = key[i] > local ? key[i] : local;
        }
        best = dpp_max(local);
    }
    float e = got > KEY_EMPTY ? expf(of_key(got) - top) : 0.f;
    if (normalize) total = dpp_sum(e);
    weight = id >= 0 ? e / total : 0.f;
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
