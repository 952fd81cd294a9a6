// The router: softmax over the experts, the k largest of every token, and the
// slots (token * k + position) in expert order, from which the chunks of an
// All-to-Allv are cut; and the gradient with respect to the logits.
//
//   p = softmax(l), ids = the k largest, w_i = p[ids_i]   (or / sum of those)
//   plain:       dl_j = p_j (g_j [j picked] - sum_i g_i w_i)
//   normalised:  dl_j = w_j (g_j - sum_i g_i w_i) at the picks, 0 elsewhere
//
// Experts differ within a row, so a workgroup of 64 rows has one bit for every
// (expert, row): a slot's place among its expert's slots is the count of bits
// below its row's, which needs no atomics whose order could matter.
#include "pccl_topk.h"

namespace pccl {
namespace {

constexpr int THREADS = 256, WAVES = 4;

template <class T, int VPL>
__device__ inline void load_row(const T *row, uint32_t experts, uint32_t lane, bool vec, float (&v)[VPL])
{
    const uint32_t e0 = lane * VPL;
    T t[VPL];
    if (vec && e0 + VPL <= experts) {
        __builtin_memcpy(t, __builtin_assume_aligned(row + e0, sizeof t < 16 ? sizeof t : 16), sizeof t);
#pragma unroll
        for (int i = 0; i < VPL; i++) v[i] = Elem<T>::get(t[i]);
        return;
    }
#pragma unroll
    for (int i = 0; i < VPL; i++) v[i] = e0 + i < experts ? Elem<T>::get(row[e0 + i]) : 0.f;
}

// Counts of the experts before each expert, for a workgroup that holds every
// expert's count in LDS; up to 4 experts a thread.
__device__ inline uint32_t scan_counts(uint32_t *base, uint32_t experts, uint32_t *sums)
{
    constexpr int PER = ROUTE_MAX_EXPERTS / THREADS;
    uint32_t c[PER], mine = 0, all;
#pragma unroll
    for (int i = 0; i < PER; i++) {
        const uint32_t e = threadIdx.x * PER + i;
        c[i] = e < experts ? base[e] : 0u;
        mine += c[i];
    }
    uint32_t at = block_scan<WAVES>(mine, sums, all);
#pragma unroll
    for (int i = 0; i < PER; i++) {
        const uint32_t e = threadIdx.x * PER + i;
        if (e < experts) base[e] = at;
        at += c[i];
    }
    __syncthreads();
    return all;
}

// The slots of one workgroup's rows in their places; base: where each
// expert's slots of these rows start.
__device__ inline void place_slots(const RouteArgs &a, const uint64_t *rows, const uint32_t *base, uint64_t row0, uint32_t n, uint32_t total)
{
    for (uint32_t s = threadIdx.x; s < n * a.topk; s += THREADS) {
        const uint32_t r = s / a.topk;
        const uint64_t slot = row0 * a.topk + s;
        const int32_t e = a.ids[slot];
        if (e >= 0) {
            const uint64_t below = rows[e] & ((1ull << r) - 1ull);
            a.order[base[e] + (uint32_t)__popcll(below)] = (int32_t)slot;
        }
        if (slot >= total) a.order[slot] = -1;
    }
}

template <class T, int VPL>
__global__ __launch_bounds__(THREADS) void k_route(RouteArgs a, bool vec, uint32_t groups)
{
    __shared__ uint64_t rows[64 * VPL];
    __shared__ uint32_t base[64 * VPL], sums[WAVES];
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    const uint64_t row0 = (uint64_t)blockIdx.x * ROUTE_ROWS;
    const uint32_t n = (uint32_t)(a.tokens - row0 < ROUTE_ROWS ? a.tokens - row0 : ROUTE_ROWS);
    for (uint32_t e = threadIdx.x; e < a.experts; e += THREADS) rows[e] = 0;
    __syncthreads();
    const T *logits = static_cast<const T *>(a.logits);
    for (uint32_t r = wave; r < n; r += WAVES) {
        const uint64_t row = row0 + r;
        float v[VPL];
        load_row<T, VPL>(logits + row * a.ld, a.experts, lane, vec, v);
        const bool there = !a.mask || a.mask[row];
        uint32_t key[VPL];
#pragma unroll
        for (int i = 0; i < VPL; i++) key[i] = there && lane * VPL + i < a.experts ? key_of(v[i]) : 0u;
        int32_t id;
        float w;
        topk_row<VPL>(key, a.topk, a.normalize, lane, id, w);
        if (lane < a.topk) {
            a.ids[row * a.topk + lane] = id;
            a.weights[row * a.topk + lane] = w;
            if (id >= 0) atomicOr((unsigned long long *)&rows[id], 1ull << r);   // LDS; bits of a set
        }
    }
    __threadfence_block();
    __syncthreads();
    if (groups > 1) {
        for (uint32_t e = threadIdx.x; e < a.experts; e += THREADS)
            a.hist[(uint64_t)e * groups + blockIdx.x] = (uint32_t)__popcll(rows[e]);
        return;
    }
    // one workgroup has every row: the counts and the order here and now
    for (uint32_t e = threadIdx.x; e < a.experts; e += THREADS) {
        const uint32_t c = (uint32_t)__popcll(rows[e]);
        base[e] = c;
        a.counts[e] = (int32_t)c;
    }
    __syncthreads();
    const uint32_t total = scan_counts(base, a.experts, sums);
    place_slots(a, rows, base, row0, n, total);
}

// One workgroup per expert: where each row group's slots start, and the count.
__global__ __launch_bounds__(THREADS) void k_route_scan(RouteArgs a, uint32_t groups)
{
    __shared__ uint32_t sums[WAVES];
    uint32_t *h = a.hist + (uint64_t)blockIdx.x * groups;
    uint32_t before = 0;
    for (uint32_t g0 = 0; g0 < groups; g0 += THREADS) {
        const uint32_t g = g0 + threadIdx.x;
        const uint32_t c = g < groups ? h[g] : 0u;
        uint32_t all;
        const uint32_t at = block_scan<WAVES>(c, sums, all);
        if (g < groups) h[g] = before + at;
        before += all;
    }
    if (threadIdx.x == 0) a.counts[blockIdx.x] = (int32_t)before;
}

__global__ __launch_bounds__(THREADS) void k_route_order(RouteArgs a, uint32_t groups)
{
    __shared__ uint64_t rows[ROUTE_MAX_EXPERTS];
    __shared__ uint32_t base[ROUTE_MAX_EXPERTS], sums[WAVES];
    const uint64_t row0 = (uint64_t)blockIdx.x * ROUTE_ROWS;
    const uint32_t n = (uint32_t)(a.tokens - row0 < ROUTE_ROWS ? a.tokens - row0 : ROUTE_ROWS);
    for (uint32_t e = threadIdx.x; e < a.experts; e += THREADS) {
        rows[e] = 0;
        base[e] = (uint32_t)a.counts[e];
    }
    __syncthreads();
    for (uint32_t s = threadIdx.x; s < n * a.topk; s += THREADS) {
        const int32_t e = a.ids[row0 * a.topk + s];
        if (e >= 0) atomicOr((unsigned long long *)&rows[e], 1ull << (s / a.topk));
    }
    const uint32_t total = scan_counts(base, a.experts, sums);
    for (uint32_t e = threadIdx.x; e < a.experts; e += THREADS) base[e] += a.hist[(uint64_t)e * groups + blockIdx.x];
    __syncthreads();
    place_slots(a, rows, base, row0, n, total);
}

template <class T, int VPL>
__global__ __launch_bounds__(THREADS) void k_route_backward(RouteBackwardArgs a, bool vec)
{
    const uint32_t lane = threadIdx.x & 63u;
    const uint64_t row = (uint64_t)blockIdx.x * WAVES + (threadIdx.x >> 6);
    if (row >= a.tokens) return;
    int32_t id = -1;
    float w = 0.f, g = 0.f;
    if (lane < a.topk) {
        const uint64_t s = row * a.topk + lane;
        id = a.ids[s];
        w = id >= 0 ? a.weights[s] : 0.f;
        g = id >= 0 ? a.dweights[s] : 0.f;
    }
    const float gw = id >= 0 ? g * w : 0.f;
    const float inner = dpp_sum(gw);
    float d[VPL];
    if (a.normalize) {
#pragma unroll
        for (int i = 0; i < VPL; i++) d[i] = 0.f;
    } else {
        float v[VPL], sum = 0.f;
        load_row<T, VPL>(static_cast<const T *>(a.logits) + row * a.ld, a.experts, lane, vec, v);
        const bool there = !a.mask || a.mask[row];
        uint32_t local = 0;
#pragma unroll
        for (int i = 0; i < VPL; i++) {
            const uint32_t k = there && lane * VPL + i < a.experts ? key_of(v[i]) : 0u;
            v[i] = k > KEY_EMPTY ? v[i] : -INFINITY;
            local = k > local ? k : local;
        }
        const uint32_t best = dpp_max(local);
        const float top = best > KEY_EMPTY ? of_key(best) : 0.f;
#pragma unroll
        for (int i = 0; i < VPL; i++) {
            v[i] = expf(v[i] - top);
            sum += v[i];
        }
        const float total = dpp_sum(sum);
        const float scale = best > KEY_EMPTY ? inner / total : 0.f;
#pragma unroll
        for (int i = 0; i < VPL; i++) d[i] = -v[i] * scale;
    }
    const float mine = a.normalize ? gw - w * inner : gw;
    for (uint32_t j = 0; j < a.topk; j++) {
        const int32_t e = __builtin_amdgcn_readlane(id, (int)j);
        const float x = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(mine), (int)j));
#pragma unroll
        for (int i = 0; i < VPL; i++)
            if (e == (int32_t)(lane * VPL + i)) d[i] += x;
    }
    T *out = static_cast<T *>(a.dlogits) + row * a.ld_d;
    const uint32_t e0 = lane * VPL;
    T t[VPL];
#pragma unroll
    for (int i = 0; i < VPL; i++) t[i] = Elem<T>::put(d[i]);
    if (vec && e0 + VPL <= a.experts) {
        __builtin_memcpy(__builtin_assume_aligned(out + e0, sizeof t < 16 ? sizeof t : 16), t, sizeof t);
        return;
    }
#pragma unroll
    for (int i = 0; i < VPL; i++)
        if (e0 + i < a.experts) out[e0 + i] = t[i];
}

// A lane's neighbouring logits are read at once where every row starts on them.
template <class T, int VPL>
bool whole(const void *p, uint64_t ld)
{
    const uint64_t unit = sizeof(T) * VPL < 16 ? sizeof(T) * VPL : 16;
    return (reinterpret_cast<uintptr_t>(p) | (ld * sizeof(T))) % unit == 0;
}

template <class T, int VPL>
hipError_t route_as(const RouteArgs &a, hipStream_t s)
{
    // without tokens one workgroup still clears the counts
    const uint32_t groups = a.tokens ? (uint32_t)((a.tokens + ROUTE_ROWS - 1) / ROUTE_ROWS) : 1u;
    k_route<T, VPL><<<dim3(groups), THREADS, 0, s>>>(a, whole<T, VPL>(a.logits, a.ld), groups);
    if (groups > 1) {
        k_route_scan<<<dim3(a.experts), THREADS, 0, s>>>(a, groups);
        k_route_order<<<dim3(groups), THREADS, 0, s>>>(a, groups);
    }
    return hipGetLastError();
}

template <class T, int VPL>
hipError_t backward_as(const RouteBackwardArgs &a, hipStream_t s)
{
    const bool vec = whole<T, VPL>(a.dlogits, a.ld_d) && (a.normalize || whole<T, VPL>(a.logits, a.ld));
    k_route_backward<T, VPL><<<dim3((uint32_t)((a.tokens + WAVES - 1) / WAVES)), THREADS, 0, s>>>(a, vec);
    return hipGetLastError();
}

template <class T>
hipError_t route_lanes(const RouteArgs &a, hipStream_t s)
{
    if (a.experts <= 64) return route_as<T, 1>(a, s);
    if (a.experts <= 128) return route_as<T, 2>(a, s);
    if (a.experts <= 256) return route_as<T, 4>(a, s);
    if (a.experts <= 512) return route_as<T, 8>(a, s);
    return route_as<T, 16>(a, s);
}
template <class T>
hipError_t backward_lanes(const RouteBackwardArgs &a, hipStream_t s)
{
    if (a.experts <= 64) return backward_as<T, 1>(a, s);
    if (a.experts <= 128) return backward_as<T, 2>(a, s);
    if (a.experts <= 256) return backward_as<T, 4>(a, s);
    if (a.experts <= 512) return backward_as<T, 8>(a, s);
    return backward_as<T, 16>(a, s);
}

}  // namespace

size_t route_workspace(uint64_t tokens, uint32_t experts)
{
    const uint64_t groups = (tokens + ROUTE_ROWS - 1) / ROUTE_ROWS;
    return groups > 1 ? (size_t)(groups * experts * sizeof(uint32_t)) : 0;
}

hipError_t launch_route(const RouteArgs &a, uint32_t dtype, hipStream_t s)
{
    if (dtype == DT_F32) return route_lanes<float>(a, s);
    if (dtype == DT_BF16) return route_lanes<__bf16>(a, s);
    return route_lanes<_Float16>(a, s);
}

hipError_t launch_route_backward(const RouteBackwardArgs &a, uint32_t dtype, hipStream_t s)
{
    if (dtype == DT_F32) return backward_lanes<float>(a, s);
    if (dtype == DT_BF16) return backward_lanes<__bf16>(a, s);
    return backward_lanes<_Float16>(a, s);
}

}  // namespace pccl
