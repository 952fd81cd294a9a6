// The router: softmax over the experts, the k largest of every token, and the
// slots (token * k + position) in expert order, from which the chunks of an
// All-to-Allv are cut; and the gradient with respect to the logits.
//
//   p = softmax(l), ids = the k largest, w_i = p[ids_i]   (or / sum of those)
//   plain:       dl_j = p_j (g_j [j picked] - sum_i g_i w_i)
//   normalised:  dl_j = w_j (g_j - sum_i g_i w_i) at the picks, 0 elsewhere
//
// Experts differ within a row, so a group of 64 rows has one bit for every
// (expert, row): a slot's place among its expert's slots is the count of bits
// below its row's, which needs no atomics whose order could matter.
#include "pccl_topk.h"

namespace pccl {
namespace {

constexpr int THREADS = 1024, WAVES = 16;

// Row groups whose counts the ordering workgroups sum up themselves (bytes, in
// 16-bit sums); beyond, a kernel between finds where each group starts.  Whole
// calls, this way and with that kernel: 256 experts, 16 groups 13.4 and 15.0 us,
// 256 15.4 and 17.1, 512 23.9 and 24.1; 64 experts, 512 groups 11.6 and 12.6;
// 1,024 experts, 256 groups 36.8 and 38.2, 512 67.3 and 62.8.
constexpr uint32_t SUMMED_GROUPS = 512;
// Groups of 64 rows of one ordering workgroup.
constexpr uint32_t ORDER_GROUPS = 4;

__host__ __device__ inline uint32_t padded_experts(uint32_t experts) { return (experts + 3u) & ~3u; }

template <class T, int V>
__device__ inline void load_row(const T *row, uint32_t experts, uint32_t sub, bool vec, T (&t)[V])
{
    const uint32_t e0 = sub * V;
    if (vec && e0 + V <= experts) {
        __builtin_memcpy(t, __builtin_assume_aligned(row + e0, sizeof t < 16 ? sizeof t : 16), sizeof t);
        return;
    }
#pragma unroll
    for (int i = 0; i < V; i++) t[i] = e0 + i < experts ? row[e0 + i] : (T)0.f;
}

// Exclusive sums over the experts of a workgroup's `base`, in place.
__device__ inline uint32_t scan_counts(uint32_t *base, uint32_t experts, uint32_t *sums)
{
    const uint32_t e = threadIdx.x;   // at most 1,024 experts
    uint32_t all;
    const uint32_t at = block_scan<WAVES>(e < experts ? base[e] : 0u, sums, all);
    if (e < experts) base[e] = at;
    __syncthreads();
    return all;
}

// Bound by the picks: 32,768 x 256 of bf16 take 9.0 us with one pick and 15 with
// eight, of which reading takes 3.  Most of a pick is in the lane, where the drawn
// key is cleared and the largest of all V is found anew; the four steps between
// lanes are the lesser part.
// The picks of 64 rows, LANES lanes a row; where one workgroup has every row,
// the counts and the order too.
template <class T, int LANES, int V>
__global__ __launch_bounds__(THREADS) void k_route(RouteArgs a, bool vec, uint32_t groups)
{
    __shared__ unsigned long long rows[LANES * V];
    __shared__ uint32_t base[LANES * V], sums[WAVES];
    constexpr int HELD = picks_held<LANES>(), PER = 64 / LANES;   // rows of a wave at a time
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, sub = lane % LANES;
    const uint64_t row0 = (uint64_t)blockIdx.x * ROUTE_ROWS;
    const uint32_t n = (uint32_t)(a.tokens - row0 < ROUTE_ROWS ? a.tokens - row0 : ROUTE_ROWS);
    for (uint32_t e = threadIdx.x; e < LANES * V; e += THREADS) rows[e] = 0;
    __syncthreads();
    const T *logits = static_cast<const T *>(a.logits);
    for (uint32_t r0 = wave * PER; r0 < n; r0 += WAVES * PER) {
        const uint32_t r = r0 + lane / LANES;
        const uint64_t row = row0 + (r < n ? r : n - 1);
        T t[V];
        load_row<T, V>(logits + row * a.ld, a.experts, sub, vec, t);
        const bool there = !a.mask || a.mask[row];
        uint32_t key[V];
#pragma unroll
        for (int i = 0; i < V; i++) key[i] = there && sub * V + i < a.experts ? Key<T>::of(t[i], sub * V + i) : 0u;
        int32_t id[HELD];
        float w[HELD];
        topk_row<T, LANES, V>(key, a.topk, a.normalize, sub, id, w);
        if (r < n) {
#pragma unroll
            for (int h = 0; h < HELD; h++) {
                const uint32_t j = sub + 16u * h;
                if (j >= a.topk) continue;
                a.ids[row * a.topk + j] = id[h];
                a.weights[row * a.topk + j] = w[h];
                if (id[h] >= 0) atomicOr(&rows[id[h]], 1ull << r);   // LDS; bits of a set
            }
        }
    }
    __threadfence_block();
    __syncthreads();
    if (groups > SUMMED_GROUPS) {
        uint32_t *hist = reinterpret_cast<uint32_t *>(a.hist);
        for (uint32_t e = threadIdx.x; e < a.experts; e += THREADS) hist[(uint64_t)e * groups + blockIdx.x] = (uint32_t)__popcll(rows[e]);
        return;
    }
    if (groups > 1) {
        const uint32_t ep = padded_experts(a.experts);
        uint8_t *hist = reinterpret_cast<uint8_t *>(a.hist) + (uint64_t)blockIdx.x * ep;
        for (uint32_t e = threadIdx.x; e < ep; e += THREADS) hist[e] = e < a.experts ? (uint8_t)__popcll(rows[e]) : 0;
        return;
    }
    for (uint32_t e = threadIdx.x; e < a.experts; e += THREADS) {
        const uint32_t c = (uint32_t)__popcll(rows[e]);
        base[e] = c;
        a.counts[e] = (int32_t)c;
    }
    __syncthreads();
    const uint32_t total = scan_counts(base, a.experts, sums);
    for (uint32_t s = threadIdx.x; s < n * a.topk; s += THREADS) {
        const int32_t e = a.ids[s];
        if (e >= 0) a.order[base[e] + (uint32_t)__popcll(rows[e] & ((1ull << (s / a.topk)) - 1ull))] = (int32_t)s;
        if (s >= total) a.order[s] = -1;
    }
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

// The order of four row groups' slots.  SUM: the workgroup adds up the groups'
// counts, those before its own and all of them; threads take four experts and
// every so many-th group.  Bound by its dependent steps (32,768 x 8 slots of 256
// experts: 9 us).
template <bool SUM>
__global__ __launch_bounds__(THREADS) void k_route_order(RouteArgs a, uint32_t groups)
{
    __shared__ unsigned long long rows[ORDER_GROUPS][ROUTE_MAX_EXPERTS];
    __shared__ uint32_t base[ROUTE_MAX_EXPERTS], start[ORDER_GROUPS][ROUTE_MAX_EXPERTS], sums[WAVES];
    const uint32_t g0 = blockIdx.x * ORDER_GROUPS;
    const uint64_t row0 = (uint64_t)g0 * ROUTE_ROWS;
    const uint32_t n = (uint32_t)(a.tokens - row0 < ORDER_GROUPS * ROUTE_ROWS ? a.tokens - row0 : ORDER_GROUPS * ROUTE_ROWS);
    const uint32_t e = threadIdx.x;
#pragma unroll
    for (uint32_t q = 0; q < ORDER_GROUPS; q++)
        if (e < a.experts) rows[q][e] = 0;
    if (e < a.experts) {
        base[e] = SUM ? 0u : (uint32_t)a.counts[e];
        start[0][e] = 0;
    }
    // everything that is read goes out at once: a thread's first two slots (all
    // of them up to eight picks) and the groups' counts
    const uint32_t slots = n * a.topk;
    const int32_t *ids = a.ids + row0 * a.topk;
    int32_t mine[2];
#pragma unroll
    for (int i = 0; i < 2; i++) mine[i] = threadIdx.x + i * THREADS < slots ? ids[threadIdx.x + i * THREADS] : -1;
    auto slot_id = [&](uint32_t s) { return s < THREADS ? mine[0] : s < 2 * THREADS ? mine[1] : ids[s]; };
    uint32_t all[2] = {0, 0}, before[2] = {0, 0};
    const uint32_t quads = padded_experts(a.experts) / 4, parts = THREADS / quads, q = threadIdx.x % quads, part = threadIdx.x / quads;
    if constexpr (SUM) {
        const uint32_t *hist = a.hist + q;
        for (uint32_t g = part; part < parts && g < groups; g += 16 * parts) {
            uint32_t w[16];
#pragma unroll
            for (uint32_t i = 0; i < 16; i++) w[i] = g + i * parts < groups ? hist[(uint64_t)(g + i * parts) * quads] : 0u;
#pragma unroll
            for (uint32_t i = 0; i < 16; i++) {
                const uint32_t even = w[i] & 0x00FF00FFu, odd = (w[i] >> 8) & 0x00FF00FFu;
                all[0] += even;
                all[1] += odd;
                before[0] += g + i * parts < g0 ? even : 0u;
                before[1] += g + i * parts < g0 ? odd : 0u;
            }
        }
    }
    __syncthreads();
    for (uint32_t s = threadIdx.x; s < slots; s += THREADS) {
        const int32_t id = slot_id(s);
        const uint32_t r = s / a.topk;
        if (id >= 0) atomicOr(&rows[r / 64][id], 1ull << (r % 64));
    }
    if constexpr (SUM) {
        if (part < parts) {
#pragma unroll
            for (uint32_t i = 0; i < 4; i++) {
                const uint32_t x = q * 4 + i, sh = (i / 2) * 16;
                if (x < a.experts) {
                    atomicAdd(&base[x], (all[i % 2] >> sh) & 0xFFFFu);      // LDS; whole numbers
                    atomicAdd(&start[0][x], (before[i % 2] >> sh) & 0xFFFFu);
                }
            }
        }
        __syncthreads();
        if (blockIdx.x == 0 && e < a.experts) a.counts[e] = (int32_t)base[e];
    }
    const uint32_t total = scan_counts(base, a.experts, sums);
    if (e < a.experts) {
        uint32_t at = base[e] + (SUM ? start[0][e] : a.hist[(uint64_t)e * groups + g0]);
#pragma unroll
        for (uint32_t q = 0; q < ORDER_GROUPS; q++) {
            start[q][e] = at;
            at += (uint32_t)__popcll(rows[q][e]);
        }
    }
    __syncthreads();
    for (uint32_t s = threadIdx.x; s < slots; s += THREADS) {
        const uint32_t r = s / a.topk;
        const uint64_t slot = row0 * a.topk + s;
        const int32_t id = slot_id(s);
        if (id >= 0) a.order[start[r / 64][id] + (uint32_t)__popcll(rows[r / 64][id] & ((1ull << (r % 64)) - 1ull))] = (int32_t)slot;
        if (slot >= total) a.order[slot] = -1;
    }
}

constexpr int BACK_THREADS = 256, BACK_WAVES = 4;

// LANES lanes a row, as in the forward pass.  32,768 x 256 of bf16, normalised:
// 7.1 us with one pick and 10 with eight, of which writing dlogits takes 3; over
// the whole row 14 and 18.  A pick is handed over by two reads across lanes and
// looked for at each of the lane's V logits; the whole row's exponentials are the
// rest.
template <class T, int LANES, int V>
__global__ __launch_bounds__(BACK_THREADS) void k_route_backward(RouteBackwardArgs a, bool vec)
{
    constexpr int HELD = picks_held<LANES>(), PER = 64 / LANES;
    const uint32_t lane = threadIdx.x & 63u, sub = lane % LANES;
    const uint64_t row = ((uint64_t)blockIdx.x * BACK_WAVES + (threadIdx.x >> 6)) * PER + lane / LANES;
    const bool in = row < a.tokens;
    const uint64_t at = in ? row : a.tokens - 1;
    int32_t id[HELD];
    float mine[HELD], w[HELD], gw = 0.f;
#pragma unroll
    for (int h = 0; h < HELD; h++) {
        const uint32_t j = sub + 16u * h;
        const uint64_t s = at * a.topk + j;
        id[h] = j < a.topk ? a.ids[s] : -1;
        w[h] = id[h] >= 0 ? a.weights[s] : 0.f;
        mine[h] = id[h] >= 0 ? w[h] * a.dweights[s] : 0.f;
        gw += mine[h];
    }
    const float inner = row_sum<LANES>(gw);
    float d[V];
    if (a.normalize) {
#pragma unroll
        for (int i = 0; i < V; i++) d[i] = 0.f;
#pragma unroll
        for (int h = 0; h < HELD; h++) mine[h] -= w[h] * inner;
    } else {
        T t[V];
        load_row<T, V>(static_cast<const T *>(a.logits) + at * a.ld, a.experts, sub, vec, t);
        const bool there = !a.mask || a.mask[at];
        uint32_t local = 0;
        float v[V], sum = 0.f;
#pragma unroll
        for (int i = 0; i < V; i++) {
            const uint32_t k = there && sub * V + i < a.experts ? Key<T>::of(t[i], sub * V + i) : 0u;
            v[i] = k > Key<T>::EMPTY ? Elem<T>::get(t[i]) : -INFINITY;
            local = k > local ? k : local;
        }
        const uint32_t best = row_max<LANES>(local);
        const bool any = best > Key<T>::EMPTY;
        const float top = any ? Key<T>::value(best) : 0.f;
#pragma unroll
        for (int i = 0; i < V; i++) {
            v[i] = expf(v[i] - top);
            sum += v[i];
        }
        const float total = row_sum<LANES>(sum);
        const float scale = any ? inner / total : 0.f;
#pragma unroll
        for (int i = 0; i < V; i++) d[i] = -v[i] * scale;
    }
    // every pick's part goes to the lane that has its expert
    for (uint32_t j = 0; j < a.topk; j++) {
        const int from = (int)(lane - sub + j % 16);
        int32_t e = __shfl(id[0], LANES == 64 ? (int)j : from);
        float x = __shfl(mine[0], LANES == 64 ? (int)j : from);
        if constexpr (HELD > 1) {
            if (j >= 16) {
                e = __shfl(id[HELD - 1], from);
                x = __shfl(mine[HELD - 1], from);
            }
        }
#pragma unroll
        for (int i = 0; i < V; i++) d[i] += e == (int32_t)(sub * V + i) ? x : 0.f;
    }
    if (!in) return;
    T *out = static_cast<T *>(a.dlogits) + row * a.ld_d;
    const uint32_t e0 = sub * V;
    T t[V];
#pragma unroll
    for (int i = 0; i < V; i++) t[i] = Elem<T>::put(d[i]);
    if (vec && e0 + V <= a.experts) {
        __builtin_memcpy(__builtin_assume_aligned(out + e0, sizeof t < 16 ? sizeof t : 16), t, sizeof t);
        return;
    }
#pragma unroll
    for (int i = 0; i < V; i++)
        if (e0 + i < a.experts) out[e0 + i] = t[i];
}

// A lane's neighbouring logits are read at once where every row starts on them.
template <class T, int V>
bool whole(const void *p, uint64_t ld)
{
    const uint64_t unit = sizeof(T) * V < 16 ? sizeof(T) * V : 16;
    return (reinterpret_cast<uintptr_t>(p) | (ld * sizeof(T))) % unit == 0;
}

struct Forward {
    template <class T, int LANES, int V>
    static hipError_t run(const RouteArgs &a, hipStream_t s)
    {
        // without tokens one workgroup still clears the counts
        const uint32_t groups = a.tokens ? (uint32_t)((a.tokens + ROUTE_ROWS - 1) / ROUTE_ROWS) : 1u;
        k_route<T, LANES, V><<<dim3(groups), THREADS, 0, s>>>(a, whole<T, V>(a.logits, a.ld), groups);
        const dim3 order((groups + ORDER_GROUPS - 1) / ORDER_GROUPS);
        if (groups > SUMMED_GROUPS) {
            k_route_scan<<<dim3(a.experts), THREADS, 0, s>>>(a, groups);
            k_route_order<false><<<order, THREADS, 0, s>>>(a, groups);
        } else if (groups > 1) {
            k_route_order<true><<<order, THREADS, 0, s>>>(a, groups);
        }
        return hipGetLastError();
    }
};

struct Backward {
    template <class T, int LANES, int V>
    static hipError_t run(const RouteBackwardArgs &a, hipStream_t s)
    {
        const bool vec = whole<T, V>(a.dlogits, a.ld_d) && (a.normalize || whole<T, V>(a.logits, a.ld));
        constexpr uint32_t per = BACK_WAVES * 64 / LANES;
        constexpr uint64_t most = most_blocks(BACK_THREADS) * per;   // rows of a launch
        for (uint64_t r = 0; r < a.tokens; r += most) {
            RouteBackwardArgs part = a;
            part.tokens = a.tokens - r < most ? a.tokens - r : most;
            if (a.logits) part.logits = static_cast<const T *>(a.logits) + r * a.ld;
            if (a.mask) part.mask += r;
            part.weights += r * a.topk;
            part.ids += r * a.topk;
            part.dweights += r * a.topk;
            part.dlogits = static_cast<T *>(a.dlogits) + r * a.ld_d;
            k_route_backward<T, LANES, V><<<dim3((uint32_t)((part.tokens + per - 1) / per)), BACK_THREADS, 0, s>>>(part, vec);
        }
        return hipGetLastError();
    }
};

// Sixteen lanes a row up to 256 experts: a reduction takes four steps instead
// of six and serves four rows.
template <class F, class T, class A>
hipError_t by_experts(const A &a, hipStream_t s)
{
    if (a.experts <= 64) return F::template run<T, 16, 4>(a, s);
    if (a.experts <= 128) return F::template run<T, 16, 8>(a, s);
    if (a.experts <= NARROW_EXPERTS) return F::template run<T, 16, 16>(a, s);
    if (a.experts <= 512) return F::template run<T, 64, 8>(a, s);
    return F::template run<T, 64, 16>(a, s);
}

template <class F, class A>
hipError_t by_type(const A &a, uint32_t dtype, hipStream_t s)
{
    if (dtype == DT_F32) return by_experts<F, float>(a, s);
    if (dtype == DT_BF16) return by_experts<F, __bf16>(a, s);
    return by_experts<F, _Float16>(a, s);
}

}  // namespace

size_t route_workspace(uint64_t tokens, uint32_t experts)
{
    const uint64_t groups = (tokens + ROUTE_ROWS - 1) / ROUTE_ROWS;
    if (groups <= 1) return 0;
    const uint64_t bytes = groups > SUMMED_GROUPS ? groups * experts * sizeof(uint32_t) : groups * padded_experts(experts);
    return (size_t)((bytes + 255) & ~255ull);
}

hipError_t launch_route(const RouteArgs &a, uint32_t dtype, hipStream_t s) { return by_type<Forward>(a, dtype, s); }
hipError_t launch_route_backward(const RouteBackwardArgs &a, uint32_t dtype, hipStream_t s) { return by_type<Backward>(a, dtype, s); }

}  // namespace pccl
