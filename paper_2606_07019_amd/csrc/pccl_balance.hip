// The router's balance loss, which keeps the counts of an expert-parallel
// All-to-Allv even, with the experts' counts and mean probabilities, and its
// gradient with respect to the logits.
//
//   p_t = softmax(l_t) over the n rows that have an expert left,
//   P_e = sum_t p_te / n,  f_e = E c_e / sum c,  loss = sum_e f_e P_e
//   dl_te = p_te (v_e - sum_i v_i p_ti) / n,  v = dloss f + dprobs
//
// The counts are whole numbers and carry no gradient.  Sums over the rows are
// split over workgroups and joined in a fixed order, in 32 bits.
#include "pccl_topk.h"

namespace pccl {
namespace {

constexpr int THREADS = 256, WAVES = 4;
constexpr uint32_t MOST_GROUPS = 512;   // workgroups that the rows are shared out to
constexpr uint32_t JOIN_EXPERTS = 16;   // experts of a joining workgroup

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

// A row's softmax in place of its logits: v and, as the result, whether the row
// has an expert left (otherwise zeros).  A NaN or plus infinity makes the row's NaN.
template <class T, int LANES, int V>
__device__ inline bool softmax(const T (&t)[V], bool there, uint32_t experts, uint32_t sub, float (&v)[V])
{
    uint32_t key[V], most = 0;
#pragma unroll
    for (int i = 0; i < V; i++) {
        key[i] = there && sub * V + i < experts ? Key<float>::of(Elem<T>::get(t[i]), 0) : 0u;
        most = key[i] > most ? key[i] : most;
    }
    most = row_max<LANES>(most);
    const bool any = most > Key<float>::EMPTY;
    const float top = Key<float>::value(most);
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < V; i++) {
        v[i] = any && key[i] > Key<float>::EMPTY ? expf(Elem<T>::get(t[i]) - top) : 0.f;
        sum += v[i];
    }
    sum = row_sum<LANES>(sum);
    const float scale = any ? 1.f / sum : 0.f;
#pragma unroll
    for (int i = 0; i < V; i++) v[i] *= scale;
    return any;
}

// What the workgroups leave for the joining one: sums of probabilities
// [groups][experts], counts [groups][experts], rows [groups]; a joining
// workgroup's sum of counts and part of the loss; how many of them are done.
struct Space {
    float *probs, *loss;
    uint32_t *counts, *rows, *done;
};
inline __host__ __device__ Space space_of(char *ws, uint32_t groups, uint32_t experts)
{
    Space s;
    s.done = reinterpret_cast<uint32_t *>(ws);
    s.loss = reinterpret_cast<float *>(ws) + 64;
    s.rows = reinterpret_cast<uint32_t *>(ws) + 128;
    s.probs = reinterpret_cast<float *>(s.rows + groups);
    s.counts = reinterpret_cast<uint32_t *>(s.probs) + (uint64_t)groups * experts;
    return s;
}

template <class T, int LANES, int V>
__global__ __launch_bounds__(THREADS) void k_balance(BalanceArgs a, bool vec)
{
    constexpr int PER = 64 / LANES;   // rows of a wave at a time
    __shared__ uint32_t hist[LANES * V], live[WAVES];
    __shared__ float sums[WAVES * PER][LANES * V];
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, sub = lane % LANES, mine = wave * PER + lane / LANES;
    for (uint32_t e = threadIdx.x; e < LANES * V; e += THREADS) hist[e] = 0;
    __syncthreads();
    const Space s = space_of(a.ws, gridDim.x, a.experts);
    if (blockIdx.x == 0 && threadIdx.x == 0) *s.done = 0;   // for the joining kernel
    float acc[V];
#pragma unroll
    for (int i = 0; i < V; i++) acc[i] = 0.f;
    uint32_t rows = 0;
    const T *logits = static_cast<const T *>(a.logits);
    for (uint64_t r0 = (uint64_t)blockIdx.x * (WAVES * PER); r0 < a.tokens; r0 += (uint64_t)gridDim.x * (WAVES * PER)) {
        const uint64_t r = r0 + mine, row = r < a.tokens ? r : a.tokens - 1;
        T t[V];
        load_row<T, V>(logits + row * a.ld, a.experts, sub, vec, t);
        const bool there = r < a.tokens && (!a.mask || a.mask[row]);
        float v[V];
        const bool any = softmax<T, LANES, V>(t, there, a.experts, sub, v);
#pragma unroll
        for (int i = 0; i < V; i++) acc[i] += v[i];
        if (!any) continue;
        rows += sub == 0;
        for (uint32_t j = sub; j < a.topk; j += LANES) {
            const uint32_t e = (uint32_t)a.ids[row * a.topk + j];
            if (e < a.experts) atomicAdd(&hist[e], 1u);   // LDS; whole numbers
        }
    }
#pragma unroll
    for (int i = 0; i < V; i++) sums[mine][sub * V + i] = acc[i];
#pragma unroll
    for (int o = 32; o; o >>= 1) rows += (uint32_t)__shfl_xor((int)rows, o);
    if (lane == 0) live[wave] = rows;
    __syncthreads();
    for (uint32_t e = threadIdx.x; e < a.experts; e += THREADS) {
        float x = sums[0][e];
#pragma unroll
        for (int w = 1; w < WAVES * PER; w++) x += sums[w][e];
        s.probs[(uint64_t)blockIdx.x * a.experts + e] = x;
        s.counts[(uint64_t)blockIdx.x * a.experts + e] = hist[e];
    }
    if (threadIdx.x == 0) s.rows[blockIdx.x] = live[0] + live[1] + live[2] + live[3];
}

// Adds up over the threads of a workgroup, in a fixed order; all get the result.
template <class S>
__device__ inline S over_all(S v, S *room)
{
    __syncthreads();
    room[threadIdx.x] = v;
    __syncthreads();
    for (uint32_t o = THREADS / 2; o; o >>= 1) {
        if (threadIdx.x < o) room[threadIdx.x] += room[threadIdx.x + o];
        __syncthreads();
    }
    return room[0];
}

// Sixteen experts a workgroup, sixteen threads an expert; the last one to be
// done adds up the loss, whose factor 1 / sum of the counts is known only then.
__global__ __launch_bounds__(THREADS) void k_balance_join(BalanceArgs a, uint32_t groups)
{
    __shared__ float fsum[THREADS];
    __shared__ uint32_t usum[THREADS];
    __shared__ uint32_t last;
    const Space s = space_of(a.ws, groups, a.experts);
    const uint32_t e = blockIdx.x * JOIN_EXPERTS + threadIdx.x % JOIN_EXPERTS, part = threadIdx.x / JOIN_EXPERTS;
    constexpr uint32_t PARTS = THREADS / JOIN_EXPERTS;
    uint32_t rows = 0;
    for (uint32_t g = threadIdx.x; g < groups; g += THREADS) rows += s.rows[g];
    rows = over_all(rows, usum);
    float p = 0.f;
    uint32_t c = 0;
    if (e < a.experts)
        for (uint32_t g = part; g < groups; g += PARTS) {
            p += s.probs[(uint64_t)g * a.experts + e];
            c += s.counts[(uint64_t)g * a.experts + e];
        }
    fsum[threadIdx.x] = p;
    __syncthreads();
    usum[threadIdx.x] = c;
    __syncthreads();
    if (part == 0) {
        for (uint32_t j = 1; j < PARTS; j++) {
            p += fsum[j * JOIN_EXPERTS + threadIdx.x];
            c += usum[j * JOIN_EXPERTS + threadIdx.x];
        }
        p = rows ? p / (float)rows : 0.f;
        if (e < a.experts) {
            a.probs[e] = p;
            a.counts[e] = (int32_t)c;
        }
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.rows = (int32_t)rows;
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) last = atomicAdd(s.done, 1u) + 1u == gridDim.x;
    __syncthreads();
    if (!last) return;
    __threadfence();
    uint32_t picks = 0;
    for (uint32_t i = threadIdx.x; i < a.experts; i += THREADS) picks += __hip_atomic_load((uint32_t *)a.counts + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    picks = over_all(picks, usum);
    float loss = 0.f;
    for (uint32_t i = threadIdx.x; i < a.experts; i += THREADS) {
        const float n = (float)__hip_atomic_load((uint32_t *)a.counts + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        loss += n * __hip_atomic_load(a.probs + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    loss = over_all(loss, fsum);
    if (threadIdx.x == 0) *a.loss = picks ? loss * ((float)a.experts / (float)picks) : 0.f;
}

template <class T, int LANES, int V>
__global__ __launch_bounds__(THREADS) void k_balance_backward(BalanceBackwardArgs a, bool vec)
{
    constexpr int PER = 64 / LANES;
    __shared__ uint32_t usum[THREADS];
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, sub = lane % LANES, mine = wave * PER + lane / LANES;
    uint32_t picks = 0;
    for (uint32_t i = threadIdx.x; i < a.experts; i += THREADS) picks += (uint32_t)a.counts[i];
    picks = over_all(picks, usum);
    const uint32_t rows = (uint32_t)*a.rows;
    const float each = rows ? 1.f / (float)rows : 0.f;
    const float unit = a.dloss && picks ? *a.dloss * ((float)a.experts / (float)picks) : 0.f;
    float g[V];   // what the experts' probabilities are worth
#pragma unroll
    for (int i = 0; i < V; i++) {
        const uint32_t e = sub * V + i;
        g[i] = e < a.experts ? (unit * (float)a.counts[e] + (a.dprobs ? a.dprobs[e] : 0.f)) * each : 0.f;
    }
    const T *logits = static_cast<const T *>(a.logits);
    for (uint64_t r0 = (uint64_t)blockIdx.x * (WAVES * PER); r0 < a.tokens; r0 += (uint64_t)gridDim.x * (WAVES * PER)) {
        const uint64_t r = r0 + mine, row = r < a.tokens ? r : a.tokens - 1;
        T t[V];
        load_row<T, V>(logits + row * a.ld, a.experts, sub, vec, t);
        float v[V], sum = 0.f;
        softmax<T, LANES, V>(t, !a.mask || a.mask[row], a.experts, sub, v);
#pragma unroll
        for (int i = 0; i < V; i++) sum += g[i] * v[i];
        sum = row_sum<LANES>(sum);
#pragma unroll
        for (int i = 0; i < V; i++) t[i] = Elem<T>::put(v[i] * (g[i] - sum));
        if (r >= a.tokens) continue;
        T *out = static_cast<T *>(a.dlogits) + row * a.ld_d;
        const uint32_t e0 = sub * V;
        if (vec && e0 + V <= a.experts) {
            __builtin_memcpy(__builtin_assume_aligned(out + e0, sizeof t < 16 ? sizeof t : 16), t, sizeof t);
            continue;
        }
#pragma unroll
        for (int i = 0; i < V; i++)
            if (e0 + i < a.experts) out[e0 + i] = t[i];
    }
}

// A lane's neighbouring logits are read at once where every row starts on them.
template <class T, int V>
bool whole(const void *p, uint64_t ld)
{
    const uint64_t unit = sizeof(T) * V < 16 ? sizeof(T) * V : 16;
    return (reinterpret_cast<uintptr_t>(p) | (ld * sizeof(T))) % unit == 0;
}

inline uint32_t rows_at_a_time(uint32_t experts) { return WAVES * (experts <= NARROW_EXPERTS ? 4u : 1u); }
inline uint32_t workgroups(uint64_t tokens, uint32_t experts)
{
    const uint64_t per = rows_at_a_time(experts), n = (tokens + per - 1) / per;
    return (uint32_t)(n < 1 ? 1 : n < MOST_GROUPS ? n : MOST_GROUPS);   // without tokens one still writes zeros
}

struct Forward {
    template <class T, int LANES, int V>
    static hipError_t run(const BalanceArgs &a, hipStream_t s)
    {
        const uint32_t groups = workgroups(a.tokens, a.experts);
        k_balance<T, LANES, V><<<dim3(groups), THREADS, 0, s>>>(a, whole<T, V>(a.logits, a.ld));
        k_balance_join<<<dim3((a.experts + JOIN_EXPERTS - 1) / JOIN_EXPERTS), THREADS, 0, s>>>(a, groups);
        return hipGetLastError();
    }
};

struct Backward {
    template <class T, int LANES, int V>
    static hipError_t run(const BalanceBackwardArgs &a, hipStream_t s)
    {
        const bool vec = whole<T, V>(a.dlogits, a.ld_d) && whole<T, V>(a.logits, a.ld);
        const uint64_t per = WAVES * 64 / LANES, n = (a.tokens + per - 1) / per;
        k_balance_backward<T, LANES, V><<<dim3((uint32_t)(n < 2048 ? n : 2048)), THREADS, 0, s>>>(a, vec);
        return hipGetLastError();
    }
};

// Sixteen lanes a row up to 256 experts, as in the router.
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

size_t balance_workspace(uint64_t tokens, uint32_t experts)
{
    const uint64_t groups = workgroups(tokens, experts);
    return (size_t)((512 + 4 * groups * (1 + 2 * (uint64_t)experts) + 255) & ~255ull);
}

hipError_t launch_balance(const BalanceArgs &a, uint32_t dtype, hipStream_t s) { return by_type<Forward>(a, dtype, s); }
hipError_t launch_balance_backward(const BalanceBackwardArgs &a, uint32_t dtype, hipStream_t s) { return by_type<Backward>(a, dtype, s); }

}  // namespace pccl
