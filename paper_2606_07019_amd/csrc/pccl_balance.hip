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

constexpr int THREADS = 1024, WAVES = 16;   // of the forward pass
constexpr uint32_t MOST_GROUPS = 256;        // workgroups that the rows are shared out to
constexpr uint32_t JOIN_EXPERTS = 16;        // experts of a joining workgroup
// Times that one workgroup takes as many rows as it can at once, by itself (256
// experts, forward pass: 128 rows 7.2 us, with joining 8.8; 256 rows 10.2 and 8.9).
constexpr uint32_t ALONE = 2;

// The logits of a lane: V in pieces of up to 16 bytes, so that a row's lanes read
// one neighbouring piece each, at any address (32,768 x 250 of bf16 backward 11.8
// us, value by value 22.6).
template <class T, int LANES, int V>
struct Share {
    static constexpr int PIECE = V * sizeof(T) < 16 ? V : 16 / sizeof(T);
    static __device__ uint32_t expert(uint32_t sub, int i) { return i / PIECE * (LANES * PIECE) + sub * PIECE + i % PIECE; }
    static __device__ void load(const T *row, uint32_t experts, uint32_t sub, T (&t)[V])
    {
#pragma unroll
        for (int i = 0; i < V; i += PIECE) {
            const uint32_t e = expert(sub, i);
            if (e + PIECE <= experts) {
                __builtin_memcpy(t + i, row + e, PIECE * sizeof(T));
                continue;
            }
#pragma unroll
            for (int j = 0; j < PIECE; j++) t[i + j] = e + j < experts ? row[e + j] : (T)-INFINITY;
        }
    }
    static __device__ void store(T *row, uint32_t experts, uint32_t sub, const T (&t)[V])
    {
#pragma unroll
        for (int i = 0; i < V; i += PIECE) {
            const uint32_t e = expert(sub, i);
            if (e + PIECE <= experts) {
                __builtin_memcpy(row + e, t + i, PIECE * sizeof(T));
                continue;
            }
#pragma unroll
            for (int j = 0; j < PIECE; j++)
                if (e + j < experts) row[e + j] = t[i + j];
        }
    }
};

// A row's softmax: v and, as the result, whether the row has an expert left
// (otherwise zeros).  Minus infinity is no expert; a NaN among the logits is lost
// in the largest but not in the sum, and makes the row's NaN, as plus infinity does.
// The instruction for 2^x as it is, without the library's steps for results below
// 2^-126, which are zero here beside a largest of 1 (32,768 x 256 of bf16, forward pass
// 14.6 us and 16.5 with expf, backward 11.5 and 13.6, each in a graph of its own).
template <class T, int LANES, int V>
__device__ inline bool softmax(const T (&t)[V], bool there, float (&v)[V])
{
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < V; i++) top = fmaxf(top, Elem<T>::get(t[i]));
    top = Key<float>::value(row_max<LANES>(Key<float>::of(top, 0)));
    top = there && top != -INFINITY ? top : 0.f;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < V; i++) {
        v[i] = __builtin_amdgcn_exp2f((Elem<T>::get(t[i]) - top) * 1.4426950408889634f);
        sum += v[i];
    }
    sum = row_sum<LANES>(sum);
    const bool any = there && sum != 0.f;   // its largest logit adds 1
    const float scale = 1.f / sum;
#pragma unroll
    for (int i = 0; i < V; i++) v[i] = any ? v[i] * scale : 0.f;
    return any;
}

// What the workgroups leave for the joining ones: sums of probabilities
// [groups][experts], counts [groups][experts], rows [groups]; and how many of the
// joining ones are done.
struct Space {
    float *probs;
    uint32_t *counts, *rows, *done;
};
constexpr uint32_t DONE_BYTES = 256;
inline __host__ __device__ Space space_of(char *ws, uint32_t groups, uint32_t experts)
{
    Space s;
    s.done = reinterpret_cast<uint32_t *>(ws);
    s.rows = reinterpret_cast<uint32_t *>(ws + DONE_BYTES);
    s.probs = reinterpret_cast<float *>(s.rows + groups);
    s.counts = reinterpret_cast<uint32_t *>(s.probs) + (uint64_t)groups * experts;
    return s;
}

// Sums over the threads of a workgroup of N waves, in a fixed order; all get them.
template <int N>
__device__ inline void over_all(uint32_t &u, float &f, uint32_t *us, float *fs)
{
#pragma unroll
    for (int o = 32; o; o >>= 1) {
        u += (uint32_t)__shfl_xor((int)u, o);
        f += __shfl_xor(f, o);
    }
    const uint32_t wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63u) == 0) {
        us[wave] = u;
        fs[wave] = f;
    }
    __syncthreads();
    u = 0;
    f = 0.f;
#pragma unroll
    for (int w = 0; w < N; w++) {
        u += us[w];
        f += fs[w];
    }
}

// LANES lanes a row, WAVES * 64 / LANES rows at a time; the next ones are read
// while these are summed up.  One workgroup by itself makes the outputs, several
// leave their sums to the joining kernels.  32,768 x 256 of bf16 9.2 to 10.8 us (17 MB
// from the device's cache): of a compute unit's busy cycles vector instructions take
// 57 %, the exponentials among them 11 %; waves wait 63 % of their time, for rows and
// at the meetings of the end.
template <class T, int LANES, int V>
__global__ __launch_bounds__(THREADS) void k_balance(BalanceArgs a)
{
    constexpr int PER = 64 / LANES;   // rows of a wave at a time
    constexpr uint32_t ROWS = WAVES * PER;
    __shared__ uint32_t hist[LANES * V], live[WAVES];
    __shared__ float sums[WAVES / 2][LANES * V];
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, sub = lane % LANES, mine = wave * PER + lane / LANES;
    for (uint32_t e = threadIdx.x; e < LANES * V; e += THREADS) hist[e] = 0;
    __syncthreads();
    const Space s = space_of(a.ws, gridDim.x, a.experts);
    if (gridDim.x > 1 && blockIdx.x == 0 && threadIdx.x == 0) *s.done = 0;   // for the joining kernel
    float acc[V];
#pragma unroll
    for (int i = 0; i < V; i++) acc[i] = 0.f;
    uint32_t rows = 0;
    const T *logits = static_cast<const T *>(a.logits);
    const uint64_t step = (uint64_t)gridDim.x * ROWS;
    struct Row {
        T t[V];
        bool there;
        int32_t id;   // of a lane's first pick
    } now, then;
    auto load = [&](Row &to, uint64_t r) {
        const uint64_t row = r < a.tokens ? r : a.tokens - 1;
        Share<T, LANES, V>::load(logits + row * a.ld, a.experts, sub, to.t);
        to.there = r < a.tokens && (!a.mask || a.mask[row]);
        to.id = sub < a.topk ? a.ids[row * a.topk + sub] : -1;
    };
    auto count = [&](int32_t id) {
        if ((uint32_t)id < a.experts) atomicAdd(&hist[id], 1u);   // LDS; whole numbers
    };
    uint64_t r0 = (uint64_t)blockIdx.x * ROWS;
    if (r0 < a.tokens) load(now, r0 + mine);
    for (; r0 < a.tokens; r0 += step) {
        if (r0 + step < a.tokens) load(then, r0 + step + mine);
        float v[V];
        const bool any = softmax<T, LANES, V>(now.t, now.there, v);
#pragma unroll
        for (int i = 0; i < V; i++) acc[i] += v[i];
        if (any) {
            rows += sub == 0;
            count(now.id);
            for (uint32_t j = sub + LANES; j < a.topk; j += LANES) count(a.ids[(r0 + mine) * a.topk + j]);
        }
        now = then;
    }
    // a wave's rows, then the upper half of the waves to the lower, then those
#pragma unroll
    for (int i = 0; i < V; i++) {
#pragma unroll
        for (int o = LANES; o < 64; o <<= 1) acc[i] += __shfl_xor(acc[i], o);
    }
    if (wave >= WAVES / 2 && lane < LANES) {
#pragma unroll
        for (int i = 0; i < V; i++) sums[wave - WAVES / 2][Share<T, LANES, V>::expert(sub, i)] = acc[i];
    }
    __syncthreads();
    if (wave < WAVES / 2 && lane < LANES) {
#pragma unroll
        for (int i = 0; i < V; i++) sums[wave][Share<T, LANES, V>::expert(sub, i)] += acc[i];
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) rows += (uint32_t)__shfl_xor((int)rows, o);
    if (lane == 0) live[wave] = rows;
    __syncthreads();
    static_assert(THREADS >= (int)ROUTE_MAX_EXPERTS, "a thread for every expert");
    float prob = 0.f;
    uint32_t picks = 0;
    if (const uint32_t e = threadIdx.x; e < a.experts) {
        float x = 0.f;
#pragma unroll
        for (uint32_t w = 0; w < WAVES / 2; w++) x += sums[w][e];
        if (gridDim.x > 1) {
            s.probs[(uint64_t)blockIdx.x * a.experts + e] = x;
            s.counts[(uint64_t)blockIdx.x * a.experts + e] = hist[e];
        } else {   // all there is; every expert has a thread of its own
            prob = x;
            picks = hist[e];
        }
    }
    uint32_t all = 0;
#pragma unroll
    for (int w = 0; w < WAVES; w++) all += live[w];
    if (gridDim.x > 1) {
        if (threadIdx.x == 0) s.rows[blockIdx.x] = all;
        return;
    }
    __syncthreads();   // the sums, which lend their room, and live have been read
    if (all) prob /= (float)all;
    if (threadIdx.x < a.experts) {
        a.probs[threadIdx.x] = prob;
        a.counts[threadIdx.x] = (int32_t)picks;
    }
    float loss = (float)picks * prob;
    over_all<WAVES>(picks, loss, live, sums[0]);
    if (threadIdx.x == 0) {
        *a.loss = picks ? loss * ((float)a.experts / (float)picks) : 0.f;
        *a.rows = (int32_t)all;
    }
}

// The workgroups' sums joined.  Few of them, and of experts: one workgroup, up to
// LOADS of them a thread (forward pass of 256 x 256, 4 workgroups, 8.9 us, with the
// kernel below 9.3; of 32,768 x 256, 256 workgroups and 64 loads, 22.0 and 14.9).
constexpr uint32_t LOADS = 16;
__global__ __launch_bounds__(THREADS) void k_balance_join(BalanceArgs a, uint32_t groups, uint32_t log_experts)
{
    __shared__ float fsum[THREADS], fs[WAVES];
    __shared__ uint32_t usum[THREADS], us[WAVES];
    const Space s = space_of(a.ws, groups, a.experts);
    const uint32_t e = threadIdx.x & ((1u << log_experts) - 1u), part = threadIdx.x >> log_experts, parts = THREADS >> log_experts;
    float p = 0.f, zero = 0.f;
    uint32_t c = 0, rows = threadIdx.x < groups ? s.rows[threadIdx.x] : 0u;
#pragma unroll
    for (uint32_t i = 0; i < LOADS; i++) {
        const uint32_t g = part + i * parts;
        const bool in = g < groups && e < a.experts;
        p += in ? s.probs[(uint64_t)g * a.experts + e] : 0.f;
        c += in ? s.counts[(uint64_t)g * a.experts + e] : 0u;
    }
    fsum[threadIdx.x] = p;
    usum[threadIdx.x] = c;
    over_all<WAVES>(rows, zero, us, fs);   // and a barrier
    p = 0.f;
    c = 0;
    if (part == 0 && e < a.experts) {
        for (uint32_t j = 0; j < parts; j++) {
            p += fsum[(j << log_experts) + e];
            c += usum[(j << log_experts) + e];
        }
        p = rows ? p / (float)rows : 0.f;
        a.probs[e] = p;
        a.counts[e] = (int32_t)c;
    }
    float loss = (float)c * p;
    uint32_t picks = c;
    __syncthreads();   // us and fs have been read
    over_all<WAVES>(picks, loss, us, fs);
    if (threadIdx.x == 0) {
        *a.loss = picks ? loss * ((float)a.experts / (float)picks) : 0.f;
        *a.rows = (int32_t)rows;
    }
}

// Many: sixteen experts a workgroup, 64 threads an expert; the last one to be
// done adds up the loss, whose factor 1 / sum of the counts is known only then.
// What it reads of the others is written past the caches before they say that they
// are done (a release of all that the caches hold takes 5 us more).
__global__ __launch_bounds__(THREADS) void k_balance_join_many(BalanceArgs a, uint32_t groups)
{
    constexpr uint32_t PARTS = THREADS / JOIN_EXPERTS, MOST = MOST_GROUPS / PARTS;
    static_assert(MOST_GROUPS <= THREADS && MOST_GROUPS % PARTS == 0, "a thread's share");
    __shared__ float fsum[PARTS][JOIN_EXPERTS + 1], fs[WAVES];
    __shared__ uint32_t usum[PARTS][JOIN_EXPERTS + 1], us[WAVES];
    __shared__ uint32_t last;
    const Space s = space_of(a.ws, groups, a.experts);
    const uint32_t mine = threadIdx.x % JOIN_EXPERTS, e = blockIdx.x * JOIN_EXPERTS + mine, part = threadIdx.x / JOIN_EXPERTS;
    float p[MOST], zero = 0.f;
    uint32_t c[MOST], rows = threadIdx.x < groups ? s.rows[threadIdx.x] : 0u;
#pragma unroll
    for (uint32_t i = 0; i < MOST; i++) {
        const uint32_t g = part + i * PARTS;
        const bool in = g < groups && e < a.experts;
        p[i] = in ? s.probs[(uint64_t)g * a.experts + e] : 0.f;
        c[i] = in ? s.counts[(uint64_t)g * a.experts + e] : 0u;
    }
#pragma unroll
    for (uint32_t i = 1; i < MOST; i++) {
        p[0] += p[i];
        c[0] += c[i];
    }
    fsum[part][mine] = p[0];
    usum[part][mine] = c[0];
    over_all<WAVES>(rows, zero, us, fs);   // and a barrier
    if (part == 0) {
        float sum = 0.f;
        uint32_t n = 0;
#pragma unroll 16
        for (uint32_t j = 0; j < PARTS; j++) {
            sum += fsum[j][mine];
            n += usum[j][mine];
        }
        if (e < a.experts) {
            __hip_atomic_store(a.probs + e, rows ? sum / (float)rows : 0.f, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            __hip_atomic_store(a.counts + e, (int32_t)n, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.rows = (int32_t)rows;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // those are there
    __syncthreads();
    if (threadIdx.x == 0) last = __hip_atomic_fetch_add(s.done, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1u == gridDim.x;
    __syncthreads();
    if (!last) return;
    uint32_t picks = 0;
    float loss = 0.f;
    for (uint32_t i = threadIdx.x; i < a.experts; i += THREADS) {
        const uint32_t n = (uint32_t)__hip_atomic_load(a.counts + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        picks += n;
        loss += (float)n * __hip_atomic_load(a.probs + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    over_all<WAVES>(picks, loss, us, fs);
    if (threadIdx.x == 0) *a.loss = picks ? loss * ((float)a.experts / (float)picks) : 0.f;
}

// The softmax again, from the logits: reading them costs less than probabilities
// that the forward pass would have to write.  Bound by its vector instructions, 77 % of
// a compute unit's busy cycles (the exponentials 12 %): 32,768 x 256 of bf16 10.6 us,
// 3.2 TB/s read and written (with 512 workgroups 15 % longer).
constexpr int BACK_THREADS = 256, BACK_WAVES = 4;
constexpr uint32_t BACK_GROUPS = 1024;   // workgroups at most

template <class T, int LANES, int V>
__global__ __launch_bounds__(BACK_THREADS) void k_balance_backward(BalanceBackwardArgs a)
{
    constexpr int PER = 64 / LANES;
    constexpr uint32_t ROWS = BACK_WAVES * PER;
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, sub = lane % LANES, mine = wave * PER + lane / LANES;
    const T *logits = static_cast<const T *>(a.logits);
    const uint64_t step = (uint64_t)gridDim.x * ROWS;
    struct Row {
        T t[V];
        bool there;
    } now, then;
    auto load = [&](Row &to, uint64_t r) {
        const uint64_t row = r < a.tokens ? r : a.tokens - 1;
        Share<T, LANES, V>::load(logits + row * a.ld, a.experts, sub, to.t);
        to.there = !a.mask || a.mask[row];
    };
    uint64_t r0 = (uint64_t)blockIdx.x * ROWS;   // below the number of tokens
    load(now, r0 + mine);
    const uint32_t rows = (uint32_t)*a.rows;
    const float dloss = a.dloss ? *a.dloss : 0.f;
    // what the experts' probabilities are worth; the lanes of a row have all experts' counts
    typedef Share<T, LANES, V> Mine;
    int32_t c[V];
    float g[V];
    uint32_t low = 0, high = 0;   // of the picks: ranks' counts together may pass 32 bits
#pragma unroll
    for (int i = 0; i < V; i += Mine::PIECE) {
        const uint32_t e = Mine::expert(sub, i);
        if (e + Mine::PIECE <= a.experts) {
            __builtin_memcpy(c + i, a.counts + e, Mine::PIECE * 4);
            if (a.dprobs) __builtin_memcpy(g + i, a.dprobs + e, Mine::PIECE * 4);
            continue;
        }
#pragma unroll
        for (int j = 0; j < Mine::PIECE; j++) {
            c[i + j] = e + j < a.experts ? a.counts[e + j] : 0;
            g[i + j] = a.dprobs && e + j < a.experts ? a.dprobs[e + j] : 0.f;
        }
    }
#pragma unroll
    for (int i = 0; i < V; i++) {
        low += (uint32_t)c[i] & 0xFFFFu;
        high += (uint32_t)c[i] >> 16;
    }
    auto add = [](uint32_t a, uint32_t b) { return a + b; };
    const uint64_t picks = ((uint64_t)reduce<LANES>(high, add) << 16) + reduce<LANES>(low, add);
    const float each = rows ? 1.f / (float)rows : 0.f;
    const float unit = picks ? dloss * ((float)a.experts / (float)picks) : 0.f;
#pragma unroll
    for (int i = 0; i < V; i++) g[i] = (unit * (float)c[i] + (a.dprobs ? g[i] : 0.f)) * each;
    for (; r0 < a.tokens; r0 += step) {
        if (r0 + step < a.tokens) load(then, r0 + step + mine);
        float v[V], sum = 0.f;
        const bool any = softmax<T, LANES, V>(now.t, now.there, v);
#pragma unroll
        for (int i = 0; i < V; i++) sum += g[i] * v[i];
        sum = row_sum<LANES>(sum);
        T t[V];
#pragma unroll
        for (int i = 0; i < V; i++) t[i] = Elem<T>::put(any ? v[i] * (g[i] - sum) : 0.f);   // whatever dloss is
        now = then;
        const uint64_t r = r0 + mine;
        if (r >= a.tokens) continue;
        Share<T, LANES, V>::store(static_cast<T *>(a.dlogits) + r * a.ld_d, a.experts, sub, t);
    }
}

inline uint32_t rows_at_a_time(uint32_t experts) { return WAVES * (experts <= NARROW_EXPERTS ? 4u : 1u); }
inline uint32_t workgroups(uint64_t tokens, uint32_t experts)
{
    const uint64_t per = rows_at_a_time(experts), n = (tokens + per - 1) / per;
    if (n <= ALONE) return 1;   // without tokens too: zeros are written
    return (uint32_t)(n < MOST_GROUPS ? n : MOST_GROUPS);
}

struct Forward {
    template <class T, int LANES, int V>
    static hipError_t run(const BalanceArgs &a, hipStream_t s)
    {
        const uint32_t groups = workgroups(a.tokens, a.experts);
        k_balance<T, LANES, V><<<dim3(groups), THREADS, 0, s>>>(a);
        if (groups == 1) return hipGetLastError();
        uint32_t log = 0;
        while ((1u << log) < a.experts) log++;
        if (groups <= LOADS * (THREADS >> log)) k_balance_join<<<dim3(1), THREADS, 0, s>>>(a, groups, log);
        else k_balance_join_many<<<dim3((a.experts + JOIN_EXPERTS - 1) / JOIN_EXPERTS), THREADS, 0, s>>>(a, groups);
        return hipGetLastError();
    }
};

struct Backward {
    template <class T, int LANES, int V>
    static hipError_t run(const BalanceBackwardArgs &a, hipStream_t s)
    {
        const uint64_t per = BACK_WAVES * 64 / LANES, n = (a.tokens + per - 1) / per;
        k_balance_backward<T, LANES, V><<<dim3((uint32_t)(n < BACK_GROUPS ? n : BACK_GROUPS)), BACK_THREADS, 0, s>>>(a);
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
    if (groups == 1) return 0;
    return (size_t)((DONE_BYTES + 4 * groups * (1 + 2 * (uint64_t)experts) + 255) & ~255ull);
}

hipError_t launch_balance(const BalanceArgs &a, uint32_t dtype, hipStream_t s) { return by_type<Forward>(a, dtype, s); }
hipError_t launch_balance_backward(const BalanceBackwardArgs &a, uint32_t dtype, hipStream_t s) { return by_type<Backward>(a, dtype, s); }

}  // namespace pccl
