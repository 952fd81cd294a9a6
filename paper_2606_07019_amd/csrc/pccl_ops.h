// Internal definitions of the operators at the ends of a collective: packing
// to microscaled 4-bit values, their product, the router and the
// mixture-of-experts layer; packing to 8 bits with a scale for 128 values, the
// products and experts' products of that, and the router's balance loss (not
// part of the ABI).
#pragma once

#include <atomic>

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace pccl {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// Element types, as in the public header.
enum : uint32_t { DT_F32 = 0, DT_BF16 = 1, DT_F16 = 2 };

// Microscaled rows: blocks of 32 values share a scale; a stored row ends on a
// whole 128 values (one matrix-instruction step of the 4-bit product), padded
// with zeros, so a row's codes are whole 64 bytes and its scales whole words.
constexpr uint32_t MX_BLOCK = 32;
constexpr uint32_t MX_STEP = 128;
inline __host__ __device__ uint64_t mx_steps(uint64_t cols) { return (cols + MX_STEP - 1) / MX_STEP; }
inline __host__ __device__ uint64_t mx_code_bytes(uint64_t cols) { return mx_steps(cols) * (MX_STEP / 2); }
inline __host__ __device__ uint64_t mx_scale_bytes(uint64_t cols) { return mx_steps(cols) * (MX_STEP / MX_BLOCK); }

// Sizes every operator takes: extents below 2^31, so that indexes of one
// extent fit 32 bits; products of two are computed in 64 bits.
constexpr uint64_t OPS_MAX_EXTENT = 0x7FFFFFFFull;

// A launch has fewer than 2^32 threads.  Kernels whose rows do not meet take
// more of them in further launches.
inline constexpr uint64_t most_blocks(uint32_t threads) { return 0xFFFFFFFFull / threads; }

// The product's k: a tile's 256 rows of codes stay within 32-bit offsets.
constexpr uint64_t MX_MAX_K = 1ull << 24;

// The router's envelope: one wave holds a row, up to 16 logits a lane.
constexpr uint32_t ROUTE_MAX_EXPERTS = 1024;
constexpr uint32_t ROUTE_MAX_TOPK = 32;
constexpr uint32_t ROUTE_ROWS = 64;   // rows of one workgroup: one bit each in an expert's row mask

// The layer's envelope: "a few tokens".
constexpr uint32_t MOE_MAX_TOKENS = 256;
constexpr uint32_t MOE_MAX_DIM = 1u << 20;   // hidden and inner size
constexpr uint64_t MOE_MAX_MATRIX = 1ull << 29;   // their product: an expert's rows stay within 32-bit offsets

struct MxQuantizeArgs {
    const void *x;
    uint64_t rows, cols, ld;
    uint8_t *codes, *scales;      // of the rows, or null
    uint8_t *codes_t, *scales_t;  // of the columns, or null
};
hipError_t launch_mx_quantize(const MxQuantizeArgs &a, uint32_t dtype, hipStream_t s);

struct MxDequantizeArgs {
    const uint8_t *codes, *scales;
    uint64_t rows, cols, ld;
    void *out;
};
hipError_t launch_mx_dequantize(const MxDequantizeArgs &a, uint32_t dtype, hipStream_t s);

struct MxMatmulArgs {
    const uint8_t *a, *as, *b, *bs;  // codes and scales of the m rows and of the n rows
    uint64_t m, n, k, ld;
    void *out;
    float *part;                     // partial sums of a split k, or null
};
size_t mx_matmul_workspace(uint64_t m, uint64_t n, uint64_t k);
bool mx_matmul_fits(uint64_t m, uint64_t n, uint64_t k);   // one launch's threads
hipError_t launch_mx_matmul(const MxMatmulArgs &a, uint32_t dtype, hipStream_t s);

struct RouteArgs {
    const void *logits;
    uint64_t tokens, ld;
    uint32_t experts, topk;
    uint32_t normalize;
    const uint8_t *mask;   // per token, 0 = no token there; or null
    float *weights;        // [tokens][topk]
    int32_t *ids;          // [tokens][topk], -1 = no expert left
    int32_t *counts;       // [experts]
    int32_t *order;        // [tokens * topk]: slots by expert, then by slot; -1 behind them
    uint32_t *hist;        // workspace: [experts][workgroups] counts, then where each starts
};
size_t route_workspace(uint64_t tokens, uint32_t experts);
hipError_t launch_route(const RouteArgs &a, uint32_t dtype, hipStream_t s);

struct RouteBackwardArgs {
    const void *logits;
    uint64_t tokens, ld, ld_d;
    uint32_t experts, topk;
    uint32_t normalize;
    const uint8_t *mask;
    const float *weights;
    const int32_t *ids;
    const float *dweights;
    void *dlogits;
};
hipError_t launch_route_backward(const RouteBackwardArgs &a, uint32_t dtype, hipStream_t s);

struct MoeArgs {
    const void *x;
    uint64_t ld_x, ld_y;
    uint32_t tokens, experts, topk, hidden, inter;
    uint32_t normalize;
    const uint8_t *mask;
    const void *router;                  // [experts][hidden]
    const void *up, *down;               // [experts][2 inter][hidden], [experts][hidden][inter]; codes if microscaled
    const uint8_t *up_scales, *down_scales;  // null: weights of x's type
    void *y;
    char *ws;
};
size_t moe_workspace(uint32_t tokens, uint32_t experts, uint32_t topk, uint32_t hidden, uint32_t inter);
hipError_t launch_moe(const MoeArgs &a, uint32_t dtype, hipStream_t s);

// Rows of 8-bit floating point: blocks of 128 values share a scale.  A stored
// row ends on a whole block, padded with zeros, and its scales on a whole word.
constexpr uint32_t F8_BLOCK = 128;
inline __host__ __device__ uint64_t f8_blocks(uint64_t cols) { return (cols + F8_BLOCK - 1) / F8_BLOCK; }
inline __host__ __device__ uint64_t f8_code_bytes(uint64_t cols) { return f8_blocks(cols) * F8_BLOCK; }
inline __host__ __device__ uint64_t f8_scale_bytes(uint64_t cols) { return (f8_blocks(cols) + 3) / 4 * 4; }

// The product's k: a tile's 256 rows of codes stay within 32-bit offsets.
constexpr uint64_t F8_MAX_K = 1ull << 23;

// Rows in expert order, cut into blocks of up to 128 rows of one expert (and of
// up to 256, for larger tiles).  The table, in words: the numbers of blocks
// before each expert and of all, the number of larger blocks, then two words a
// block (its first row; its expert and rows, expert | rows << 16), no rows in
// those that are not used; then the larger blocks the same way.
inline __host__ __device__ uint64_t groups_blocks(uint64_t experts, uint64_t rows, uint32_t block)
{
    return rows / block + (experts < rows ? experts : rows);
}
struct GroupsArgs {
    const int32_t *counts;
    uint64_t rows;
    uint32_t experts, pad;
    uint64_t blocks, blocks2;    // of 128 rows, of 256
    int32_t *table;
};
inline __host__ __device__ uint64_t groups_words(uint64_t experts, uint64_t rows)
{
    return experts + 2 + 2 * groups_blocks(experts, rows, 128) + 2 * groups_blocks(experts, rows, 256);
}
hipError_t launch_groups(const GroupsArgs &a, hipStream_t s);

struct F8QuantizeArgs {
    const void *x;
    uint64_t batch, rows, cols, ld;   // `batch` matrices, one behind the other
    uint8_t *codes, *scales;          // of the rows, or null
    uint8_t *codes_t, *scales_t;      // of the columns, or null
    uint32_t tiles;                   // a scale for 128 x 128 values, the same for rows and columns
    uint32_t experts;                 // of the blocks of rows
    const int32_t *groups;            // the columns' blocks are those of this table; or null
};
hipError_t launch_f8_quantize(const F8QuantizeArgs &a, uint32_t dtype, hipStream_t s);

struct F8DequantizeArgs {
    const uint8_t *codes, *scales;
    uint64_t rows, cols, ld;
    void *out;
};
hipError_t launch_f8_dequantize(const F8DequantizeArgs &a, uint32_t dtype, hipStream_t s);

struct F8MatmulArgs {
    const uint8_t *a, *as, *b, *bs;  // codes and scales of the m rows and of the n rows
    uint64_t m, n, k, ld;
    void *out;
    float *part;                     // partial sums of a split k, or null
    const int32_t *groups;           // experts' products: the table
    uint64_t rows;                   // of all experts
    uint32_t experts;
};
size_t f8_matmul_workspace(uint64_t m, uint64_t n, uint64_t k);
bool f8_matmul_fits(uint64_t m, uint64_t n, uint64_t k);   // one launch's threads
hipError_t launch_f8_matmul(const F8MatmulArgs &a, uint32_t dtype, hipStream_t s);
// out [rows][n]: rows of a times their expert's b [n][k]
bool f8_experts_fit(uint64_t rows, uint32_t experts, uint64_t n);
hipError_t launch_f8_expert_matmul(const F8MatmulArgs &a, uint32_t dtype, hipStream_t s);
// out [experts][m][n]: m rows of a times n rows of b over each expert's blocks
bool f8_gradients_fit(uint32_t experts, uint64_t m, uint64_t n);
hipError_t launch_f8_expert_gradient(const F8MatmulArgs &a, uint32_t dtype, hipStream_t s);

struct BalanceArgs {
    const void *logits;
    uint64_t tokens, ld;
    uint32_t experts, topk;
    const uint8_t *mask;
    const int32_t *ids;
    float *loss, *probs;
    int32_t *counts, *rows;
    char *ws;
};
size_t balance_workspace(uint64_t tokens, uint32_t experts);
hipError_t launch_balance(const BalanceArgs &a, uint32_t dtype, hipStream_t s);

struct BalanceBackwardArgs {
    const void *logits;
    uint64_t tokens, ld, ld_d;
    uint32_t experts, pad;
    const uint8_t *mask;
    const int32_t *counts, *rows;
    const float *dloss, *dprobs;   // either may be null
    void *dlogits;
};
hipError_t launch_balance_backward(const BalanceBackwardArgs &a, uint32_t dtype, hipStream_t s);

#ifdef __HIPCC__
// Lets a kernel have `bytes` of LDS on the current device, once for each device.
template <auto Kernel>
inline hipError_t allow_lds(uint32_t bytes)
{
    static std::atomic<uint64_t> devices{0};
    int d = 0;
    hipError_t e = hipGetDevice(&d);
    if (e != hipSuccess) return e;
    const uint64_t bit = 1ull << (d % 64);
    if (d < 64 && (devices.load(std::memory_order_acquire) & bit)) return hipSuccess;
    e = hipFuncSetAttribute(reinterpret_cast<const void *>(Kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e == hipSuccess) devices.fetch_or(bit, std::memory_order_release);
    return e;
}

// ---- device helpers -------------------------------------------------------

template <class T>
struct Elem;
template <>
struct Elem<float> {
    static __device__ float get(float v) { return v; }
    static __device__ float put(float v) { return v; }
};
template <>
struct Elem<__bf16> {
    static __device__ float get(__bf16 v) { return (float)v; }
    static __device__ __bf16 put(float v) { return (__bf16)v; }  // to nearest, ties to even
};
template <>
struct Elem<_Float16> {
    static __device__ float get(_Float16 v) { return (float)v; }
    static __device__ _Float16 put(float v) { return (_Float16)v; }
};

// The scale byte as the float 2^(byte - 127) whose exponent the conversion
// instructions read; NaN for 255.
__device__ inline float mx_scale(uint32_t byte)
{
    return __uint_as_float(byte == 255u ? 0x7FC00000u : byte << 23);
}
#endif

}  // namespace pccl
