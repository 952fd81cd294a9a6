// C ABI of the operators at the ends of a collective: argument checks and
// launches.  The work runs in pccl_mx.hip, pccl_mx_matmul.hip, pccl_route.hip
// and pccl_moe.hip.
#include <cstdarg>
#include <cstdio>
#include <exception>

#include "pccl.h"
#include "pccl_ops.h"

namespace pccl {
int ctx_device(const pccl_ctx *c);
void ctx_set_error(pccl_ctx *c, const char *text);
}  // namespace pccl

using namespace pccl;

namespace {

pccl_status fail(pccl_ctx *c, pccl_status st, const char *fmt, ...) __attribute__((format(printf, 3, 4)));
pccl_status fail(pccl_ctx *c, pccl_status st, const char *fmt, ...)
{
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    ctx_set_error(c, buf);
    return st;
}

typedef unsigned long long ull;

bool aligned(const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }
size_t elem_bytes(pccl_dtype t) { return t == PCCL_F32 ? 4 : 2; }

// The body of an entry point: no exception crosses the ABI.
template <class F>
pccl_status entry(pccl_ctx *c, F &&body)
{
    if (!c) return PCCL_EINVAL;
    try {
        ctx_set_error(c, "");
        return body();
    } catch (const std::exception &ex) {
        return fail(c, PCCL_EINTERNAL, "exception: %s", ex.what());
    } catch (...) {
        return fail(c, PCCL_EINTERNAL, "unknown exception");
    }
}

#define NEED(cond, ...)                                            \
    do {                                                           \
        if (!(cond)) return fail(c, PCCL_EINVAL, __VA_ARGS__);     \
    } while (0)
#define LIMIT(cond, ...)                                               \
    do {                                                               \
        if (!(cond)) return fail(c, PCCL_EUNSUPPORTED, __VA_ARGS__);   \
    } while (0)

// The context's device for the launches of a call; the caller's again at its end.
class OnDevice {
public:
    pccl_status enter(pccl_ctx *c)
    {
        int now = 0;
        hipError_t e = hipGetDevice(&now);
        if (e == hipSuccess && now != ctx_device(c)) {
            e = hipSetDevice(ctx_device(c));
            if (e == hipSuccess) before_ = now;
        }
        return e == hipSuccess ? PCCL_OK : fail(c, PCCL_EDEVICE, "no device: %s", hipGetErrorString(e));
    }
    ~OnDevice()
    {
        if (before_ >= 0) (void)hipSetDevice(before_);
    }

private:
    int before_ = -1;
};

pccl_status launched(pccl_ctx *c, hipError_t e, const char *what)
{
    return e == hipSuccess ? PCCL_OK : fail(c, PCCL_EDEVICE, "%s: %s", what, hipGetErrorString(e));
}

// A matrix argument: `ld` elements from row to row, elements of `bytes` bytes.
pccl_status check_rows(pccl_ctx *c, const char *name, const void *p, uint64_t rows, uint64_t cols, uint64_t ld, size_t bytes)
{
    LIMIT(rows <= OPS_MAX_EXTENT && cols <= OPS_MAX_EXTENT, "%s: %llu x %llu (limit 2^31 - 1 either way)", name, (ull)rows, (ull)cols);
    if (rows == 0 || cols == 0) return PCCL_OK;
    NEED(p, "%s is null", name);
    NEED(aligned(p, bytes), "%s is not aligned to its elements", name);
    NEED(ld >= cols, "%s: row stride %llu below the row's %llu elements", name, (ull)ld, (ull)cols);
    LIMIT(ld <= OPS_MAX_EXTENT, "%s: row stride %llu (limit 2^31 - 1)", name, (ull)ld);
    return PCCL_OK;
}

// A packed argument.
pccl_status check_packed(pccl_ctx *c, const char *name, const void *codes, const void *scales)
{
    NEED(codes && scales, "%s: codes or scales are null", name);
    NEED(aligned(codes, 16) && aligned(scales, 4), "%s: codes need 16-byte, scales 4-byte alignment", name);
    return PCCL_OK;
}

// A launch of `blocks` workgroups must stay below 2^32 threads.
pccl_status check_grid(pccl_ctx *c, uint64_t blocks, uint32_t threads)
{
    LIMIT(blocks <= most_blocks(threads), "%llu workgroups in one launch (limit %llu)", (ull)blocks, (ull)most_blocks(threads));
    return PCCL_OK;
}

pccl_status check_space(pccl_ctx *c, const void *ws, size_t have, size_t need)
{
    if (need == 0) return PCCL_OK;
    NEED(ws, "workspace is null (%llu bytes needed)", (ull)need);
    NEED(aligned(ws, 256), "workspace is not 256-byte aligned");
    if (have < need) return fail(c, PCCL_ENOMEM, "workspace of %llu bytes, %llu needed", (ull)have, (ull)need);
    return PCCL_OK;
}

#define TRY(expr)                             \
    do {                                      \
        const pccl_status st_ = (expr);       \
        if (st_ != PCCL_OK) return st_;       \
    } while (0)

pccl_status check_picks(pccl_ctx *c, uint64_t tokens, uint32_t experts, uint32_t topk)
{
    NEED(experts > 0, "no experts");
    NEED(topk > 0 && topk <= experts, "topk %u of %u experts", topk, experts);
    LIMIT(experts <= ROUTE_MAX_EXPERTS, "%u experts (limit %u)", experts, ROUTE_MAX_EXPERTS);
    LIMIT(topk <= ROUTE_MAX_TOPK, "topk %u (limit %u)", topk, ROUTE_MAX_TOPK);
    LIMIT(tokens <= OPS_MAX_EXTENT / topk, "%llu tokens with %u picks each (limit 2^31 - 1 slots)", (ull)tokens, topk);
    return PCCL_OK;
}

pccl_status check_dtype(pccl_ctx *c, pccl_dtype t)
{
    NEED(t == PCCL_F32 || t == PCCL_BF16 || t == PCCL_F16, "unknown element type %d", (int)t);
    return PCCL_OK;
}

pccl_status check_layer(pccl_ctx *c, uint32_t tokens, uint32_t experts, uint32_t topk, uint32_t hidden, uint32_t inter)
{
    TRY(check_picks(c, tokens, experts, topk));
    LIMIT(tokens <= MOE_MAX_TOKENS, "%u tokens (limit %u)", tokens, MOE_MAX_TOKENS);
    NEED(hidden > 0 && inter > 0, "hidden %u, inter %u", hidden, inter);
    LIMIT(hidden <= MOE_MAX_DIM && inter <= MOE_MAX_DIM, "hidden %u, inter %u (limit %u)", hidden, inter, MOE_MAX_DIM);
    LIMIT((uint64_t)hidden * inter <= MOE_MAX_MATRIX, "hidden %u x inter %u (limit 2^29 values)", hidden, inter);
    return PCCL_OK;
}

}  // namespace

extern "C" {

pccl_status pccl_mx_quantize(pccl_ctx *c, const void *x, pccl_dtype dtype, uint64_t rows, uint64_t cols, uint64_t ld,
                             uint8_t *codes, uint8_t *scales, uint8_t *codes_t, uint8_t *scales_t, void *hip_stream)
{
    return entry(c, [&]() -> pccl_status {
        TRY(check_dtype(c, dtype));
        TRY(check_rows(c, "x", x, rows, cols, ld, elem_bytes(dtype)));
        if (rows == 0 || cols == 0) return PCCL_OK;   // what is written is empty too, and has no address
        NEED(codes || scales || codes_t || scales_t, "no output");
        if (codes || scales) TRY(check_packed(c, "rows", codes, scales));
        if (codes_t || scales_t) TRY(check_packed(c, "columns", codes_t, scales_t));
        if (codes_t) TRY(check_grid(c, ((rows + 127) / 128) * ((cols + 127) / 128), 256));
        OnDevice device;
        TRY(device.enter(c));
        const MxQuantizeArgs a{x, rows, cols, ld, codes, scales, codes_t, scales_t};
        return launched(c, launch_mx_quantize(a, dtype, (hipStream_t)hip_stream), "mx_quantize");
    });
}

pccl_status pccl_mx_dequantize(pccl_ctx *c, const uint8_t *codes, const uint8_t *scales, uint64_t rows, uint64_t cols,
                               void *out, pccl_dtype dtype, uint64_t ld, void *hip_stream)
{
    return entry(c, [&]() -> pccl_status {
        TRY(check_dtype(c, dtype));
        TRY(check_rows(c, "out", out, rows, cols, ld, elem_bytes(dtype)));
        if (rows == 0 || cols == 0) return PCCL_OK;
        TRY(check_packed(c, "input", codes, scales));
        OnDevice device;
        TRY(device.enter(c));
        const MxDequantizeArgs a{codes, scales, rows, cols, ld, out};
        return launched(c, launch_mx_dequantize(a, dtype, (hipStream_t)hip_stream), "mx_dequantize");
    });
}

pccl_status pccl_mx_matmul_workspace(pccl_ctx *c, uint64_t m, uint64_t n, uint64_t k, size_t *out_bytes)
{
    return entry(c, [&]() -> pccl_status {
        NEED(out_bytes, "out_bytes is null");
        *out_bytes = 0;
        LIMIT(m <= OPS_MAX_EXTENT && n <= OPS_MAX_EXTENT && k <= MX_MAX_K, "%llu x %llu x %llu (limits 2^31 - 1, 2^31 - 1, 2^24)", (ull)m, (ull)n, (ull)k);
        if (m && n) *out_bytes = mx_matmul_workspace(m, n, k);
        return PCCL_OK;
    });
}

pccl_status pccl_mx_matmul(pccl_ctx *c, const uint8_t *a_codes, const uint8_t *a_scales, const uint8_t *b_codes,
                           const uint8_t *b_scales, uint64_t m, uint64_t n, uint64_t k, void *out, pccl_dtype dtype,
                           uint64_t ld, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    return entry(c, [&]() -> pccl_status {
        TRY(check_dtype(c, dtype));
        LIMIT(k <= MX_MAX_K, "k = %llu (limit 2^24)", (ull)k);
        TRY(check_rows(c, "out", out, m, n, ld, elem_bytes(dtype)));
        if (m == 0 || n == 0) return PCCL_OK;
        if (k) {
            TRY(check_packed(c, "a", a_codes, a_scales));
            TRY(check_packed(c, "b", b_codes, b_scales));
        }
        LIMIT(mx_matmul_fits(m, n, k), "%llu x %llu (limit 2^23 - 1 tiles of 256 x 256)", (ull)m, (ull)n);
        TRY(check_space(c, workspace, workspace_bytes, mx_matmul_workspace(m, n, k)));
        OnDevice device;
        TRY(device.enter(c));
        const MxMatmulArgs a{a_codes, a_scales, b_codes, b_scales, m, n, k, ld, out, (float *)workspace};
        return launched(c, launch_mx_matmul(a, dtype, (hipStream_t)hip_stream), "mx_matmul");
    });
}

pccl_status pccl_moe_route_workspace(pccl_ctx *c, uint64_t tokens, uint32_t experts, uint32_t topk, size_t *out_bytes)
{
    return entry(c, [&]() -> pccl_status {
        NEED(out_bytes, "out_bytes is null");
        *out_bytes = 0;
        TRY(check_picks(c, tokens, experts, topk));
        *out_bytes = route_workspace(tokens, experts);
        return PCCL_OK;
    });
}

pccl_status pccl_moe_route(pccl_ctx *c, const void *logits, pccl_dtype dtype, uint64_t tokens, uint32_t experts, uint64_t ld,
                           uint32_t topk, int normalize, const uint8_t *token_mask, float *weights, int32_t *ids,
                           int32_t *counts, int32_t *order, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    return entry(c, [&]() -> pccl_status {
        TRY(check_dtype(c, dtype));
        TRY(check_picks(c, tokens, experts, topk));
        TRY(check_rows(c, "logits", logits, tokens, experts, ld, elem_bytes(dtype)));
        NEED(counts && aligned(counts, 4), "counts are null or misaligned");
        if (tokens) {
            NEED(weights && aligned(weights, 4), "weights are null or misaligned");
            NEED(ids && aligned(ids, 4), "ids are null or misaligned");
            NEED(order && aligned(order, 4), "order is null or misaligned");
        }
        TRY(check_grid(c, (tokens + ROUTE_ROWS - 1) / ROUTE_ROWS, 1024));
        TRY(check_space(c, workspace, workspace_bytes, route_workspace(tokens, experts)));
        OnDevice device;
        TRY(device.enter(c));
        const RouteArgs a{logits, tokens, ld, experts, topk, normalize ? 1u : 0u, token_mask, weights, ids, counts, order, (uint32_t *)workspace};
        return launched(c, launch_route(a, dtype, (hipStream_t)hip_stream), "moe_route");
    });
}

pccl_status pccl_moe_route_backward(pccl_ctx *c, const void *logits, pccl_dtype dtype, uint64_t tokens, uint32_t experts,
                                    uint64_t ld, uint32_t topk, int normalize, const uint8_t *token_mask,
                                    const float *weights, const int32_t *ids, const float *dweights, void *dlogits,
                                    uint64_t ld_d, void *hip_stream)
{
    return entry(c, [&]() -> pccl_status {
        TRY(check_dtype(c, dtype));
        TRY(check_picks(c, tokens, experts, topk));
        if (!normalize) TRY(check_rows(c, "logits", logits, tokens, experts, ld, elem_bytes(dtype)));
        TRY(check_rows(c, "dlogits", dlogits, tokens, experts, ld_d, elem_bytes(dtype)));
        if (tokens == 0) return PCCL_OK;
        NEED(weights && aligned(weights, 4), "weights are null or misaligned");
        NEED(ids && aligned(ids, 4), "ids are null or misaligned");
        NEED(dweights && aligned(dweights, 4), "dweights are null or misaligned");
        OnDevice device;
        TRY(device.enter(c));
        const RouteBackwardArgs a{logits, tokens, ld, ld_d, experts, topk, normalize ? 1u : 0u, token_mask, weights, ids, dweights, dlogits};
        return launched(c, launch_route_backward(a, dtype, (hipStream_t)hip_stream), "moe_route_backward");
    });
}

pccl_status pccl_moe_layer_workspace(pccl_ctx *c, uint32_t tokens, uint32_t experts, uint32_t topk, uint32_t hidden,
                                     uint32_t inter, size_t *out_bytes)
{
    return entry(c, [&]() -> pccl_status {
        NEED(out_bytes, "out_bytes is null");
        *out_bytes = 0;
        TRY(check_layer(c, tokens, experts, topk, hidden, inter));
        if (tokens) *out_bytes = moe_workspace(tokens, experts, topk, hidden, inter);
        return PCCL_OK;
    });
}

pccl_status pccl_moe_layer(pccl_ctx *c, const void *x, pccl_dtype dtype, uint64_t ld_x, uint32_t tokens, uint32_t experts,
                           uint32_t topk, uint32_t hidden, uint32_t inter, int normalize, const uint8_t *token_mask,
                           const void *router, const void *up, const uint8_t *up_scales, const void *down,
                           const uint8_t *down_scales, void *y, uint64_t ld_y, void *workspace, size_t workspace_bytes,
                           void *hip_stream)
{
    return entry(c, [&]() -> pccl_status {
        NEED(dtype == PCCL_BF16 || dtype == PCCL_F16, "element type %d: bf16 or f16 is needed", (int)dtype);
        TRY(check_layer(c, tokens, experts, topk, hidden, inter));
        TRY(check_rows(c, "x", x, tokens, hidden, ld_x, 2));
        TRY(check_rows(c, "y", y, tokens, hidden, ld_y, 2));
        NEED(router && aligned(router, 2), "router weights are null or misaligned");
        NEED((up_scales == nullptr) == (down_scales == nullptr), "either both or neither of up and down are packed");
        if (up_scales) {
            TRY(check_packed(c, "up", up, up_scales));
            TRY(check_packed(c, "down", down, down_scales));
        } else {
            NEED(up && aligned(up, 2), "up is null or misaligned");
            NEED(down && aligned(down, 2), "down is null or misaligned");
        }
        if (tokens == 0) return PCCL_OK;
        TRY(check_space(c, workspace, workspace_bytes, moe_workspace(tokens, experts, topk, hidden, inter)));
        OnDevice device;
        TRY(device.enter(c));
        const MoeArgs a{x, ld_x, ld_y, tokens, experts, topk, hidden, inter, normalize ? 1u : 0u, token_mask, router, up, down,
                        up_scales, down_scales, y, (char *)workspace};
        return launched(c, launch_moe(a, dtype, (hipStream_t)hip_stream), "moe_layer");
    });
}

}  // extern "C"
