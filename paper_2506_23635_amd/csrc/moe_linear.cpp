// moe_linear.cpp -- the C-ABI of the plain product in e4m3 and of coding rows
// (include/moe.h, "Products in e4m3"): checks, the buffers' division, launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <new>
#include <string>

#include "../../include/moe.h"
#include "moe_common.h"

namespace {

constexpr int kFewTokens = 16;          // rows of one MFMA B operand
constexpr int kRowTile = 128;           // rows of a tile of a product with ranges of K; ...
constexpr int kSplitRows = 64;          // ... up to these rows there are always such tiles
constexpr int kMostSplit = 16384;       // ... and beyond these none has ranges (two feature tiles at least)
constexpr int kFeatures = 256;          // packed features come in multiples of a tile's
constexpr int64_t kMostStride = 1ll << 32;   // elements between rows (offsets stay below 2^63)
constexpr int64_t kMostBlocks = 1ll << 31;   // that moe_quantize_e4m3 codes in a call
constexpr size_t kAlign = 256;

size_t align_up(size_t v, size_t a) { return (v + a - 1) / a * a; }
bool misaligned(const void* p) { return ((uintptr_t)p & 15u) != 0; }

bool overlap(const void* a, size_t na, const void* b, size_t nb)
{
    const uintptr_t p = (uintptr_t)a, q = (uintptr_t)b;
    return p < q + nb && q < p + na;
}

struct Layout {
    int K, N;                           // padded
    size_t scales_off, weight_bytes, parts_off, ws_bytes;
};

// Ranges of K of a call with T rows (more than kFewTokens).
int n_split(const Layout& L, int T)
{
    return moe_gemm_mid_tiles(T, 1, 1, 1, L.N) ? moe_gemm_linear_split(T, L.K, L.N) : 1;
}

const char* check_config(const moe_linear_config* c)
{
    constexpr int kMost = 1 << 20;
    if (!c) return "config is NULL";
    if (c->in_dim < 16 || c->in_dim > kMost || c->in_dim % 16) return "in_dim must be a multiple of 16 in [16, 2^20]";
    if (c->out_dim < 16 || c->out_dim > kMost || c->out_dim % 16) return "out_dim must be a multiple of 16 in [16, 2^20]";
    if (c->max_tokens < 1 || c->max_tokens > kMost) return "max_tokens must be in [1, 2^20]";
    if (align_up(c->in_dim, 256) * align_up(c->out_dim, 256) > INT32_MAX)
        return "in_dim * out_dim must stay below 2^31 (32-bit offsets)";
    if ((size_t)c->max_tokens * align_up(c->in_dim, moe::kBlock) * 2 > INT32_MAX)
        return "max_tokens * in_dim * 2 must stay below 2^31 (32-bit offsets)";
    if (c->flags) return "flags must be 0";
    return nullptr;
}

Layout make_layout(const moe_linear_config* c)
{
    Layout L{};
    L.K = (int)align_up(c->in_dim, moe::kBlock);
    L.N = (int)align_up(c->out_dim, kFeatures);
    const size_t quads = moe::scale_quads(L.K);
    L.scales_off = (size_t)L.K * L.N;
    L.weight_bytes = align_up(L.scales_off + (size_t)(L.N / moe::kBlock) * quads * 4, kAlign);
    // rows on the e4m3 grid, then the sums of the ranges of K, for the call that
    // needs the most: calls whose last row tile is the same have as many ranges
    L.parts_off = align_up((size_t)c->max_tokens * L.K * 2, kAlign);
    size_t parts = 0;
    for (int rows = kSplitRows; rows <= kMostSplit; rows += rows < kRowTile ? kRowTile - rows : kRowTile) {
        const int T = std::min(rows, c->max_tokens), n = T > kFewTokens ? n_split(L, T) : 1;
        if (n > 1) parts = std::max(parts, (size_t)n * T * c->out_dim * 4);
        if (T == c->max_tokens) break;
    }
    L.ws_bytes = align_up(L.parts_off + parts, kAlign);
    return L;
}

thread_local std::string g_init_error;

}  // namespace

struct moe_linear {
    moe_linear_config cfg;
    Layout L;
    uint8_t *weights, *workspace;
    bool loaded;
    std::string err;
};

namespace {

moe_status fail(moe_linear* ctx, moe_status s, const std::string& msg)
{
    if (ctx) ctx->err = msg;
    else g_init_error = msg;
    return s;
}

moe_status hip_fail(moe_linear* ctx, hipError_t e, const char* what)
{
    return fail(ctx, MOE_E_HIP, std::string(what) + ": " + hipGetErrorString(e));
}

}  // namespace

extern "C" {

moe_status moe_quantize_e4m3(const void* x, int64_t ld, int32_t type, int32_t T, int32_t n, uint8_t* codes,
                             uint8_t* scales, moe_stream_t stream)
{
    if (type != MOE_T_F32 && type != MOE_T_BF16) return MOE_E_ARG;
    if (T < 0) return MOE_E_ARG;
    if (n < 16 || n % 16 || n > 1 << 24 || T > 1 << 24) return MOE_E_SHAPE;
    if ((int64_t)T * ((n + moe::kBlock - 1) / moe::kBlock) > kMostBlocks) return MOE_E_SHAPE;
    if (T == 0) return MOE_OK;
    if (!x || !codes || !scales || ld < n || ld > kMostStride) return MOE_E_ARG;
    const int size = type == MOE_T_F32 ? 4 : 2, blocks = (n + moe::kBlock - 1) / moe::kBlock;
    if (misaligned(x) || misaligned(codes) || (T > 1 && ld % (16 / size))) return MOE_E_ALIGN;
    const size_t x_bytes = ((size_t)(T - 1) * (size_t)ld + n) * size, c_bytes = (size_t)T * n, s_bytes = (size_t)T * blocks;
    if (overlap(x, x_bytes, codes, c_bytes) || overlap(x, x_bytes, scales, s_bytes) ||
        overlap(codes, c_bytes, scales, s_bytes))
        return MOE_E_ARG;
    const hipError_t e = moe_launch_quantize(x, ld, type == MOE_T_BF16, T, nullptr, n, n, codes, scales, nullptr,
                                             static_cast<hipStream_t>(stream));
    return e == hipSuccess ? MOE_OK : MOE_E_HIP;
}

size_t moe_linear_weight_bytes(const moe_linear_config* cfg)
{
    return check_config(cfg) ? 0 : make_layout(cfg).weight_bytes;
}

size_t moe_linear_workspace_bytes(const moe_linear_config* cfg)
{
    return check_config(cfg) ? 0 : make_layout(cfg).ws_bytes;
}

moe_status moe_linear_init(const moe_linear_config* cfg, void* weights, void* workspace, moe_linear** out)
{
    if (!out) return fail(nullptr, MOE_E_ARG, "out is NULL");
    *out = nullptr;
    if (const char* why = check_config(cfg)) return fail(nullptr, MOE_E_SHAPE, why);
    if (!weights || !workspace) return fail(nullptr, MOE_E_ARG, "weights or workspace is NULL");
    if (((uintptr_t)weights & (kAlign - 1)) || ((uintptr_t)workspace & (kAlign - 1)))
        return fail(nullptr, MOE_E_ALIGN, "weights and workspace must be 256-byte aligned");
    moe_linear* c = new (std::nothrow) moe_linear();
    if (!c) return fail(nullptr, MOE_E_ARG, "out of host memory");
    c->cfg = *cfg;
    c->L = make_layout(cfg);
    c->weights = static_cast<uint8_t*>(weights);
    c->workspace = static_cast<uint8_t*>(workspace);
    *out = c;
    return MOE_OK;
}

moe_status moe_linear_load(moe_linear* ctx, const uint16_t* w, moe_stream_t stream)
{
    if (!ctx) return MOE_E_ARG;
    if (!w) return fail(ctx, MOE_E_ARG, "w is NULL");
    if (misaligned(w)) return fail(ctx, MOE_E_ALIGN, "w must be 16-byte aligned");
    const hipError_t e = moe_launch_pack_e4m3(w, ctx->cfg.in_dim, ctx->cfg.out_dim, ctx->L.K, ctx->L.N, ctx->weights,
                                              ctx->weights + ctx->L.scales_off, 1, 0, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(ctx, e, "pack kernel launch");
    ctx->loaded = true;
    return MOE_OK;
}

moe_status moe_linear_forward(moe_linear* ctx, const uint16_t* x, int64_t ldx, void* y, int32_t type, int32_t T,
                              moe_stream_t stream)
{
    if (!ctx) return MOE_E_ARG;
    const moe_linear_config& c = ctx->cfg;
    if (T < 0) return fail(ctx, MOE_E_ARG, "T is negative");
    if (T > c.max_tokens) return fail(ctx, MOE_E_CAPACITY, "T exceeds max_tokens");
    if (type != MOE_T_F32 && type != MOE_T_BF16) return fail(ctx, MOE_E_ARG, "type is no moe_type");
    if (!ctx->loaded) return fail(ctx, MOE_E_STATE, "no weights loaded");
    if (T == 0) return MOE_OK;
    if (!x || !y) return fail(ctx, MOE_E_ARG, "x or y is NULL");
    if (ldx < c.in_dim || ldx > kMostStride) return fail(ctx, MOE_E_ARG, "ldx is below in_dim or above 2^32");
    if (misaligned(x) || misaligned(y) || (T > 1 && ldx % 8))
        return fail(ctx, MOE_E_ALIGN, "x, its rows and y must be 16-byte aligned");
    if (overlap(x, ((size_t)(T - 1) * (size_t)ldx + c.in_dim) * 2, y, (size_t)T * c.out_dim * (type == MOE_T_F32 ? 4 : 2)))
        return fail(ctx, MOE_E_ARG, "y overlaps x");
    hipStream_t s = static_cast<hipStream_t>(stream);
    uint16_t* xq = reinterpret_cast<uint16_t*>(ctx->workspace);
    const bool raw = moe_e4m3_linear_raw(T, ctx->L.K);
    hipError_t e = hipSuccess;
    if (!raw) e = moe_launch_quantize(x, ldx, 1, T, nullptr, c.in_dim, ctx->L.K, nullptr, nullptr, xq, s);
    if (e != hipSuccess) return hip_fail(ctx, e, "quantize kernel launch");
    float* y32 = type == MOE_T_F32 ? static_cast<float*>(y) : nullptr;
    uint16_t* y16 = type == MOE_T_F32 ? nullptr : static_cast<uint16_t*>(y);
    if (T <= kFewTokens) {
        moe::E4m3Args a{};
        a.w = ctx->weights;
        a.ws = ctx->weights + ctx->L.scales_off;
        a.x = raw ? x : xq;
        a.ldx = ldx;
        a.raw_K = raw ? c.in_dim : 0;
        a.K = ctx->L.K;
        a.N = c.out_dim;
        a.T = T;
        a.y32 = y32;
        a.y16 = y16;
        e = moe_launch_e4m3_linear_few(&a, s);
    } else {
        moe::GemmArgs a{};
        a.experts = ctx->weights;
        a.expert_bytes = ctx->L.scales_off;
        a.scales = ctx->weights + ctx->L.scales_off;
        a.H = xq;
        a.O = y32;
        a.y16 = y16;
        a.f = ctx->L.K;
        a.d = ctx->L.N;
        a.n_out = c.out_dim;
        a.n_local = 1;
        a.T = a.max_rows = T;
        a.mid = moe_gemm_mid_tiles(T, 1, 1, 1, ctx->L.N);
        a.k_split = n_split(ctx->L, T);
        a.mid_rows = moe_gemm_mid_rows(T, 1, 1, 1, ctx->L.N, a.k_split, 1);
        if (a.k_split > 1) {
            a.O = reinterpret_cast<float*>(ctx->workspace + ctx->L.parts_off);
            a.split_stride = (uint64_t)T * c.out_dim;
        }
        e = moe_launch_gemm_linear(&a, s);
        if (e == hipSuccess && a.k_split > 1)
            e = moe_launch_linear_sum(a.O, a.k_split, (int64_t)a.split_stride, (int64_t)a.split_stride, y32, y16, s);
    }
    if (e != hipSuccess) return hip_fail(ctx, e, "product kernel launch");
    return MOE_OK;
}

void moe_linear_destroy(moe_linear* ctx) { delete ctx; }

const char* moe_linear_last_error(const moe_linear* ctx)
{
    return ctx ? ctx->err.c_str() : g_init_error.c_str();
}

}  // extern "C"
