// moe_e4m3.hip -- 8-bit floating point for the experts and for plain products
// (include/moe.h, "Products in e4m3"): coding rows and weights, and the products
// of few rows (many rows: moe_prefill.hip).
//
// A code times its scale, a power of two, has 4 significant bits, so it is a
// bf16 exactly, and products of two of them are exact in fp32.  The matrix
// products therefore run on the bf16 instructions, weights decoded in registers
// (v_cvt_scalef32_pk_bf16_fp8: two codes and their scale), rows kept as bf16
// values on the e4m3 grid.  The matrix instructions that take 8-bit operands
// would do the same work at twice the rate, but their sums are not fp32 sums:
// within a lane's terms they are aligned to the largest and lose what lies below
// 2^-13 of it (profiles/e4m3_mfma_sums.txt: 16x16x32 and the scaled 16x16x128 and
// 32x32x64, beside bf16's, which keep 2^-24).  A product of 333 x 1040 x 1488 came
// out 4.9e-5 from its fp64 value so, where fp32 sums leave 1e-7, and it moves silu(G) U
// across rounding borders before the down product.
#include <cmath>
#include <cstring>

#include "e4m3.h"
#include "moe_common.h"

namespace moe {

// ------------------------------------------------------------------ coding --

// Rows to codes and scales, or (codes NULL) to the bf16 values that these stand
// for: 16 lanes per block of 128, 8 elements each.  Rows are read once and written
// once: 2048 x 6144 from bf16 to codes, 38 MB, in 7.5 to 8.1 us, 4.7 to 5.0 TB/s (two
// blocks per thread at a time 7.5, four 9.0).  Values from n to n_pad are zeros.  n_rows
// (device memory): rows that are written, of at most T; or NULL.  Blocks are counted
// in 32 bits (a division in 64 per block took longer than the rest).
template <bool kBf16>
__global__ __launch_bounds__(256) void quantize_kernel(const void* __restrict__ x, int64_t ld, uint32_t T,
                                                       const int32_t* __restrict__ n_rows, int n, int n_pad,
                                                       uint8_t* __restrict__ codes, uint8_t* __restrict__ scales,
                                                       uint16_t* __restrict__ values)
{
    const uint32_t blocks = (uint32_t)((n + kBlock - 1) / kBlock), units = T * blocks;
    const int piece = threadIdx.x % 16;
    const int64_t rows = n_rows ? (int64_t)*n_rows : (int64_t)T;
    for (uint32_t u = blockIdx.x * 16 + threadIdx.x / 16; u < units; u += gridDim.x * 16) {
        const int64_t t = (int64_t)(u / blocks);
        const int b = (int)(u - (uint32_t)t * blocks), k = b * kBlock + piece * 8;
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (k < n) {
            if constexpr (kBf16) {
                unpack8(*reinterpret_cast<const u32x4_t*>(static_cast<const uint16_t*>(x) + t * ld + k), v);
            } else {
                const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(x) + t * ld + k);
                const float4 p0 = p[0], p1 = p[1];
                v[0] = p0.x; v[1] = p0.y; v[2] = p0.z; v[3] = p0.w;
                v[4] = p1.x; v[5] = p1.y; v[6] = p1.z; v[7] = p1.w;
            }
        }
        const Coded c = code_block(v);
        if (t >= rows) continue;
        if (codes) {
            if (k < n) *reinterpret_cast<uint2*>(codes + t * n + k) = make_uint2(c.lo, c.hi);
            if (piece == 0) scales[t * (int64_t)blocks + b] = (uint8_t)(c.e + 127);
        } else if (k < n_pad) {
            *reinterpret_cast<u32x4_t*>(values + t * n_pad + k) = decode8(c.lo, c.hi, exp2i(c.e));
        }
    }
}

// Weights src bf16 [K][N] to the packed layout and the scales of their 128 x 128
// blocks, one block per workgroup: feature n goes to row tile (n / 16) rt_mul +
// rt_add.  Rows and features past K and N (up to whole blocks) are zeros.
__global__ __launch_bounds__(256) void pack_e4m3_kernel(const uint16_t* __restrict__ src, int K, int N,
                                                        uint8_t* __restrict__ dst, uint8_t* __restrict__ scales,
                                                        int KT, int scale_ld, int rt_mul, int rt_add)
{
    __shared__ uint16_t tile[kBlock][kBlock + 2];
    __shared__ float s_max[4];
    const int n0 = blockIdx.x * kBlock, kt = blockIdx.y, k0 = kt * kBlock, tid = threadIdx.x;
    float amax = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = i * 16 + tid / 16, c = tid % 16 * 8;
        u32x4_t v = {0u, 0u, 0u, 0u};
        if (k0 + r < K && n0 + c < N) v = *reinterpret_cast<const u32x4_t*>(src + (int64_t)(k0 + r) * N + n0 + c);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            *reinterpret_cast<uint32_t*>(&tile[r][c + 2 * j]) = v[j];
            const float lo = __uint_as_float(v[j] << 16), hi = __uint_as_float(v[j] & 0xFFFF0000u);
            if (finite(lo)) amax = fmaxf(amax, fabsf(lo));
            if (finite(hi)) amax = fmaxf(amax, fabsf(hi));
        }
    }
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) amax = fmaxf(amax, __shfl_xor(amax, o, 64));
    if (tid % 64 == 0) s_max[tid / 64] = amax;
    __syncthreads();
    const int e = scale_exponent(fmaxf(fmaxf(s_max[0], s_max[1]), fmaxf(s_max[2], s_max[3])));
    // the last block's workgroup also clears the bytes up to the row's end
    if (tid == 0) scales[(int64_t)blockIdx.x * scale_ld + kt] = (uint8_t)(e + 127);
    else if (kt + 1 == (int)gridDim.y && kt + tid < scale_ld) scales[(int64_t)blockIdx.x * scale_ld + kt + tid] = 0;
    const float inv = exp2i(-e);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        // granule c % 4 of the block's K tile c / 4: K 8 g .. 8 g + 7 and 32 on
        const int g = i * 256 + tid, n = g % kBlock, c = g / kBlock;
        u32x4_t w;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int k = c / 4 * kTileK8 + j / 2 * 32 + c % 4 * 8 + j % 2 * 4;
            float v[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] = bf16_to_f32(tile[k + q][n]);
            w[j] = code4(v, inv);
        }
        const int64_t rt = (int64_t)((n0 + n) / kTileRows) * rt_mul + rt_add;
        *reinterpret_cast<u32x4_t*>(dst + tile_offset8(rt, kt * 2 + c / 4, KT) + c % 4 * 256 + n % kTileRows * 16) = w;
    }
}

// The sums of a plain product's ranges of K, in their order; count is a multiple
// of 16.
__global__ __launch_bounds__(256) void linear_sum_kernel(const float* __restrict__ parts, int n, int64_t stride,
                                                         int64_t count, float* __restrict__ y32,
                                                         uint16_t* __restrict__ y16)
{
    const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (i >= count) return;
    float4 v = *reinterpret_cast<const float4*>(parts + i);
    for (int q = 1; q < n; ++q) {
        const float4 p = *reinterpret_cast<const float4*>(parts + q * stride + i);
        v = make_float4(v.x + p.x, v.y + p.y, v.z + p.z, v.w + p.w);
    }
    if (y32)
        *reinterpret_cast<float4*>(y32 + i) = v;
    else
        *reinterpret_cast<uint2*>(y16 + i) = make_uint2(cvt_pk_bf16(v.x, v.y), cvt_pk_bf16(v.z, v.w));
}

// --------------------------------------------------------------- few rows --
//
// At most 16 rows per expert (or of a plain product): the weights are streamed
// once, one 16-feature tile (gate/up: the tiles of both) per workgroup, the K
// tiles dealt to its waves in turn, as in the bf16 decode kernels.  The weight
// tile is the A operand, the rows are the B operand.

constexpr int kFewWaves = 8;

// kFewLinearRaw: rows as they come; every workgroup rounds them itself, into LDS,
// while its first weights are on their way
enum { kFewGateUp = 0, kFewDown = 1, kFewLinear = 2, kFewLinearRaw = 3 };

// K tiles per wave in flight, of each row tile (d 6144, f 10752, one token, where a
// wave has 12 K tiles of gate and up and 21 of down: gate/up 76.4 us with 3, 78.1
// with 4, 78.9 with 6; down 45.4 with 4, 43.0 with 7, 52.4 with 11; 6144 to 8192
// features 7.2 with 4, 7.6 with 6.  4 or 16 waves instead of 8: 2 to 15 % slower.)
constexpr int few_unroll(int mode) { return mode == kFewGateUp ? 3 : mode == kFewDown ? 7 : 4; }

template <int kMode>
__global__ __launch_bounds__(64 * kFewWaves) void few_kernel(E4m3Args a)
{
    constexpr int kM = kMode == kFewGateUp ? 2 : 1;      // row tiles per workgroup
    constexpr bool kExperts = kMode == kFewGateUp || kMode == kFewDown;
    constexpr bool kRaw = kMode == kFewLinearRaw;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    f32x4_t* s_red = reinterpret_cast<f32x4_t*>(lds);    // [kM][(kFewWaves - 1) * 64]
    uint16_t* s_x = reinterpret_cast<uint16_t*>(lds + kM * (kFewWaves - 1) * 64 * sizeof(f32x4_t));   // kRaw: [T][K]
    const int n_tiles = a.N / kTileRows, slot = blockIdx.x / n_tiles, p = blockIdx.x % n_tiles;
    int ge = 0, e = 0;
    if (kExperts) {
        if (slot >= a.active[0]) return;
        ge = a.active[1 + slot];
        e = ge - a.e_begin;
    }
    const int lane = threadIdx.x % 64, w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), j = lane % 16, g = lane / 16;
    const int KT = a.K / kTileK8, scale_ld = scale_quads(a.K) * 4;
    const uint64_t at = (uint64_t)e * a.expert_bytes;
    const uint8_t* pw[kM];
#pragma unroll
    for (int i = 0; i < kM; ++i) pw[i] = a.w + at + tile_offset8(p * kM + i, 0, KT) + lane * 16;
    const uint8_t* ps[2] = {a.ws + at + (int64_t)(p * kTileRows / kBlock) * scale_ld,
                            kM == 2 ? a.ws_up + at + (int64_t)(p * kTileRows / kBlock) * scale_ld : nullptr};
    // kUnroll K tiles at a time, w, w + kFewWaves, ...; past the last one they are
    // the last one again, with rows of zeros.  Lane u loads the scale of tile u.
    constexpr int kUnroll = few_unroll(kMode);
    u32x4_t wt[kM][kUnroll];
    int sc[kM];
    auto fetch = [&](int kt) {
        const int mine = min(kt + lane % kUnroll * kFewWaves, KT - 1);
#pragma unroll
        for (int i = 0; i < kM; ++i) sc[i] = ps[i][mine / 2];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
#pragma unroll
            for (int i = 0; i < kM; ++i)
                wt[i][u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(
                    pw[i] + (int64_t)min(kt + u * kFewWaves, KT - 1) * (kGroup8 * kTileBytes)));
    };
    // the weights' addresses are known before the rows'
    if (w < KT) fetch(w);
    const int m = kExperts ? a.counts[ge] : a.T, row0 = kExperts ? a.offsets[ge] : 0;
    const bool live = j < m;
    const uint16_t* px;
    if constexpr (kRaw) {
        const int blocks = a.K / kBlock;
        for (int u = threadIdx.x / 16; u < m * blocks; u += 64 * kFewWaves / 16) {
            const int t = u / blocks, k = u % blocks * kBlock + threadIdx.x % 16 * 8;
            float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            if (k < a.raw_K) unpack8(*reinterpret_cast<const u32x4_t*>(a.x + t * a.ldx + k), v);
            *reinterpret_cast<u32x4_t*>(&s_x[t * a.K + k]) = round_block(v);
        }
        __syncthreads();
        px = s_x + (live ? j * a.K : 0) + g * 8;
    } else {
        const int64_t row = live ? (kMode == kFewGateUp ? a.row_token[row0 + j] : row0 + j) : 0;
        px = a.x + row * a.K + g * 8;
    }
    f32x4_t acc[kM];
#pragma unroll
    for (int i = 0; i < kM; ++i) acc[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    for (int kt = w; kt < KT; kt += kUnroll * kFewWaves) {
        u32x4_t xb[kUnroll][2];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int t = kt + u * kFewWaves;
            xb[u][0] = xb[u][1] = u32x4_t{0u, 0u, 0u, 0u};
            if (live && t < KT) {
                xb[u][0] = *reinterpret_cast<const u32x4_t*>(px + t * kTileK8);
                xb[u][1] = *reinterpret_cast<const u32x4_t*>(px + t * kTileK8 + 32);
            }
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
#pragma unroll
            for (int i = 0; i < kM; ++i) {
                const float scale = __int_as_float(__builtin_amdgcn_readlane(sc[i], u) << 23);
                acc[i] = mfma16x16x32(decode8(wt[i][u][0], wt[i][u][1], scale), xb[u][0], acc[i]);
                acc[i] = mfma16x16x32(decode8(wt[i][u][2], wt[i][u][3], scale), xb[u][1], acc[i]);
            }
        if (kt + kUnroll * kFewWaves < KT) fetch(kt + kUnroll * kFewWaves);
    }
    constexpr int kRed = (kFewWaves - 1) * 64;
#pragma unroll
    for (int i = 0; i < kM; ++i)
        if (w > 0) s_red[i * kRed + (w - 1) * 64 + lane] = acc[i];
    __syncthreads();
    if (w > 0 || !live) return;
#pragma unroll
    for (int i = 0; i < kM; ++i)
        for (int q = 0; q + 1 < kFewWaves; ++q) acc[i] += s_red[i * kRed + q * 64 + lane];
    const int64_t out = (int64_t)(row0 + j) * a.N + p * kTileRows + g * 4;
    if constexpr (kMode == kFewGateUp)
        *reinterpret_cast<float4*>(a.h32 + out) =
            make_float4(silu_mul(acc[0][0], acc[1][0]), silu_mul(acc[0][1], acc[1][1]),
                        silu_mul(acc[0][2], acc[1][2]), silu_mul(acc[0][3], acc[1][3]));
    else if (kMode == kFewDown || a.y32)
        *reinterpret_cast<float4*>(a.y32 + out) = make_float4(acc[0][0], acc[0][1], acc[0][2], acc[0][3]);
    else
        *reinterpret_cast<uint2*>(a.y16 + out) =
            make_uint2(cvt_pk_bf16(acc[0][0], acc[0][1]), cvt_pk_bf16(acc[0][2], acc[0][3]));
}

}  // namespace moe

extern "C" {

// At most 2^31 blocks in all (and 16 of each of up to 65536 workgroups past them).
hipError_t moe_launch_quantize(const void* x, int64_t ld, int bf16, int64_t T, const int32_t* n_rows, int n,
                               int n_pad, uint8_t* codes, uint8_t* scales, uint16_t* values, hipStream_t s)
{
    const int64_t units = T * ((n + moe::kBlock - 1) / moe::kBlock), wgs = (units + 15) / 16;
    const dim3 grid((unsigned)(wgs < 65536 ? wgs : 65536)), block(256);
    const auto kernel = bf16 ? moe::quantize_kernel<true> : moe::quantize_kernel<false>;
    hipLaunchKernelGGL(kernel, grid, block, 0, s, x, ld, (uint32_t)T, n_rows, n, n_pad, codes, scales, values);
    return hipGetLastError();
}

hipError_t moe_launch_pack_e4m3(const uint16_t* src, int K, int N, int K_pad, int N_pad, uint8_t* dst,
                                uint8_t* scales, int rt_mul, int rt_add, hipStream_t s)
{
    hipLaunchKernelGGL(moe::pack_e4m3_kernel, dim3(N_pad / moe::kBlock, K_pad / moe::kBlock), dim3(256), 0, s, src, K,
                       N, dst, scales, K_pad / moe::kTileK8, moe::scale_quads(K_pad) * 4, rt_mul, rt_add);
    return hipGetLastError();
}

static size_t few_lds(int row_tiles) { return (size_t)row_tiles * (moe::kFewWaves - 1) * 64 * sizeof(moe::f32x4_t); }

hipError_t moe_launch_e4m3_gateup_few(const moe::E4m3Args* a, int n_slots, hipStream_t s)
{
    hipLaunchKernelGGL(moe::few_kernel<moe::kFewGateUp>, dim3(n_slots * (a->N / moe::kTileRows)),
                       dim3(64 * moe::kFewWaves), few_lds(2), s, *a);
    return hipGetLastError();
}

hipError_t moe_launch_e4m3_down_few(const moe::E4m3Args* a, int n_slots, hipStream_t s)
{
    hipLaunchKernelGGL(moe::few_kernel<moe::kFewDown>, dim3(n_slots * (a->N / moe::kTileRows)),
                       dim3(64 * moe::kFewWaves), few_lds(1), s, *a);
    return hipGetLastError();
}

// Whether a plain product of T rows rounds them itself: one or two rows that take
// at most 32 KiB of LDS (so that two workgroups still share a CU), rounded by
// every workgroup in a round or two of its threads.
int moe_e4m3_linear_raw(int T, int K) { return T <= 2 && (int64_t)T * K * 2 <= 32768; }

hipError_t moe_launch_e4m3_linear_few(const moe::E4m3Args* a, hipStream_t s)
{
    const dim3 grid(a->N / moe::kTileRows), block(64 * moe::kFewWaves);
    if (a->raw_K)
        hipLaunchKernelGGL(moe::few_kernel<moe::kFewLinearRaw>, grid, block, few_lds(1) + (size_t)a->T * a->K * 2, s, *a);
    else
        hipLaunchKernelGGL(moe::few_kernel<moe::kFewLinear>, grid, block, few_lds(1), s, *a);
    return hipGetLastError();
}

hipError_t moe_launch_linear_sum(const float* parts, int n, int64_t stride, int64_t count, float* y32, uint16_t* y16,
                                 hipStream_t s)
{
    hipLaunchKernelGGL(moe::linear_sum_kernel, dim3((unsigned)((count / 4 + 255) / 256)), dim3(256), 0, s, parts, n, stride,
                       count, y32, y16);
    return hipGetLastError();
}

// The same coding and layout on the host, for weights in host memory (K and N
// multiples of 128).
void moe_pack_e4m3_host(const uint16_t* src, int K, int N, uint8_t* dst, uint8_t* scales, int rt_mul, int rt_add)
{
    const int KT = K / moe::kTileK8, scale_ld = moe::scale_quads(K) * 4;
    auto value = [](uint16_t b) {
        const uint32_t u = (uint32_t)b << 16;
        float f;
        std::memcpy(&f, &u, 4);
        return f;
    };
    for (int n0 = 0; n0 < N; n0 += moe::kBlock)
        for (int kb = 0; kb < K / moe::kBlock; ++kb) {
            const uint16_t* block = src + (size_t)kb * moe::kBlock * N + n0;
            float amax = 0.f;
            for (int k = 0; k < moe::kBlock; ++k)
                for (int n = 0; n < moe::kBlock; ++n) {
                    const float v = std::fabs(value(block[(size_t)k * N + n]));
                    if (std::isfinite(v) && v > amax) amax = v;
                }
            // the least e with amax <= 448 * 2^e = 1.75 * 2^(e + 8)
            int e = moe::kExpMin;
            while (e < moe::kExpMax && amax > std::ldexp(448.0, e)) ++e;
            scales[(size_t)(n0 / moe::kBlock) * scale_ld + kb] = (uint8_t)(e + 127);
            const float inv = std::ldexp(1.f, -e);
            for (int n = 0; n < moe::kBlock; ++n)
                for (int k = 0; k < moe::kBlock; ++k) {
                    const float x = value(block[(size_t)k * N + n]);
                    const float v = std::fmin(std::fabs(x) * inv, 448.f);
                    uint8_t c;
                    if (!std::isfinite(x)) {
                        c = 0x7F;
                    } else if (v < 0x1p-6f) {
                        c = (uint8_t)(v * 512.f + 0x1.8p23f - 0x1.8p23f);    // to nearest even; 8: the least normal code
                    } else {
                        uint32_t u;                                          // 20 bits rounded off the mantissa
                        std::memcpy(&u, &v, 4);
                        c = (uint8_t)(((u + 0x7FFFFu + (u >> 20 & 1)) >> 20) - ((127 - 7) << 3));
                    }
                    if (std::signbit(x)) c |= 0x80;
                    const size_t rt = (size_t)((n0 + n) / moe::kTileRows) * rt_mul + rt_add;
                    const int q = k % moe::kTileK8;        // in the K tile: granule, half and byte of it
                    dst[moe::tile_offset8(rt, kb * 2 + k / moe::kTileK8, KT) + q % 32 / 8 * 256 +
                        n % moe::kTileRows * 16 + q / 32 * 8 + q % 8] = c;
                }
        }
}

}  // extern "C"
