// attn_paged.hip -- kernels of the paged cache (include/attn.h): appending a
// batch's keys and values with the rotation, and causal attention over pages.
//
//   unpack_kernel  a batch's arrays from pinned host memory to the workspace
//   append_kernel  q rotated to bf16, k rotated and v to their slots (of e4m3
//                  pages the scales too)
//   attend_kernel  attention: few() of up to 16 query rows per key/value head,
//                  tile() of blocks of 128 or 64
//   merge_kernel   adds the partial sums of rows whose positions were shared out
#include <cmath>
#include <type_traits>

#include "attn_paged.h"
#include "e4m3.h"
#include "attn_weights.h"
#include "moe_common.h"

namespace paged {

using moe::base2;
using moe::code4;
using moe::decay;
using moe::decode8;
using moe::exp2i;
using moe::f32x4_t;
using moe::far_scores;
using moe::finite;
using moe::kExpMax;
using moe::kExpMin;
using moe::scale_exponent;
using moe::u32x4_t;

typedef __attribute__((__vector_size__(16 * sizeof(float)))) float f32x16_t;

__device__ inline u32x4_t ld16(const void* p) { return *reinterpret_cast<const u32x4_t*>(p); }

typedef __attribute__((__vector_size__(2 * sizeof(uint32_t)))) uint32_t u32x2_t;
__device__ inline u32x4_t ld16_nt(const void* p) { return __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p)); }
__device__ inline u32x2_t ld8_nt(const void* p) { return __builtin_nontemporal_load(reinterpret_cast<const u32x2_t*>(p)); }

__device__ inline f32x16_t mfma32x32x16(const u32x4_t a, const u32x4_t b, f32x16_t c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(moe::bf16x8_t, a),
                                                   __builtin_bit_cast(moe::bf16x8_t, b), c, 0, 0, 0);
}

// A load through the scalar cache, of what no kernel writes while this one
// runs and whose address is the same for the whole wave.  (Left to the
// compiler these are vector loads, as the kernel also stores, and the wait for
// a page number becomes a wait for every key and value in flight.)
template <class T>
__device__ __forceinline__ T uniform_load(const T* p)
{
    return *(const __attribute__((address_space(4))) T*)p;
}

template <class T>
__device__ __forceinline__ T uniform_struct(const T* p)
{
    static_assert(sizeof(T) % 16 == 0);
    T r;
    u32x4_t* d = reinterpret_cast<u32x4_t*>(&r);
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) / 16); ++i) d[i] = uniform_load(reinterpret_cast<const u32x4_t*>(p) + i);
    return r;
}

// The maximum over lanes l, l ^ 32 and over l, l ^ 16 (halves and rows
// swapped between two registers: no LDS)
__device__ __forceinline__ float max32(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

__device__ __forceinline__ float max16(float v)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// barrier for LDS traffic only: global loads stay in flight across it
__device__ __forceinline__ void lds_barrier()
{
    constexpr int kWaitLgkm = 0xC07F;   // lgkmcnt 0; vmcnt and expcnt at their maxima
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(kWaitLgkm);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// of the batch on the device, 0 where a launch is not made for as many tokens
__device__ __forceinline__ int count(const Args& a, const int32_t* n)
{
    return uniform_load(&a.hdr->T) == a.T ? uniform_load(n) : 0;
}

// ------------------------------------------------------------------ batch --

// All arrays in one pass over the host memory: the link's latency once, 4 to 7
// us for a batch (array after array 9 to 12).
__global__ __launch_bounds__(256) void unpack_kernel(Unpack u)
{
    for (uint64_t at = ((uint64_t)blockIdx.x * 256 + threadIdx.x) * 16; at < u.bytes; at += (uint64_t)gridDim.x * 4096) {
        uint64_t dst = 0;                    // of the last segment that begins at or before it
#pragma unroll
        for (int s = 0; s < kSegments; ++s)
            if (u.seg[s].src <= at) dst = u.seg[s].dst + (at - u.seg[s].src);
        *reinterpret_cast<u32x4_t*>(u.dst + dst) = ld16(u.src + at);
    }
}

// ----------------------------------------------------------------- append --

// cos and sin of pos * inv_freq.  The angle is formed and reduced to the
// nearest multiple k of pi / 2 in fp64 (pi / 2 in two parts; k below 2^25);
// what is left, r in [-pi / 4, pi / 4], goes through the Taylor series to r^9
// and r^10 in fp32, which leave out less than 2^-28 and 2^-33.  The result is off
// by less than 2^-23 and the angle's own error, |angle| 2^-51 (inv_freq and the
// product rounded to fp64): absolute, as the rotated values need it; near a zero
// that can be many ulp.  (With the library's sincosf, and the new values held
// in registers between the scale and the codes, pieces of six prompts of 200 to
// 900 tokens took 24.3 us into e4m3 pages; so they take 17.7.)
__device__ inline float2 rotation(int pos, double inv_freq)
{
    constexpr double kHalfPiHi = 1.57079632679489655800e+00;   // pi / 2 rounded to fp64
    constexpr double kHalfPiLo = 6.12323399573676603587e-17;   // pi / 2 - kHalfPiHi
    constexpr double kInvHalfPi = 6.36619772367581382433e-01;
    const double ang = (double)pos * inv_freq;
    const double k = rint(ang * kInvHalfPi);
    const float r = (float)fma(-k, kHalfPiLo, fma(-k, kHalfPiHi, ang));
    const int quarter = (int)k;
    const float x = r * r;
    float s = fmaf(x, 1.0f / 362880.0f, -1.0f / 5040.0f);
    s = fmaf(x, s, 1.0f / 120.0f);
    s = fmaf(x, s, -1.0f / 6.0f);
    s = fmaf(r * x, s, r);
    float c = fmaf(x, -1.0f / 3628800.0f, 1.0f / 40320.0f);
    c = fmaf(x, c, -1.0f / 720.0f);
    c = fmaf(x, c, 1.0f / 24.0f);
    c = fmaf(x, c, -0.5f);
    c = fmaf(x, c, 1.0f);
    const float cq = quarter & 1 ? s : c, sq = quarter & 1 ? c : s;
    return make_float2((quarter + 1) & 2 ? -cq : cq, quarter & 2 ? -sq : sq);
}

// Four consecutive features f .. f + 3 (f a multiple of 4) of head `head` of
// token t.  Packed rows hold a query or key head's features f and f + hd/2
// eight apart in tiles of 16 (moe::rope_row).
template <bool kPacked>
__device__ inline float4 load4(const Source& x, int t, int head, int f, int hd, int n_rotated)
{
    if constexpr (kPacked) {
        const int n = head * hd + f;
        const float* src = static_cast<const float*>(x.x) + t * x.ld + (head < n_rotated ? moe::rope_row(n, hd) : n);
        float4 v = *reinterpret_cast<const float4*>(src);
        for (int k = 1; k < x.n_split; ++k) {
            const float4 p = *reinterpret_cast<const float4*>(src + k * x.stride);
            v.x += p.x; v.y += p.y; v.z += p.z; v.w += p.w;
        }
        return v;
    } else {
        const int64_t i = t * x.ld + head * hd + f;
        if (!x.bf16) return *reinterpret_cast<const float4*>(static_cast<const float*>(x.x) + i);
        const uint2 w = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(x.x) + i);
        return make_float4(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xFFFF0000u),
                           __uint_as_float(w.y << 16), __uint_as_float(w.y & 0xFFFF0000u));
    }
}

__device__ inline uint2 pack_bf16x4(const float* v)
{
    return make_uint2(moe::cvt_pk_bf16(v[0], v[1]), moe::cvt_pk_bf16(v[2], v[3]));
}

// Eight values of one head: a piece of four rotation pairs (lo: features f ..
// f + 3, hi: their partners), or of a value head eight features f .. f + 7.
struct Piece {
    float lo[4], hi[4];
};

template <bool kPacked>
__device__ inline Piece load_piece(const Source& x, int t, int head, int f, int hd, int n_rotated, bool turn)
{
    const float4 a = load4<kPacked>(x, t, head, f, hd, n_rotated);
    const float4 b = load4<kPacked>(x, t, head, turn ? f + hd / 2 : f + 4, hd, n_rotated);
    return Piece{{a.x, a.y, a.z, a.w}, {b.x, b.y, b.z, b.w}};
}

__device__ inline void turn_pair(float& a, float& b, float2 cs)
{
    const float x = a, y = b;
    a = x * cs.x - y * cs.y;
    b = y * cs.x + x * cs.y;
}

// q of a token t (and with bf16 pages its k and v): one workgroup per run of
// 256 pieces.  The token's rotations, one per frequency, are formed once per
// workgroup.  Bound by memory: 2048 tokens of 8192 fp32 values, 100.7 MB read
// and written, take 18.4 us (5.5 TB/s; a plain copy here does 4.9).
template <bool kPacked>
__device__ __forceinline__ void append_rows(const Args& a, const Source& x, uint16_t* __restrict__ q, int t, int run)
{
    __shared__ float2 s_cs[64];
    const Token tok = a.tok[t];
    const int hd = a.hd, half = hd / 2, P = hd / 8;      // pieces per head
    if ((int)threadIdx.x < half) s_cs[threadIdx.x] = rotation(tok.pos, a.freq[threadIdx.x]);
    const int e = run * 256 + threadIdx.x;
    const int head = e / P, n_rotated = a.H + a.G;
    const bool live = head < (a.e4m3 ? a.H : a.H + 2 * a.G);
    const bool turn = head < n_rotated;
    const int f = turn ? e % P * 4 : e % P * 8;
    Piece v{};
    if (live) v = load_piece<kPacked>(x, t, head, f, hd, n_rotated, turn);
    __syncthreads();
    if (!live || uniform_load(&a.hdr->T) != a.T) return;
    if (turn) {
#pragma unroll
        for (int i = 0; i < 4; ++i) turn_pair(v.lo[i], v.hi[i], s_cs[f + i]);
    }
    uint16_t* dst;
    if (head < a.H) {
        dst = q + ((int64_t)t * a.H + head) * hd;
    } else {
        if (tok.page < 0) return;            // (a graph replayed on a batch that append itself refuses)
        const int g = turn ? head - a.H : head - n_rotated;
        const int64_t row = ((int64_t)tok.page * a.G + g) << a.shift | (tok.pos & ((1 << a.shift) - 1));
        dst = reinterpret_cast<uint16_t*>(turn ? a.k : a.v) + row * hd;
    }
    *reinterpret_cast<uint2*>(dst + f) = pack_bf16x4(v.lo);
    *reinterpret_cast<uint2*>(dst + f + (turn ? half : 4)) = pack_bf16x4(v.hi);
}

// codes rounded again for a scale that grew: value * ratio, ratio a power of two
__device__ inline uint32_t recode4(uint32_t c, float ratio)
{
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, false);
    const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, true);
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(lo[0] * ratio, lo[1] * ratio, 0, false);
    r = __builtin_amdgcn_cvt_pk_fp8_f32(hi[0] * ratio, hi[1] * ratio, r, true);
    return (uint32_t)r;
}

// e4m3 pages: one workgroup per page with new tokens, key/value head and K or
// V, so that the page's scale has one writer and needs no atomics.  The new
// values' maximum gives the scale, then they are coded.  A thread takes a
// piece of a token; more tokens than one pass takes (16 at 128 dims) are read
// and rotated a second time (held in registers instead, they left the queries'
// workgroups half of the waves per CU).  Six pieces of 200 to 900 tokens, 73.5
// MB, take 17.8 us with their queries, 4.1 TB/s.
template <bool kPacked>
__device__ __forceinline__ void append_codes(const Args& a, const Source& x, int n_blocks)
{
    __shared__ float s_max[4];
    const int G = a.G, hd = a.hd, P = hd / 8;
    const int per_pass = 256 / P;
    const int tj = threadIdx.x / P, pc = threadIdx.x % P;
    const int n_tasks = count(a, &a.hdr->n_pages) * G * 2;
    for (int task = blockIdx.x; task < n_tasks; task += n_blocks) {
        const PageWork w = uniform_struct(a.pages + task / (2 * G));
        const int g = task / 2 % G;
        const bool turn = task % 2 == 0;
        const int head = a.H + g + (turn ? 0 : G), f = pc * (turn ? 4 : 8);
        const int64_t pg = (int64_t)w.page * G + g;
        uint8_t* base = (turn ? a.k : a.v) + (pg << a.shift) * hd;
        float* scale = (turn ? a.k_scale : a.v_scale) + pg;
        int e_old = kExpMin;
        if (w.slot0 > 0) e_old = min(max((int)(__float_as_uint(*scale) >> 23 & 255u) - 127, kExpMin), kExpMax);
        auto load = [&](int j) {
            Piece v = load_piece<kPacked>(x, w.tok0 + j, head, f, hd, a.H + G, turn);
            if (turn) {
                const int pos = a.tok[w.tok0 + j].pos;
#pragma unroll
                for (int i = 0; i < 4; ++i) turn_pair(v.lo[i], v.hi[i], rotation(pos, a.freq[f + i]));
            }
            return v;
        };
        Piece v{};
        float amax = 0.f;
        for (int j = tj; j < w.n; j += per_pass) {
            v = load(j);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (finite(v.lo[i])) amax = fmaxf(amax, fabsf(v.lo[i]));
                if (finite(v.hi[i])) amax = fmaxf(amax, fabsf(v.hi[i]));
            }
        }
        for (int off = 32; off >= 1; off >>= 1) amax = fmaxf(amax, __shfl_xor(amax, off, 64));
        if ((threadIdx.x & 63) == 0) s_max[threadIdx.x >> 6] = amax;
        __syncthreads();
        amax = fmaxf(fmaxf(s_max[0], s_max[1]), fmaxf(s_max[2], s_max[3]));
        const int e = max(e_old, scale_exponent(amax));
        if (threadIdx.x == 0) *scale = exp2i(e);
        if (w.slot0 > 0 && e > e_old) {
            const float ratio = exp2i(max(e_old - e, -126));
            for (int i = threadIdx.x; i < w.slot0 * hd / 16; i += 256) {
                u32x4_t c = ld16(base + i * 16);
#pragma unroll
                for (int k = 0; k < 4; ++k) c[k] = recode4(c[k], ratio);
                *reinterpret_cast<u32x4_t*>(base + i * 16) = c;
            }
        }
        const float inv = exp2i(-e);
        for (int j = tj; j < w.n; j += per_pass) {
            if (w.n > per_pass) v = load(j);
            uint8_t* dst = base + (w.slot0 + j) * hd + f;
            *reinterpret_cast<uint32_t*>(dst) = code4(v.lo, inv);
            *reinterpret_cast<uint32_t*>(dst + (turn ? hd / 2 : 4)) = code4(v.hi, inv);
        }
        __syncthreads();                                 // s_max is written again
    }
}

// The first n_code workgroups code pages (longer work first), the others take
// the tokens' runs, n_runs each.
template <bool kPacked, bool kE4m3>
__global__ __launch_bounds__(256) void append_kernel(Args a, Source x, uint16_t* __restrict__ q, int n_code,
                                                     int n_runs)
{
    const int b = (int)blockIdx.x - (kE4m3 ? n_code : 0);
    if (kE4m3 && b < 0) append_codes<kPacked>(a, x, n_code);
    else append_rows<kPacked>(a, x, q, b / n_runs, b % n_runs);
}

// ----------------------------------------------------------------- attend --

// Four rows of 16 dims, 16-bit, transposed on their way from LDS: lane n of
// each 16 supplies the address of dims 4 (n % 4) .. + 3 of row n / 4 and gets
// dim n of the four rows.
__device__ __forceinline__ uint2 transposed(const uint8_t* p)
{
    typedef short s16x4_t __attribute__((ext_vector_type(4)));
    return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                         (__attribute__((address_space(3))) s16x4_t*)const_cast<uint8_t*>(p)));
}

// 16 bytes a lane from base + offset (below `bytes`, a wave's range) straight
// to LDS, lane after lane from dst on.  In assembly, because after the
// compiler's builtin the next LDS read, whatever it reads, waits for the load;
// it writes no register, and the caller waits for it (vmcnt) before the barrier
// that hands the rows on.  m0 and memory are declared as changed (m0 is a register
// that the compiler never hands out and only sets for instructions that read it,
// of which a warning reminds; none here do).
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void load_to_lds(const uint8_t* base, uint32_t bytes, uint8_t* dst, int offset)
{
    const uint64_t b = (uint64_t)(uintptr_t)base;
    // buffer descriptor: base, no stride, its size, raw dword data (gfx9 family)
    const u32x4_t d = {(uint32_t)b, (uint32_t)(b >> 32) & 0xFFFFu, bytes, 0x00020000u};
    const uint32_t at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)dst;
    // (the pause: a scalar register that a vector instruction has just written)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                 :
                 : "s"(__builtin_amdgcn_readfirstlane(at)), "v"(offset), "s"(d)
                 : "m0", "memory");
}
#pragma clang diagnostic pop

// the same into registers
__device__ __forceinline__ u32x4_t load_16(const uint8_t* base, uint32_t bytes, int offset)
{
    const __amdgpu_buffer_rsrc_t d = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(base), 0, (int)bytes, 0x00020000);
    return __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(d, offset, 0, 0));
}

// of two bf16: bits all ones in the halves that are not finite
__device__ inline uint32_t bad_halves(uint32_t w)
{
    return ((w & 0x7F80u) == 0x7F80u ? 0xFFFFu : 0u) | ((w & 0x7F800000u) == 0x7F800000u ? 0xFFFF0000u : 0u);
}

constexpr uint32_t kOnes = 0x3F803F80u;      // two bf16 ones

// few(): up to 16 query rows (tokens of a sequence times the heads of
// one key/value head) over one range of positions, 4 waves taking the range's
// 32-position steps in turn, each with a maximum and sums of its own, merged
// through LDS at the end.
//
// Scores, weights and sums stay in registers (the bf16 variant at head_dim 128
// fills all 256 and spills three to scratch; the scalars spill to vector
// registers).  Scores transposed, S^T = K Q^T, with
// v_mfma_f32_16x16x32_bf16: lane (r, g) = (lane % 16, lane / 16) supplies K of
// position r and Q of row r, and ends with the scores of row r at positions
// 16 s + 4 g + i of sub-block s.  O^T += V^T P^T takes them as they are: its B
// operand wants eight positions per lane, in any order that V follows, and
// gets {4 g + i, 16 + 4 g + i}; the lane loads V of those eight positions at
// dims D r .. D r + D - 1 (D = hd / 16, whole rows per 16 lanes) and output
// block i takes dim D r + i for row r: an 8 x D transposition inside the lane.
// P enters as two bf16 terms (the second the rounding of what the first left:
// 16 bits), since the matrix cores have time: the loads bound the kernel (64
// sequences of 8000 to 16000 positions in bf16 484 us, 6.5 TB/s, where a plain
// read does 7.1; one token after 131071 in e4m3 45 us, 6.0: a share takes some 3
// us to its first scores).
// b, nb: this workgroup among those that take such shares, and their number (it
// takes the runs of shares that begin with shares b, b + nb, ... of the list).
template <int HD>
struct FewLds {
    float o[4][kFewRows][HD + 4];            // the waves' sums, maxima and weights
    float m[4][kFewRows], l[4][kFewRows];
};

template <int HD, bool kE4m3>
__device__ __forceinline__ void few(const Args& a, const uint16_t* __restrict__ q, uint16_t* __restrict__ out,
                                    float scale2, FewLds<HD>& lds, int b, int nb)
{
    constexpr int NC = HD / 32;              // MFMA K steps of the scores
    constexpr int D = HD / 16;               // dims per lane of V
    constexpr int ES = kE4m3 ? 1 : 2;
    constexpr int KW = kE4m3 ? HD / 64 : NC; // 16-byte loads per K row and lane
    constexpr int VW = D * ES / 4;           // words per V row and lane
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, g = lane >> 4;
    const int group = a.H / a.G, P = 1 << a.shift;
    // (the first share is read along with the count, not after it: the list
    // has room for every workgroup of the grid)
    Item im = uniform_struct(a.few + b);
    const int n_first = count(a, &a.hdr->n_few);
    for (int it = b, first = b; it < n_first || it != first;) {
        if (it != b) im = uniform_struct(a.few + it);
        const int32_t* table = a.table + im.table;
        const int R = im.rows, kvh = im.kvh, n_pos = im.n_pos;
        const bool row_ok = r < R;
        const int t = (row_ok ? r : 0) / group, j = kvh * group + (row_ok ? r : 0) % group;
        const int lim = row_ok ? im.pos0 + t : n_pos;    // the row's last position
        u32x4_t qf[NC];
        {
            const uint16_t* qr = q + ((int64_t)(im.tok0 + t) * a.H + j) * HD;
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const int d = kE4m3 ? c / 2 * 64 + g * 16 + c % 2 * 8 : c * 32 + g * 8;
                const u32x4_t v = ld16(qr + d);
                qf[c] = row_ok ? v : u32x4_t{0u, 0u, 0u, 0u};
            }
        }
        f32x4_t o[D];
#pragma unroll
        for (int i = 0; i < D; ++i) o[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        float m = -INFINITY, l = 0.f;
        // One set of registers for the loads: the next step's K is loaded into
        // them as soon as the scores are formed, its V once V is transposed.
        u32x4_t kr[2][KW];
        uint32_t vr[8][VW];
        float ksc[2], vsc[2];
        // pages of the step at p0; a sub-block past the sequence's end reads
        // the end's page
        auto pages = [&](int p0, int (&pg)[2]) {
#pragma unroll
            for (int s = 0; s < 2; ++s) pg[s] = uniform_load(table + (min(p0 + 16 * s, n_pos - 1) >> a.shift));
        };
        // rows past the sequence's last position read that position (masked
        // for every row); a sub-block without a page reads page 0 and is
        // cleared before use
        auto fetch_k = [&](int p0, const int (&pg)[2]) {
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const int pb = min(p0 + 16 * s, (n_pos - 1) & ~15);
                const int64_t head = (int64_t)max(pg[s], 0) * a.G + kvh;
                const int64_t row = (head << a.shift) + (pb & (P - 1)) + min(r, n_pos - 1 - pb);
                const uint8_t* kb = a.k + row * (HD * ES) + g * 16;
#pragma unroll
                for (int c = 0; c < KW; ++c) kr[s][c] = ld16_nt(kb + c * 64);
                if constexpr (kE4m3) ksc[s] = uniform_load(a.k_scale + head);
            }
        };
        auto fetch_v = [&](int p0, const int (&pg)[2]) {
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const int pb = min(p0 + 16 * s, (n_pos - 1) & ~15);
                const int64_t head = (int64_t)max(pg[s], 0) * a.G + kvh;
                const uint8_t* vb = a.v + ((head << a.shift) + (pb & (P - 1))) * (HD * ES) + r * (D * ES);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint8_t* src = vb + min(4 * g + i, n_pos - 1 - pb) * (HD * ES);
                    uint32_t* dst = vr[s * 4 + i];
                    if constexpr (VW == 4) {
                        const u32x4_t u = ld16_nt(src);
                        dst[0] = u[0]; dst[1] = u[1]; dst[2] = u[2]; dst[3] = u[3];
                    } else if constexpr (VW == 2) {
                        const u32x2_t u = ld8_nt(src);
                        dst[0] = u[0]; dst[1] = u[1];
                    } else {
                        dst[0] = *reinterpret_cast<const uint32_t*>(src);
                    }
                }
                if constexpr (kE4m3) vsc[s] = uniform_load(a.v_scale + head);
            }
        };
        // two dims of the lane's position i, as bf16
        auto dims = [&](int i, int k) -> uint32_t {
            if constexpr (kE4m3) {
                const uint32_t c = vr[i][k / 2];
                return __builtin_bit_cast(uint32_t, k % 2 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, vsc[i / 4], true)
                                                          : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, vsc[i / 4], false));
            } else {
                return vr[i][k];
            }
        };
        constexpr int step = 4 * kTile;
        int p0 = im.begin + w * kTile;
        int pg[2], pn[2];
        // One step: scores, softmax, P V.  kMore: the next step's loads are
        // issued on the way (static: loads behind a branch would make every
        // wait for V a wait for the next K too).  kMasked: some row does not
        // see some position of the step, or a page is missing.
        auto advance = [&](auto more, auto mask) {
            constexpr bool kMore = decltype(more)::value, kMasked = decltype(mask)::value;
            f32x4_t sc[2];
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                sc[s] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    u32x4_t kf;
                    if constexpr (kE4m3) kf = decode8(kr[s][c / 2][c % 2 * 2], kr[s][c / 2][c % 2 * 2 + 1], ksc[s]);
                    else kf = kr[s][c];
                    sc[s] = moe::mfma16x16x32(kf, qf[c], sc[s]);
                }
            }
            if constexpr (kMore) fetch_k(p0 + step, pn);
            auto unseen = [&](int s, int i) { return pg[s] < 0 || p0 + 16 * s + 4 * g + i > lim; };
            if constexpr (kMasked) {
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (unseen(s, i)) sc[s][i] = -INFINITY;
            }
            float mx = m;
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int i = 0; i < 4; ++i) mx = fmaxf(mx, sc[s][i]);
            mx = max32(max16(mx));
            if (__ballot(mx != m)) {
                const float alpha = decay(m, mx, scale2);
                l *= alpha;
#pragma unroll
                for (int i = 0; i < D; ++i) o[i] *= alpha;
                m = mx;
            }
            const float ms = far_scores(sc, m, m == -INFINITY ? 0.f : base2(m, scale2));
            u32x4_t p1, p2;
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const float pa = __builtin_amdgcn_exp2f(fmaf(sc[s][2 * i], scale2, -ms));
                    const float pb = __builtin_amdgcn_exp2f(fmaf(sc[s][2 * i + 1], scale2, -ms));
                    l += pa + pb;
                    const uint32_t hw = moe::cvt_pk_bf16(pa, pb);
                    p1[2 * s + i] = hw;
                    p2[2 * s + i] = moe::cvt_pk_bf16(pa - __uint_as_float(hw << 16), pb - __uint_as_float(hw & 0xFFFF0000u));
                }
            // dim D r + i of the lane's eight positions
            u32x4_t vt[D];
#pragma unroll
            for (int k = 0; k < D / 2; ++k)
#pragma unroll
                for (int n = 0; n < 4; ++n) {
                    const uint32_t lo = dims(2 * n, k), hi = dims(2 * n + 1, k);
                    vt[2 * k][n] = __builtin_amdgcn_perm(hi, lo, 0x05040100u);
                    vt[2 * k + 1][n] = __builtin_amdgcn_perm(hi, lo, 0x07060302u);
                }
            if constexpr (kMore) fetch_v(p0 + step, pn);
            if constexpr (kMasked) {
                // values without a page are zeros; and a value that is not
                // finite among positions that some rows do not see is taken
                // out, since 0 times it would still reach those, while the
                // rows that see it (counted by a product of zeros and ones)
                // get a NaN
                uint32_t bad = 0u;
#pragma unroll
                for (int i = 0; i < D; ++i)
#pragma unroll
                    for (int n = 0; n < 4; ++n) {
                        if (pg[n / 2] < 0) vt[i][n] = 0u;
                        bad |= bad_halves(vt[i][n]);
                    }
                if (__ballot(bad != 0u)) {
                    u32x4_t seen;
#pragma unroll
                    for (int s = 0; s < 2; ++s)
#pragma unroll
                        for (int i = 0; i < 2; ++i)
                            seen[2 * s + i] = (unseen(s, 2 * i) ? 0u : kOnes & 0xFFFFu) |
                                              (unseen(s, 2 * i + 1) ? 0u : kOnes & 0xFFFF0000u);
#pragma unroll
                    for (int i = 0; i < D; ++i) {
                        u32x4_t ind;
#pragma unroll
                        for (int n = 0; n < 4; ++n) {
                            const uint32_t x = bad_halves(vt[i][n]);
                            ind[n] = x & kOnes;
                            vt[i][n] &= ~x;
                        }
                        const f32x4_t count = moe::mfma16x16x32(ind, seen, f32x4_t{0.f, 0.f, 0.f, 0.f});
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (count[e] > 0.f) o[i][e] = NAN;
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < D; ++i) o[i] = moe::mfma16x16x32(vt[i], p1, o[i]);
#pragma unroll
            for (int i = 0; i < D; ++i) o[i] = moe::mfma16x16x32(vt[i], p2, o[i]);
        };
        // steps that every row sees whole, one after another without a pause;
        // then the sequence's last ones (and all of one with missing pages)
        const int clean = im.holes ? -1 : min(im.end, im.pos0 + 1) - kTile;   // the last start of such a step
        if (p0 <= clean) {
            pages(p0, pg);
            pages(p0 + step, pn);
            fetch_k(p0, pg);
            fetch_v(p0, pg);
            for (; p0 + step <= clean; p0 += step) {
                advance(std::true_type{}, std::false_type{});
                pages(p0 + 2 * step, pn);
            }
            advance(std::false_type{}, std::false_type{});
            p0 += step;
        }
        for (; p0 < im.end; p0 += step) {
            pages(p0, pg);
            if (pg[0] < 0 && pg[1] < 0) continue;
            fetch_k(p0, pg);
            fetch_v(p0, pg);
            advance(std::false_type{}, std::true_type{});
        }
        l += __shfl_xor(l, 16, 64);
        l += __shfl_xor(l, 32, 64);
        if (row_ok) {
            if (g == 0) {
                lds.m[w][r] = m;
                lds.l[w][r] = l;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int i = 0; i < D; i += 4)
                    *reinterpret_cast<float4*>(&lds.o[w][r][D * (4 * g + e) + i]) =
                        make_float4(o[i][e], o[i + 1][e], o[i + 2][e], o[i + 3][e]);
        }
        __syncthreads();
        // the waves' sums in wave order: thread (row, eight or four dims)
        const int row = threadIdx.x >> 4, d0 = (threadIdx.x & 15) * D;
        if (row < R) {
            float M = fmaxf(fmaxf(lds.m[0][row], lds.m[1][row]), fmaxf(lds.m[2][row], lds.m[3][row]));
            float L = 0.f, v[D];
#pragma unroll
            for (int i = 0; i < D; ++i) v[i] = 0.f;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float mk = lds.m[k][row];
                // (a wave that has seen only NaN has no maximum, and NaN sums)
                const float f = decay(mk, M, scale2);
                L = fmaf(lds.l[k][row], f, L);
#pragma unroll
                for (int i = 0; i < D; ++i) v[i] = fmaf(lds.o[k][row][d0 + i], f, v[i]);
            }
            if (im.slot >= 0) {
                float* dst = a.few_part + ((int64_t)im.slot * kFewRows + row) * (HD + kPartPad);
#pragma unroll
                for (int i = 0; i < D; i += 4)
                    *reinterpret_cast<float4*>(dst + d0 + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
                if (d0 == 0) {
                    dst[HD] = M;
                    dst[HD + 1] = L;
                }
            } else {
                const int tt = row / group, jj = kvh * group + row % group;
                uint16_t* dst = out + ((int64_t)(im.tok0 + tt) * a.H + jj) * HD + d0;
                const float inv = M == -INFINITY ? 0.f : 1.0f / L;
#pragma unroll
                for (int i = 0; i < D; ++i) v[i] *= inv;
#pragma unroll
                for (int i = 0; i < D; i += 4) *reinterpret_cast<uint2*>(dst + i) = pack_bf16x4(v + i);
            }
        }
        __syncthreads();                                 // the LDS sums are written again
        if (im.next < 0) first += nb;
        it = im.next < 0 ? first : im.next;
    }
}

// tile(): blocks of 128 or 64 query rows (kPG = 1 or 2 position groups:
// the 4 / kPG waves of a group own 32 rows each) over one range of positions
// in steps of 64, whose K and V rows are in LDS as bf16, two steps in turn, so
// that one barrier a step is enough; the query rows stay in registers.
// v_mfma_f32_32x32x16_bf16: S^T = K Q^T leaves lane (c, h) = (lane % 32,
// lane / 32) the scores of row c at positions 8 i + 4 h + e of a 32-position
// block, which O^T += V^T P^T takes from the registers, V^T being read in the
// same order by transposing LDS reads (ds_read_b64_tr_b16: 16 lanes read four
// rows of 16 dims, and lane n ends with dim n of the four).
//
// Rows are brought piece by piece beside the matrix products: bf16 rows of the
// next step straight from memory to LDS, e4m3 codes of the step after that to
// registers, decoded to LDS a step later.  A row's 16-byte chunks are swapped
// about by its number, so that neither the 32 rows of a K read nor the four of
// a V read meet in the same banks.
//
// P enters as two bf16 terms, as in few(): a weight is off by 2^-16 of itself at
// most.  (One term, off by 2^-8, would save a third of the matrix instructions,
// a prompt of 2048 tokens 85 -> 67 us, but the result's error would then be half
// as large again as its own rounding, and change with the kind of share that a
// row happens to be in.)  The exponent's reference m only
// follows the maximum when some score is more than 2^kLazy above it: the
// weights are then at most 2^kLazy, which changes nothing in fp32 or bf16, and
// most steps need no rescaling and no exchange between lanes.
//
// A wave in its matrix products goes before its SIMD's other wave, so that the
// two fall out of step and one's softmax runs beside the other's products (a
// prompt of 2048 tokens, with one term: 66.7 us, at equal priority 70.3).
//
// Bound by what does not run beside the products.  A prompt of 2048 tokens at 48
// heads of 128 takes 80 to 85 us (610 to 645 TFLOP/s of the 51.6 GFLOP below the
// diagonal; the matrix cores, which the second term keeps busy half as long
// again, are busy in 57 % of the cycles), 500 tokens after 7001 on e4m3 pages 140
// to 147 with their merge, which is some 13 of it.
constexpr float kLazy = 8.f;

template <int HD>
struct TileLds {
    uint8_t rows[4 * kStep * HD * 2];        // K and V of two steps; then the other position group's sums
    uint32_t bad;                            // a value of V is not finite, where it is masked for some rows
};

template <int HD, bool kE4m3, int kPG>
__device__ __forceinline__ void tile(const Args& a, const uint16_t* __restrict__ q, uint16_t* __restrict__ out,
                                     float scale2, TileLds<HD>& shared, int wg, int n_wg)
{
    constexpr int KQ = HD / 16;              // 16-dim K steps of the score MFMAs
    constexpr int DB = HD / 32;              // 32-dim blocks of the output
    constexpr int kP = kStep;
    constexpr int NB = kP / 32 / kPG;        // 32-position blocks per wave and step
    constexpr int kRowWaves = 4 / kPG;       // waves on different rows
    constexpr int RB = HD * 2;               // bytes of a row in LDS
    constexpr int ES = kE4m3 ? 1 : 2;
    constexpr int kHalf = kP * RB;           // K or V of a step
    constexpr int kBuf = 2 * kHalf;
    constexpr int kMergeBytes = (4 - kRowWaves) * (DB * 16 + 2) * 64 * 4;
    static_assert(sizeof shared.rows >= 2 * kBuf && sizeof shared.rows >= kMergeBytes);
    uint8_t* lds = shared.rows;
    const int group = a.H / a.G, P = 1 << a.shift;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c = lane & 31, h = lane >> 5;
    const int pg = w / kRowWaves;                        // the wave's position group
    const Item* items = a.tile[kPG - 1];
    Item im = uniform_struct(items + wg);
    const int n_items = count(a, &a.hdr->n_tile[kPG - 1]);
    const u32x4_t zero = {0u, 0u, 0u, 0u};
    // chunk of row r is at chunk ^ k_key(r) of K, ^ v_key(r) of V (rows of 64
    // dims: two share the 256 bytes of all banks)
    auto k_key = [](int r) { return HD == 128 ? r & 15 : r >> 1 & 7; };
    auto v_key = [](int r) { return HD == 128 ? (r & 3) * 4 : (r >> 1 & 1) * 4; };
    const int k_off = (pg * NB * 32 + c) * RB + (h ^ k_key(c)) * 16;          // K step k: ^ k * 32
    const int vrow = 4 * h + (c & 15) / 4;               // the lane's V row of 8
    int v_off[DB];
#pragma unroll
    for (int b = 0; b < DB; ++b)
        v_off[b] = kHalf + (pg * NB * 32 + vrow) * RB +
                   ((b * 4 + c / 16 * 2 + (c >> 1 & 1)) ^ v_key(vrow)) * 16 + (c & 1) * 8;
    constexpr int RW = kP / 4;                           // rows of a step that a wave brings
    constexpr int CL = RW * HD * ES / 1024;              // 16-byte pieces of K per lane and step
    constexpr int LR = 1024 / (HD * ES);                 // rows per 64 pieces
    constexpr int PR = HD * ES / 16;                     // pieces per row
    constexpr int DC = kE4m3 ? 2 : 1;                    // LDS chunks per piece
    const int k_in = (lane % PR * DC ^ k_key(RW * w) ^ k_key(lane / PR)) * 16, v_in = (lane % PR * DC ^ v_key(lane / PR)) * 16;
    u32x4_t kc[CL], vc[CL];                              // e4m3: the next step's codes
    float ksc = 0.f, vsc = 0.f, ksc_in = 0.f, vsc_in = 0.f;
    for (int it = wg; it < n_items; it += n_wg) {
        if (it != wg) im = uniform_struct(items + it);
        const int32_t* table = a.table + im.table;
        const int kvh = im.kvh, n_pos = im.n_pos, R = im.rows;
        const int row_w0 = w % kRowWaves * 32;           // the wave's first row in the block
        const int row = row_w0 + c;
        const bool wave_ok = row_w0 < R, row_ok = row < R;
        const int gr = im.row0 + (row_ok ? row : 0);     // the lane's row of the sequence
        const int t = gr / group, j = kvh * group + gr % group;
        const int lim = im.pos0 + t;
        const int lim_w0 = im.pos0 + (im.row0 + row_w0) / group;
        const int lim_b0 = im.pos0 + im.row0 / group;    // last position of the block's first row
        u32x4_t qf[KQ];
        {
            const uint16_t* qrow = q + ((int64_t)(im.tok0 + t) * a.H + j) * HD + h * 8;
#pragma unroll
            for (int k = 0; k < KQ; ++k) {
                const u32x4_t v = ld16(qrow + k * 16);
                qf[k] = row_ok ? v : zero;
            }
        }
        f32x16_t o[DB];
#pragma unroll
        for (int b = 0; b < DB; ++b) o[b] = f32x16_t{};
        float m = -INFINITY, ms = 0.f, thr = -INFINITY, l = 0.f;
        // Wave w brings RW rows of a later step from RW w on, which lie in one
        // page, piece by piece between its matrix products: K's pieces, then
        // V's.  Positions past the sequence's end are its last one (masked for
        // every row); without a page they are zeros.
        const uint8_t *kb_in = nullptr, *vb_in = nullptr;
        uint32_t in_bytes = 0;
        int last = 0;
        auto locate = [&](int p0) {
            const int pb = min(p0 + RW * w, (n_pos - 1) & ~(RW - 1));
            last = n_pos - 1 - pb;
            const int page = uniform_load(table + (pb >> a.shift));
            const int64_t head = (int64_t)max(page, 0) * a.G + kvh;
            const int64_t at = ((head << a.shift) + (pb & (P - 1))) * (HD * ES);
            kb_in = a.k + at;
            vb_in = a.v + at;
            in_bytes = page < 0 ? 0u : RW * HD * ES;     // (a read past the size gives zero)
            if constexpr (kE4m3) {
                ksc_in = uniform_load(a.k_scale + head);
                vsc_in = uniform_load(a.v_scale + head);
            }
        };
        // bf16: piece i of the located step straight to LDS
        auto load_piece = [&](int i, int to) {
            const bool v = i >= CL;
            const int x = i % CL;
            const int off = min(x * LR + lane / PR, last) * RB + (v ? v_in ^ v_key(x * LR) * 16 : k_in ^ k_key(x * LR) * 16);
            load_to_lds(v ? vb_in : kb_in, in_bytes, lds + to + (v ? kHalf : 0) + w * RW * RB + x * 1024, off);
        };
        // e4m3: the located step's codes into registers, and from there
        // (piece i: row i LR + lane / PR, whose key is that of lane / PR ^ that
        // of i LR) to LDS
        auto load_codes = [&] {
#pragma unroll
            for (int i = 0; i < CL; ++i) {
                const int off = min(i * LR + lane / PR, last) * HD + lane % PR * 16;
                kc[i] = load_16(kb_in, in_bytes, off);
                vc[i] = load_16(vb_in, in_bytes, off);
            }
            ksc = ksc_in;
            vsc = vsc_in;
        };
        auto decode_piece = [&](int i, int to) {
            const bool v = i >= CL;
            const int x = i % CL;
            uint8_t* dst = lds + to + (v ? kHalf : 0) + (w * RW + x * LR + lane / PR) * RB;
            const int off = v ? v_in ^ v_key(x * LR) * 16 : k_in ^ k_key(x * LR) * 16;
            const u32x4_t& c = v ? vc[x] : kc[x];
            const float scale = v ? vsc : ksc;
            *reinterpret_cast<u32x4_t*>(dst + off) = decode8(c[0], c[1], scale);
            *reinterpret_cast<u32x4_t*>(dst + (off ^ 16)) = decode8(c[2], c[3], scale);
        };
        const int first = im.begin, end = im.end;
        const int p_last = first + (end - first - 1) / kP * kP;   // the last step; past it, it is brought again
        // a step that some row of the block does not see whole
        auto partly_seen = [&](int p0) { return p0 + kP - 1 > lim_b0 || im.holes; };
        __syncthreads();                                 // the last item's LDS reads are done
        if (threadIdx.x == 0) shared.bad = 0u;
        locate(first);
        if constexpr (kE4m3) {
            load_codes();
#pragma unroll
            for (int i = 0; i < 2 * CL; ++i) decode_piece(i, 0);
            locate(min(first + kP, p_last));
            load_codes();
        } else {
#pragma unroll
            for (int i = 0; i < 2 * CL; ++i) load_piece(i, 0);
        }
        // The step's start, the same for every wave: its rows have arrived
        // from every wave, and every wave is done with the last step's.  Of a
        // step that is only partly seen, values of V that are not finite are
        // taken out (0 times one would still reach the rows that do not see it).
        auto begin_step = [&](int p0, int buf) {
            __builtin_amdgcn_s_waitcnt(kE4m3 ? 0xC07F : 0x0070);   // lgkmcnt 0, and vmcnt 0 where LDS is loaded
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            locate(min(p0 + (kE4m3 ? 2 : 1) * kP, p_last));
            if (partly_seen(p0)) {
                uint32_t bad = 0u;
#pragma unroll
                for (int i = 0; i < RW * RB / 1024; ++i) {
                    u32x4_t* d = reinterpret_cast<u32x4_t*>(lds + buf + kHalf + w * RW * RB + i * 1024 + lane * 16);
                    u32x4_t v = *d;
                    uint32_t any = 0u;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const uint32_t x = bad_halves(v[k]);
                        any |= x;
                        v[k] &= ~x;
                    }
                    if (any) *d = v;
                    bad |= any;
                }
                if (bad) shared.bad = 1u;
                lds_barrier();
            }
        };
        // what is brought beside K step k of the scores
        auto bring = [&](int k, int to) {
            if constexpr (kE4m3) {
#pragma unroll
                for (int i = 0; i < 2 * CL; ++i)
                    if (i * (KQ - 1) / (2 * CL) == k) decode_piece(i, to);
                if (k == KQ - 1) load_codes();
            } else {
#pragma unroll
                for (int i = 0; i < 2 * CL; ++i)
                    if (i * KQ / (2 * CL) == k) load_piece(i, to);
            }
        };
        int buf = 0;
        if (!wave_ok) {                                  // no rows: this wave only brings its share
            for (int p0 = first; p0 < end; p0 += kP, buf ^= kBuf) {
                begin_step(p0, buf);
#pragma unroll
                for (int k = 0; k < KQ; ++k) bring(k, buf ^ kBuf);
            }
        } else {
            for (int p0 = first; p0 < end; p0 += kP, buf ^= kBuf) {
                begin_step(p0, buf);
                const uint8_t* kb = lds + buf;
                // K fragments are read kAhead K steps before their products, an
                // LDS access taking as long as several of these
                f32x16_t sc[NB];
                constexpr int kAhead = KQ < 4 ? KQ : 4;
                u32x4_t kf[kAhead][NB];
                auto read_k = [&](int k) {
#pragma unroll
                    for (int pb = 0; pb < NB; ++pb)
                        kf[k % kAhead][pb] = *reinterpret_cast<const u32x4_t*>(kb + (k_off ^ (k * 32)) + pb * 32 * RB);
                };
#pragma unroll
                for (int k = 0; k < kAhead; ++k) read_k(k);
                __builtin_amdgcn_s_setprio(1);
                // V of the first 16 positions, and then always 16 ahead
                u32x4_t av[2][DB];
                auto read_v = [&](int i) {
#pragma unroll
                    for (int b = 0; b < DB; ++b) {
                        const uint8_t* p = kb + v_off[b] + i * 16 * RB;
                        const uint2 v0 = transposed(p), v1 = transposed(p + 8 * RB);
                        av[i % 2][b] = u32x4_t{v0.x, v0.y, v1.x, v1.y};
                    }
                };
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int k = 0; k < KQ; ++k) {
#pragma unroll
                    for (int pb = 0; pb < NB; ++pb)
                        sc[pb] = mfma32x32x16(kf[k % kAhead][pb], qf[k], k ? sc[pb] : f32x16_t{});
                    if (k + kAhead < KQ) read_k(k + kAhead);
                    else if (k == KQ - 1) read_v(0);
                    bring(k, buf ^ kBuf);
                    __builtin_amdgcn_sched_barrier(0);
                }
                __builtin_amdgcn_s_setprio(0);
                const int pw0 = p0 + pg * NB * 32;       // the wave's first position
                if (pw0 + NB * 32 - 1 > lim_w0 || im.holes) {
                    uint32_t holes = 0u;                 // runs of 16 positions without a page
                    if (im.holes) {
#pragma unroll
                        for (int i = 0; i < kP / 16; ++i)
                            if (uniform_load(table + (min(p0 + 16 * i, n_pos - 1) >> a.shift)) < 0) holes |= 1u << i;
                    }
                    const int seen = lim - pw0 - 4 * h;
#pragma unroll
                    for (int pb = 0; pb < NB; ++pb)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const int at = pb * 32 + 8 * (i / 4) + i % 4;
                            if (at > seen || (holes >> (pg * NB * 2 + at / 16) & 1u)) sc[pb][i] = -INFINITY;
                        }
                }
                float mx = -INFINITY;
#pragma unroll
                for (int pb = 0; pb < NB; ++pb)
#pragma unroll
                    for (int i = 0; i < 16; ++i) mx = fmaxf(mx, sc[pb][i]);
                if (__ballot(mx > thr)) {
                    mx = fmaxf(m, max32(mx));
                    const float alpha = decay(m, mx, scale2);
                    l *= alpha;
#pragma unroll
                    for (int b = 0; b < DB; ++b) o[b] *= alpha;
                    m = mx;
                    ms = mx == -INFINITY ? 0.f : base2(mx, scale2);
                    thr = mx + kLazy / scale2;
                }
                const float ref = far_scores(sc, m, ms);
                // the weights of 16 positions are formed beside the products
                // of the 16 before, two scores to a product
                u32x4_t bt[2], rt[2];
                auto weights = [&](int i, int e) {
                    const float pa = __builtin_amdgcn_exp2f(fmaf(sc[i / 2][i % 2 * 8 + 2 * e], scale2, -ref));
                    const float pb = __builtin_amdgcn_exp2f(fmaf(sc[i / 2][i % 2 * 8 + 2 * e + 1], scale2, -ref));
                    l += pa + pb;
                    const uint32_t hw = moe::cvt_pk_bf16(pa, pb);
                    bt[i % 2][e] = hw;
                    rt[i % 2][e] = moe::cvt_pk_bf16(pa - __uint_as_float(hw << 16), pb - __uint_as_float(hw & 0xFFFF0000u));
                };
#pragma unroll
                for (int e = 0; e < 4; ++e) weights(0, e);
                __builtin_amdgcn_sched_barrier(0);
                __builtin_amdgcn_s_setprio(1);
#pragma unroll
                for (int i = 0; i < 2 * NB; ++i) {
                    if (i + 1 < 2 * NB) read_v(i + 1);
#pragma unroll
                    for (int b = 0; b < DB; ++b) {
                        o[b] = mfma32x32x16(av[i % 2][b], bt[i % 2], o[b]);
                        o[b] = mfma32x32x16(av[i % 2][b], rt[i % 2], o[b]);
                        if (i + 1 < 2 * NB) {
#pragma unroll
                            for (int e = b * 4 / DB; e < (b + 1) * 4 / DB; ++e) weights(i + 1, e);
                        }
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
                __builtin_amdgcn_s_setprio(0);
            }
        }
        // (what was brought again is done with the LDS)
        __builtin_amdgcn_s_waitcnt(0x0070);
        __syncthreads();
        if (shared.bad) {
            // the rows that see a value that was taken out get a NaN in its dim
            for (int p0 = first; p0 < end; p0 += kP) {
                if (!partly_seen(p0)) continue;
                for (int p = p0; p < min(p0 + kP, end); ++p) {
                    const int pgv = uniform_load(table + (p >> a.shift));
                    if (pgv < 0) continue;
                    const uint8_t* vrow = a.v + ((((int64_t)pgv * a.G + kvh) << a.shift) + (p & (P - 1))) * (HD * ES);
#pragma unroll
                    for (int b = 0; b < DB; ++b)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const int d = b * 32 + 8 * (i / 4) + 4 * h + i % 4;
                            bool bad;
                            if constexpr (kE4m3) bad = (vrow[d] & 0x7F) == 0x7F;
                            else bad = (reinterpret_cast<const uint16_t*>(vrow)[d] & 0x7F80) == 0x7F80;
                            if (bad && p <= lim) o[b][i] = NAN;
                        }
                }
            }
        }
        l += __shfl_xor(l, 32, 64);
        if constexpr (kPG > 1) {
            // the other position group's sums, merged by group 0
            float* mg = reinterpret_cast<float*>(lds);
            __syncthreads();
            if (pg > 0) {
                float* dst = mg + (w - kRowWaves) * (DB * 16 + 2) * 64 + lane;
#pragma unroll
                for (int b = 0; b < DB; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i) dst[(b * 16 + i) * 64] = o[b][i];
                dst[DB * 16 * 64] = m;
                dst[(DB * 16 + 1) * 64] = l;
            }
            __syncthreads();
            if (pg > 0) continue;
#pragma unroll
            for (int k = 1; k < kPG; ++k) {
                const float* src = mg + ((k - 1) * kRowWaves + w) * (DB * 16 + 2) * 64 + lane;
                const float m2 = src[DB * 16 * 64], l2 = src[(DB * 16 + 1) * 64];
                const float mn = fmaxf(m, m2);
                const float f1 = decay(m, mn, scale2), f2 = decay(m2, mn, scale2);
#pragma unroll
                for (int b = 0; b < DB; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        o[b][i] = fmaf(src[(b * 16 + i) * 64], f2, o[b][i] * f1);
                l = fmaf(l2, f2, l * f1);
                m = mn;
            }
        }
        if (!row_ok) continue;
        // lane: dims 32 b + 8 i + 4 h + e of its row (register 4 i + e)
        if (im.slot >= 0) {
            float* dst = a.tile_part + ((int64_t)im.slot * 128 + row) * (HD + kPartPad);
#pragma unroll
            for (int b = 0; b < DB; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    *reinterpret_cast<float4*>(dst + b * 32 + 8 * i + 4 * h) =
                        make_float4(o[b][4 * i], o[b][4 * i + 1], o[b][4 * i + 2], o[b][4 * i + 3]);
            if (h == 0) {
                dst[HD] = m;
                dst[HD + 1] = l;
            }
            continue;
        }
        const float inv = m == -INFINITY ? 0.f : 1.0f / l;
        uint16_t* dst = out + ((int64_t)(im.tok0 + t) * a.H + j) * HD + 4 * h;
#pragma unroll
        for (int b = 0; b < DB; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float v[4] = {o[b][4 * i] * inv, o[b][4 * i + 1] * inv, o[b][4 * i + 2] * inv, o[b][4 * i + 3] * inv};
                *reinterpret_cast<uint2*>(dst + b * 32 + 8 * i) = pack_bf16x4(v);
            }
    }
}

// The attention's launch.  kKinds: the kinds of shares that the batch has, 1
// few(), 2 and 4 tile() on blocks of 128 and 64 rows; with several kinds the
// workgroups that take them come in turn, eight at a time (one per XCD), so
// that the ones that wait for memory and the ones that multiply share the CUs
// (24 sequences with one token and two with 150 to 300, after up to 3000
// positions: 62 to 63 us with the merge; as two calls 36 and 44).
struct Split {
    int few, tile[2];                        // workgroups / 8 of each kind
};

template <int HD, bool kE4m3, int kKinds>
__global__ __launch_bounds__(256, 2) void attend_kernel(Args a, const uint16_t* __restrict__ q,
                                                        uint16_t* __restrict__ out, float scale2, Split n)
{
    union Lds {
        FewLds<HD> few;
        TileLds<HD> tile;
    };
    __shared__ __attribute__((aligned(1024)))
    uint8_t mem[kKinds == 1 ? sizeof(FewLds<HD>) : kKinds == 7 ? sizeof(Lds) : sizeof(TileLds<HD>)];
    FewLds<HD>& fl = *reinterpret_cast<FewLds<HD>*>(mem);
    TileLds<HD>& tl = *reinterpret_cast<TileLds<HD>*>(mem);
    const int b = blockIdx.x, nb = gridDim.x;
    if constexpr (kKinds == 1) {
        few<HD, kE4m3>(a, q, out, scale2, fl, b, nb);
    } else if constexpr (kKinds == 2) {
        tile<HD, kE4m3, 1>(a, q, out, scale2, tl, b, nb);
    } else if constexpr (kKinds == 4) {
        tile<HD, kE4m3, 2>(a, q, out, scale2, tl, b, nb);
    } else {
        const int x = b / kXcds, tiles = n.tile[0] + n.tile[1], all = tiles + n.few;
        const int before = (int)((int64_t)x * tiles / all);
        if ((int)((int64_t)(x + 1) * tiles / all) == before)
            few<HD, kE4m3>(a, q, out, scale2, fl, (x - before) * kXcds + b % kXcds, n.few * kXcds);
        else if (before < n.tile[0])
            tile<HD, kE4m3, 1>(a, q, out, scale2, tl, before * kXcds + b % kXcds, n.tile[0] * kXcds);
        else
            tile<HD, kE4m3, 2>(a, q, out, scale2, tl, (before - n.tile[0]) * kXcds + b % kXcds, n.tile[1] * kXcds);
    }
}

// merge_kernel: the partial sums of a row's slots, weighted by their maxima,
// added in slot order.  Up to kWaveSlots slots a wave takes a row (lane s the
// maximum and weight of slot s, then every lane its dims of all slots); more,
// a workgroup does, wave w adding slots w, w + 4, ..., the waves' sums in wave
// order.  A slot without weight holds zeros.
//
// A workgroup takes four rows of an entry of few()'s, or one where some row has
// many slots, and eight of tile()'s (sixteen with two slots); `chunks` workgroups
// an entry of 16 or 128 rows.  A wave loads as many slots as its variant has
// room for, 2, 5, 8 or 16: rows of few slots would otherwise read slot 0 again
// for the rest (five ranges are what pieces of some hundred tokens behind a long
// prefix get).  Bound by its reads, which mostly come from the last-level cache: five
// ranges of 500 tokens' rows, 65 MB, take 13.4 us (one row a wave 15.4); few
// slots, by latency, 3.7 to 5.
constexpr int kWaveSlots = 16;
constexpr int kMaxSlots = kFewRuns;          // the most of one row

struct MergeGrid {
    int few, few_chunks, tile_chunks;        // workgroups / few_chunks for few()'s entries
    int few_rows, tile_rows;                 // rows of a workgroup
};

template <int HD>
__global__ __launch_bounds__(256) void merge_kernel(Args a, uint16_t* __restrict__ out, float scale2, MergeGrid g)
{
    constexpr int D = HD / 64;
    __shared__ float s_f[kMaxSlots], s_red[2][4], s_sum[4][HD];
    const int group = a.H / a.G, lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int b = blockIdx.x, few_wgs = g.few * g.few_chunks;
    const bool tiles = b >= few_wgs;
    const int chunks = tiles ? g.tile_chunks : g.few_chunks, rows = tiles ? g.tile_rows : g.few_rows;
    const int x = tiles ? b - few_wgs : b;
    const int entries = tiles ? ((int)gridDim.x - few_wgs) / chunks : g.few;   // taken at once
    const int row0 = x % chunks * rows;
    const Merge* list = a.merge[tiles];
    const float* part = tiles ? a.tile_part : a.few_part;
    const int stride = (tiles ? 128 : kFewRows) * (HD + kPartPad);
    Merge mg = uniform_struct(list + x / chunks);
    const int last = count(a, &a.hdr->n_merge[tiles]);
    for (int it = x / chunks; it < last; it += entries) {
        if (it != x / chunks) mg = uniform_struct(list + it);
        const int n = mg.n;
        const float* base = part + (int64_t)mg.slot0 * stride;
        auto load = [&](const float* row, int s, float (&v)[D]) {
            const float* p = row + (int64_t)s * stride + lane * D;
            if constexpr (D == 2) {
                const float2 t = *reinterpret_cast<const float2*>(p);
                v[0] = t.x;
                v[1] = t.y;
            } else {
                v[0] = p[0];
            }
        };
        auto write = [&](int row, const float (&acc)[D], float L) {
            const float inv = L > 0.f || L != L ? 1.0f / L : 0.f;      // no weight at all: zeros
            const int gr = mg.row0 + row, t = gr / group, j = mg.kvh * group + gr % group;
            uint16_t* dst = out + ((int64_t)(mg.tok0 + t) * a.H + j) * HD + lane * D;
            if constexpr (D == 2) *reinterpret_cast<uint32_t*>(dst) = moe::cvt_pk_bf16(acc[0] * inv, acc[1] * inv);
            else dst[0] = moe::f32_to_bf16(acc[0] * inv);
        };
        if (n <= kWaveSlots) {
            // `most` slots (past n: slot 0 with factor 0), their sums loaded
            // along with the maxima
            auto add_all = [&](auto most, auto rows_at_once) {
                constexpr int kMost = decltype(most)::value, kRows = decltype(rows_at_once)::value;
                const int end = min(mg.rows, row0 + rows);
                for (int r0 = row0 + w; r0 < end; r0 += 4 * kRows) {
                    float2 ml[kRows];
                    float v[kRows][kMost][D];
#pragma unroll
                    for (int k = 0; k < kRows; ++k) {                      // (past the end: r0 again)
                        const int row = r0 + 4 * k < end ? r0 + 4 * k : r0;
                        const float* pr = base + row * (HD + kPartPad);
                        ml[k] = make_float2(-INFINITY, 0.f);
                        if (lane < n) ml[k] = *reinterpret_cast<const float2*>(pr + (int64_t)lane * stride + HD);
#pragma unroll
                        for (int s = 0; s < kMost; ++s) load(pr, s < n ? s : 0, v[k][s]);
                    }
#pragma unroll
                    for (int k = 0; k < kRows; ++k) {
                        float M = ml[k].x;
                        for (int off = kWaveSlots / 2; off >= 1; off >>= 1) M = fmaxf(M, __shfl_xor(M, off, 64));
                        const float f = decay(ml[k].x, M, scale2);
                        float L = ml[k].y * f;
                        for (int off = kWaveSlots / 2; off >= 1; off >>= 1) L += __shfl_xor(L, off, 64);
                        L = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(L)));
                        float acc[D] = {};
#pragma unroll
                        for (int s = 0; s < kMost; ++s) {
                            const float fs = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f), s));
#pragma unroll
                            for (int e = 0; e < D; ++e) acc[e] = fmaf(v[k][s][e], fs, acc[e]);
                        }
                        if (r0 + 4 * k < end) write(r0 + 4 * k, acc, L);
                    }
                }
            };
            using std::integral_constant;
            if (!tiles) {                                // four rows for four waves
                if (n <= 5) add_all(integral_constant<int, 5>{}, integral_constant<int, 1>{});
                else add_all(integral_constant<int, kWaveSlots>{}, integral_constant<int, 1>{});
            } else if (n <= 2) {
                add_all(integral_constant<int, 2>{}, integral_constant<int, 4>{});
            } else if (n <= 5) {
                add_all(integral_constant<int, 5>{}, integral_constant<int, 2>{});
            } else if (n <= 8) {
                add_all(integral_constant<int, 8>{}, integral_constant<int, 2>{});
            } else {
                add_all(integral_constant<int, kWaveSlots>{}, integral_constant<int, 1>{});
            }
            continue;
        }
        for (int row = row0; row < min(mg.rows, row0 + rows); ++row) {
            const float* pr = base + row * (HD + kPartPad);
            // thread s: slot s (and s + 256, ..., which are read twice)
            auto ml_of = [&](int s) { return *reinterpret_cast<const float2*>(pr + (int64_t)s * stride + HD); };
            const float2 own = (int)threadIdx.x < n ? ml_of(threadIdx.x) : make_float2(-INFINITY, 0.f);
            float M = own.x, L = 0.f;
            for (int s = threadIdx.x + 256; s < n; s += 256) M = fmaxf(M, ml_of(s).x);
            for (int off = 32; off >= 1; off >>= 1) M = fmaxf(M, __shfl_xor(M, off, 64));
            if (lane == 0) s_red[0][w] = M;
            __syncthreads();
            M = fmaxf(fmaxf(s_red[0][0], s_red[0][1]), fmaxf(s_red[0][2], s_red[0][3]));
            for (int s = threadIdx.x; s < n; s += 256) {
                const float2 ml = s < 256 ? own : ml_of(s);
                const float f = decay(ml.x, M, scale2);
                s_f[s] = f;
                L = fmaf(ml.y, f, L);
            }
            for (int off = 32; off >= 1; off >>= 1) L += __shfl_xor(L, off, 64);
            if (lane == 0) s_red[1][w] = L;
            __syncthreads();
            L = ((s_red[1][0] + s_red[1][1]) + s_red[1][2]) + s_red[1][3];
            float acc[D] = {};
            // sixteen slots of a wave at a time, all loads together (past n:
            // slot 0 with factor 0)
            for (int s = w; s < n; s += 64) {
#pragma unroll
                for (int u = 0; u < 16; ++u) {
                    const int z = s + 4 * u;
                    float v[D];
                    load(pr, z < n ? z : 0, v);
#pragma unroll
                    for (int e = 0; e < D; ++e) acc[e] = fmaf(v[e], z < n ? s_f[z] : 0.f, acc[e]);
                }
            }
#pragma unroll
            for (int e = 0; e < D; ++e) s_sum[w][lane * D + e] = acc[e];
            __syncthreads();
            if (w == 0) {
#pragma unroll
                for (int e = 0; e < D; ++e) {
                    const int d = lane * D + e;
                    acc[e] = ((s_sum[0][d] + s_sum[1][d]) + s_sum[2][d]) + s_sum[3][d];
                }
                write(row, acc, L);
            }
            __syncthreads();                             // the LDS sums are written again
        }
    }
}

}  // namespace paged

extern "C" {

hipError_t attn_paged_launch_unpack(const paged::Unpack* u, hipStream_t s)
{
    const uint64_t blocks = (u->bytes / 16 + 255) / 256;
    hipLaunchKernelGGL(paged::unpack_kernel, dim3((unsigned)(blocks < 1 ? 1 : blocks > 256 ? 256 : blocks)), dim3(256), 0, s, *u);
    return hipGetLastError();
}

hipError_t attn_paged_launch_append(const paged::Args* a, const paged::Source* x, uint16_t* q, int T,
                                    int n_pages, hipStream_t s)
{
    const int pieces = (a->e4m3 ? a->H : a->H + 2 * a->G) * a->hd / 8, runs = (pieces + 255) / 256;
    const int codes = a->e4m3 ? n_pages * a->G * 2 : 0;
    const dim3 grid(codes + T * runs);
#define APPEND(PACKED, E) hipLaunchKernelGGL((paged::append_kernel<PACKED, E>), grid, dim3(256), 0, s, *a, *x, q, codes, runs)
    if (x->packed) {
        if (a->e4m3) APPEND(true, true);
        else APPEND(true, false);
    } else {
        if (a->e4m3) APPEND(false, true);
        else APPEND(false, false);
    }
#undef APPEND
    return hipGetLastError();
}

static float scale2(int hd) { return (float)(1.4426950408889634 / sqrt((double)hd)); }

hipError_t attn_paged_launch_attend(const paged::Args* a, const uint16_t* q, uint16_t* out, const int* n, hipStream_t s)
{
    auto groups = [](int v) { return (v + paged::kXcds - 1) / paged::kXcds; };
    const paged::Split sp{groups(n[0]), {groups(n[1]), groups(n[2])}};
    const int kinds = (n[0] ? 1 : 0) | (n[1] ? 2 : 0) | (n[2] ? 4 : 0);
    if (!kinds) return hipSuccess;
    const bool one = kinds == 1 || kinds == 2 || kinds == 4;
    const int grid = one ? n[0] + n[1] + n[2] : (sp.few + sp.tile[0] + sp.tile[1]) * paged::kXcds;
#define ATTEND(HD, E, K) hipLaunchKernelGGL((paged::attend_kernel<HD, E, K>), dim3(grid), dim3(256), 0, s, *a, q, out, scale2(HD), sp)
#define ATTEND_ALL(HD, E) \
    do { \
        if (kinds == 1) ATTEND(HD, E, 1); \
        else if (kinds == 2) ATTEND(HD, E, 2); \
        else if (kinds == 4) ATTEND(HD, E, 4); \
        else ATTEND(HD, E, 7); \
    } while (0)
    if (a->hd == 128) {
        if (a->e4m3) ATTEND_ALL(128, true);
        else ATTEND_ALL(128, false);
    } else {
        if (a->e4m3) ATTEND_ALL(64, true);
        else ATTEND_ALL(64, false);
    }
#undef ATTEND_ALL
#undef ATTEND
    return hipGetLastError();
}

hipError_t attn_paged_launch_merge(const paged::Args* a, uint16_t* out, const int* n, const int* slots, int few_rows,
                                   hipStream_t s)
{
    // four rows to a workgroup, or one where some row has many slots
    paged::MergeGrid g{};
    g.few_rows = slots[0] <= paged::kWaveSlots ? 4 : 1;
    g.tile_rows = slots[1] <= 2 ? 16 : 8;
    g.few = n[0];
    g.few_chunks = (few_rows + g.few_rows - 1) / g.few_rows;
    g.tile_chunks = 128 / g.tile_rows;
    const dim3 grid(g.few * g.few_chunks + n[1] * g.tile_chunks);
    if (grid.x == 0) return hipSuccess;
    if (a->hd == 128) hipLaunchKernelGGL(paged::merge_kernel<128>, grid, dim3(256), 0, s, *a, out, scale2(128), g);
    else hipLaunchKernelGGL(paged::merge_kernel<64>, grid, dim3(256), 0, s, *a, out, scale2(64), g);
    return hipGetLastError();
}

}  // extern "C"
