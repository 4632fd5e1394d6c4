// moe_route.hip -- the router (paper Sec. 3.1: its output decides which
// experts receive a token), top-k selection (Sec. 2.1: 4 of 16), the gate
// weights, and the token -> expert permutation.
//
// Logits.  The product of a bf16 activation and an fp32 router weight is
// exact in fp64, so the kernels accumulate in fp64 and round once to fp32:
// the logit equals the fp32 rounding of the exact dot product except when
// that sum lies within a few fp64 ulps of an fp32 rounding boundary.  The
// router weight is held transposed in the arena (wrT [E][d], d contiguous) so
// that every load is 16 bytes.
//
// Kernels
//   router_kernel (+ sum_select_kernel): logits of many tokens on the fp64 matrix
//       cores.
//   route_partials_kernel + route_finish_kernel (T <= 16, E <= 16,
//       T*k <= 64): partial logits over a few workgroups, then one workgroup
//       sums them in fixed order, selects and permutes.
//   route_one_kernel: both in one launch where one workgroup forms the logits
//       anyway (d <= 512).
//   select_kernel: selection and weights from fp32 logits, router_kernel's or the
//       caller's.
//   permute_kernel: the permutation and the list of token tiles.
// The kernels that select have a second form for a layer with a routing policy
// (choose below), select_kernel's is policy_select_kernel.
//
// Selection: the k largest logits, ties to the lower expert id, slots ordered
// by (logit desc, id asc); weights = softmax over the selected logits (fp32).
// Permutation: prefix sums per local expert over pairs in (token, slot)
// order, which gives rows grouped by expert, then token -- no atomic decides
// a row, so the order is deterministic.
#include <algorithm>

#include "../../include/moe.h"
#include "e4m3.h"
#include "moe_common.h"

namespace moe {

constexpr int kRouteThreads = 1024;
constexpr int kRouteWaves = kRouteThreads / kWave;
// Selection and weights for token t from logits l[0..E) (any address space).
// The logits, the chosen ids and their exponentials stay in registers
// (kMaxE and kMaxK bound the static arrays; E <= 64 always).
constexpr int kMaxK = 8;

template <int kMaxE>
__device__ __forceinline__ void select_token(const float* l, int E, int k, int* ids, float* w)
{
    float lv[kMaxE];
#pragma unroll
    for (int e = 0; e < kMaxE; ++e) lv[e] = e < E ? l[e] : 0.f;
    uint64_t taken = 0;
    float ps[kMaxK];
    float lmax = 0.f, z = 0.f;
    for (int j = 0; j < k; ++j) {
        int best = -1;
        float bv = 0.f;
#pragma unroll
        for (int e = 0; e < kMaxE; ++e) {
            const bool ok = e < E && !((taken >> e) & 1ull);
            if (ok && (best < 0 || lv[e] > bv)) { best = e; bv = lv[e]; }
        }
        taken |= 1ull << best;
        if (j == 0) lmax = bv;
        const float p = expf(bv - lmax);
        z += p;
        ids[j] = best;
#pragma unroll
        for (int q = 0; q < kMaxK; ++q)
            if (q == j) ps[q] = p;
        if (j >= kMaxK) w[j] = p;   // normalised below
    }
    const float inv = 1.0f / z;
#pragma unroll
    for (int q = 0; q < kMaxK; ++q)
        if (q < k) w[q] = ps[q] * inv;
    for (int j = kMaxK; j < k; ++j) w[j] = w[j] * inv;
}

// selection of token t into the routing view (inlined: as a call it spills
// callee-saved registers to scratch)
__device__ __forceinline__ void select_token_any(const float* l, int t, int E, int k, const RouteView& rv)
{
    int* ids = rv.topk_idx + (int64_t)t * k;
    float* w = rv.topk_w + (int64_t)t * k;
    if (E <= 16) select_token<16>(l, E, k, ids, w);
    else select_token<64>(l, E, k, ids, w);
}

// The value of v in lane q of this lane's W consecutive ones (W 64: q is the same
// for the wave).
template <int W>
__device__ __forceinline__ double from_lane(double v, int q)
{
    if constexpr (W == kWave) {
        const uint64_t u = __builtin_bit_cast(uint64_t, v);
        const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)u, q);
        const uint32_t hi = __builtin_amdgcn_readlane((int)(uint32_t)(u >> 32), q);
        return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
    } else {
        return __shfl(v, q, W);
    }
}

template <int W>
__device__ __forceinline__ float from_lane(float v, int q)
{
    if constexpr (W == kWave)
        return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), q));
    else
        return __shfl(v, q, W);
}

template <int W>
__device__ __forceinline__ double sum_lanes(double v)
{
#pragma unroll
    for (int o = W / 2; o >= 1; o >>= 1) v += __shfl_xor(v, o, W);
    return v;
}

template <int W>
__device__ __forceinline__ double max_lanes(double v)
{
#pragma unroll
    for (int o = W / 2; o >= 1; o >>= 1) v = fmax(v, __shfl_xor(v, o, W));
    return v;
}

// Selection and weights of one token under a policy, by W lanes (16 or 64, at
// least E), lane e holding expert e's logit.  Each lane forms its expert's score
// and choice value and counts the experts that go before it; the k first write
// their slots.  All of it in fp64: next to a border the choice would otherwise
// hang on the last bit of an exp, and scores of far logits would tie.  A whole
// wave compares its experts through scalar registers.
template <int W>
__device__ __forceinline__ void choose(const Policy& p, float logit, int e, int E, int k, int* ids, float* w)
{
    constexpr int kAtOnce = 8;            // lanes read at once (those past E are closed)
    const bool live = e < E;
    const double l = live ? (double)logit : -INFINITY;
    // exp(l - m) of the lanes that take part; nothing but -inf gives zeros, a NaN stays one
    auto exp_from = [&](double m, bool in) { return !in || (m == -INFINITY && l == l) ? 0.0 : exp(l - m); };
    double s = l;
    if (p.score == MOE_SCORE_SOFTMAX) {
        const double x = exp_from(max_lanes<W>(l), live);
        const double z = sum_lanes<W>(x);
        s = z == 0.0 ? 0.0 : x / z;
    } else if (p.score == MOE_SCORE_SIGMOID) {
        s = 1.0 / (1.0 + exp(-l));
    }
    double c = s + (live && p.balance ? (double)p.balance[e] : 0.0);
    if (c != c) c = -INFINITY;
    const float order = logit == logit ? logit : -INFINITY;   // among equal c
    bool open = live;
    if (p.top_groups < p.n_groups) {
        const int n = E / p.n_groups, g = min(e, E - 1) / n;
        double b1 = -INFINITY, b2 = -INFINITY;                // the two largest c of the group
        if ((n & (n - 1)) == 0) {
            b1 = c;
            for (int o = 1; o < n; o <<= 1) {                 // groups are aligned runs of lanes
                const double o1 = __shfl_xor(b1, o, W), o2 = __shfl_xor(b2, o, W);
                b2 = fmax(fmin(b1, o1), fmax(b2, o2));
                b1 = fmax(b1, o1);
            }
        } else {
            for (int q0 = 0; q0 < E; q0 += kAtOnce)
#pragma unroll
                for (int q = q0; q < q0 + kAtOnce; ++q) {
                    const double cq = from_lane<W>(c, q);
                    const double v = q >= g * n && q < g * n + n ? cq : -INFINITY;
                    b2 = fmax(b2, fmin(b1, v));
                    b1 = fmax(b1, v);
                }
        }
        double value = p.group_best == 2 ? b1 + b2 : b1;
        if (value != value) value = -INFINITY;
        int before = 0;
        for (int q = 0; q < p.n_groups; ++q) {
            const double v = from_lane<W>(value, q * n);
            before += v > value || (v == value && q < g) ? 1 : 0;
        }
        open = live && before < p.top_groups;
    }
    // how many come before: those of a larger c, and (only where some c are equal)
    // those of the same c with a larger logit, or the same and a lower id.  A
    // closed expert's c is NaN here, which no comparison holds for.
    const double key = open ? c : NAN;
    int rank = 0, upto = 0;
    for (int q0 = 0; q0 < E; q0 += kAtOnce)
#pragma unroll
        for (int q = q0; q < q0 + kAtOnce; ++q) {
            const double cq = from_lane<W>(key, q);
            rank += cq > c ? 1 : 0;
            upto += cq >= c ? 1 : 0;
        }
    if (__ballot(open && upto > rank + 1))
        for (int q = 0; q < E; ++q) {
            const double cq = from_lane<W>(key, q);
            const float lq = from_lane<W>(order, q);
            rank += cq == c && (lq > order || (lq == order && q < e)) ? 1 : 0;
        }
    const bool in = open && rank < k;
    double v = in ? s : 0.0;
    if (p.score == MOE_SCORE_SELECTED) v = exp_from(max_lanes<W>(in ? l : -INFINITY), in);
    if (p.renormalize || p.score == MOE_SCORE_SELECTED) {
        const double z = sum_lanes<W>(v);
        v = z == 0.0 ? 0.0 : v / z;
    }
    if (in) {
        ids[rank] = e;
        w[rank] = (float)(v * (double)p.scale);
    }
}

// barrier for LDS traffic only: waits for this wave's LDS operations, not for
// its outstanding global stores (which a __syncthreads() release would)
__device__ __forceinline__ void lds_barrier()
{
    constexpr int kWaitLgkm = 0xC07F;   // lgkmcnt 0; vmcnt and expcnt at their maxima
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(kWaitLgkm);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

__device__ inline void fma8(double& acc, const u32x4_t xv, const float4 w0, const float4 w1)
{
    acc = fma((double)__uint_as_float(xv[0] << 16), (double)w0.x, acc);
    acc = fma((double)__uint_as_float(xv[0] & 0xFFFF0000u), (double)w0.y, acc);
    acc = fma((double)__uint_as_float(xv[1] << 16), (double)w0.z, acc);
    acc = fma((double)__uint_as_float(xv[1] & 0xFFFF0000u), (double)w0.w, acc);
    acc = fma((double)__uint_as_float(xv[2] << 16), (double)w1.x, acc);
    acc = fma((double)__uint_as_float(xv[2] & 0xFFFF0000u), (double)w1.y, acc);
    acc = fma((double)__uint_as_float(xv[3] << 16), (double)w1.z, acc);
    acc = fma((double)__uint_as_float(xv[3] & 0xFFFF0000u), (double)w1.w, acc);
}

constexpr int kSmallT = 16;

// Decode routing (T <= 16, E <= 16, T*k <= 64) in two launches.
// route_partials_kernel spreads the logits over n_wg workgroups, each owning
// d/n_wg of the reduction axis (8-wide groups, thread = (expert tid%16, group
// tid/16)); per workgroup the partials are reduced in fixed order (lane
// butterfly, then over the 16 waves through LDS) and written to the
// workspace.  route_finish_kernel, one workgroup, sums the n_wg partials in
// workgroup order, selects, weighs and permutes.  The kernel boundary orders
// the two: measured, it costs less than a release fence, a device-scope
// ticket and an acquire inside one launch (~9 us of a 14 us kernel).
constexpr int kDecE = 16;
constexpr int kDecPairs = 64;
constexpr int kDecMaxWg = 16;   // partial sums read in one batch (d <= 8192)

struct DecodeRouteArgs {
    const uint16_t* x;
    const float* wrT;
    const float* bias;
    double* partial;          // [n_wg][kSmallT][kDecE]
    int T, d, E, k, e_begin, n_local, tile_rows, n_wg;
    uint16_t* xq;             // x rounded to the e4m3 grid (workgroups from n_wg on), or NULL
    Policy policy;
    RouteView rv;
};

// The fp64 sums of this workgroup's share of the reduction axis, thread
// (t, ee) = (tid / 16, tid % 16) < (T, 16) ending with token t and expert ee's.
// kT tokens' loads are issued together, those past T re-reading token T - 1
// (with each token's load in a branch of its own, 16 tokens waited for 16
// loads in turn: 7.2 us at d 256).
template <int kT>
__device__ __forceinline__ double partial_logits(const DecodeRouteArgs& a)
{
    __shared__ double wsum[kRouteWaves][kT][kDecE];
    const int T = a.T, E = a.E, d = a.d;
    const int tid = threadIdx.x;
    const int lane = tid & 63, wid = tid >> 6;
    const int e = tid & 15;
    double acc[kT];
#pragma unroll
    for (int t = 0; t < kT; ++t) acc[t] = 0.0;
    // 8-element groups blockIdx*64 + tid/16, then + n_wg*64, ... (one pass
    // when the grid covers d, several for a single workgroup)
    for (int g = blockIdx.x * (kRouteThreads / kDecE) + (tid >> 4); e < E && g < d / 8;
         g += a.n_wg * (kRouteThreads / kDecE)) {
        const float4 w0 = *reinterpret_cast<const float4*>(a.wrT + (int64_t)e * d + g * 8);
        const float4 w1 = *reinterpret_cast<const float4*>(a.wrT + (int64_t)e * d + g * 8 + 4);
        u32x4_t xv[kT];
#pragma unroll
        for (int t = 0; t < kT; ++t)
            xv[t] = *reinterpret_cast<const u32x4_t*>(a.x + (int64_t)min(t, T - 1) * d + g * 8);
#pragma unroll
        for (int t = 0; t < kT; ++t) fma8(acc[t], xv[t], w0, w1);
    }
    // lanes l, l^16, l^32, l^48 hold the same expert: fixed-order butterfly
#pragma unroll
    for (int t = 0; t < kT; ++t) {
        double v = acc[t];
        v += __shfl_xor(v, 16, 64);
        v += __shfl_xor(v, 32, 64);
        if (lane < kDecE) wsum[wid][t][lane] = v;
    }
    __syncthreads();
    double v = 0.0;
    if (tid < T * kDecE)
        for (int w = 0; w < kRouteWaves; ++w) v += wsum[w][tid / kDecE][tid % kDecE];
    return v;
}

// x on the e4m3 grid, for experts in that form: the work of the workgroups behind
// those that form logits or place pairs, 64 blocks of 128 each (a launch of its own
// is 4 us).
constexpr int kRoundBlocks = kRouteThreads / 16;
__device__ __forceinline__ void round_x(const uint16_t* x, uint16_t* xq, int T, int d, int wg)
{
    const int u = wg * kRoundBlocks + threadIdx.x / 16;
    if (u >= T * (d / kBlock)) return;                   // 16 lanes at once
    const int64_t at = (int64_t)u * kBlock + threadIdx.x % 16 * 8;
    float v[8];
    unpack8(*reinterpret_cast<const u32x4_t*>(x + at), v);
    *reinterpret_cast<u32x4_t*>(xq + at) = round_block(v);
}

template <int kT>
__global__ __launch_bounds__(kRouteThreads) void route_partials_kernel(DecodeRouteArgs a)
{
    if ((int)blockIdx.x >= a.n_wg) {
        round_x(a.x, a.xq, a.T, a.d, blockIdx.x - a.n_wg);
        return;
    }
    const double v = partial_logits<kT>(a);
    const int tid = threadIdx.x;
    if (tid < a.T * kDecE) a.partial[(int64_t)blockIdx.x * kSmallT * kDecE + tid] = v;
}

template <bool kPolicy>
__device__ __forceinline__ void finish_route(const DecodeRouteArgs& a, float (&lg)[kSmallT][kDecE]);

// logits, selection and permutation in LDS, then every routing output
// written at the end (global stores are not waited for inside the
// workgroup).  Every step is spread over threads: one (token, expert) pair
// per thread.
template <bool kPolicy>
__global__ __launch_bounds__(kRouteThreads) void route_finish_kernel(DecodeRouteArgs a)
{
    __shared__ float lg[kSmallT][kDecE];
    const int T = a.T, E = a.E;
    const int tid = threadIdx.x;
    if (tid < T * kDecE) {
        const int t = tid / kDecE, ee = tid % kDecE;
        if (ee < E) {
            // the partials of all workgroups loaded at once, summed in
            // workgroup order
            double pv[kDecMaxWg];
#pragma unroll
            for (int w = 0; w < kDecMaxWg; ++w)
                pv[w] = w < a.n_wg ? __builtin_nontemporal_load(
                                         &a.partial[((int64_t)w * kSmallT + t) * kDecE + ee])
                                   : 0.0;
            double v = 0.0;
#pragma unroll
            for (int w = 0; w < kDecMaxWg; ++w)
                if (w < a.n_wg) v += pv[w];
            for (int w = kDecMaxWg; w < a.n_wg; ++w)
                v += __builtin_nontemporal_load(&a.partial[((int64_t)w * kSmallT + t) * kDecE + ee]);
            float l = (float)v;
            if (a.bias) l = __fadd_rn(l, a.bias[ee]);
            lg[t][ee] = l;
        }
    }
    finish_route<kPolicy>(a, lg);
}

// Both halves in one launch where one workgroup forms the logits anyway
// (d <= 512): small layer (d 256, f 512, 8 experts, top-2) at 1 token 19.8 ->
// 16.3 us, at 16 tokens 21.1 -> 18.8.
template <int kT, bool kPolicy>
__global__ __launch_bounds__(kRouteThreads) void route_one_kernel(DecodeRouteArgs a)
{
    __shared__ float lg[kSmallT][kDecE];
    if (blockIdx.x > 0) {
        round_x(a.x, a.xq, a.T, a.d, blockIdx.x - 1);
        return;
    }
    const double v = partial_logits<kT>(a);
    const int tid = threadIdx.x, t = tid / kDecE, ee = tid % kDecE;
    if (t < a.T && ee < a.E) {
        float l = (float)v;
        if (a.bias) l = __fadd_rn(l, a.bias[ee]);
        lg[t][ee] = l;
    }
    finish_route<kPolicy>(a, lg);
}

template <bool kPolicy>
__device__ __forceinline__ void finish_route(const DecodeRouteArgs& a, float (&lg)[kSmallT][kDecE])
{
    __shared__ int s_ids[kDecPairs];
    __shared__ float s_w[kDecPairs];
    __shared__ int s_rank[kSmallT][kDecE];
    __shared__ int s_cnt[kDecE];
    __shared__ int s_off[kDecE + 1];
    const int T = a.T, E = a.E, k = a.k;
    const int tid = threadIdx.x;
    const int lane = tid & 63, wid = tid >> 6;
    lds_barrier();
    if constexpr (kPolicy) {
        // 16 lanes per token
        if (tid < T * kDecE) {
            const int t = tid / kDecE, e = tid % kDecE;
            choose<kDecE>(a.policy, lg[t][min(e, E - 1)], e, E, k, &s_ids[t * k], &s_w[t * k]);
        }
    } else {
        // rank of expert e in its token's order (logit descending, id ascending):
        // the experts before e with a logit >= its own and those after it with a
        // larger one; rank < k selects it at slot rank.  A row holding a NaN
        // takes the sequential scan instead (its order is scan-dependent).
        if (tid < T * kDecE) {
            const int t = tid / kDecE, e = tid % kDecE;
            if (e < E) {
                const float le = lg[t][e];
                int r = 0;
                bool ordered = true;
                for (int q = 0; q < E; ++q) {
                    const float lq = lg[t][q];
                    ordered = ordered && lq == lq;
                    r += q < e ? (lq >= le ? 1 : 0) : (lq > le ? 1 : 0);
                }
                s_rank[t][e] = ordered ? r : -1;
                if (ordered && r < k) s_ids[t * k + r] = e;
            }
        }
        lds_barrier();
        if (tid < T) {
            const int t = tid;
            if (s_rank[t][0] < 0) {
                select_token<kDecE>(&lg[t][0], E, k, &s_ids[t * k], &s_w[t * k]);
            } else {
                // weights in slot order, as the sequential selection forms them
                const float lmax = lg[t][s_ids[t * k]];
                float z = 0.f;
                for (int j2 = 0; j2 < k; ++j2) {
                    const float p = expf(lg[t][s_ids[t * k + j2]] - lmax);
                    s_w[t * k + j2] = p;
                    z += p;
                }
                const float inv = 1.0f / z;
                for (int j2 = 0; j2 < k; ++j2) s_w[t * k + j2] = s_w[t * k + j2] * inv;
            }
        }
    }
    lds_barrier();
    const int P = T * k;
    const int lo = a.e_begin, hi = a.e_begin + a.n_local;
    if (tid < E) {
        int c = 0;
        if (tid >= lo && tid < hi)
            for (int p = 0; p < P; ++p) c += (s_ids[p] == tid);
        s_cnt[tid] = c;
    }
    lds_barrier();
    // per expert: its first row, active-list slot and first tile, from
    // prefix sums over the experts before it (lanes 0..15 of wave 0)
    if (wid == 0) {
        const int c = tid < E ? s_cnt[tid] : 0;
        const int nz = c > 0 ? 1 : 0;
        const int tl = (c + a.tile_rows - 1) / a.tile_rows;
        int run = c, na = nz, nt = tl;
#pragma unroll
        for (int off = 1; off < kDecE; off <<= 1) {
            const int r1 = __shfl_up(run, off, 64), n1 = __shfl_up(na, off, 64),
                      t1 = __shfl_up(nt, off, 64);
            if (lane >= off) { run += r1; na += n1; nt += t1; }
        }
        run -= c; na -= nz; nt -= tl;   // exclusive
        if (tid < E) {
            s_off[tid] = run;
            a.rv.counts[tid] = c;
            a.rv.offsets[tid] = run;
            if (c > 0) {
                a.rv.active[1 + na] = tid;
                for (int r = 0; r < c; r += a.tile_rows) {
                    a.rv.tiles[2 * nt] = tid;
                    a.rv.tiles[2 * nt + 1] = run + r;
                    ++nt;
                }
            }
            if (tid == E - 1) {
                a.rv.offsets[E] = run + c;
                a.rv.active[0] = na + nz;
                *a.rv.n_tiles = nt;
            }
        }
    }
    lds_barrier();
    if (tid < P) {
        const int ee = s_ids[tid];
        a.rv.topk_idx[tid] = ee;
        a.rv.topk_w[tid] = s_w[tid];
        if (ee >= lo && ee < hi) {
            int rank = 0;
            for (int p = 0; p < tid; ++p) rank += (s_ids[p] == ee);
            const int r = s_off[ee] + rank;
            a.rv.pair_row[tid] = r;
            a.rv.row_token[r] = tid / k;
        } else {
            a.rv.pair_row[tid] = -1;
        }
    }
    if (tid < T * kDecE) {
        const int t = tid / kDecE, ee = tid % kDecE;
        if (ee < E) a.rv.logits[(int64_t)t * E + ee] = lg[t][ee];
    }
}

// Logits of many tokens, on the fp64 matrix cores.  A workgroup takes 16 tokens
// (kTiles times) x 16 experts and every n_split-th 512 elements of the reduction
// axis, its 16 waves 32 of them each; a wave's step is eight v_mfma_f64_16x16x4_f64,
// lane l holding eight elements of token l % 16 and of expert l % 16, those from 8 (l
// / 16) on, and instruction i taking the i-th of all four runs.  A step's loads are
// issued before the multiplications of the step before.  The waves' sums meet in
// LDS and are added in wave order; with several ranges (few tokens: one workgroup
// alone multiplies 10 us long at d 6144) they go to the workspace, and
// sum_select_kernel adds them in order.  Every conversion to fp64 serves 16
// products; four tokens x eight experts per wave on the vector unit, 64 lanes along
// the axis and a transpose-reduce at the end, took 17 us for 17 to 500 tokens of d
// 6144 and 16 experts, 26 for 2048, 92 for 8000, 81 for 2048 and 64 experts.
constexpr int kRmWaves = 16;
constexpr int kRmStep = 32;
constexpr int kRmAxis = kRmWaves * kRmStep;
constexpr int kRmWg = 256;         // workgroups that n_split aims at: one per CU
constexpr int kRmManyWg = 512;     // workgroups of 16 tokens from which on they take 32
typedef double f64x4_t __attribute__((ext_vector_type(4)));

template <int kTiles>              // of 16 tokens
__global__ __launch_bounds__(64 * kRmWaves) void router_kernel(const uint16_t* __restrict__ x,
                                                               const float* __restrict__ wrT,
                                                               const float* __restrict__ bias, int T, int d, int E,
                                                               float* __restrict__ logits, double* __restrict__ part)
{
    __shared__ double s_part[kRmWaves][4][64];
    const int tid = threadIdx.x, lane = tid % 64, w = tid / 64;
    const int t0 = blockIdx.x * (16 * kTiles), e0 = blockIdx.y * 16;
    // tokens past T and experts past E: the last ones again, their sums dropped
    const uint16_t* px[kTiles];
#pragma unroll
    for (int n = 0; n < kTiles; ++n) px[n] = x + (int64_t)min(t0 + n * 16 + lane % 16, T - 1) * d + lane / 16 * 8;
    const float* pw = wrT + (int64_t)min(e0 + lane % 16, E - 1) * d + lane / 16 * 8;
    struct Step {
        u32x4_t x[kTiles];
        float4 w0, w1;
    };
    auto fetch = [&](Step& s, int k) {
#pragma unroll
        for (int n = 0; n < kTiles; ++n) s.x[n] = *reinterpret_cast<const u32x4_t*>(px[n] + k);
        s.w0 = *reinterpret_cast<const float4*>(pw + k);
        s.w1 = *reinterpret_cast<const float4*>(pw + k + 4);
    };
    f64x4_t acc[kTiles];
#pragma unroll
    for (int n = 0; n < kTiles; ++n) acc[n] = f64x4_t{0.0, 0.0, 0.0, 0.0};
    auto multiply = [&](const Step& s) {
        const float wv[8] = {s.w0.x, s.w0.y, s.w0.z, s.w0.w, s.w1.x, s.w1.y, s.w1.z, s.w1.w};
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int n = 0; n < kTiles; ++n) {
                const float xv = __uint_as_float(i % 2 ? s.x[n][i / 2] & 0xFFFF0000u : s.x[n][i / 2] << 16);
                acc[n] = __builtin_amdgcn_mfma_f64_16x16x4f64((double)xv, (double)wv[i], acc[n], 0, 0, 0);
            }
    };
    const int all = kRmAxis * gridDim.z;
    Step s0, s1;
    int k = blockIdx.z * kRmAxis + w * kRmStep;
    if (k < d) fetch(s0, k);
    for (; k < d; k += 2 * all) {
        fetch(s1, min(k + all, d - kRmStep));
        multiply(s0);
        if (k + all >= d) break;
        fetch(s0, min(k + 2 * all, d - kRmStep));
        multiply(s1);
    }
    // lane l holds tokens l / 16 + 4 i of expert l % 16
#pragma unroll
    for (int n = 0; n < kTiles; ++n) {
        if (n > 0) __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) s_part[w][i][lane] = acc[n][i];
        __syncthreads();
        if (tid < 256) {
            const int i = tid / 64, t = t0 + n * 16 + lane / 16 + 4 * i, e = e0 + lane % 16;
            double v = 0.0;
#pragma unroll
            for (int q = 0; q < kRmWaves; ++q) v += s_part[q][i][lane];
            if (part) {
                const int64_t rows = (int64_t)gridDim.x * (16 * kTiles);
                part[(blockIdx.z * rows + t) * (gridDim.y * 16) + e] = v;
            } else if (t < T && e < E) {
                float l = (float)v;
                if (bias) l = __fadd_rn(l, bias[e]);
                logits[(int64_t)t * E + e] = l;
            }
        }
    }
}

// The logits of router_kernel's ranges (n of them, rows x ld apart), and the
// selection: one wave per token, lane e its expert e.
template <bool kPolicy>
__global__ __launch_bounds__(256) void sum_select_kernel(const double* __restrict__ part, int n, int64_t rows, int ld,
                                                         const float* __restrict__ bias, int T, int E, int k,
                                                         Policy policy, RouteView rv)
{
    __shared__ float lg[256 / kWave][kWave];
    const int lane = threadIdx.x % kWave, w = threadIdx.x / kWave, t = blockIdx.x * (256 / kWave) + w;
    if (t >= T) return;
    constexpr int kAtOnce = 8;                           // ranges' sums in flight
    double v = 0.0;
    for (int z0 = 0; z0 < n; z0 += kAtOnce) {
        double p[kAtOnce];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) p[i] = part[(min(z0 + i, n - 1) * rows + t) * ld + min(lane, E - 1)];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i)
            if (z0 + i < n) v += p[i];
    }
    float l = (float)v;
    if (bias) l = __fadd_rn(l, bias[min(lane, E - 1)]);
    if (lane < E) rv.logits[(int64_t)t * E + lane] = l;
    if constexpr (kPolicy) {
        choose<kWave>(policy, l, lane, E, k, rv.topk_idx + (int64_t)t * k, rv.topk_w + (int64_t)t * k);
    } else {
        lg[w][lane] = l;                                 // (read by the wave that wrote it)
        __builtin_amdgcn_wave_barrier();
        if (lane == 0) select_token_any(&lg[w][0], t, E, k, rv);
    }
}

// Selection from fp32 logits (copied into the routing view, where they are not
// there already): one thread per token.
__global__ __launch_bounds__(256) void select_kernel(const float* logits_in, int T,
                                                     int E, int k, RouteView rv)
{
    const int t = blockIdx.x * blockDim.x + threadIdx.x;
    if (t >= T) return;
    const float* l = logits_in + (int64_t)t * E;
    if (logits_in != rv.logits)
        for (int e = 0; e < E; ++e) rv.logits[(int64_t)t * E + e] = l[e];
    select_token_any(l, t, E, k, rv);
}

// The same under a policy: one wave per token.
__global__ __launch_bounds__(256) void policy_select_kernel(const float* logits_in, int T, int E, int k,
                                                            Policy policy, RouteView rv)
{
    const int t = blockIdx.x * (256 / kWave) + threadIdx.x / kWave, lane = threadIdx.x % kWave;
    if (t >= T) return;
    const float l = logits_in[(int64_t)t * E + min(lane, E - 1)];
    if (lane < E && logits_in != rv.logits) rv.logits[(int64_t)t * E + lane] = l;
    choose<kWave>(policy, l, lane, E, k, rv.topk_idx + (int64_t)t * k, rv.topk_w + (int64_t)t * k);
}

// Expert-grouped permutation of the T*k pairs, rows grouped by local expert, then
// by pair (token, slot) order.  A workgroup places a chunk of 1024 pairs (or of
// several rounds of 1024, where there are more than kPermMaxWg chunks).  It
// counts every pair's expert, those of earlier chunks apart, so that it knows the
// experts' first rows and how many rows the chunks before it take of each, without
// a launch or a wait between workgroups; the ids are 4 bytes a pair and lie in the
// L2.  A pair's place among its round's is the number of equal ids before it: in
// its wave by ballots over the id's bits, of the waves before by their counts.
// Deterministic: the counts are sums, and no atomic decides a row.  (One workgroup
// that placed all pairs, 8192 at a time with packed counters of 16 experts: 18 us
// for 8192 pairs of 16 experts, 68 for 16384 of 64.)
constexpr int kPermMaxWg = 1024;
constexpr int kPermCopies = 4;       // histograms, by lane: fewer lanes meet at one counter

struct PermArgs {
    int T, E, k, e_begin, n_local, tile_rows;
    int chunk;                       // pairs per workgroup, a multiple of kRouteThreads
    int n_wg;                        // workgroups that place pairs; those behind them ...
    const uint16_t* x;               // ... round x [T, d] to xq, or there are none
    uint16_t* xq;
    int d;
    RouteView rv;
};

__global__ __launch_bounds__(kRouteThreads) void permute_kernel(PermArgs a)
{
    __shared__ int hist[2][kPermCopies][64];     // all pairs, pairs of earlier chunks
    __shared__ int cursor[64];
    __shared__ int wcount[kRouteWaves][64];
    const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
    const int E = a.E, k = a.k, P = a.T * a.k;
    const int lo = a.e_begin, hi = a.e_begin + a.n_local;
    const RouteView& rv = a.rv;
    if ((int)blockIdx.x >= a.n_wg) {
        round_x(a.x, a.xq, a.T, a.d, blockIdx.x - a.n_wg);
        return;
    }
    const int c0 = (int)blockIdx.x * a.chunk, c1 = min(c0 + a.chunk, P);
    if (tid < 2 * kPermCopies * 64) (&hist[0][0][0])[tid] = 0;
    lds_barrier();
    constexpr int kLoads = 8;                    // ids in flight per thread
    for (int p0 = tid; p0 < P; p0 += kRouteThreads * kLoads) {
        int ids[kLoads];
#pragma unroll
        for (int i = 0; i < kLoads; ++i) ids[i] = rv.topk_idx[min(p0 + i * kRouteThreads, P - 1)];
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int p = p0 + i * kRouteThreads, e = ids[i];
            if (p < P && e >= lo && e < hi) {
                atomicAdd(&hist[0][lane % kPermCopies][e], 1);
                if (p < c0) atomicAdd(&hist[1][lane % kPermCopies][e], 1);
            }
        }
    }
    lds_barrier();
    // the experts' first rows (wave 0); workgroup 0 also writes the counts, the
    // active list and the tiles
    if (wid == 0) {
        int c = 0, earlier = 0;
#pragma unroll
        for (int i = 0; i < kPermCopies; ++i) {
            c += hist[0][i][lane];
            earlier += hist[1][i][lane];
        }
        const int nz = c > 0 ? 1 : 0;
        const int tl = (c + a.tile_rows - 1) / a.tile_rows;
        int run = c, na = nz, nt = tl;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int r1 = __shfl_up(run, off, 64), n1 = __shfl_up(na, off, 64),
                      t1 = __shfl_up(nt, off, 64);
            if (lane >= off) { run += r1; na += n1; nt += t1; }
        }
        run -= c; na -= nz; nt -= tl;   // exclusive
        cursor[lane] = run + earlier;
        if (lane < E && blockIdx.x == 0) {
            rv.counts[lane] = c;
            rv.offsets[lane] = run;
            if (c > 0) {
                rv.active[1 + na] = lane;
                for (int r = 0; r < c; r += a.tile_rows) {
                    rv.tiles[2 * nt] = lane;
                    rv.tiles[2 * nt + 1] = run + r;
                    ++nt;
                }
            }
            if (lane == E - 1) {
                rv.offsets[E] = run + c;
                rv.active[0] = na + nz;
                *rv.n_tiles = nt;
            }
        }
    }
    for (int r0 = c0; r0 < c1; r0 += kRouteThreads) {
        const int p = r0 + tid;
        const int id = p < c1 ? rv.topk_idx[p] : -1;
        const bool mine = id >= lo && id < hi;
        uint64_t same = __ballot(mine);          // the wave's pairs of the same expert
#pragma unroll
        for (int bit = 0; bit < 6; ++bit) {
            const uint64_t set = __ballot(id >> bit & 1);
            same &= id >> bit & 1 ? set : ~set;
        }
        const int before = __popcll(same & ((1ull << lane) - 1));
        (&wcount[0][0])[tid] = 0;
        lds_barrier();                           // (and the cursors are written)
        if (mine && before == 0) wcount[wid][id] = __popcll(same);
        lds_barrier();
        int row = -1;
        if (mine) {
            row = cursor[id] + before;
            for (int w = 0; w < wid; ++w) row += wcount[w][id];
            rv.row_token[row] = p / k;
        }
        if (p < c1) rv.pair_row[p] = row;
        lds_barrier();                           // every thread has read the cursors
        if (tid < 64) {
            int n = 0;
#pragma unroll
            for (int w = 0; w < kRouteWaves; ++w) n += wcount[w][tid];
            cursor[tid] += n;
        }
        lds_barrier();                           // ... and the waves' counts
    }
}

// wrT[e][i] = wr[i][e]
__global__ __launch_bounds__(256) void transpose_router_kernel(const float* __restrict__ wr, int d,
                                                               int E, float* __restrict__ wrT)
{
    const int64_t n = (int64_t)d * E;
    for (int64_t o = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; o < n;
         o += (int64_t)gridDim.x * blockDim.x) {
        const int64_t e = o / d, i = o % d;
        wrT[o] = wr[i * E + e];
    }
}

}  // namespace moe

extern "C" int moe_route_decode_ok(int T, int E, int k)
{
    return T >= 1 && T <= moe::kSmallT && E <= moe::kDecE && T * k <= moe::kDecPairs;
}

extern "C" int moe_route_decode_wgs(int d) { return (d / 8 + 63) / 64; }

// workgroups that round x [T, d]
static int round_wgs(int T, int d) { return (T * (d / moe::kBlock) + moe::kRoundBlocks - 1) / moe::kRoundBlocks; }



extern "C" hipError_t moe_launch_route_decode(const uint16_t* x, const float* wrT,
                                              const float* bias, double* partial, int T, int d,
                                              int E, int k, int e_begin, int n_local, int tile_rows,
                                              const moe::Policy* policy, uint16_t* xq,
                                              const moe::RouteView* rv, hipStream_t s)
{
    moe::DecodeRouteArgs a{};
    a.policy = *policy;
    a.xq = xq;
    const int n_round = xq ? round_wgs(T, d) : 0;
    a.x = x; a.wrT = wrT; a.bias = bias; a.partial = partial;
    a.T = T; a.d = d; a.E = E; a.k = k;
    a.e_begin = e_begin; a.n_local = n_local; a.tile_rows = tile_rows;
    a.rv = *rv;
    a.n_wg = moe_route_decode_wgs(d);
    using Kernel = void (*)(moe::DecodeRouteArgs);
    auto by_tokens = [T](Kernel k1, Kernel k2, Kernel k4, Kernel k8, Kernel k16) {
        return T == 1 ? k1 : T == 2 ? k2 : T <= 4 ? k4 : T <= 8 ? k8 : k16;
    };
    if (a.n_wg == 1) {
        const Kernel one =
            policy->on ? by_tokens(moe::route_one_kernel<1, true>, moe::route_one_kernel<2, true>,
                                   moe::route_one_kernel<4, true>, moe::route_one_kernel<8, true>,
                                   moe::route_one_kernel<moe::kSmallT, true>)
                       : by_tokens(moe::route_one_kernel<1, false>, moe::route_one_kernel<2, false>,
                                   moe::route_one_kernel<4, false>, moe::route_one_kernel<8, false>,
                                   moe::route_one_kernel<moe::kSmallT, false>);
        hipLaunchKernelGGL(one, dim3(1 + n_round), dim3(moe::kRouteThreads), 0, s, a);
        return hipGetLastError();
    }
    const Kernel partials = by_tokens(moe::route_partials_kernel<1>, moe::route_partials_kernel<2>,
                                      moe::route_partials_kernel<4>, moe::route_partials_kernel<8>,
                                      moe::route_partials_kernel<moe::kSmallT>);
    hipLaunchKernelGGL(partials, dim3(a.n_wg + n_round), dim3(moe::kRouteThreads), 0, s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const Kernel finish = policy->on ? moe::route_finish_kernel<true> : moe::route_finish_kernel<false>;
    hipLaunchKernelGGL(finish, dim3(1), dim3(moe::kRouteThreads), 0, s, a);
    return hipGetLastError();
}

static hipError_t launch_select(const float* logits, int T, int E, int k, const moe::Policy* policy,
                                const moe::RouteView* rv, hipStream_t s)
{
    if (policy->on)
        hipLaunchKernelGGL(moe::policy_select_kernel, dim3((T + 3) / 4), dim3(256), 0, s, logits, T, E, k, *policy, *rv);
    else
        hipLaunchKernelGGL(moe::select_kernel, dim3((T + 255) / 256), dim3(256), 0, s, logits, T, E, k, *rv);
    return hipGetLastError();
}

// Ranges of the reduction axis that router_kernel takes for T tokens.
static int router_split(int T, int d, int E)
{
    const int64_t wgs = (int64_t)((T + 15) / 16) * ((E + 15) / 16);
    return (int)std::max<int64_t>(1, std::min<int64_t>(moe::kRmWg / wgs, d / moe::kRmAxis));
}

// Workspace of the partial logits of up to max_tokens tokens: the decode routing's,
// and router_kernel's, whose ranges are as many as fit kRmWg workgroups.
extern "C" size_t moe_route_partial_bytes(int max_tokens, int d, int E)
{
    const size_t tiles = (size_t)((max_tokens + 15) / 16) * ((E + 15) / 16) * std::max(1, d / moe::kRmAxis);
    const size_t few = (size_t)moe_route_decode_wgs(d) * moe::kSmallT * moe::kDecE;
    return std::max(few, std::min<size_t>(tiles, moe::kRmWg) * 16 * 16) * sizeof(double);
}

extern "C" hipError_t moe_launch_router_select(const uint16_t* x, const float* wrT,
                                               const float* bias, double* partial, int T, int d, int E, int k,
                                               const moe::Policy* policy,
                                               const moe::RouteView* rv, hipStream_t s)
{
    const int n_e = (E + 15) / 16, n_t = (T + 15) / 16, n = router_split(T, d, E);
    double* part = n > 1 ? partial : nullptr;
    if ((int64_t)n_t * n_e >= moe::kRmManyWg)
        hipLaunchKernelGGL(moe::router_kernel<2>, dim3((n_t + 1) / 2, n_e), dim3(64 * moe::kRmWaves), 0, s, x, wrT, bias, T, d,
                           E, rv->logits, part);
    else
        hipLaunchKernelGGL(moe::router_kernel<1>, dim3(n_t, n_e, n), dim3(64 * moe::kRmWaves), 0, s, x, wrT, bias, T, d, E,
                           rv->logits, part);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (!part) return launch_select(rv->logits, T, E, k, policy, rv, s);
    const auto kernel = policy->on ? moe::sum_select_kernel<true> : moe::sum_select_kernel<false>;
    hipLaunchKernelGGL(kernel, dim3((T + 3) / 4), dim3(256), 0, s, part, n, (int64_t)n_t * 16, n_e * 16, bias, T, E, k,
                       *policy, *rv);
    return hipGetLastError();
}

extern "C" hipError_t moe_launch_route(const float* logits_in, int T, int E, int k, int e_begin,
                                       int n_local, int tile_rows, const moe::Policy* policy,
                                       const uint16_t* x, int d, uint16_t* xq, const moe::RouteView* rv,
                                       hipStream_t s)
{
    if (logits_in) {
        const hipError_t e = launch_select(logits_in, T, E, k, policy, rv, s);
        if (e != hipSuccess) return e;
    }
    moe::PermArgs a{};
    a.T = T; a.E = E; a.k = k;
    a.e_begin = e_begin; a.n_local = n_local; a.tile_rows = tile_rows;
    a.rv = *rv;
    const int64_t rounds = ((int64_t)T * k + moe::kRouteThreads - 1) / moe::kRouteThreads;
    const int per_wg = (int)((rounds + moe::kPermMaxWg - 1) / moe::kPermMaxWg);
    a.chunk = per_wg * moe::kRouteThreads;
    a.n_wg = (int)((rounds + per_wg - 1) / per_wg);
    a.x = x;
    a.xq = xq;
    a.d = d;
    hipLaunchKernelGGL(moe::permute_kernel, dim3(a.n_wg + (xq ? round_wgs(T, d) : 0)), dim3(moe::kRouteThreads), 0, s, a);
    return hipGetLastError();
}

extern "C" hipError_t moe_launch_transpose_router(const float* wr, int d, int E, float* wrT,
                                                  hipStream_t s)
{
    const int64_t n = (int64_t)d * E;
    int grid = (int)std::min<int64_t>((n + 255) / 256, 4096);
    hipLaunchKernelGGL(moe::transpose_router_kernel, dim3(grid), dim3(256), 0, s, wr, d, E, wrT);
    return hipGetLastError();
}
