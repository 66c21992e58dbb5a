// The mixture-of-experts layer's routing: router logits, Top-K and gates of
// every token, and the control block of the experts' kernel set to zero.
//
//   z = W^R x,  S = TopK(z) (score descending, index ascending),
//   g_e = exp(z_e - max z) / sum exp(z - max z), divided by its sum over S on request
//
// A cluster of eight CTAs takes 16 tokens: each CTA multiplies one eighth of d
// for all experts and the CTAs' partial logits are summed, in rank order,
// through distributed shared memory; then a warp takes a token.  Splitting d
// reads every element of x and W^R once per cluster (one token of N = 128,
// d = 2048: 64 KB of W^R a CTA, against 512 KB on one), and the sum of eight short
// chains is nearer to the exact logit than one long one.
#pragma once

#include "crc_device.cuh"

namespace crc {

constexpr int kRouteTokens = 16;     // tokens of a cluster: the rows of one m16n8k16
constexpr int kRouteCtas = 8;        // portable cluster size
constexpr int kRouteThreads = 256;
constexpr int kMoeMaxN = 128;

struct MoeRouteArgs {
    const uint16_t* x;               // bf16, rows ldx apart (null: scores given, no x)
    const uint16_t* w;               // bf16 [N][d]
    const float* scores;             // fp32 rows lds apart, or null
    long long ldx, lds;
    int M, N, K, d;
    int renorm;
    uint8_t* ids;                    // [M][K]
    float* gates;                    // [M][K]
    uint8_t* ids_out;                // the caller's, or null
    float* gates_out;
    float* xscale;                   // [M] power-of-two scale of x's row, or null
    uint32_t* ctrl;                  // zeroed
    int ctrl_words;
};

__device__ __forceinline__ void pdl_launch_dependents() {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}
__device__ __forceinline__ void pdl_wait() {
    asm volatile("griddepcontrol.wait;" ::: "memory");
}

// Scores as integers in the same order; NaN lowest, 0 left for "none".
__device__ __forceinline__ uint32_t score_key(float v) {
    if (v != v) return 1u;
    const uint32_t b = __float_as_uint(v + 0.0f);          // -0 -> +0
    return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float score_of(uint32_t key) {
    if (key == 1u) return __uint_as_float(0x7fc00000u);
    return __uint_as_float((key & 0x80000000u) ? key & 0x7fffffffu : ~key);
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
    return v;
}

// One warp: Top-K and gates of a token; lane i holds the scores of experts
// i, i + 32, ... (those < N).  probs: the scores are probabilities.
__device__ __forceinline__ void route_token(const float (&v)[4], int N, int K, bool probs,
                                            int renorm, int lane, uint8_t* ids, float* gates,
                                            uint8_t* ids_out, float* gates_out) {
    uint32_t key[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) key[i] = lane + 32 * i < N ? score_key(v[i]) : 0u;
    float mx = 0.f, total = 1.f, chosen = 0.f, mine = 0.f;
    int my_id = 0;
    for (int k = 0; k < K; ++k) {
        const uint32_t best = __reduce_max_sync(
            kFull, max(max(key[0], key[1]), max(key[2], key[3])));
        uint32_t at = 0xffu;
#pragma unroll
        for (int i = 3; i >= 0; --i)
            if (key[i] == best) at = (uint32_t)(lane + 32 * i);
        const uint32_t e = __reduce_min_sync(kFull, at);    // ties to the lowest index
        if (k == 0 && !probs) {
            mx = score_of(best);
            float s = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (lane + 32 * i < N) s += expf(v[i] - mx);
            total = warp_sum(s);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if ((uint32_t)(lane + 32 * i) == e) key[i] = 0u;
        const float z = score_of(best);
        const float p = probs ? z : expf(z - mx) / total;
        chosen += p;
        if (lane == k) {
            mine = p;
            my_id = (int)e;
        }
    }
    if (lane < K) {
        if (renorm) mine /= chosen;
        ids[lane] = (uint8_t)my_id;
        gates[lane] = mine;
        if (ids_out) ids_out[lane] = (uint8_t)my_id;
        if (gates_out) gates_out[lane] = mine;
    }
}

__device__ __forceinline__ void mma_bf16_16x8x16(float (&c)[4], uint32_t a0, uint32_t a1,
                                                 uint32_t a2, uint32_t a3, uint32_t b0,
                                                 uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
        "{%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ float dsm_f32(uint32_t addr) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr));
    return v;
}

__device__ __forceinline__ void zero_ctrl(const MoeRouteArgs& a) {
    if (blockIdx.x == 0)
        for (int i = threadIdx.x; i < a.ctrl_words; i += blockDim.x) a.ctrl[i] = 0u;
}

// The power-of-two scale that brings a row's largest value into [128, 256): two
// e4m3 pieces, hi + lo / 16, then hold a bf16 x exactly down to 2^-13 of the row's
// largest and to 2^-21 of it below.
// NaN for a row with an infinity or a NaN, which makes its results NaN.
__device__ __forceinline__ float split_scale(float amax) {
    const uint32_t ex = __float_as_uint(amax) >> 23;
    if (ex >= 255u) return __uint_as_float(0x7fc00000u);
    return __uint_as_float((ex < 8u ? 1u : ex - 7u) << 23);
}

__global__ void __launch_bounds__(kRouteThreads)
    moe_route_kernel(MoeRouteArgs a) {
    __shared__ float part[kRouteTokens][kMoeMaxN];
    __shared__ float amax_sm[kRouteTokens];
    zero_ctrl(a);
    pdl_launch_dependents();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = (int)cluster_ctarank();
    const int t0 = (int)(blockIdx.x / kRouteCtas) * kRouteTokens;
    const int g = lane >> 2, t = lane & 3;
    // this CTA's chunks of 32 elements of d
    const int nch = (a.d + 31) / 32;
    const int c0 = nch * rank / kRouteCtas, c1 = nch * (rank + 1) / kRouteCtas;
    const int tiles = a.N / 8;                       // tiles of 8 experts: this warp's warp, warp + 8
    const bool lo = warp < tiles, hi = warp + 8 < tiles;
    const bool r0 = t0 + g < a.M, r1 = t0 + g + 8 < a.M;
    const uint16_t* x0 = a.x + (long long)(r0 ? t0 + g : 0) * a.ldx + 8 * t;
    const uint16_t* x1 = a.x + (long long)(r1 ? t0 + g + 8 : 0) * a.ldx + 8 * t;
    const uint16_t* w0 = a.w + (size_t)(lo ? warp * 8 + g : 0) * a.d + 8 * t;
    const uint16_t* w1 = a.w + (size_t)(hi ? (warp + 8) * 8 + g : 0) * a.d + 8 * t;
    float acc0[4] = {}, acc1[4] = {};
    float am0 = 0.f, am1 = 0.f;
    if (lo) {
        const uint4 zero = make_uint4(0, 0, 0, 0);
        // The order of k inside a product is free as long as both operands share
        // it: a thread's 16 contiguous bytes of a row serve two k16 steps.
#pragma unroll 8
        for (int c = c0; c < c1; ++c) {
            const bool in = 32 * c + 8 * t < a.d;
            const uint4 xa = in && r0 ? *reinterpret_cast<const uint4*>(x0 + 32 * c) : zero;
            const uint4 xb = in && r1 ? *reinterpret_cast<const uint4*>(x1 + 32 * c) : zero;
            const uint4 wa = in ? *reinterpret_cast<const uint4*>(w0 + 32 * c) : zero;
            const uint4 wb = in && hi ? *reinterpret_cast<const uint4*>(w1 + 32 * c) : zero;
            mma_bf16_16x8x16(acc0, xa.x, xb.x, xa.y, xb.y, wa.x, wa.y);
            mma_bf16_16x8x16(acc0, xa.z, xb.z, xa.w, xb.w, wa.z, wa.w);
            if (hi) {
                mma_bf16_16x8x16(acc1, xa.x, xb.x, xa.y, xb.y, wb.x, wb.y);
                mma_bf16_16x8x16(acc1, xa.z, xb.z, xa.w, xb.w, wb.z, wb.w);
            }
            if (a.xscale && warp == 0) {
                const uint32_t ua[4] = {xa.x, xa.y, xa.z, xa.w}, ub[4] = {xb.x, xb.y, xb.z, xb.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    // magnitudes as integers: a NaN counts as the largest
                    am0 = __uint_as_float(max(__float_as_uint(am0),
                                              max(ua[i] << 16 & 0x7fffffffu,
                                                  ua[i] & 0x7fff0000u)));
                    am1 = __uint_as_float(max(__float_as_uint(am1),
                                              max(ub[i] << 16 & 0x7fffffffu,
                                                  ub[i] & 0x7fff0000u)));
                }
            }
        }
        const int n = warp * 8 + 2 * t;
        part[g][n] = acc0[0];
        part[g][n + 1] = acc0[1];
        part[g + 8][n] = acc0[2];
        part[g + 8][n + 1] = acc0[3];
        if (hi) {
            part[g][n + 64] = acc1[0];
            part[g][n + 65] = acc1[1];
            part[g + 8][n + 64] = acc1[2];
            part[g + 8][n + 65] = acc1[3];
        }
    }
    if (a.xscale && warp == 0) {
#pragma unroll
        for (int o = 1; o < 4; o <<= 1) {
            am0 = __uint_as_float(max(__float_as_uint(am0),
                                      __shfl_xor_sync(kFull, __float_as_uint(am0), o)));
            am1 = __uint_as_float(max(__float_as_uint(am1),
                                      __shfl_xor_sync(kFull, __float_as_uint(am1), o)));
        }
        if (t == 0) {
            amax_sm[g] = am0;
            amax_sm[g + 8] = am1;
        }
    }
    cluster_sync();
    // tokens rank and rank + 8 of the cluster: a warp each
    const int tok = rank + 8 * warp;
    if (warp < 2 && t0 + tok < a.M) {
        float v[4] = {0.f, 0.f, 0.f, 0.f};
        float am = 0.f;
#pragma unroll
        for (int r = 0; r < kRouteCtas; ++r) {
            const uint32_t at = cluster_map(&part[tok][0], (uint32_t)r);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (lane + 32 * i < a.N) v[i] += dsm_f32(at + 4u * (lane + 32 * i));
            if (a.xscale) am = __uint_as_float(max(__float_as_uint(am),
                                  __float_as_uint(dsm_f32(cluster_map(&amax_sm[tok], r)))));
        }
        const size_t m = (size_t)(t0 + tok);
        if (a.xscale && lane == 0) a.xscale[m] = split_scale(am);
        route_token(v, a.N, a.K, false, a.renorm, lane, a.ids + m * a.K, a.gates + m * a.K,
                    a.ids_out ? a.ids_out + m * a.K : nullptr,
                    a.gates_out ? a.gates_out + m * a.K : nullptr);
    }
    cluster_sync();                  // no CTA leaves while its partial logits are read
}

// The same from given probabilities: a warp a token.
__global__ void __launch_bounds__(kRouteThreads)
    moe_topk_kernel(MoeRouteArgs a) {
    zero_ctrl(a);
    pdl_launch_dependents();
    const int lane = threadIdx.x & 31;
    const long long m = (long long)blockIdx.x * (kRouteThreads / 32) + (threadIdx.x >> 5);
    if (m >= a.M) return;
    float v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        v[i] = lane + 32 * i < a.N ? a.scores[m * a.lds + lane + 32 * i] : 0.f;
    if (a.xscale) {
        const uint16_t* x = a.x + m * a.ldx;
        uint32_t am = 0;
        for (int i = 8 * lane; i < a.d; i += 256) {
            const uint4 u = *reinterpret_cast<const uint4*>(x + i);
            const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) am = max(am, max(w[j] << 16 & 0x7fffffffu, w[j] & 0x7fff0000u));
        }
        am = __reduce_max_sync(kFull, am);
        if (lane == 0) a.xscale[m] = split_scale(__uint_as_float(am));
    }
    route_token(v, a.N, a.K, true, a.renorm, lane, a.ids + m * a.K, a.gates + m * a.K,
                a.ids_out ? a.ids_out + m * a.K : nullptr,
                a.gates_out ? a.gates_out + m * a.K : nullptr);
}

}  // namespace crc
