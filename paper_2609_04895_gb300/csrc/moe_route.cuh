// The mixture-of-experts layer's routing: router logits, Top-K and gates of
// every token, and the control block of the experts' kernel set to zero.
//
//   z = W^R x,  S = TopK(z) (score descending, index ascending),
//   g_e = exp(z_e - max z) / sum exp(z - max z), divided by its sum over S on request
//
// A cluster of eight CTAs takes 16 tokens: each CTA multiplies one eighth of d
// for all experts and puts its partial logits into the shared memory of the CTA
// that owns the token (rank = token mod 8), where a warp sums them in rank order.
// Splitting d reads every element of x and W^R once per cluster (N = 128, d = 2048: 64 KB
// of W^R a CTA, against 512 KB on one), and the sum of eight short chains is nearer to
// the exact logit than one long one.  mma.sync and not tcgen05: 16 tokens are an eighth
// of its smallest full tile, and what bounds this kernel is latency: 64 tokens, N = 128,
// d = 2048 take 5 us, 2 of them the trip to memory, 1 the Top-K's rounds of two
// reductions each.
#pragma once

#include "crc_device.cuh"
#include "pdl.cuh"

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
    float* logits;                   // [M][N], moe_logits_kernel only
    uint8_t* ids;                    // [M][K]
    float* gates;                    // [M][K]
    uint8_t* ids_out;                // the caller's, or null
    float* gates_out;
    float* xscale;                   // [M] power-of-two scale of x's row, or null
    uint32_t* ctrl;                  // zeroed
    int ctrl_words;
};

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
    uint32_t mine = 0u, top = 0u;     // lane k: the k-th choice
    int my_id = 0;
    for (int k = 0; k < K; ++k) {
        const uint32_t best = __reduce_max_sync(
            kFull, max(max(key[0], key[1]), max(key[2], key[3])));
        uint32_t at = 0xffu;
#pragma unroll
        for (int i = 3; i >= 0; --i)
            if (key[i] == best) at = (uint32_t)(lane + 32 * i);
        const uint32_t e = __reduce_min_sync(kFull, at);    // ties to the lowest index
        if (k == 0) top = best;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if ((uint32_t)(lane + 32 * i) == e) key[i] = 0u;
        if (lane == k) {
            mine = best;
            my_id = (int)e;
        }
    }
    float p = lane < K ? score_of(mine) : 0.f;
    if (!probs) {
        const float mx = score_of(top);
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (lane + 32 * i < N) s += expf(v[i] - mx);
        s = warp_sum(s);
        p = lane < K ? expf(p - mx) / s : 0.f;
    }
    if (renorm) p /= warp_sum(p);
    if (lane < K) {
        ids[lane] = (uint8_t)my_id;
        gates[lane] = p;
        if (ids_out) ids_out[lane] = (uint8_t)my_id;
        if (gates_out) gates_out[lane] = p;
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

// Largest magnitude of eight bf16, as the bits of a float: a NaN counts as the largest.
__device__ __forceinline__ uint32_t max_abs(const uint4& v) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) m = max(m, max(w[i] << 16 & 0x7fffffffu, w[i] & 0x7fff0000u));
    return m;
}

__device__ __forceinline__ void dsm_store2(uint32_t addr, float x, float y) {
    asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(addr), "f"(x), "f"(y)
                 : "memory");
}
__device__ __forceinline__ void dsm_store(uint32_t addr, uint32_t v) {
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}

__device__ __forceinline__ void zero_ctrl(const MoeRouteArgs& a) {
    if (blockIdx.x == 0 && blockIdx.y == 0)
        for (int i = threadIdx.x; i < a.ctrl_words; i += blockDim.x) a.ctrl[i] = 0u;
}

// A warp multiplies two tiles of 8 experts; with fewer than 128 experts the
// warps that are left split d further.
__global__ void __launch_bounds__(kRouteThreads)
    moe_route_kernel(MoeRouteArgs a) {
    constexpr int WARPS = kRouteThreads / 32, BATCH = 8;
    // partial logits of this CTA's two tokens: [token / 8][rank][warp][16 experts]
    __shared__ float part[2][kRouteCtas][WARPS * 16];
    __shared__ uint32_t amax[2][kRouteCtas][WARPS];
    asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");
    pdl_begin();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = (int)cluster_ctarank();
    const int t0 = (int)(blockIdx.x / kRouteCtas) * kRouteTokens;
    const int g = lane >> 2, t = lane & 3;
    const int pairs = a.N / 16, split = WARPS / pairs;     // tile pairs; warps a pair
    const int pair = warp / split;
    float acc0[4] = {}, acc1[4] = {};
    uint32_t am0 = 0, am1 = 0;
    if (pair < pairs) {
        // this warp's chunks of 32 elements of d
        const int nch = (a.d + 31) / 32, slices = kRouteCtas * split;
        const int slice = rank * split + warp % split;
        const int c0 = nch * slice / slices, c1 = nch * (slice + 1) / slices;
        const bool r0 = t0 + g < a.M, r1 = t0 + g + 8 < a.M;
        const uint16_t* x0 = a.x + (long long)(r0 ? t0 + g : 0) * a.ldx + 8 * t;
        const uint16_t* x1 = a.x + (long long)(r1 ? t0 + g + 8 : 0) * a.ldx + 8 * t;
        const uint16_t* w0 = a.w + (size_t)(pair * 16 + g) * a.d + 8 * t;
        const uint16_t* w1 = w0 + (size_t)8 * a.d;
        const uint4 zero = make_uint4(0, 0, 0, 0);
        // Every load of a batch is asked for before the first is used: one token is
        // bound by the latency of memory.
        for (int c = c0; c < c1; c += BATCH) {
            uint4 xa[BATCH], xb[BATCH], wa[BATCH], wb[BATCH];
#pragma unroll
            for (int i = 0; i < BATCH; ++i) {
                const int k = 32 * (c + i);
                const bool in = c + i < c1 && k + 8 * t < a.d;
                wa[i] = in ? *reinterpret_cast<const uint4*>(w0 + k) : zero;
                wb[i] = in ? *reinterpret_cast<const uint4*>(w1 + k) : zero;
                xa[i] = in && r0 ? *reinterpret_cast<const uint4*>(x0 + k) : zero;
                xb[i] = in && r1 ? *reinterpret_cast<const uint4*>(x1 + k) : zero;
            }
            // The order of k inside a product is free as long as both operands share
            // it: a thread's 16 contiguous bytes of a row serve two k16 steps.
#pragma unroll
            for (int i = 0; i < BATCH; ++i) {
                if (c + i >= c1) break;
                mma_bf16_16x8x16(acc0, xa[i].x, xb[i].x, xa[i].y, xb[i].y, wa[i].x, wa[i].y);
                mma_bf16_16x8x16(acc1, xa[i].x, xb[i].x, xa[i].y, xb[i].y, wb[i].x, wb[i].y);
                mma_bf16_16x8x16(acc0, xa[i].z, xb[i].z, xa[i].w, xb[i].w, wa[i].z, wa[i].w);
                mma_bf16_16x8x16(acc1, xa[i].z, xb[i].z, xa[i].w, xb[i].w, wb[i].z, wb[i].w);
                if (a.xscale) {
                    am0 = max(am0, max_abs(xa[i]));
                    am1 = max(am1, max_abs(xb[i]));
                }
            }
        }
    }
    if (a.xscale) {
#pragma unroll
        for (int o = 1; o < 4; o <<= 1) {
            am0 = max(am0, __shfl_xor_sync(kFull, am0, o));
            am1 = max(am1, __shfl_xor_sync(kFull, am1, o));
        }
    }
    zero_ctrl(a);
    asm volatile("barrier.cluster.wait;" ::: "memory");     // every CTA has begun
    {
        // rows g and g + 8 are tokens of CTA g
        const uint32_t at = cluster_map(&part[0][rank][warp * 16 + 2 * t], (uint32_t)g);
        const uint32_t next = (uint32_t)sizeof part[0];
        if (t0 + g < a.M) {
            dsm_store2(at, acc0[0], acc0[1]);
            dsm_store2(at + 32, acc1[0], acc1[1]);
            if (a.xscale && t == 0) dsm_store(cluster_map(&amax[0][rank][warp], (uint32_t)g), am0);
        }
        if (t0 + g + 8 < a.M) {
            dsm_store2(at + next, acc0[2], acc0[3]);
            dsm_store2(at + next + 32, acc1[2], acc1[3]);
            if (a.xscale && t == 0) dsm_store(cluster_map(&amax[1][rank][warp], (uint32_t)g), am1);
        }
    }
    cluster_sync();                  // nothing is written to this CTA after it
    const int tok = rank + 8 * warp;
    if (warp >= 2 || t0 + tok >= a.M) return;
    float v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[i] = 0.f;
        const int e = lane + 32 * i;
        if (e >= a.N) continue;
        for (int w = 0; w < split; ++w)
#pragma unroll
            for (int r = 0; r < kRouteCtas; ++r)
                v[i] += part[warp][r][((e >> 4) * split + w) * 16 + (e & 15)];
    }
    const size_t m = (size_t)(t0 + tok);
    if (a.xscale) {                  // the warps without a tile pair have left zeros
        const uint32_t* am = &amax[warp][0][0];
        const uint32_t top = __reduce_max_sync(kFull, max(am[lane], am[lane + 32]));
        if (lane == 0) a.xscale[m] = split_scale(__uint_as_float(top));
    }
    route_token(v, a.N, a.K, false, a.renorm, lane, a.ids + m * a.K, a.gates + m * a.K,
                a.ids_out ? a.ids_out + m * a.K : nullptr,
                a.gates_out ? a.gates_out + m * a.K : nullptr);
}

// Few choices: the logits alone, a warp an (expert, token); every CTA of the experts' kernel
// then takes the Top-K itself (one token, N = 128, d = 2048: 4.9 us from this kernel's
// start to the tables, against 6.9 with the Top-K in the cluster above).
__global__ void __launch_bounds__(kRouteThreads)
    moe_logits_kernel(MoeRouteArgs a) {
    constexpr int BATCH = 16;         // rows of 4096 elements at once
    pdl_begin();
    zero_ctrl(a);
    const int lane = threadIdx.x & 31;
    const int e = (int)blockIdx.x * (kRouteThreads / 32) + (threadIdx.x >> 5);
    if (e >= a.N) return;
    const uint16_t* w = a.w + (size_t)e * a.d;
    const int m = (int)blockIdx.y;
    const uint16_t* x = a.x + m * a.ldx;
    float acc0 = 0.f, acc1 = 0.f;
    uint32_t am = 0;
    for (int k0 = 8 * lane; k0 < a.d; k0 += 256 * BATCH) {
        uint4 wv[BATCH], xv[BATCH];
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const int k = k0 + 256 * i;
            const uint4 zero = make_uint4(0, 0, 0, 0);
            wv[i] = k < a.d ? *reinterpret_cast<const uint4*>(w + k) : zero;
            xv[i] = k < a.d ? *reinterpret_cast<const uint4*>(x + k) : zero;
        }
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const uint32_t wu[4] = {wv[i].x, wv[i].y, wv[i].z, wv[i].w};
            const uint32_t xu[4] = {xv[i].x, xv[i].y, xv[i].z, xv[i].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                acc0 = fmaf(__uint_as_float(wu[j] << 16), __uint_as_float(xu[j] << 16), acc0);
                acc1 = fmaf(__uint_as_float(wu[j] & 0xffff0000u),
                            __uint_as_float(xu[j] & 0xffff0000u), acc1);
            }
            if (a.xscale && e == 0) am = max(am, max_abs(xv[i]));
        }
    }
    const float z = warp_sum(acc0 + acc1);
    if (lane == 0) a.logits[m * a.N + e] = z;
    if (a.xscale && e == 0) {
        am = __reduce_max_sync(kFull, am);
        if (lane == 0) a.xscale[m] = split_scale(__uint_as_float(am));
    }
}

// The same from given probabilities: a warp a token.
__global__ void __launch_bounds__(kRouteThreads)
    moe_topk_kernel(MoeRouteArgs a) {
    pdl_begin();
    zero_ctrl(a);
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
        for (int i = 8 * lane; i < a.d; i += 256)
            am = max(am, max_abs(*reinterpret_cast<const uint4*>(x + i)));
        am = __reduce_max_sync(kFull, am);
        if (lane == 0) a.xscale[m] = split_scale(__uint_as_float(am));
    }
    route_token(v, a.N, a.K, true, a.renorm, lane, a.ids + m * a.K, a.gates + m * a.K,
                a.ids_out ? a.ids_out + m * a.K : nullptr,
                a.gates_out ? a.gates_out + m * a.K : nullptr);
}

}  // namespace crc
