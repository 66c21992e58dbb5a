// Products of a few rows with matrices in 4 bits: y = W_e x for every choice of an expert
// e, W = scale * code with one bf16 scale for G columns of a row (rows4.cu writes both).
//
// Mathematics.  For a group q of columns, part = sum over it of code * x is formed first,
// exactly as products (4 by 8 significant bits) and in fp32 as a sum, and y += scale_q part
// in fp32, so no weight is rounded.  A code becomes a bf16 number by two bit operations (its
// four bits with the top one turned over, put below the exponent of 128, are 136 + code) and
// the subtraction of 136, which is exact.
//
// What it should be bound by is bytes, half of one a weight and 2 / G for the scale.  At 6.8 TB/s
// an SM has to turn over some 47 weights a clock, more than scalar fp32 instructions could (about 3
// a weight), so the fragments of mma.sync m16n8k16 are filled from the packed words in registers:
// the eight columns of the product are eight choices of the same expert.  (tcgen05 was not tried.
// Widened codes could go to its A operand in shared memory or TMEM, a group's sums to columns of
// their own.  But a step of 16 columns of a pair's 256 rows takes some 105 clocks in
// group_matmul.cuh whatever its N up to 200, operands in shared memory: 20 weights a clock and SM,
// no more than here.  How long one with A in TMEM takes has not been measured.)  It reaches 20 to
// 25 weights a clock: 64 tokens' second product (128 experts, 105 MB) takes 39 us, 35 of them with
// the loads left out and 22 with the products left out: what bounds it are two bit operations, a
// shift and a subtraction for two weights, and the legacy tensor path.  One token's (14 MB) takes
// 10 us: 5 are the launch and the choices' order, and eight experts are too few boxes a warp to
// fill the rest.
//
// A persistent grid: each CTA brings the choices into their experts' order once, and its warps take
// tiles of 32 rows (with gate and up: 16 rows of each) of the active experts in turn.  A warp's
// codes and scales come by TMA into a ring of its own, 256 columns a time, across the ends of its
// tiles; with too few tiles for the warps, 2, 4 or 8 warps share a tile's columns and their sums
// are added in a fixed order (another one for another number of warps: of 2048 columns one bf16
// result in 6000 rounds the other way).  Half a box's words, scales and x are loaded before they
// are used (41 us against 49).  Two CTAs an SM leave 128 registers a thread: with 20 warps of 96 it
// took 45 us.
#include <cudaTypedefs.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "crc_device.cuh"
#include "crc_internal.h"
#include "pdl.cuh"

namespace crc {

PFN_cuTensorMapEncodeTiled_v12000 encode_fn();      // router.cu

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kCtas = 2;                             // CTAs of an SM
constexpr int kBoxCols = 256;                        // columns of a stage: 128 bytes a row
constexpr int kCodeBytes = 32 * 128;                 // a stage's codes: two tiles of 16 rows
constexpr int kScaleBytes = 2 * 256;                 // and scales, at most 8 groups x 32 rows
constexpr int kStageBytes = kCodeBytes + kScaleBytes;
constexpr int kStages = 2;
constexpr int kMaxChoices = 8192;
constexpr int kMaxTokens = 1024;
constexpr int kMaxExperts = 256;
constexpr int kBins = kMaxExperts + 1;               // the last: choices without a slot
constexpr int kSums = kWarps * 8 * 33;               // floats: what the warps of a tile found

inline bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

struct Matvec4Args {
    const uint16_t* x;
    const uint8_t* topk;         // [E], NULL: every choice takes expert 0
    const int32_t* slot;         // [N] or NULL
    uint16_t* y;                 // [E][out]
    uint32_t* err;
    long long ldx;
    int x_div;                   // the row of x of choice c is c / x_div
    int E, N, slots;
    int n, k;                    // rows (of y too) and columns of a matrix
    int glu;
    int splits;                  // warps that share a tile's columns: 1, 2, 4, 8
    int tiles;                   // tiles of 32 (glu: 16) rows of an expert
};

__device__ __forceinline__ void mma_bf16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0,
                                         uint32_t b1, const float (&c)[4]) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
        "{%8,%9}, {%10,%11,%12,%13};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(c[0]), "f"(c[1]),
          "f"(c[2]), "f"(c[3]));
}

// Codes i and i + 4 of a word (i by the shift before) as bf16.  (Taken as steps of 2^-133 in the
// low bits of a bf16 and scaled up by an fma, two codes need no shift, but that took 5 to 9%
// longer.)
__device__ __forceinline__ uint32_t widen2(uint32_t w) {
    uint32_t r;
    asm("lop3.b32 %0, %1, 0x000f000f, 0x43084308, 0x6a;" : "=r"(r) : "r"(w));
    const __nv_bfloat162 v = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&r),
                                     __floats2bfloat162_rn(136.f, 136.f));
    return *reinterpret_cast<const uint32_t*>(&v);
}

__device__ __forceinline__ float lds_bf16(uint32_t addr) {
    uint16_t v;
    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(addr));
    return __uint_as_float((uint32_t)v << 16);
}
__device__ __forceinline__ uint32_t lds32(uint32_t addr) {
    uint32_t v;
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(addr));
    return v;
}

// One lane of a converged warp.
__device__ __forceinline__ uint32_t elected() {
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(r));
    return r;
}
// Issued by the lane whose `lead` is set, in code that the whole warp runs.
__device__ __forceinline__ void tma_load_4d_by(uint32_t lead, void* dst, const CUtensorMap* map,
                                               uint64_t* bar, int c0, int c1, int c2, int c3,
                                               uint64_t policy) {
    asm volatile(
        "{\n\t.reg .pred e;\n\tsetp.ne.b32 e, %8, 0;\n\t"
        "@e cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
        ".L2::cache_hint [%0], [%1, {%2, %3, %4, %5}], [%6], %7;\n\t}" ::"r"(smem_u32(dst)),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(c2), "r"(c3),
        "r"(smem_u32(bar)), "l"(policy), "r"(lead)
        : "memory");
}

// The choices in their experts' order: shared memory.
struct Order {
    int first[kBins + 1];        // of an expert's choices in the list
    int next[kBins];
    int slot[kMaxExperts];
    uint16_t active[kMaxExperts];   // experts with choices and a slot
    int actives;
};

// A tile of an expert's rows for up to NT * 8 of its choices: one pass over the weights.
struct Pass {
    int item;                    // of the warp's turns; its expert's tile has a pass or more
    int slot, tile, at, end;     // the matrix, its rows' tile, the choices in the list
};

// The x of a half box (128 columns) for NT * 8 choices, as the fragments want it: lane (g, t)
// has columns 8 t .. of each 32 of choice g.  Zeros behind the last column.
template <int NT>
struct Half {
    uint4 v[NT][4];
    __device__ __forceinline__ void load(const Matvec4Args& a, const uint16_t* const (&xrow)[NT],
                                         int col0) {
        if (col0 + 128 <= a.k) {
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    v[j][c] = __ldg(reinterpret_cast<const uint4*>(xrow[j] + col0 + c * 32));
        } else {
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    v[j][c] = make_uint4(0, 0, 0, 0);
                    if (col0 + c * 32 < a.k)
                        v[j][c] = __ldg(reinterpret_cast<const uint4*>(xrow[j] + col0 + c * 32));
                }
        }
    }
};

// 128 columns of a warp's two row tiles for NT * 8 choices; acc[tile][nt][4] in the
// fragments' order.  (Columns behind the last are zeros in x, codes and scales.)
template <int G, int NT>
__device__ __forceinline__ void half_products(uint32_t codes, uint32_t scales, int tile_scales,
                                              int group_scales, int half, const Half<NT>& x,
                                              float (&acc)[2][NT][4]) {
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const float none[4] = {0.f, 0.f, 0.f, 0.f};
    constexpr int kPer = G / 32, kGroups = 4 / kPer;   // steps of a group, groups of a half
    // tile rows g and g + 8: 128-byte rows, 16-byte pieces at piece ^ (row % 8)
    const uint32_t cw = codes + g * 128 + t * 4;
    const uint32_t cs = scales + g * 2 + half * kGroups * group_scales;
    uint32_t w[4][2][2];
    float sc[kGroups][2][2];
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int tile = 0; tile < 2; ++tile) {
            const uint32_t at = cw + tile * 2048 + (((half * 4 + c) ^ g) << 4);
            w[c][tile][0] = lds32(at);
            w[c][tile][1] = lds32(at + 1024);
        }
#pragma unroll
    for (int q = 0; q < kGroups; ++q)
#pragma unroll
        for (int tile = 0; tile < 2; ++tile) {
            const uint32_t at = cs + tile * tile_scales + q * group_scales;
            sc[q][tile][0] = lds_bf16(at);
            sc[q][tile][1] = lds_bf16(at + 16);
        }
    float part[2][NT][4];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        uint32_t b[NT][4];
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            // columns i and i + 4 of the eight, as the codes of a word lie
            const uint4 v = x.v[j][c];
            b[j][0] = __byte_perm(v.x, v.z, 0x5410);
            b[j][1] = __byte_perm(v.x, v.z, 0x7632);
            b[j][2] = __byte_perm(v.y, v.w, 0x5410);
            b[j][3] = __byte_perm(v.y, v.w, 0x7632);
        }
#pragma unroll
        for (int tile = 0; tile < 2; ++tile) {
            const uint32_t w0 = w[c][tile][0], w1 = w[c][tile][1];
            const uint32_t lo[4] = {widen2(w0), widen2(w1), widen2(w0 >> 4), widen2(w1 >> 4)};
            const uint32_t hi[4] = {widen2(w0 >> 8), widen2(w1 >> 8), widen2(w0 >> 12),
                                    widen2(w1 >> 12)};
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                if (c % kPer == 0)
                    mma_bf16(part[tile][j], lo, b[j][0], b[j][1], none);
                else
                    mma_bf16(part[tile][j], lo, b[j][0], b[j][1], part[tile][j]);
                mma_bf16(part[tile][j], hi, b[j][2], b[j][3], part[tile][j]);
                if (c % kPer == kPer - 1)
#pragma unroll
                    for (int v = 0; v < 4; ++v)
                        acc[tile][j][v] = fmaf(sc[c / kPer][tile][v / 2], part[tile][j][v],
                                               acc[tile][j][v]);
            }
        }
    }
}

__device__ __forceinline__ float silu_up(float gate, float up) {
    return __fdividef(gate, 1.f + __expf(-gate)) * up;
}

struct Ring {
    uint8_t* codes;
    uint8_t* scales;
    uint64_t* full;
    uint32_t turn;               // boxes consumed
};

// One pass: the products of this warp's boxes, then y.  x is the first half box's, and the next
// pass's when it returns (`advance` goes there, false at the end).  `refill` issues the next box
// of the warp's stream into a stage that was read.  `ok` turns false when a wait runs out: the
// warp then only keeps the barriers of the warps that share its tiles.
template <int G, int NT, class F, class N>
__device__ __forceinline__ bool pass_products(const Matvec4Args& a, Ring& ring, Pass& pass,
                                              const uint16_t* (&xrow)[NT], Half<NT>& x,
                                              const uint32_t* list, float* sums, int& buf,
                                              bool& ok, F refill, N advance) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int split = warp % a.splits;
    const int boxes = (a.k + kBoxCols - 1) / kBoxCols;
    const Pass it = pass;
    const int count = min(NT * 8, it.end - it.at);
    list += it.at;
    float acc[2][NT][4] = {};
    // a stage's scales: [groups][32], with gate and up [2][groups][16]
    const int tile_scales = a.glu ? kBoxCols / G * 32 : 32, group_scales = a.glu ? 32 : 64;
    for (int box = split; box < boxes; box += a.splits) {
        const int s = ring.turn % kStages, col0 = box * kBoxCols;
        if (ok) ok = mbar_wait_warp(&ring.full[s], (ring.turn / kStages) & 1);
        if (!ok) latch_error(a.err, CRC_ETIMEOUT);
        const uint32_t codes = smem_u32(ring.codes + s * kCodeBytes);
        const uint32_t scales = smem_u32(ring.scales + s * kScaleBytes);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            Half<NT> ahead;
            ahead.load(a, xrow, half ? (box + a.splits) * kBoxCols : col0 + 128);
            half_products<G, NT>(codes, scales, tile_scales, group_scales, half, x, acc);
            x = ahead;
        }
        if (ok) {
            ++ring.turn;
            __syncwarp();                              // every lane has read the stage
            refill(s);
        }
    }
    // (between the halves of the last box it came 5% dearer: 44 us, not 41, for 64 tokens)
    const bool more = advance();
    if (more) x.load(a, xrow, split * kBoxCols);
    const int each = a.glu ? 16 : 32, row0 = it.tile * each;
    if (a.splits == 1) {
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const int i = j * 8 + 2 * t + (v & 1), r = row0 + g + (v >> 1) * 8;
                if (i >= count || !ok) continue;
                uint16_t* y = a.y + (long long)(list[i] & 0xffffu) * a.n;
                if (a.glu) {
                    if (r < a.n)
                        y[r] = __bfloat16_as_ushort(
                            __float2bfloat16_rn(silu_up(acc[0][j][v], acc[1][j][v])));
                } else {
                    if (r < a.n) y[r] = __bfloat16_as_ushort(__float2bfloat16_rn(acc[0][j][v]));
                    if (r + 16 < a.n)
                        y[r + 16] = __bfloat16_as_ushort(__float2bfloat16_rn(acc[1][j][v]));
                }
            }
        return more;
    }
    if constexpr (NT == 1) {
        // sums[buf][warp][choice][32 rows]; a buffer is written again behind the next barrier
        float* mine = sums + buf * kSums;
        buf ^= 1;
#pragma unroll
        for (int tile = 0; tile < 2; ++tile)
#pragma unroll
            for (int v = 0; v < 4; ++v)
                mine[(warp * 8 + 2 * t + (v & 1)) * 33 + tile * 16 + g + (v >> 1) * 8] =
                    acc[tile][0][v];
        const int w0 = warp - split;
        named_sync(1 + w0 / a.splits, a.splits * 32);
        for (int o = split * 32 + lane; o < each * count; o += a.splits * 32) {
            const int i = o / each, r = o % each;
            if (row0 + r >= a.n) continue;
            float v = 0.f, u = 0.f;
            for (int w = w0; w < w0 + a.splits; ++w) {
                v += mine[(w * 8 + i) * 33 + r];
                if (a.glu) u += mine[(w * 8 + i) * 33 + r + 16];
            }
            if (a.glu) v = silu_up(v, u);
            a.y[(long long)(list[i] & 0xffffu) * a.n + row0 + r] =
                __bfloat16_as_ushort(__float2bfloat16_rn(v));
        }
    }
    return more;
}

// NT: choices of a pass over the weights, in eights.
template <int G, int NT>
__global__ void __launch_bounds__(kThreads, kCtas)
    matvec4_kernel(const __grid_constant__ CUtensorMap mw, const __grid_constant__ CUtensorMap ms,
                   Matvec4Args a) {
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    __shared__ uint64_t full[kWarps][kStages];
    __shared__ Order order;
    uint8_t* smem = reinterpret_cast<uint8_t*>(
        (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    Ring ring;
    ring.codes = smem + warp * kStages * kCodeBytes;
    ring.scales = smem + kWarps * kStages * kCodeBytes + warp * kStages * kScaleBytes;
    ring.full = full[warp];
    ring.turn = 0;
    float* sums = reinterpret_cast<float*>(smem + kWarps * kStages * kStageBytes);
    uint32_t* list = reinterpret_cast<uint32_t*>(sums + (a.splits > 1 ? 2 * kSums : 0));
    for (int e = threadIdx.x; e <= a.N; e += kThreads) order.next[e] = 0;
    if (threadIdx.x == 0) {
        // (one thread: the fence, without which TMA need not see a barrier, is for those that the
        // thread itself has set up)
        for (int i = 0; i < kWarps * kStages; ++i) mbar_init(&full[0][0] + i, 1);
        fence_mbar_init();
        tma_prefetch_desc(&mw);
        tma_prefetch_desc(&ms);
    }
    pdl_begin();
    // (this thread's first choice and slot are asked for together)
    const int id0 = a.topk && (int)threadIdx.x < a.E ? a.topk[threadIdx.x] : 0;
    for (int e = threadIdx.x; e < a.N; e += kThreads) {
        const int slot = a.slot ? a.slot[e] : e;
        order.slot[e] = slot >= 0 && slot < a.slots ? slot : -1;
    }
    __syncthreads();
    const auto bin_of = [&](int c) {
        const int id = c == (int)threadIdx.x ? id0 : a.topk ? a.topk[c] : 0;
        return id < a.N && order.slot[id] >= 0 ? id : a.N;
    };
    for (int c = threadIdx.x; c < a.E; c += kThreads) atomicAdd(&order.next[bin_of(c)], 1);
    __syncthreads();
    if (warp == 0) {
        constexpr int kEach = (kBins + 31) / 32;
        int n = 0, active = 0;                         // this lane's bins
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int e = lane * kEach + i;
            if (e > a.N) continue;
            n += order.next[e];
            active += e < a.N && order.next[e] > 0;
        }
        int n0 = n, a0 = active;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int un = __shfl_up_sync(kFull, n0, o), ua = __shfl_up_sync(kFull, a0, o);
            if (lane >= o) {
                n0 += un;
                a0 += ua;
            }
        }
        if (lane == 31) order.actives = a0;
        n0 -= n;
        a0 -= active;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int e = lane * kEach + i;
            if (e > a.N) continue;
            const int count = order.next[e];
            order.first[e] = n0;
            order.next[e] = n0;
            n0 += count;
            if (e == a.N)
                order.first[e + 1] = n0;
            else if (count)
                order.active[a0++] = (uint16_t)e;
        }
    }
    __syncthreads();
    // (the row of x, the choice), in any order, another one in each CTA: a choice's result does
    // not depend on its column of the fragments, nor on its pass, and one warp makes all passes
    // of a tile
    for (int c = threadIdx.x; c < a.E; c += kThreads)
        list[atomicAdd(&order.next[bin_of(c)], 1)] = (uint32_t)(c / a.x_div) << 16 | (uint32_t)c;
    __syncthreads();

    // the choices without a slot: zeros.  (By their numbers: the list's order is this CTA's.)
    if (order.first[a.N + 1] > order.first[a.N])
        for (int c = blockIdx.x; c < a.E; c += gridDim.x)
            if (bin_of(c) == a.N)
                for (int o = threadIdx.x; o < a.n / 8; o += kThreads)
                    *(reinterpret_cast<uint4*>(a.y + (long long)c * a.n) + o) =
                        make_uint4(0, 0, 0, 0);

    const int items = order.actives * a.tiles;
    const int groups = kWarps / a.splits;              // groups of warps of a CTA
    // (the warps of the last, partial turn lie in all CTAs)
    const int first = warp / a.splits * gridDim.x + blockIdx.x, step = gridDim.x * groups;
    const int boxes = (a.k + kBoxCols - 1) / kBoxCols, split = warp % a.splits;
    const int each = a.glu ? 16 : 32;
    // To the warp's next pass, from item `first - step` with nothing left on the way.
    const auto advance = [&](Pass& p) {
        p.at += NT * 8;
        if (p.at < p.end) return true;
        if (p.item + step >= items) return false;
        p.item += step;
        const int e = order.active[p.item / a.tiles];
        p.tile = p.item % a.tiles;
        p.slot = order.slot[e];
        p.at = order.first[e];
        p.end = order.first[e + 1];
        return true;
    };
    // the warp's stream of boxes, issued kStages before they are taken
    const uint32_t lead = elected();
    const uint64_t pol = l2_evict_first_policy();
    Pass ahead = {};
    ahead.item = first - step;
    int nbox = boxes;
    uint32_t issued = 0;
    const auto refill = [&](int s) {
        if (nbox >= boxes) {
            if (!advance(ahead)) return;
            nbox = split;
        }
        if (lead)
            mbar_arrive_expect_tx(&ring.full[s], kCodeBytes + 2 * 32 * (kBoxCols / G));
        tma_load_4d_by(lead, ring.codes + s * kCodeBytes, &mw, &ring.full[s], nbox * 128,
                       ahead.tile * each, 0, ahead.slot, pol);
        tma_load_4d_by(lead, ring.scales + s * kScaleBytes, &ms, &ring.full[s], ahead.tile * each,
                       nbox * (kBoxCols / G), 0, ahead.slot, pol);
        nbox += a.splits;
        ++issued;
    };
#pragma unroll
    for (int s = 0; s < kStages; ++s) refill(s);
    int buf = 0;
    bool ok = true;
    Pass pass = {};
    pass.item = first - step;
    const uint16_t* xrow[NT];
    const auto next_pass = [&] {
        if (!advance(pass)) return false;
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            // (columns of the fragments without a choice: the first one's x, not stored)
            const int i = pass.at + j * 8 + (lane >> 2);
            xrow[j] = a.x + (long long)(list[i < pass.end ? i : pass.at] >> 16) * a.ldx +
                      (lane & 3) * 8;
        }
        return true;
    };
    bool more = next_pass();
    Half<NT> x;
    if (more) x.load(a, xrow, split * kBoxCols);       // on its way while the codes are
    while (more)
        more = pass_products<G, NT>(a, ring, pass, xrow, x, list, sums, buf, ok, refill,
                                    next_pass);
    // never leave with copies in flight
    if (!ok)
        for (uint32_t n = ring.turn; n < issued; ++n)
            mbar_wait_warp(&ring.full[n % kStages], (n / kStages) & 1);
}

size_t smem_bytes(int splits, int E) {
    return 1024 + (size_t)kWarps * kStages * kStageBytes + (splits > 1 ? 2 * kSums * 4 : 0) +
           (size_t)E * 4 + 16;
}

template <int G, int NT>
int launch(const CUtensorMap& mw, const CUtensorMap& ms, const Matvec4Args& a, dim3 grid,
           cudaStream_t st) {
    auto kern = matvec4_kernel<G, NT>;
    const size_t most = smem_bytes(8, kMaxChoices);
    static PerDevice ready;
    const int up = ready.get(current_device(), [&] {
        return cuda_status(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                (int)most)) == CRC_OK;
    });
    if (!up) return CRC_ECUDA;
    cudaError_t e;
    {
        ProfScope prof(CRC_KERNEL_MATVEC4, st);
        e = launch_dependent(kern, grid, kThreads, smem_bytes(a.splits, a.E), st, 1, mw, ms,
                             a);
    }
    note_launch();
    return cuda_status(e);
}

int check_matvec4(const crc_matvec4_weights* w) {
    if (!w || w->reserved != 0) return CRC_EINVAL;
    if (w->N < 1 || w->n < 1 || w->k < 1 || w->slots < 1) return CRC_EINVAL;
    if (w->glu != 0 && w->glu != 1) return CRC_EINVAL;
    if (w->group != 32 && w->group != 64 && w->group != 128) return CRC_EUNSUPPORTED;
    if (w->N > kMaxExperts || w->n % 8 != 0 || w->k % w->group != 0 || w->n > 65536 ||
        w->k > 32768)
        return CRC_EUNSUPPORTED;
    if (!w->codes_dev || !w->scale_dev || !aligned(w->codes_dev, 16) ||
        !aligned(w->scale_dev, 16) || !aligned(w->expert_slot_dev, 4))
        return CRC_EINVAL;
    const int64_t half = (int64_t)w->n * (w->k / 2), sc = (int64_t)w->n * (w->k / w->group) * 2;
    const int64_t parts = w->glu ? 2 : 1;
    if (w->codes_stride % 16 || w->scale_stride % 16 || w->codes_stride < parts * half ||
        w->scale_stride < parts * sc)
        return CRC_EINVAL;
    if (w->codes_stride >= (1ll << 40) || w->scale_stride >= (1ll << 40)) return CRC_EUNSUPPORTED;
    if (!w->expert_slot_dev && w->N > w->slots) return CRC_EINVAL;
    return CRC_OK;
}

// Codes as (k / 2, n, gate / up, slots), a box of 128 bytes x 32 rows, with gate and up 16 of
// each; scales as (n, k / G, gate / up, slots), the same rows x the groups of 256 columns.
bool make_maps(CUtensorMap* mw, CUtensorMap* ms, const crc_matvec4_weights& w) {
    auto enc = encode_fn();
    if (!enc) return false;
    const cuuint64_t k2 = w.k / 2, n = w.n, groups = w.k / w.group, slots = w.slots;
    const cuuint64_t parts = w.glu ? 2 : 1;
    const cuuint32_t ones[4] = {1, 1, 1, 1};
    const cuuint64_t dw[4] = {k2, n, parts, slots};
    const cuuint64_t sw[3] = {k2, n * k2, (cuuint64_t)w.codes_stride};
    const cuuint32_t rows = w.glu ? 16 : 32, halves = w.glu ? 2 : 1;
    const cuuint32_t bw[4] = {128, rows, halves, 1};
    const cuuint64_t ds[4] = {n, groups, parts, slots};
    const cuuint64_t ss[3] = {n * 2, n * groups * 2, (cuuint64_t)w.scale_stride};
    const cuuint32_t bs[4] = {rows, (cuuint32_t)(kBoxCols / w.group), halves, 1};
    return enc(mw, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, const_cast<uint8_t*>(w.codes_dev), dw, sw, bw,
               ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
               CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS &&
           enc(ms, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<uint16_t*>(w.scale_dev), ds, ss,
               bs, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE,
               CU_TENSOR_MAP_L2_PROMOTION_NONE,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace
}  // namespace crc

using namespace crc;

extern "C" int crc_matvec4(const crc_matvec4_weights* w, const uint16_t* x_dev, int64_t x_stride,
                           int32_t x_per_choice, const uint8_t* topk_dev, int32_t M, int32_t K,
                           uint16_t* y_dev, void* stream) {
    const int rc = check_matvec4(w);
    if (rc) return rc;
    if (M < 0 || K < 1 || (x_per_choice != 0 && x_per_choice != 1)) return CRC_EINVAL;
    if (x_stride < w->k || x_stride % 8 != 0) return CRC_EINVAL;
    if (M == 0) return CRC_OK;
    if (!topk_dev && (K != 1 || w->expert_slot_dev)) return CRC_EINVAL;
    if (M > kMaxTokens || K > 32 || M * K > kMaxChoices) return CRC_EUNSUPPORTED;
    if (!x_dev || !y_dev || !aligned(x_dev, 16) || !aligned(y_dev, 16)) return CRC_EINVAL;
    CUtensorMap mw, ms;
    if (!make_maps(&mw, &ms, *w)) return CRC_ECUDA;
    Matvec4Args a = {};
    a.x = x_dev;
    a.topk = topk_dev;
    a.slot = w->expert_slot_dev;
    a.y = y_dev;
    a.err = device_error_word();
    a.ldx = x_stride;
    a.x_div = x_per_choice ? 1 : K;
    a.E = M * K;
    a.N = topk_dev ? w->N : 1;
    a.slots = w->slots;
    a.n = w->n;
    a.k = w->k;
    a.glu = w->glu;
    const int each = a.glu ? 16 : 32;
    a.tiles = (a.n + each - 1) / each;
    // 2, 4 or 8 warps share a tile's columns where that ends the last turn of the warps earlier:
    // turns times boxes, and one more for a turn's beginning and end.  (Experts that some choice
    // takes are at most E and N.)
    const int boxes = (a.k + kBoxCols - 1) / kBoxCols;
    const long long items = (long long)(a.E < a.N ? a.E : a.N) * a.tiles;
    const long long warps = (long long)sm_count() * kCtas * kWarps;
    const bool few = a.E < 8ll * a.N;              // choices of an expert, on average
    a.splits = 1;
    long long least = 0;
    for (int s = 1; s <= (few ? kWarps : 1) && s <= boxes; s *= 2) {
        const long long turns = (items * s + warps - 1) / warps;
        const long long cost = turns * ((boxes + s - 1) / s + 1);
        if (s == 1 || cost < least) {
            least = cost;
            a.splits = s;
        }
    }
    // (A pass over the weights takes 8 choices, 16 where the mean over all N experts is 8 or more: it
    // is not known here how many each has.  So a liked expert of a smaller batch is read, from L2,
    // once for every 8 of its choices; and from that mean on a warp has a tile to itself, which leaves
    // most of the GPU without work where the matrices are few and small.)
    const long long ctas = (items * a.splits + kWarps - 1) / kWarps;
    const long long room = (long long)sm_count() * kCtas;
    const dim3 grid((unsigned)(ctas < room ? ctas : room));
    cudaStream_t st = static_cast<cudaStream_t>(stream);
#define CRC_G(G) (few ? launch<G, 1>(mw, ms, a, grid, st) : launch<G, 2>(mw, ms, a, grid, st))
    return w->group == 32 ? CRC_G(32) : w->group == 64 ? CRC_G(64) : CRC_G(128);
#undef CRC_G
}
