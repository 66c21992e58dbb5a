// Matrix products grouped by expert: what their kernels share.  The rows of a call lie in
// their experts' order, expert e's are offsets[e] .. offsets[e + 1] - 1, known on the device
// only, so every CTA plans its own share of the work from them.
#pragma once

#include <cuda_bf16.h>

#include "crc_device.cuh"
#include "pdl.cuh"

namespace crc {

constexpr int kGroupMaxExperts = 256;

// ---------------------------------------------------------------------------
// tcgen05 operands whose rows lie across the contraction (MN-major)
// ---------------------------------------------------------------------------
// 64 elements of M (or N) a 128-byte row, one row for each step of the contraction, 128-byte
// swizzle: the layout that TMA writes for a box of 64 columns x 64 rows.  The next 64 elements
// of M are `chunk` bytes on, the next eight steps of the contraction 1024; 16 steps further
// the start address is 2048 bytes on.
__device__ __forceinline__ uint64_t sw128_mnmajor_desc(uint32_t smem_addr, uint32_t chunk) {
    uint64_t d = 0;
    d |= (uint64_t)((smem_addr >> 4) & 0x3FFFu);  // start address
    d |= (uint64_t)((chunk >> 4) & 0x3FFFu) << 16;
    d |= (uint64_t)(1024u >> 4) << 32;
    d |= (uint64_t)1u << 46;                      // descriptor version for tcgen05
    d |= (uint64_t)2u << 61;                      // 128-byte swizzle
    return d;
}
// Bits of the instruction descriptor: A, B with their rows across the contraction.
constexpr uint32_t kIdescMnA = 1u << 15, kIdescMnB = 1u << 16;

// e4m3 A and B, fp32 D.
__host__ __device__ constexpr uint32_t idesc_e4m3_f32_mn(int M, int N) {
    return (1u << 4) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

// One lane of a converged warp.
__device__ __forceinline__ uint32_t elected() {
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(r));
    return r;
}
// An arrival by the lane whose `lead` is set.  (As a branch of that lane, in the warps that gather
// rows: 217 us instead of 189 for the first product of 4096 tokens of 128 experts.)
__device__ __forceinline__ void arrive_by(uint64_t* bar, uint32_t lead) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %1, 0;\n\t"
        "@p mbarrier.arrive.shared::cta.b64 _, [%0];\n\t}" ::"r"(smem_u32(bar)),
        "r"(lead)
        : "memory");
}
// Issued by the lane whose `lead` is set, in code that the whole warp runs: the descriptors
// stay in uniform registers, where the instruction wants them.  (In a branch of one lane each
// MMA took 85 ns, whatever its columns.)
template <bool W8, bool Pair>
__device__ __forceinline__ void umma_by(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc,
                                        uint32_t idesc, uint32_t accumulate, uint32_t lead) {
#define CRC_UMMA(group, kind)                                                                 \
    asm volatile("{\n\t.reg .pred p, e;\n\t"                                                 \
                 "setp.ne.b32 p, %4, 0;\n\t"                                                  \
                 "setp.ne.b32 e, %5, 0;\n\t"                                                  \
                 "@e tcgen05.mma." group "." kind " [%0], %1, %2, %3, p;\n\t}\n" ::"r"(d_tmem), \
                 "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate), "r"(lead)               \
                 : "memory")
    if constexpr (Pair && W8)
        CRC_UMMA("cta_group::2", "kind::f8f6f4");
    else if constexpr (Pair)
        CRC_UMMA("cta_group::2", "kind::f16");
    else if constexpr (W8)
        CRC_UMMA("cta_group::1", "kind::f8f6f4");
    else
        CRC_UMMA("cta_group::1", "kind::f16");
#undef CRC_UMMA
}
__device__ __forceinline__ void commit_pair_by(uint64_t* bar, uint32_t lead) {
    asm volatile(
        "{\n\t.reg .pred e;\n\t"
        "setp.ne.b32 e, %2, 0;\n\t"
        "@e tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster"
        ".b64 [%0], %1;\n\t}" ::"r"(smem_u32(bar)),
        "h"((uint16_t)3), "r"(lead)
        : "memory");
}
__device__ __forceinline__ void commit_by(uint64_t* bar, uint32_t lead) {
    asm volatile(
        "{\n\t.reg .pred e;\n\t"
        "setp.ne.b32 e, %1, 0;\n\t"
        "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(
            smem_u32(bar)),
        "r"(lead)
        : "memory");
}

template <bool Pair>
__device__ __forceinline__ void commit_of(uint64_t* bar, uint32_t lead) {
    if constexpr (Pair)
        commit_pair_by(bar, lead);
    else
        commit_by(bar, lead);
}

// ---------------------------------------------------------------------------
// TMA
// ---------------------------------------------------------------------------
__device__ __forceinline__ uint64_t l2_normal_policy() {
    uint64_t p;
    asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(p));
    return p;
}
// (bar: a shared::cluster address, with Pair of either CTA.  Issued by the lane whose `lead` is
// set, in code that the whole warp runs.)
#define CRC_TMA_LOAD(dim, group, mode, coords, ...)                                        \
    asm volatile("{\n\t.reg .pred e;\n\tsetp.ne.b32 e, %3, 0;\n\t"                          \
                 "@e cp.async.bulk.tensor." dim group ".shared::cluster.global." mode          \
                 ".mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, " coords "], [%2], " \
                 "%4;\n\t}" ::"r"(smem_u32(dst)),                                             \
                 "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(lead), "l"(policy),      \
                 __VA_ARGS__                                                                  \
                 : "memory")
template <bool Pair>
__device__ __forceinline__ void tma_load_5d_of(uint32_t lead, void* dst, const CUtensorMap* map,
                                               uint32_t bar, int c0, int c1, int c2, int c3,
                                               int c4, uint64_t policy) {
    if constexpr (Pair)
        CRC_TMA_LOAD("5d", ".cta_group::2", "tile", "{%5, %6, %7, %8, %9}", "r"(c0), "r"(c1),
                     "r"(c2), "r"(c3), "r"(c4));
    else
        CRC_TMA_LOAD("5d", "", "tile", "{%5, %6, %7, %8, %9}", "r"(c0), "r"(c1), "r"(c2),
                     "r"(c3), "r"(c4));
}
template <bool Pair>
__device__ __forceinline__ void tma_load_3d_of(uint32_t lead, void* dst, const CUtensorMap* map,
                                               uint32_t bar, int c0, int c1, int c2,
                                               uint64_t policy) {
    if constexpr (Pair)
        CRC_TMA_LOAD("3d", ".cta_group::2", "tile", "{%5, %6, %7}", "r"(c0), "r"(c1), "r"(c2));
    else
        CRC_TMA_LOAD("3d", "", "tile", "{%5, %6, %7}", "r"(c0), "r"(c1), "r"(c2));
}
template <bool Pair>
__device__ __forceinline__ void tma_load_2d_of(uint32_t lead, void* dst, const CUtensorMap* map,
                                               uint32_t bar, int c0, int c1, uint64_t policy) {
    if constexpr (Pair)
        CRC_TMA_LOAD("2d", ".cta_group::2", "tile", "{%5, %6}", "r"(c0), "r"(c1));
    else
        CRC_TMA_LOAD("2d", "", "tile", "{%5, %6}", "r"(c0), "r"(c1));
}
// Four rows of a matrix, columns c0 on (the map's box is one row high).
template <bool Pair>
__device__ __forceinline__ void tma_gather4_of(uint32_t lead, void* dst, const CUtensorMap* map,
                                               uint32_t bar, int c0, const int (&r)[4],
                                               uint64_t policy) {
    if constexpr (Pair)
        CRC_TMA_LOAD("2d", ".cta_group::2", "tile::gather4", "{%5, %6, %7, %8, %9}", "r"(c0),
                     "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]));
    else
        CRC_TMA_LOAD("2d", "", "tile::gather4", "{%5, %6, %7, %8, %9}", "r"(c0), "r"(r[0]),
                     "r"(r[1]), "r"(r[2]), "r"(r[3]));
}
__device__ __forceinline__ void tma_store_3d(const CUtensorMap* map, const void* src, int c0,
                                             int c1, int c2) {
    asm volatile(
        "cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(
            reinterpret_cast<uint64_t>(map)),
        "r"(smem_u32(src)), "r"(c0), "r"(c1), "r"(c2)
        : "memory");
}

// ---------------------------------------------------------------------------
// an accumulator's transpose
// ---------------------------------------------------------------------------
// 16 lanes x 32 columns of TMEM: v[4 i + 2 h + b] is lane t / 4 + 8 h, column 8 i + 2 (t % 4) + b
// of thread t, the fragments of 8 x 8 matrices that stmatrix takes.
__device__ __forceinline__ void tmem_ld_frag(uint32_t taddr, float (&v)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.16x256b.x4.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]),
          "=f"(v[7]), "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]),
          "=f"(v[13]), "=f"(v[14]), "=f"(v[15])
        : "r"(taddr));
}
// Four 8 x 8 matrices of bf16, stored by columns: 16 bytes at the address that lane 8 m + c
// gives are column c of matrix m.
__device__ __forceinline__ void store_transposed(uint32_t addr, const uint32_t (&r)[4]) {
    asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(
                     addr),
                 "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3])
                 : "memory");
}

// ---------------------------------------------------------------------------
// the rows of every expert, and a share of the work
// ---------------------------------------------------------------------------
struct GroupRows {
    const int32_t* offsets;      // [N + 1]
    const int32_t* rows;         // [E] or NULL: row i of x
    uint32_t* err;
    int E, N, K;                 // row i reads x's row rows[i] / K, or i
    int x_rows;
};

// The row of x that sorted row i reads.  What is out of x is an error, and reads row 0.
__device__ __forceinline__ int source_row(const GroupRows& r, int i) {
    if (!r.rows) return i;
    const int c = r.rows[i];
    const int s = c / r.K;
    if (c >= 0 && s < r.x_rows) return s;
    latch_error(r.err, CRC_EDEVICE);
    return 0;
}

struct GroupPlan {                         // shared memory
    long long cost[kGroupMaxExperts + 1];  // of the experts before each
    int begin[kGroupMaxExperts], count[kGroupMaxExperts];
};

// Fills the plan: cost_of(rows) is an expert's.  All threads of the CTA; ends in a barrier.
template <class F>
__device__ __forceinline__ void make_plan(GroupPlan& p, const GroupRows& r, F cost_of) {
    for (int e = threadIdx.x; e < r.N; e += blockDim.x) {
        int b = r.offsets[e], n = r.offsets[e + 1];
        if (b < 0 || n < b || n > r.E) {                 // not offsets of these rows
            latch_error(r.err, CRC_EDEVICE);
            b = n = 0;
        }
        p.begin[e] = b;
        p.count[e] = n - b;
    }
    __syncthreads();
    if (threadIdx.x < 32) {
        constexpr int kEach = kGroupMaxExperts / 32;
        const int lane = threadIdx.x;
        long long v[kEach], sum = 0;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int e = lane * kEach + i;
            v[i] = sum;
            if (e < r.N) sum += cost_of(p.count[e]);
        }
        long long incl = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long u = __shfl_up_sync(kFull, incl, o);
            if (lane >= o) incl += u;
        }
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int e = lane * kEach + i;
            if (e < r.N) p.cost[e] = incl - sum + v[i];
        }
        if (lane == 31) p.cost[r.N] = incl;
    }
    __syncthreads();
}

// The expert in whose share of the cost `at` lies, at < cost[N].
__device__ __forceinline__ int expert_at(const GroupPlan& p, int N, long long at) {
    int lo = 0, hi = N;                                  // cost[lo] <= at < cost[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (p.cost[mid] <= at)
            lo = mid;
        else
            hi = mid;
    }
    return lo;
}

}  // namespace crc
