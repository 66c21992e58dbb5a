// The experts' products of the mixture-of-experts layer for a few tokens, one
// persistent kernel:
//
//   h_r = silu(G_e x_t) * (U_e x_t)      for every choice r = (token t, expert e)
//   y_r = D_e h_r,   out_t = sum over t's choices of g_r y_r
//
// A few tokens read every active expert's weights once and multiply each by a
// handful of rows, so the kernel is built to stream weights: they are the A
// operand (128 weight rows of one tcgen05.mma), the rows that take the expert
// its N columns (16 at least).  TMA fetches blocks of 128 rows x 256 bytes of
// weights into a ring that holds as much as shared memory has room for; 8-bit
// weights go to the tensor cores as they lie in memory.  256 bytes and not one
// 128-byte swizzle row: a block costs the MMA warp 150 ns beside its MMAs and their
// commit (70 ns for 128 bytes), which bounds a CTA's stream when few run.
//
// Work items, claimed in order from one counter, so that a CTA waits only for
// items that running CTAs hold (no co-residency is needed):
//   1. (row tile, 64 elements of f): gate and up rows of the same elements in one
//      128-row block, 16 and 16 to a warp's quarter of TMEM, so that silu(gate)
//      meets up by one exchange inside the warp; h goes to the workspace;
//   2. (row tile, 128 elements of d): waits until h of the tile is complete (its
//      weights are on their way meanwhile), y goes to the workspace in fp32;
//   then all CTAs add up the choices of their share of the tokens, in rank order.
//
// What bounds it is memory: 64 Qwen3-shaped tokens read 1208 MB in 178 us, 6.8 TB/s; a
// call is 8 us longer before the first block (routing, tables) and 3 behind the last.
// One token (75 MB, 24 us with its routing) is a chain of latencies: weights 8 us, h to
// the other CTAs 3, y and its sum 4.
//
// Rows wider than the weights go in two pieces, hi and lo, as two columns of the same
// product (columns cost nothing: an MMA reads 128 weight rows for 16 as for 64).  h is
// kept in fp32 and multiplied as hi + lo in bf16 (16 significant bits); one bf16 made
// the error of the bf16 output 1.4 times that of its own rounding.  With 8-bit weights a
// row is x / s = hi + lo / 16 in e4m3, s a power of two from the row's largest value: a
// bf16 x exactly down to 2^-13 of that value, h to 2^-9 of each element and 2^-21 of the
// largest (6e-4 of an element in the mean square).  No weight is converted.  With tiles of
// 16 rows the row warps split on the way into shared memory, for every item anew.  With
// more rows that would bound the kernel (three conversions a pair of elements), so
// rows are split once, by items of their own before either phase, and the pieces are
// copied: 200 tokens of the d = 4096 shape 423 -> 378 us, 1000 Qwen3-shaped 423 -> 288
// (with h in fp32 between the products, as now, 386 and 333).
#pragma once

#include <cuda_bf16.h>

#include "crc_device.cuh"
#include "moe_route.cuh"

namespace crc {

constexpr int kMoeThreads = 512;     // warps 0 TMA, 1 MMA, 2-3 idle, 4-7 epilogue, 8-15 rows
constexpr int kMoeMaxTiles = 256;    // row tiles of NT: N + M K / NT at most, M K <= 128 NT
constexpr int kItemRing = 4;
// Control words: the next item; phase-2 items done; warps done splitting x; phase-1
// items done and warps done splitting h, by row tile.
constexpr int kCtrlNext = 0, kCtrlDone2 = 1, kCtrlXSplit = 2, kCtrlDone1 = 3;
constexpr int kCtrlHSplit = kCtrlDone1 + kMoeMaxTiles;
constexpr int kCtrlWords = kCtrlHSplit + kMoeMaxTiles;
constexpr int kSplitUnits = 512;     // 16-element units that an item splits, at least
// Choices of which a warp has one a lane, of tokens of which each warp has one at most.
constexpr int kFewChoices = 32, kFewTokens = 16;
__host__ __device__ inline bool few_choices(int M, int K) {
    return M * K <= kFewChoices && M <= kFewTokens;
}

template <bool W8, int NT>
struct MoeCfg {
    // a block: two halves of 128 bytes (one swizzle row) of 128 weight rows
    static constexpr int A_HALF = 128 * 128, A_BYTES = 2 * A_HALF;
    static constexpr int BK = W8 ? 256 : 128;                  // elements of a block's row
    static constexpr int COLS = 2 * NT;                        // accumulator columns: two pieces
    static constexpr int B_HALF = COLS * 128, B_BYTES = 2 * B_HALF;
    static constexpr int SB = NT == 64 ? 2 : 3;
    static constexpr int LIST = 128 * NT;                      // choices (M K) at most
    static constexpr int TMEM_COLS = 2 * COLS;                 // two accumulators
    static constexpr int TABLE_BYTES = 3 * 128 * 4 + 3 * kMoeMaxTiles * 2 + LIST * 2 +
                                       kItemRing * NT * 4 + kFewChoices * 5 + 64;
    static constexpr int BAR_BYTES = 512;
    static constexpr int SA =
        (232448 - 1024 - BAR_BYTES - TABLE_BYTES - SB * B_BYTES) / A_BYTES;
    static constexpr int SMEM = 1024 + BAR_BYTES + TABLE_BYTES + SB * B_BYTES + SA * A_BYTES;
    static constexpr int DEPTH = NT > 16 ? 1 : W8 ? 2 : 3;     // row blocks a thread has in flight
    static constexpr bool PRE = W8 && NT > 16;                 // rows are split by items of their own
    static_assert(SA > SB && SA <= 16, "weight ring");
};

struct MoeArgs {
    const uint8_t* x;                // rows: bf16, or e4m3 with `x_split` 0 and 8-bit weights
    long long x_bytes;               // bytes between rows
    const float* xs;                 // [M] scale of x's rows (8-bit weights)
    int x_split;                     // 8-bit weights: x is bf16 and goes in two pieces
    const uint8_t* ids;              // [M][K]
    const float* gates;              // [M][K]
    const float* logits;             // [M][N], few choices: ids and gates are taken here
    uint8_t* ids_out;                // then the caller's, or null
    float* gates_out;
    int renorm;
    const int32_t* expert_slot;      // [N] or null
    const float *s13, *s2;           // scales of 8-bit weight rows, slots s13_stride floats apart
    long long s13_stride, s2_stride;
    float* h;                        // [M K][f], rows by expert
    float* y;                        // [M K][d], rows by choice
    uint8_t *xq, *hq;                // [M][hi, lo][d], [M K][hi, lo][f]: rows split once
    uint32_t* hmax;                  // [M K] largest magnitude of h's rows, zeroed (8-bit weights)
    uint32_t* ctrl;                  // kCtrlWords, zeroed
    uint32_t* err;
    __nv_bfloat16* out;              // [M][d]
    int M, N, K, d, f, slots;
    int kb1, kb2;                    // blocks of d, of f
    int ft, dt;                      // items a row tile: ceil(f / 64), ceil(d / 128)
};

// All of 128 threads, with their writes and reads before it ordered before those after.
// It has no limit of its own: every warp of a group makes the same calls, and one last
// call when it has ended or given up, after which (all false) nobody makes another.
__device__ __forceinline__ bool group_all(bool ok, int id) {
    uint32_t all;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\t"
        "barrier.cta.red.and.pred q, %2, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}\n"
        : "=r"(all)
        : "r"((uint32_t)ok), "r"(id)
        : "memory");
    return all != 0;
}

// One lane of a converged warp.
__device__ __forceinline__ uint32_t elect_lane() {
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(r));
    return r;
}
// D[tmem] (+)= A[smem] * B[smem]^T, issued by the lane whose `lead` is set.
template <bool W8>
__device__ __forceinline__ void umma(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc,
                                     uint32_t idesc, uint32_t accumulate, uint32_t lead) {
    if constexpr (W8)
        asm volatile(
            "{\n\t.reg .pred p, e;\n\t"
            "setp.ne.b32 p, %4, 0;\n\t"
            "setp.ne.b32 e, %5, 0;\n\t"
            "@e tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}\n" ::"r"(d_tmem),
            "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate), "r"(lead)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p, e;\n\t"
            "setp.ne.b32 p, %4, 0;\n\t"
            "setp.ne.b32 e, %5, 0;\n\t"
            "@e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}\n" ::"r"(d_tmem),
            "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate), "r"(lead)
            : "memory");
}
// Whether the phase of that parity has completed, without waiting (try_wait may
// suspend the thread).
__device__ __forceinline__ bool mbar_test(uint64_t* bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}\n"
        : "=r"(ok)
        : "r"(smem_u32(bar)), "r"(parity)
        : "memory");
    return ok != 0;
}
__device__ __forceinline__ void umma_commit_by(uint64_t* bar, uint32_t lead) {
    asm volatile(
        "{\n\t.reg .pred e;\n\t"
        "setp.ne.b32 e, %1, 0;\n\t"
        "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(
            smem_u32(bar)),
        "r"(lead)
        : "memory");
}
// Instruction descriptor, kind::f8f6f4: e4m3 A and B (K-major), fp32 D, M x N.
__device__ __forceinline__ uint32_t idesc_e4m3_f32(int M, int N) {
    return (1u << 4) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

__device__ __forceinline__ void tma_load_5d(void* dst, const CUtensorMap* map, uint64_t* bar,
                                            int c0, int c1, int c2, int c3, int c4,
                                            uint64_t policy) {
    asm volatile(
        "cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
        ".L2::cache_hint [%0], [%1, {%2, %3, %4, %5, %6}], [%7], %8;" ::"r"(smem_u32(dst)),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(c4),
        "r"(smem_u32(bar)), "l"(policy)
        : "memory");
}
__device__ __forceinline__ uint64_t l2_evict_normal_policy() {
    uint64_t p;
    asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(p));
    return p;
}

// One more, behind this warp's writes (after a __syncwarp).
__device__ __forceinline__ void add_release(uint32_t* p) {
    asm volatile("red.release.gpu.global.add.u32 [%0], 1;" ::"l"(p) : "memory");
}
__device__ __forceinline__ uint32_t ld_acquire(const uint32_t* p) {
    uint32_t v;
    asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}
// Adds one to a word in shared memory; acquires what was released there before.
__device__ __forceinline__ uint32_t add_cta(uint32_t* p) {
    uint32_t was;
    asm volatile("atom.acq_rel.cta.shared::cta.add.u32 %0, [%1], 1;"
                 : "=r"(was)
                 : "r"(smem_u32(p))
                 : "memory");
    return was;
}
// Wait until *p reaches n; false on timeout.
__device__ __forceinline__ bool wait_count(const uint32_t* p, uint32_t n) {
    if (ld_acquire(p) >= n) return true;
    const uint64_t t0 = globaltimer_ns();
    while (true) {
#pragma unroll 1
        for (int i = 0; i < 256; ++i)
            if (ld_acquire(p) >= n) return true;
        if (globaltimer_ns() - t0 > kWaitLimitNs) return false;
    }
}

// Two floats as e4m3 pieces: hi, and lo = 16 (v - hi).
__device__ __forceinline__ void split_floats(float a, float b, uint32_t& hi, uint32_t& lo) {
    uint16_t h, l;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(h) : "f"(b), "f"(a));
    uint32_t back;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(back) : "h"(h));
    float fa, fb;
    asm("{\n\t.reg .b16 x, y;\n\tmov.b32 {x, y}, %2;\n\tcvt.f32.f16 %0, x;\n\tcvt.f32.f16 %1, y;\n\t}"
        : "=f"(fa), "=f"(fb)
        : "r"(back));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;"
        : "=h"(l)
        : "f"((b - fb) * 16.f), "f"((a - fa) * 16.f));
    hi = h;
    lo = l;
}
// Sixteen bf16 -> sixteen bytes of each piece.
__device__ __forceinline__ void split16(const uint4 (&v)[2], float inv, uint4& hi, uint4& lo) {
    const uint32_t w[8] = {v[0].x, v[0].y, v[0].z, v[0].w, v[1].x, v[1].y, v[1].z, v[1].w};
    uint32_t ho[4], lw[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t h0, l0, h1, l1;
        split_floats(__uint_as_float(w[2 * i] << 16) * inv,
                     __uint_as_float(w[2 * i] & 0xffff0000u) * inv, h0, l0);
        split_floats(__uint_as_float(w[2 * i + 1] << 16) * inv,
                     __uint_as_float(w[2 * i + 1] & 0xffff0000u) * inv, h1, l1);
        ho[i] = h0 | h1 << 16;
        lw[i] = l0 | l1 << 16;
    }
    hi = make_uint4(ho[0], ho[1], ho[2], ho[3]);
    lo = make_uint4(lw[0], lw[1], lw[2], lw[3]);
}

// Sixteen floats -> sixteen bytes of each e4m3 piece; eight -> eight bf16 of each
// bf16 piece, hi + lo.
__device__ __forceinline__ void split16(const uint4 (&v)[4], float inv, uint4& hi, uint4& lo) {
    uint32_t ho[4], lw[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t h0, l0, h1, l1;
        split_floats(__uint_as_float(v[i].x) * inv, __uint_as_float(v[i].y) * inv, h0, l0);
        split_floats(__uint_as_float(v[i].z) * inv, __uint_as_float(v[i].w) * inv, h1, l1);
        ho[i] = h0 | h1 << 16;
        lw[i] = l0 | l1 << 16;
    }
    hi = make_uint4(ho[0], ho[1], ho[2], ho[3]);
    lo = make_uint4(lw[0], lw[1], lw[2], lw[3]);
}
__device__ __forceinline__ void split8(const uint4 (&v)[2], uint4& hi, uint4& lo) {
    const uint32_t w[8] = {v[0].x, v[0].y, v[0].z, v[0].w, v[1].x, v[1].y, v[1].z, v[1].w};
    uint32_t ho[4], lw[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float a = __uint_as_float(w[2 * i]), b = __uint_as_float(w[2 * i + 1]);
        const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
        const __nv_bfloat162 l =
            __floats2bfloat162_rn(a - __low2float(h), b - __high2float(h));
        ho[i] = *reinterpret_cast<const uint32_t*>(&h);
        lw[i] = *reinterpret_cast<const uint32_t*>(&l);
    }
    hi = make_uint4(ho[0], ho[1], ho[2], ho[3]);
    lo = make_uint4(lw[0], lw[1], lw[2], lw[3]);
}

template <bool W8, int NT>
struct MoeShared {
    using Cfg = MoeCfg<W8, NT>;
    uint8_t *a, *b;
    uint64_t *a_full, *a_empty, *b_full, *t_full, *t_empty, *i_full, *i_empty, *drain;
    uint32_t* tmem_slot;
    int* items;
    uint32_t* ended;       // [4] epilogue warps that have ended an item, by its turn
    float* hscale;         // [kItemRing][NT] scales of h's rows (8-bit weights)
    float* few_gates;      // [kFewChoices]
    uint8_t* few_ids;      // [kFewChoices]
    int* slot;             // [128] slot of each expert, -1 without
    int* start;            // [128] first row of each expert
    int* count;            // [128] rows of each expert, then [0] = row tiles
    uint16_t *tile_e, *tile_row, *tile_rows;   // [kMoeMaxTiles]
    uint16_t* list;        // choices sorted by expert, then by token

    __device__ __forceinline__ explicit MoeShared(uint8_t* base) {
        a = base;
        b = a + Cfg::SA * Cfg::A_BYTES;
        uint8_t* p = b + Cfg::SB * Cfg::B_BYTES;
        a_full = reinterpret_cast<uint64_t*>(p);
        a_empty = a_full + Cfg::SA;
        b_full = a_empty + Cfg::SA;
        t_full = b_full + Cfg::SB;
        t_empty = t_full + 2;
        i_full = t_empty + 2;
        i_empty = i_full + kItemRing;
        drain = i_empty + kItemRing;
        tmem_slot = reinterpret_cast<uint32_t*>(drain + 1);
        items = reinterpret_cast<int*>(tmem_slot + 1);
        ended = reinterpret_cast<uint32_t*>(items + kItemRing);
        static_assert((2 * Cfg::SA + Cfg::SB + 4 + 2 * kItemRing + 1) * 8 + 20 + 4 * kItemRing <=
                          Cfg::BAR_BYTES,
                      "barrier space");
        slot = reinterpret_cast<int*>(p + Cfg::BAR_BYTES);
        start = slot + 128;
        count = start + 128;
        tile_e = reinterpret_cast<uint16_t*>(count + 128);
        tile_row = tile_e + kMoeMaxTiles;
        tile_rows = tile_row + kMoeMaxTiles;
        list = tile_rows + kMoeMaxTiles;
        hscale = reinterpret_cast<float*>(list + Cfg::LIST);
        few_gates = hscale + kItemRing * NT;
        few_ids = reinterpret_cast<uint8_t*>(few_gates + kFewChoices);
    }
};

// Sorts the choices by expert, then by token, and cuts each expert's rows into tiles of
// NT.  Every CTA builds the same tables.  All threads.
//
// One warp does it when the choices are one a lane (one token of up to 32 choices,
// four of 8), without the general form's barriers.
template <bool W8, int NT>
__device__ __forceinline__ void build_small_tables(const MoeArgs& a, const MoeShared<W8, NT>& s) {
    const int lane = threadIdx.x & 31, E = a.M * a.K;
    int e = 128;
    if (lane < E) e = a.logits ? s.few_ids[lane] : __ldcg(a.ids + lane);
    if (e < 128 && s.slot[e] < 0) e = 128;
    const uint32_t peers = __match_any_sync(kFull, e);
    const bool lead = e < 128 && lane == __ffs(peers) - 1;
    const uint32_t leads = __ballot_sync(kFull, lead);
    int pos = __popc(peers & ((1u << lane) - 1u)), row0 = 0, tile = 0;
    for (uint32_t rest = leads; rest; rest &= rest - 1) {
        const int l = __ffs(rest) - 1;
        const int other = __shfl_sync(kFull, e, l);
        const int n = __popc(__shfl_sync(kFull, peers, l));
        if (other < e) {
            row0 += n;
            ++tile;
        }
    }
    if (e < 128) s.list[row0 + pos] = (uint16_t)lane;
    if (lead) {                      // an expert has one row a token at most: one tile
        s.tile_e[tile] = (uint16_t)e;
        s.tile_row[tile] = (uint16_t)row0;
        s.tile_rows[tile] = (uint16_t)__popc(peers);
    }
    if (lane == 0) s.count[0] = __popc(leads);
}

template <bool W8, int NT>
__device__ __forceinline__ void build_tables(const MoeArgs& a, const MoeShared<W8, NT>& s,
                                             int slot_e) {
    using Cfg = MoeCfg<W8, NT>;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int E = a.M * a.K;
    const bool few = few_choices(a.M, a.K), route = few && a.logits && warp < a.M;
    float v[4];                       // asked for before the slots are waited for
    if (route) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int e = lane + 32 * i;
            v[i] = e < a.N ? __ldcg(a.logits + warp * a.N + e) : 0.f;
        }
    }
    if (threadIdx.x < 128) s.slot[threadIdx.x] = slot_e >= 0 && slot_e < a.slots ? slot_e : -1;
    if (few) {
        if (route) {                  // Top-K and gates, a warp a token
            const int r = warp * a.K;
            const bool out = blockIdx.x == 0;
            route_token(v, a.N, a.K, false, a.renorm, lane, s.few_ids + r, s.few_gates + r,
                        out && a.ids_out ? a.ids_out + r : nullptr,
                        out && a.gates_out ? a.gates_out + r : nullptr);
        }
        __syncthreads();
        if (warp == 0) build_small_tables<W8, NT>(a, s);
        __syncthreads();
        return;
    }
    // Scratch in the weight ring, which is not in use yet: for every expert the set
    // of its tokens as bits, with the count of those before each word.  (An expert is
    // chosen once a token at most.)
    const int words = (a.M + 31) / 32;
    uint32_t* set = reinterpret_cast<uint32_t*>(s.a);                  // [128][words]
    uint16_t* before = reinterpret_cast<uint16_t*>(set + 128 * words); // [128][words]
    static_assert(128 * 32 * 6 <= Cfg::SA * Cfg::A_BYTES, "scratch");
    for (int i = threadIdx.x; i < 128 * words; i += kMoeThreads) set[i] = 0u;
    // a thread's choices: four neighbours in each of `quads` words, all asked at once
    constexpr int QUADS = (Cfg::LIST + 4 * kMoeThreads - 1) / (4 * kMoeThreads);
    uint32_t ids[QUADS];
#pragma unroll
    for (int q = 0; q < QUADS; ++q) {
        const int i = 4 * (threadIdx.x + q * kMoeThreads);
        ids[q] = i < E ? __ldcg(reinterpret_cast<const uint32_t*>(a.ids) + i / 4) : 0u;
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < QUADS; ++q) {
        const int i = 4 * (threadIdx.x + q * kMoeThreads);
        int tok = i / a.K, k = i - tok * a.K;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int e = (int)(ids[q] >> (8 * j) & 0xffu);
            if (i + j < E && s.slot[e] >= 0) atomicOr(&set[e * words + (tok >> 5)], 1u << (tok & 31));
            if (++k == a.K) k = 0, ++tok;
        }
    }
    __syncthreads();
    if (threadIdx.x < 128) {
        const int e = threadIdx.x;
        int n = 0;
        for (int w = 0; w < words; ++w) {
            before[e * words + w] = (uint16_t)n;
            n += __popc(set[e * words + w]);
        }
        s.count[e] = n;
    }
    __syncthreads();
    if (warp == 0) {                 // exclusive sums over experts: rows and tiles
        int c[4], rows = 0, tiles = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            c[i] = s.count[4 * lane + i];
            rows += c[i];
            tiles += (c[i] + NT - 1) / NT;
        }
        int r = rows, t = tiles;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int ur = __shfl_up_sync(kFull, r, o), ut = __shfl_up_sync(kFull, t, o);
            if (lane >= o) {
                r += ur;
                t += ut;
            }
        }
        const int all = __shfl_sync(kFull, t, 31);
        r -= rows;
        t -= tiles;
        __syncwarp();
        if (lane == 0) s.count[0] = all;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            s.start[4 * lane + i] = r;
            for (int k = 0; k < c[i]; k += NT, ++t) {
                s.tile_e[t] = (uint16_t)(4 * lane + i);
                s.tile_row[t] = (uint16_t)(r + k);
                s.tile_rows[t] = (uint16_t)(c[i] - k < NT ? c[i] - k : NT);
            }
            r += c[i];
        }
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < QUADS; ++q) {
        const int i = 4 * (threadIdx.x + q * kMoeThreads);
        int tok = i / a.K, k = i - tok * a.K;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int e = (int)(ids[q] >> (8 * j) & 0xffu);
            if (i + j < E && s.slot[e] >= 0) {
                const int at = e * words + (tok >> 5);
                s.list[s.start[e] + before[at] + __popc(set[at] & ((1u << (tok & 31)) - 1u))] =
                    (uint16_t)(i + j);
            }
            if (++k == a.K) k = 0, ++tok;
        }
    }
    // the ring's stages go from generic reads and writes to TMA
    fence_proxy_async_smem();
    __syncthreads();
}

// A work item.
enum { kGateUp = 0, kDown = 1, kSplitX = 2, kSplitH = 3 };
struct MoeItem {
    int kind, tile, j;       // kGateUp: 64 elements of f; kDown: 128 elements of d;
    int e, row0, rows;       // kSplitX: all tokens; kSplitH: the tile's rows; j: the part of them
    bool ok;                 // checking builds: within the arrays (else nothing is written)
};
// First items of the kinds, in the order kSplitX, kGateUp, kSplitH, kDown.  Everything
// that follows waits for the splits, so they are cut into items for all CTAs, x as a
// whole, h each tile's rows into `parts` (200 tokens of d = f = 2880, 32 experts, 8-bit:
// 174 us with 16 tokens of x and one tile of h an item, 168 so).
struct MoeItems {
    int gate_up, split_h, down, end, parts;
    template <bool W8, int NT>
    __device__ __forceinline__ static MoeItems of(const MoeArgs& a, int tiles) {
        MoeItems n;
        const int ctas = (int)gridDim.x;
        n.gate_up = MoeCfg<W8, NT>::PRE && a.x_split && tiles
                        ? min(ctas, (a.M * (a.d / 16) + kSplitUnits - 1) / kSplitUnits)
                        : 0;
        n.parts = MoeCfg<W8, NT>::PRE && tiles
                      ? max(1, min((ctas + tiles - 1) / tiles,
                                   a.M * a.K / tiles * (a.f / 16) / kSplitUnits))
                      : 1;
        n.split_h = n.gate_up + tiles * a.ft;
        n.down = n.split_h + (MoeCfg<W8, NT>::PRE ? tiles * n.parts : 0);
        n.end = n.down + tiles * a.dt;
        return n;
    }
};
template <bool W8, int NT>
__device__ __forceinline__ MoeItem moe_item(const MoeArgs& a, const MoeShared<W8, NT>& s,
                                            const MoeItems& n, int i) {
    MoeItem it;
    it.j = 0;
    if (i >= n.down) {
        it.kind = kDown;
        it.tile = (i - n.down) / a.dt;
        it.j = i - n.down - it.tile * a.dt;
    } else if (MoeCfg<W8, NT>::PRE && i >= n.split_h) {
        it.kind = kSplitH;
        it.tile = (i - n.split_h) / n.parts;
        it.j = i - n.split_h - it.tile * n.parts;
    } else if (!MoeCfg<W8, NT>::PRE || i >= n.gate_up) {
        it.kind = kGateUp;
        it.tile = (i - n.gate_up) / a.ft;
        it.j = i - n.gate_up - it.tile * a.ft;
    } else {
        it.kind = kSplitX;
        it.tile = it.e = it.row0 = 0;
        it.j = i;
        it.rows = a.M;
        it.ok = true;
        return it;
    }
    it.e = s.tile_e[it.tile];
    it.row0 = s.tile_row[it.tile];
    it.rows = s.tile_rows[it.tile];
    it.ok = CRC_IN_BOUNDS(it.tile < s.count[0] && it.e < a.N && s.slot[it.e] >= 0 &&
                              s.slot[it.e] < a.slots && it.rows > 0 && it.rows <= NT &&
                              it.row0 + it.rows <= a.M * a.K,
                          a.err);
    if (!it.ok) {                    // what is read with it all the same is in the tables
        it.e = it.row0 = 0;
        it.rows = 1;
    }
    return it;
}

// A row group's place in the ring of row blocks.  Two groups of four warps take
// the blocks alternately.  Block n takes the place of block n - SB, which is free
// once that block's MMAs are complete: the weight stage of the same block says so
// (SB < SA, so that stage cannot have moved on by two phases), and one commit a
// block serves both rings.
template <bool W8, int NT>
struct RowRing {
    using Cfg = MoeCfg<W8, NT>;
    int next;                        // this group's next block, counted over all items
    int stage, free;                 // its place; the weight stage of block next - SB
    uint32_t free_phase = 0;
    __device__ __forceinline__ explicit RowRing(int group)
        : next(group), stage(group), free(group - Cfg::SB) {}
    __device__ __forceinline__ void advance() {
        next += 2;
        stage += 2;
        if (stage >= Cfg::SB) stage -= Cfg::SB;
        free += 2;
        if (free >= Cfg::SA) {
            free -= Cfg::SA;
            free_phase ^= 1;
        }
    }
};

// A group's row blocks of one item into the ring (four warps).  base: the item's
// first block, counted over all items.  A thread's unit is 16 bytes of one row's
// 256: chunk tid % 16 of rows tid / 16, + 8, ...  MODE kCopy: as they are; kSplit: bf16
// elements become hi and lo (8-bit weights); kSplitF: fp32 elements do (h); kPieces:
// hi and lo are copied, K bytes apart.
enum { kCopy = 0, kSplit = 1, kPieces = 2, kSplitF = 3 };
template <bool W8, int NT, int MODE>
__device__ __forceinline__ bool produce_rows(const MoeShared<W8, NT>& s, const uint8_t* (&src)[NT / 8],
                                             const float (&inv)[NT / 8], uint32_t have, int n8,
                                             int base, int kb, int K, int tid,
                                             RowRing<W8, NT>& ring) {
    using Cfg = MoeCfg<W8, NT>;
    constexpr int U = NT / 8, D = Cfg::DEPTH;
    constexpr int V = MODE == kCopy ? 1 : MODE == kSplitF && W8 ? 4 : 2;   // loads a unit
    constexpr int STEP = MODE == kPieces ? 256 : 256 * V;      // bytes of a row's block
    constexpr int CE = W8 ? 16 : 8;                            // elements of a unit
    const int chunk = tid & 15, lane = tid & 31;
    uint4 v[D][U][V];
    auto load = [&](int k, uint4 (&r)[U][V]) {
        const bool in = k * Cfg::BK + chunk * CE < K;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int q = 0; q < V; ++q)
                r[u][q] = in && (have >> u & 1u)
                              ? __ldcg(reinterpret_cast<const uint4*>(
                                    src[u] + (size_t)k * STEP + q * (MODE == kPieces ? K : 16)))
                              : make_uint4(0, 0, 0, 0);
    };
    const int first = ring.next - base;
#pragma unroll
    for (int i = 0; i < D; ++i) load(first + 2 * i, v[i]);
    for (int k0 = first; k0 < kb; k0 += 2 * D) {
#pragma unroll
        for (int i = 0; i < D; ++i) {
            const int k = k0 + 2 * i;
            if (k >= kb) break;
            if (ring.next >= Cfg::SB && !mbar_wait_warp(&s.a_empty[ring.free], ring.free_phase))
                return false;
            uint8_t* dst = s.b + ring.stage * Cfg::B_BYTES + (chunk >> 3) * Cfg::B_HALF;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (!(have >> u & 1u)) continue;
                const int row = (tid >> 4) + 8 * u;
                if constexpr (MODE != kCopy) {
                    uint4 hi = v[i][u][0], lo = v[i][u][V - 1];
                    if constexpr (MODE == kSplitF && !W8)
                        split8(v[i][u], hi, lo);
                    else if constexpr (MODE != kPieces)
                        split16(v[i][u], inv[u], hi, lo);
                    const int low = n8 + row;
                    *reinterpret_cast<uint4*>(dst + row * 128 + (((chunk ^ row) & 7) << 4)) = hi;
                    *reinterpret_cast<uint4*>(dst + low * 128 + (((chunk ^ low) & 7) << 4)) = lo;
                } else {
                    *reinterpret_cast<uint4*>(dst + row * 128 + (((chunk ^ row) & 7) << 4)) =
                        v[i][u][0];
                }
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&s.b_full[ring.stage]);
            ring.advance();
            if (k + 2 * D < kb) load(k + 2 * D, v[i]);
        }
    }
    return true;
}

// n elements (a multiple of 16) of `rows` rows, bf16 (V = 2) or fp32 (V = 4), into two e4m3
// pieces: a thread a chunk of 16.  src(r), inv(r): row r and 1 / its scale; dst: rows
// of hi and lo, n bytes each.
template <int V, class Src, class Inv>
__device__ __forceinline__ void split_rows(int rows, int n, int thread, int threads, Src src, Inv inv,
                                           uint8_t* dst) {
    constexpr int D = 4 / V;                        // chunks in flight
    const int chunks = n / 16, all = rows * chunks;
    for (int i0 = thread; i0 < all; i0 += D * threads) {
        uint4 v[D][V];
        float s[D];
#pragma unroll
        for (int u = 0; u < D; ++u) {
            const int i = i0 + u * threads;
            if (i >= all) break;
            const int r = i / chunks, c = i - r * chunks;
            const uint4* at = reinterpret_cast<const uint4*>(src(r)) + V * c;
#pragma unroll
            for (int j = 0; j < V; ++j) v[u][j] = __ldcg(at + j);
            s[u] = inv(r);
        }
#pragma unroll
        for (int u = 0; u < D; ++u) {
            const int i = i0 + u * threads;
            if (i >= all) break;
            const int r = i / chunks, c = i - r * chunks;
            uint4 hi, lo;
            split16(v[u], s[u], hi, lo);
            uint8_t* to = dst + (size_t)r * 2 * n + 16 * c;
            *reinterpret_cast<uint4*>(to) = hi;
            *reinterpret_cast<uint4*>(to + n) = lo;
        }
    }
}

// Gates of up to eight choices from r on; a bit for each whose expert has a slot.
struct Gates {
    float g[8];
    uint32_t have;
    template <class Shared>
    __device__ __forceinline__ void load(const MoeArgs& a, const Shared& s, int r, int n) {
        have = 0;
        int id[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            id[k] = 0;
            g[k] = 0.f;
            if (k >= n) continue;
            id[k] = a.logits ? s.few_ids[r + k] : __ldcg(a.ids + r + k);
            g[k] = a.logits ? s.few_gates[r + k] : __ldcg(a.gates + r + k);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k < n && s.slot[id[k]] >= 0) have |= 1u << k;
    }
};

template <bool W8, int NT>
__global__ void __launch_bounds__(kMoeThreads, 1)
    moe_experts_kernel(const __grid_constant__ CUtensorMap map13,
                       const __grid_constant__ CUtensorMap map2, MoeArgs a) {
    using Cfg = MoeCfg<W8, NT>;
    extern __shared__ uint8_t smem_raw[];
    MoeShared<W8, NT> s(reinterpret_cast<uint8_t*>(
        (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023)));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int i = 0; i < Cfg::SA; ++i) {
            mbar_init(&s.a_full[i], 1);
            mbar_init(&s.a_empty[i], 1);
        }
        for (int i = 0; i < Cfg::SB; ++i) mbar_init(&s.b_full[i], 4);
        for (int i = 0; i < 2; ++i) {
            mbar_init(&s.t_full[i], 1);
            mbar_init(&s.t_empty[i], 4);
        }
        for (int i = 0; i < kItemRing; ++i) {
            mbar_init(&s.i_full[i], 1);
            mbar_init(&s.i_empty[i], 13);        // MMA, 4 epilogue, 8 row warps
        }
        for (int i = 0; i < 4; ++i) s.ended[i] = 0;
        mbar_init(s.drain, 1);
        fence_mbar_init();
        tma_prefetch_desc(&map13);
        tma_prefetch_desc(&map2);
    }
    if (warp == 1) {
        tmem_alloc(s.tmem_slot, Cfg::TMEM_COLS);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *s.tmem_slot;

    pdl_begin();                      // the choices and the zeroed counters are in place
    int next = 0;
    if (threadIdx.x == 0) next = (int)atomicAdd(&a.ctrl[kCtrlNext], 1u);
    int slot_e = -1;                  // of expert threadIdx.x
    if (threadIdx.x < a.N) slot_e = a.expert_slot ? __ldcg(a.expert_slot + threadIdx.x) : threadIdx.x;
    build_tables<W8, NT>(a, s, slot_e);
    const int tiles = s.count[0];
    const MoeItems items = MoeItems::of<W8, NT>(a, tiles);

    if (warp == 0) {
        // ------------------------------------------------------ weights by TMA
        if (lane == 0) {
            const uint64_t once = l2_evict_first_policy(), again = l2_evict_normal_policy();
            int stage = 0, issued = 0, islot = 0;
            uint32_t phase = 0, iphase = 0;
            bool failed = false;
            while (!failed) {
                const int item = next < items.end ? next : -1;
                if (!mbar_wait(&s.i_empty[islot], iphase ^ 1)) {
                    failed = true;
                    break;
                }
                s.items[islot] = item;
                mbar_arrive(&s.i_full[islot]);
                if (++islot == kItemRing) {
                    islot = 0;
                    iphase ^= 1;
                }
                if (item < 0) break;
                const MoeItem it = moe_item<W8, NT>(a, s, items, item);
                if (it.kind >= kSplitX) {
                    next = (int)atomicAdd(&a.ctrl[kCtrlNext], 1u);
                    continue;
                }
                const int slot = it.ok ? s.slot[it.e] : 0;
                // an expert with several row tiles (all but the last are full) is
                // read again, from L2
                const uint64_t pol = it.rows == NT ? again : once;
                const int kb = it.kind == kDown ? a.kb2 : a.kb1;
                const int first = stage;
                const uint32_t first_phase = phase;
                for (int k = 0; k < kb; ++k) {
                    if (!mbar_wait(&s.a_empty[stage], phase ^ 1)) {
                        failed = true;
                        break;
                    }
                    mbar_arrive_expect_tx(&s.a_full[stage], Cfg::A_BYTES);
                    uint8_t* dst = s.a + stage * Cfg::A_BYTES;
#pragma unroll
                    for (int half = 0; half < 2; ++half) {     // past the row's end: zeros
                        const int x = k * Cfg::BK + half * (Cfg::BK / 2);
                        if (it.kind == kGateUp)
                            tma_load_5d(dst + half * Cfg::A_HALF, &map13, &s.a_full[stage], x, 0, 0,
                                        it.j * 4, slot, pol);
                        else
                            tma_load_3d(dst + half * Cfg::A_HALF, &map2, &s.a_full[stage], x,
                                        it.j * 128, slot, pol);
                    }
                    ++issued;
                    if (++stage == Cfg::SA) {
                        stage = 0;
                        phase ^= 1;
                    }
                }
                if (failed) break;
                // Of the last items, the next is claimed once this one's first block is
                // consumed: a CTA that waits for h would otherwise take items that idle CTAs
                // could have (one Qwen3-shaped token: all 128 down items on 56 CTAs).
                if (kb <= Cfg::SA && items.end - item <= 2 * (int)gridDim.x &&
                    !mbar_wait(&s.a_empty[first], first_phase)) {
                    failed = true;
                    break;
                }
                next = (int)atomicAdd(&a.ctrl[kCtrlNext], 1u);
            }
            if (failed) latch_error(a.err, CRC_ETIMEOUT);
            // Never leave with copies in flight.
            for (int k = issued < Cfg::SA ? issued : Cfg::SA; k > 0; --k) {
                if (--stage < 0) {
                    stage = Cfg::SA - 1;
                    phase ^= 1;
                }
                if (!mbar_wait(&s.a_full[stage], phase)) latch_error(a.err, CRC_ETIMEOUT);
            }
        }
    } else if (warp == 1) {
        // ------------------------------------------------------ MMA
        // The whole warp walks the blocks with uniform control flow and one lane
        // issues: descriptors then live in uniform registers.
        const uint32_t lead = elect_lane();
        const uint64_t a0 = sw128_kmajor_desc(smem_u32(s.a)), b0 = sw128_kmajor_desc(smem_u32(s.b));
        const MoeItems my = MoeItems::of<W8, NT>(a, __reduce_max_sync(kFull, tiles));
        int stage = 0, bstage = 0, islot = 0, acc = 0;
        uint32_t phase = 0, bphase = 0, iphase = 0, aphase = 0;
        bool failed = false;
        while (true) {
            if (__any_sync(kFull, !mbar_wait(&s.i_full[islot], iphase))) {
                failed = true;
                break;
            }
            const int item = __reduce_max_sync(kFull, s.items[islot]);
            if (lead) mbar_arrive(&s.i_empty[islot]);
            if (++islot == kItemRing) {
                islot = 0;
                iphase ^= 1;
            }
            if (item < 0) break;
            if (Cfg::PRE && (item < my.gate_up || (item >= my.split_h && item < my.down))) continue;
            const bool second = item >= my.down;
            const int rows = __reduce_max_sync(kFull, moe_item<W8, NT>(a, s, my, item).rows);
            const bool split = second || (W8 && a.x_split);
            const int n = split ? 2 * ((rows + 7) & ~7) : (rows + 15) & ~15;
            const uint32_t idesc = W8 ? idesc_e4m3_f32(128, n) : idesc_bf16_f32(128, n);
            if (__any_sync(kFull, !mbar_wait(&s.t_empty[acc], aphase ^ 1))) {
                failed = true;
                break;
            }
            tc_fence_after();
            const uint32_t dt = tmem + (uint32_t)(acc * Cfg::COLS);
            const int kb = second ? a.kb2 : a.kb1;
            bool there = false;
            for (int k = 0; k < kb; ++k) {
                if (!there) {
                    const bool ok = mbar_wait(&s.b_full[bstage], bphase) &&
                                    mbar_wait(&s.a_full[stage], phase);
                    if (__any_sync(kFull, !ok)) {
                        failed = true;
                        break;
                    }
                }
                tc_fence_after();
                const uint64_t ad = a0 + (uint64_t)(stage * (Cfg::A_BYTES >> 4));
                const uint64_t bd = b0 + (uint64_t)(bstage * (Cfg::B_BYTES >> 4));
                uint64_t* free = &s.a_empty[stage];
                if (++stage == Cfg::SA) {
                    stage = 0;
                    phase ^= 1;
                }
                if (++bstage == Cfg::SB) {
                    bstage = 0;
                    bphase ^= 1;
                }
                // the next block is asked for before this one's MMAs: the answer takes as
                // long as they do
                const bool next = mbar_test(&s.b_full[bstage], bphase) &
                                  mbar_test(&s.a_full[stage], phase) & (k + 1 < kb);
#pragma unroll
                for (int q = 0; q < 8; ++q)             // 32 bytes of K a step
                    umma<W8>(dt, ad + (q >> 2) * (Cfg::A_HALF >> 4) + 2 * (q & 3),
                             bd + (q >> 2) * (Cfg::B_HALF >> 4) + 2 * (q & 3), idesc, (k | q) != 0,
                             lead);
                umma_commit_by(free, lead);
                there = __all_sync(kFull, next);
            }
            if (failed) break;
            umma_commit_by(&s.t_full[acc], lead);
            acc ^= 1;
            if (acc == 0) aphase ^= 1;
        }
        if (failed && lead) latch_error(a.err, CRC_ETIMEOUT);
        // All issued MMAs must be complete before TMEM is released.
        umma_commit_by(s.drain, lead);
        if (!mbar_wait(s.drain, 0)) latch_error(a.err, CRC_ETIMEOUT);
    } else if (warp >= 8) {
        // ------------------------------------------------------ rows
        const int tid = threadIdx.x & 127;
        RowRing<W8, NT> ring((warp - 8) >> 2);
        int islot = 0, base = 0;
        uint32_t iphase = 0;
        bool failed = false, apart = true;   // apart: the group does not know of it yet
        const int group = 1 + ((warp - 8) >> 2);
        while (true) {
            if (!mbar_wait_warp(&s.i_full[islot], iphase)) {
                failed = true;
                break;
            }
            const int item = s.items[islot], ring_slot = islot;
            __syncwarp();
            if (lane == 0) mbar_arrive(&s.i_empty[islot]);
            if (++islot == kItemRing) {
                islot = 0;
                iphase ^= 1;
            }
            if (item < 0) break;
            const MoeItem it = moe_item<W8, NT>(a, s, items, item);
            // what the item reads: x in pieces, h of the whole tile, h in pieces
            const bool x_pieces = Cfg::PRE && a.x_split && it.kind == kGateUp;
            if (x_pieces || it.kind == kSplitH || it.kind == kDown) {
                const uint32_t* at = &a.ctrl[x_pieces ? kCtrlXSplit
                                             : Cfg::PRE && it.kind == kDown ? kCtrlHSplit + it.tile
                                                                            : kCtrlDone1 + it.tile];
                const uint32_t n = x_pieces ? 8u * items.gate_up
                                   : Cfg::PRE && it.kind == kDown ? 8u * items.parts
                                                                  : (uint32_t)a.ft;
                // One thread asks for its four warps: the answers and the counters' own adds
                // queue at the same place in L2 (one token, every warp asking: 24.9 us, so
                // 23.7; 8-bit 20.6 and 19.2).
                bool ok = true;
                if (tid == 0) ok = wait_count(at, n);
                if (!group_all(ok, group)) {
                    failed = true;
                    apart = false;
                    break;
                }
            }
            if (Cfg::PRE && it.kind >= kSplitX) {
                const int t = it.j * 256 + threadIdx.x - 256;
                const int rows = it.ok ? it.rows : 0;
                if (it.kind == kSplitX)
                    split_rows<2>(rows, a.d, t, 256 * items.gate_up,
                                  [&](int r) { return a.x + (it.row0 + r) * a.x_bytes; },
                               [&](int r) { return 1.f / __ldcg(a.xs + it.row0 + r); },
                               a.xq + (size_t)it.row0 * 2 * a.d);
                else
                    split_rows<4>(rows, a.f, t, 256 * items.parts,
                               [&](int r) { return a.h + (size_t)(it.row0 + r) * a.f; },
                               [&](int r) {
                                   return 1.f / split_scale(__uint_as_float(
                                                    __ldcg(a.hmax + it.row0 + r)));
                               },
                               a.hq + (size_t)it.row0 * 2 * a.f);
                __syncwarp();
                if (lane == 0)
                    add_release(&a.ctrl[it.kind == kSplitX ? kCtrlXSplit : kCtrlHSplit + it.tile]);
                continue;
            }
            const bool down = it.kind == kDown;
            const bool split = down || (W8 && a.x_split);
            const int n8 = (it.rows + 7) & ~7;
            const uint8_t* src[NT / 8];
            float inv[NT / 8];
            uint32_t have = 0;
#pragma unroll
            for (int u = 0; u < NT / 8; ++u) {
                const int r = (tid >> 4) + 8 * u;
                src[u] = nullptr;
                inv[u] = 1.f;
                if (r >= it.rows || !it.ok) continue;
                have |= 1u << u;
                if (down) {
                    const size_t row = (size_t)(it.row0 + r);
                    src[u] = Cfg::PRE ? a.hq + row * 2 * a.f
                                      : reinterpret_cast<const uint8_t*>(a.h + row * a.f);
                    if (W8) {
                        const float hs = split_scale(__uint_as_float(__ldcg(a.hmax + row)));
                        inv[u] = 1.f / hs;
                        // for the epilogue, from the group whose block is the item's first
                        if (ring.next == base && (tid & 15) == 0) s.hscale[ring_slot * NT + r] = hs;
                    }
                } else {
                    const int tok = s.list[it.row0 + r] / a.K;
                    src[u] = x_pieces ? a.xq + (size_t)tok * 2 * a.d : a.x + tok * a.x_bytes;
                    if (W8 && !Cfg::PRE && split) inv[u] = 1.f / __ldcg(a.xs + tok);
                }
                src[u] += (tid & 15) * (Cfg::PRE || !split ? 16 : !down ? 32 : W8 ? 64 : 32);
            }
            const int kb = down ? a.kb2 : a.kb1, K = down ? a.f : a.d;
            bool ok;
            if (!split)
                ok = produce_rows<W8, NT, kCopy>(s, src, inv, have, n8, base, kb, K, tid, ring);
            else if (Cfg::PRE || !down)
                ok = produce_rows<W8, NT, !W8 ? kCopy : Cfg::PRE ? kPieces : kSplit>(
                    s, src, inv, have, n8, base, kb, K, tid, ring);
            else
                ok = produce_rows<W8, NT, Cfg::PRE ? kPieces : kSplitF>(s, src, inv, have, n8, base,
                                                                        kb, K, tid, ring);
            if (!ok) {
                failed = true;
                break;
            }
            base += kb;
        }
        if (apart) group_all(!failed, group);
        if (failed && lane == 0) latch_error(a.err, CRC_ETIMEOUT);
    } else if (warp >= 4) {
        // ------------------------------------------------------ epilogue
        const int quarter = warp & 3;
        int islot = 0, acc = 0, turn = 0;
        uint32_t iphase = 0, aphase = 0;
        bool failed = false;
        while (true) {
            if (!mbar_wait_warp(&s.i_full[islot], iphase)) {
                failed = true;
                break;
            }
            const int item = s.items[islot];
            if (item < 0) break;
            const MoeItem it = moe_item<W8, NT>(a, s, items, item);
            if (Cfg::PRE && it.kind >= kSplitX) {
                __syncwarp();
                if (lane == 0) mbar_arrive(&s.i_empty[islot]);
                if (++islot == kItemRing) {
                    islot = 0;
                    iphase ^= 1;
                }
                continue;
            }
            const bool down = it.kind == kDown;
            const int slot = s.slot[it.e];
            const bool split = down || (W8 && a.x_split);
            const int n8 = (it.rows + 7) & ~7;
            // this lane's weight row: an element of f (gate in the low half of the
            // warp, up in the high half), or of d
            const int wrow = down ? it.j * 128 + quarter * 32 + lane
                                  : it.j * 64 + quarter * 16 + (lane & 15);
            const bool in = it.ok && wrow < (down ? a.d : a.f);
            float sw = 1.f;
            if (W8 && in)
                sw = down ? a.s2[slot * a.s2_stride + wrow]
                          : a.s13[slot * a.s13_stride + (lane >> 4) * a.f + wrow];
            // scales of the rows: lane l holds those of rows l, l + 32
            constexpr int RS = (NT + 31) / 32;
            float rs[RS];
            if (W8 && !down) {
#pragma unroll
                for (int u = 0; u < RS; ++u) {
                    const int r = lane + 32 * u;
                    rs[u] = r < it.rows ? __ldcg(a.xs + s.list[it.row0 + r] / a.K) : 0.f;
                }
            }
            if (!mbar_wait_warp(&s.t_full[acc], aphase)) {
                failed = true;
                break;
            }
            tc_fence_after();
            if (W8 && down) {
#pragma unroll
                for (int u = 0; u < RS; ++u) {
                    const int r = lane + 32 * u;
                    rs[u] = r < it.rows ? s.hscale[islot * NT + r] : 0.f;
                }
            }
            __syncwarp();             // the item's place is free when its scales are read
            if (lane == 0) mbar_arrive(&s.i_empty[islot]);
            if (++islot == kItemRing) {
                islot = 0;
                iphase ^= 1;
            }
            const uint32_t tb =
                tmem + (uint32_t)(acc * Cfg::COLS) + ((uint32_t)(quarter * 32) << 16);
#pragma unroll 1
            for (int c0 = 0; c0 < it.rows; c0 += 16) {
                float v[16];
                tmem_ld16f(tb + c0, v);
                if (split) {
                    float lo[16];
                    tmem_ld16f(tb + n8 + c0, lo);
                    tmem_ld_wait();
                    pin16(v);
                    pin16(lo);
#pragma unroll
                    for (int i = 0; i < 16; ++i) v[i] = fmaf(lo[i], W8 ? 0.0625f : 1.f, v[i]);
                } else {
                    tmem_ld_wait();
                    pin16(v);
                }
                if (c0 + 16 >= it.rows) {          // read whole: hand it back
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&s.t_empty[acc]);
                }
                const int n = it.rows - c0 < 16 ? it.rows - c0 : 16;
                if (W8) {
                    const float r = RS == 2 && c0 >= 32 ? rs[RS - 1] : rs[0];
#pragma unroll
                    for (int c = 0; c < 16; ++c)
                        v[c] *= sw * __shfl_sync(kFull, r, (c0 & 16) + c);
                }
                if (!down) {
                    uint32_t top[8] = {};
#pragma unroll
                    for (int c = 0; c < 16; c += 2) {
                        if (c >= n) break;
                        // low half: column c, high half: column c + 1
                        const float got =
                            __shfl_xor_sync(kFull, lane < 16 ? v[c + 1] : v[c], 16);
                        const float gate = lane < 16 ? v[c] : got, up = lane < 16 ? got : v[c + 1];
                        const float hv = __fdividef(gate, 1.f + __expf(-gate)) * up;
                        const int col = c + (lane >> 4);
                        const bool mine = in && col < n;
                        if (mine) a.h[(size_t)(it.row0 + c0 + col) * a.f + wrow] = hv;
                        if (W8)
                            top[c / 2] = mine ? __float_as_uint(hv) & 0x7fffffffu : 0u;
                    }
                    if (W8) {
                        // the largest of 16 lanes for eight columns at once: each exchange
                        // halves the columns that a lane keeps
#pragma unroll
                        for (int o = 8, m = 4; o > 1; o >>= 1, m >>= 1)
#pragma unroll
                            for (int i = 0; i < m; ++i) {
                                const bool upper = lane & o;
                                const uint32_t keep = upper ? top[i + m] : top[i];
                                const uint32_t give = upper ? top[i] : top[i + m];
                                top[i] = max(keep, __shfl_xor_sync(kFull, give, o));
                            }
                        const uint32_t m = max(top[0], __shfl_xor_sync(kFull, top[0], 1));
                        const int col = 2 * ((lane & 8 ? 4 : 0) + (lane & 4 ? 2 : 0) +
                                             (lane & 2 ? 1 : 0)) + (lane >> 4);
                        if (!(lane & 1) && col < n && m) atomicMax(a.hmax + it.row0 + c0 + col, m);
                    }
                } else {
#pragma unroll
                    for (int c = 0; c < 16; ++c) {
                        if (c >= n) break;
                        if (in) a.y[(size_t)s.list[it.row0 + c0 + c] * a.d + wrow] = v[c];
                    }
                }
            }
            acc ^= 1;
            if (acc == 0) aphase ^= 1;
            __syncwarp();
            // the last of the four warps adds for all
            if (lane == 0 && add_cta(&s.ended[turn & 3]) % 4 == 3)
                add_release(&a.ctrl[down ? kCtrlDone2 : kCtrlDone1 + it.tile]);
            ++turn;
        }
        if (failed && lane == 0) latch_error(a.err, CRC_ETIMEOUT);
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, Cfg::TMEM_COLS);
    }

    // -------------------------------------------------------- the choices' sum
    // Four elements of d of one token a thread; all loads of eight choices are under
    // way at once, and the first gates before the last y is there.
    const int quads = a.d / 4;
    const long long all = (long long)a.M * quads;
    long long i = (long long)blockIdx.x * kMoeThreads + threadIdx.x;
    int tok = i < all ? (int)(i / quads) : 0;
    Gates gates;
    if (i < all) gates.load(a, s, tok * a.K, a.K);
    if (threadIdx.x == 0) {
        const bool ok = wait_count(&a.ctrl[kCtrlDone2], (uint32_t)(tiles * a.dt));
        if (!ok) latch_error(a.err, CRC_ETIMEOUT);
        s.items[0] = ok;
    }
    __syncthreads();
    if (!s.items[0]) return;
    while (i < all) {
        const int c = (int)(i - (long long)tok * quads) * 4;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int k0 = 0; k0 < a.K; k0 += 8) {
            const int r = tok * a.K + k0;
            if (k0) gates.load(a, s, r, a.K - k0);
            float4 y[8];
#pragma unroll
            for (int k = 0; k < 8; ++k)
                y[k] = gates.have >> k & 1u
                           ? __ldcg(reinterpret_cast<const float4*>(a.y + (size_t)(r + k) * a.d + c))
                           : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                if (!(gates.have >> k & 1u)) continue;
                o.x = fmaf(gates.g[k], y[k].x, o.x);
                o.y = fmaf(gates.g[k], y[k].y, o.y);
                o.z = fmaf(gates.g[k], y[k].z, o.z);
                o.w = fmaf(gates.g[k], y[k].w, o.w);
            }
        }
        const __nv_bfloat162 p = __floats2bfloat162_rn(o.x, o.y), q = __floats2bfloat162_rn(o.z, o.w);
        uint2 w;
        w.x = *reinterpret_cast<const uint32_t*>(&p);
        w.y = *reinterpret_cast<const uint32_t*>(&q);
        *reinterpret_cast<uint2*>(a.out + (size_t)tok * a.d + c) = w;
        i += (long long)gridDim.x * kMoeThreads;
        if (i >= all) break;
        tok = (int)(i / quads);
        gates.load(a, s, tok * a.K, a.K);
    }
}

}  // namespace crc
