// Products of ragged groups of rows with their expert's matrix, D = W_e X_e^T.
//
//   y_i = W_e x_row(i)                         (or silu(G_e x) * (U_e x), gate and up in W)
//   dx_i = W_e^T dy_i                          (TW: the matrix's rows lie across the contraction)
//
// The matrix's rows are the 256 rows (A) of a CTA pair's tcgen05.mma, the expert's rows its N
// columns, 16 to 256 of them in steps of 16: rows come in ragged numbers, so a tile is as wide
// as they are, to the next 16.  (With the rows as A, an expert's last tile of 128 or 256 would
// be half empty on average.)  TMA stages 128-byte pieces of the contraction: 128 matrix rows a
// CTA, and half of the tile's rows, gathered four at a time where they are a token's.  Two
// accumulators in TMEM, so that one is drained while the next tile's products run.  With few
// rows the matrices bound the call, and CTAs by themselves (128 matrix rows, up to 128 rows)
// leave fewer of them without a tile.
//
// 8-bit rows hold four significant bits.  Rows in two pieces (split), x = s (hi + lo), hold bf16's:
// the pieces have one scale, so both go to the same accumulator, hi and lo in turn beside the same
// piece of the matrix.  A prompt of a layer with 8-bit experts (both products and all around them;
// bf16 experts / one piece / two): 64 Qwen3-shaped tokens 193 / 113 / 162 us, 1000 234 / 152 / 203,
// 4096 327 / 256 / 340; out is off by 4.5e-2 of itself with one piece, by 3e-3 with two.
//
// Work: tiles of (expert, matrix rows, rows), in that order, dealt to the CTAs in turn: those
// running together work on the same experts and find their rows and matrices in L2.  (In equal
// shares of neighbouring tiles, each pair on experts of its own, the first product of 4096 tokens
// took 348 us, not 189.)
//
// What bounds it: up to some hundred tokens the matrices' bytes (1000 tokens of the d = 4096
// shape 466 us, 6.5 TB/s).  With a few hundred rows an expert, loads in flight: six stages of
// 32 KB (three: 253 us, four 215, five 198, six 191 for 4096 tokens' gate and up, whose bytes
// and flops take 128 and 106), and in long runs power (207 us at 1785 MHz and 1360 W).
#pragma once

#include "group.cuh"

namespace crc {

// Warps 0 weights, 1 MMA, 2 rows in order, 4-7 epilogue, 8-15 gathered rows.
constexpr int kGmThreads = 512;
constexpr int kGmGatherWarps = 8;
constexpr int kGmStages = 6;
constexpr int kGmA = 128 * 128, kGmB = 128 * 128, kGmStage = kGmA + kGmB;   // bytes, a CTA
constexpr int kGmUnit = 16, kGmTileUnits = 16;       // rows of a unit, units of a pair's tile
constexpr int kGmStaging = 2 * 32 * 256;   // two pieces of 32 rows x 128 columns of y
constexpr int kGmScales = 2 * 256 * 4;     // the scales of a tile's rows, of two tiles
// Rows of a TMA box of x in order: eight for a CTA with less than 32, which load in time what they
// hold (the second product of one token of 32 experts of 5760 x 2880, 4 of them read, 22 us with
// boxes of 32 and 12.3 now; of 128 of 1536 x 2048, 9.0 and 6.3).
constexpr int kGmBoxRows = 32, kGmLastRows = 8;

struct GroupArgs {
    GroupRows r;
    uint16_t* y;                 // [E][out]
    const float* xs;             // [x_rows] scales of e4m3 rows
    const float* ws;             // e4m3: [N][out], with gate and up [N][2][out]
    long long ws_stride;         // floats
    int kblocks;                 // 128-byte pieces of the contraction
    int split;                   // 1: e4m3 rows in two pieces, each matrix piece taken twice
    int lo;                      // elements from a row's hi to its lo
    int out;                     // columns of y
    int ftiles;                  // tiles of 256 matrix rows, 128 of a CTA by itself
};

struct GroupTile {
    int e, ft, row, rows;        // expert, tile of matrix rows, first row of x in order, rows
};

// Tiles of an expert with `count` rows.
template <bool Pair>
__device__ __forceinline__ long long group_tiles(int count, int ftiles) {
    constexpr int kRows = kGmUnit * kGmTileUnits / (Pair ? 1 : 2);
    return (long long)ftiles * ((count + kRows - 1) / kRows);
}

// Tile `i` of the call, i < cost[N]: an expert's rows in equal tiles, one after the other for
// each tile of its matrix.
template <bool Pair>
__device__ __forceinline__ GroupTile group_tile(const GroupPlan& p, int N, int ftiles,
                                                long long i) {
    constexpr int kUnits = kGmTileUnits / (Pair ? 1 : 2);
    GroupTile t;
    t.e = expert_at(p, N, i);
    const int count = p.count[t.e], units = (count + kGmUnit - 1) / kGmUnit;
    const int pieces = (units + kUnits - 1) / kUnits;
    const int in = (int)(i - p.cost[t.e]);
    const int size = (units + pieces - 1) / pieces, unit = in % pieces * size;
    t.ft = in / pieces;
    t.row = p.begin[t.e] + unit * kGmUnit;
    t.rows = min(size * kGmUnit, count - unit * kGmUnit);
    return t;
}

// The first columns of the matrix and of x that piece kb of the contraction reads; of a split row's hi
// and lo in turn.  (Behind the last column of hi, lo's begins; the matrix's are zeros there.)
template <bool W8>
__device__ __forceinline__ int w_column(const GroupArgs& a, int kb) {
    return W8 ? (kb >> a.split) * 128 : kb * 64;
}
template <bool W8>
__device__ __forceinline__ int x_column(const GroupArgs& a, int kb) {
    return w_column<W8>(a, kb) + (W8 ? (kb & a.split) * a.lo : 0);
}

// All of 128 threads; orders what they did before it before what they do after.  It has no
// limit of its own: the epilogue's warps make the same calls until one outcome is false.
__device__ __forceinline__ bool group4_all(bool ok, int id) {
    uint32_t all;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\t"
        "barrier.cta.red.and.pred q, %2, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}\n"
        : "=r"(all)
        : "r"((uint32_t)ok), "r"(id)
        : "memory");
    return all != 0;
}

__device__ __forceinline__ float gm_silu_up(float gate, float up) {
    return __fdividef(gate, 1.f + __expf(-gate)) * up;
}

// Rows that a CTA of the tile loads, of `half` that are its: those there are, to the next `unit`,
// one of them at least, so that the ring waits for it.  (What the columns behind them hold does
// not matter: a column of the product is a row's own.)
__device__ __forceinline__ int loaded_rows(const GroupTile& t, int half, int rank, int unit) {
    return (min(max(t.rows - rank * half, 1), half) + unit - 1) / unit * unit;
}

struct GroupSmem {
    static constexpr size_t bytes() {
        return 1024 + (size_t)kGmStages * kGmStage + kGmStaging + kGmScales + sizeof(GroupPlan) + 512;
    }
};

// W8: e4m3 rows and matrices.  GLU: gate and up, 16 and 16 rows of a quarter of TMEM.
// TW: the matrix is [contraction][matrix rows].  Pair: on CTA pairs, else on CTAs by themselves.
template <bool W8, bool GLU, bool TW, bool Pair>
__global__ void __launch_bounds__(kGmThreads, 1)
    group_matmul_kernel(const __grid_constant__ CUtensorMap mw,
                        const __grid_constant__ CUtensorMap mx,
                        const __grid_constant__ CUtensorMap mx8, GroupArgs a) {
    constexpr int kCtas = Pair ? 2 : 1;                // CTAs of a tile
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>(
        (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t* staging = smem + kGmStages * kGmStage;
    float* scales = reinterpret_cast<float*>(staging + kGmStaging);
    GroupPlan& plan = *reinterpret_cast<GroupPlan*>(staging + kGmStaging + kGmScales);
    uint64_t* full_bar = reinterpret_cast<uint64_t*>(
        reinterpret_cast<uint8_t*>(&plan) + (sizeof(GroupPlan) + 15) / 16 * 16);
    uint64_t* empty_bar = full_bar + kGmStages;
    uint64_t* tfull_bar = empty_bar + kGmStages;
    uint64_t* tempty_bar = tfull_bar + 2;
    uint64_t* drain_bar = tempty_bar + 2;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drain_bar + 1);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = Pair ? cluster_ctarank() : 0u;
    const bool leader = rank == 0u;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kGmStages; ++s) {
            mbar_init(&full_bar[s], 2);                // the matrix's producer and the rows'
            mbar_init(&empty_bar[s], 1 + (a.r.rows ? kGmGatherWarps : 0));
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(&tfull_bar[s], 1);
            mbar_init(&tempty_bar[s], 4 * kCtas);      // four warps of each CTA
        }
        mbar_init(drain_bar, 1);
        fence_mbar_init();
        tma_prefetch_desc(&mw);
        tma_prefetch_desc(&mx);
        tma_prefetch_desc(&mx8);
    }
    if (warp == 1) {
        if constexpr (Pair) {
            tmem_alloc_pair(tmem_slot, 512);
            tmem_relinquish_pair();
        } else {
            tmem_alloc(tmem_slot, 512);
            tmem_relinquish();
        }
    }
    pdl_begin();
    make_plan(plan, a.r, [&](int n) { return group_tiles<Pair>(n, a.ftiles); });
    tc_fence_before();
    __syncthreads();
    if constexpr (Pair) cluster_sync();   // the peer's barriers exist before any remote use
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;

    const int pair = (int)blockIdx.x / kCtas, pairs = (int)gridDim.x / kCtas;
    const long long tiles = plan.cost[a.r.N];

    if (warp == 0) {
        // ---------------------------------------------------------- matrix rows
        const uint32_t lead = elected();
        const uint64_t pol = l2_normal_policy();
        // both CTAs' loads of a stage complete on the even CTA's barrier
        const uint32_t lead_full = Pair ? cluster_map(&full_bar[0], 0u) : smem_u32(&full_bar[0]);
        int stage = 0, issued = 0;
        uint32_t phase = 0;
        bool ok = true;
        for (long long i = pair; i < tiles && ok; i += pairs) {
            const GroupTile t = group_tile<Pair>(plan, a.r.N, a.ftiles, i);
            for (int kb = 0; kb < a.kblocks; ++kb) {
                ok = __all_sync(kFull, mbar_wait_cluster(&empty_bar[stage], phase ^ 1));
                if (!ok) {
                    latch_error(a.r.err, CRC_ETIMEOUT);
                    break;
                }
                uint8_t* sa = smem + stage * kGmStage;
                if (leader && lead) mbar_arrive_expect_tx(&full_bar[stage], kCtas * kGmA);
                const uint32_t fb = lead_full + (uint32_t)(stage * 8);
                if constexpr (TW) {
                    const int f0 = (t.ft * kCtas + (int)rank) * 128;
                    tma_load_3d_of<Pair>(lead, sa, &mw, fb, f0, kb * 64, t.e, pol);
                    tma_load_3d_of<Pair>(lead, sa + 8192, &mw, fb, f0 + 64, kb * 64, t.e, pol);
                } else if constexpr (GLU) {
                    // four times 16 gate rows and the 16 up rows beside them
                    tma_load_5d_of<Pair>(lead, sa, &mw, fb, w_column<W8>(a, kb), 0, 0,
                                        (t.ft * kCtas + (int)rank) * 4, t.e, pol);
                } else {
                    tma_load_3d_of<Pair>(lead, sa, &mw, fb, w_column<W8>(a, kb),
                                        (t.ft * kCtas + (int)rank) * 128, t.e, pol);
                }
                ++issued;
                if (++stage == kGmStages) {
                    stage = 0;
                    phase ^= 1;
                }
            }
        }
        // Never leave with copies in flight (the even CTA's barriers see both CTAs'
        // loads; the odd one stays for the final cluster barrier).
        if (leader && lead) {
            int s = stage;
            uint32_t ph = phase;
            for (int k = 0; k < min(issued, kGmStages); ++k) {
                if (--s < 0) {
                    s = kGmStages - 1;
                    ph ^= 1;
                }
                if (!mbar_wait_cluster(&full_bar[s], ph)) latch_error(a.r.err, CRC_ETIMEOUT);
            }
        }
    } else if (warp == 2 && !a.r.rows) {
        // ---------------------------------------------------------- rows in order
        const uint32_t lead = elected();
        const uint64_t pol = l2_normal_policy();
        const uint32_t lead_full = Pair ? cluster_map(&full_bar[0], 0u) : smem_u32(&full_bar[0]);
        int stage = 0;
        uint32_t phase = 0;
        bool ok = true;
        for (long long i = pair; i < tiles && ok; i += pairs) {
            const GroupTile t = group_tile<Pair>(plan, a.r.N, a.ftiles, i);
            const int half = (t.rows + kGmUnit - 1) / kGmUnit * (kGmUnit / kCtas);
            const int first = t.row + (int)rank * half;                // this CTA's rows
            const int unit = half < kGmBoxRows ? kGmLastRows : kGmBoxRows;
            const int mine = loaded_rows(t, half, (int)rank, unit);
            const int all = loaded_rows(t, half, 0, unit) +
                            (Pair ? loaded_rows(t, half, 1, unit) : 0);
            for (int kb = 0; kb < a.kblocks; ++kb) {
                ok = __all_sync(kFull, mbar_wait_cluster(&empty_bar[stage], phase ^ 1));
                if (!ok) {
                    latch_error(a.r.err, CRC_ETIMEOUT);
                    break;
                }
                uint8_t* sb = smem + stage * kGmStage + kGmA;
                if (leader && lead)
                    mbar_arrive_expect_tx(&full_bar[stage], all * 128);
                const uint32_t fb = lead_full + (uint32_t)(stage * 8);
                for (int b = 0; b < mine; b += unit)
                    tma_load_2d_of<Pair>(lead, sb + b * 128, unit == kGmBoxRows ? &mx : &mx8, fb,
                                         x_column<W8>(a, kb), first + b, pol);
                if (++stage == kGmStages) {
                    stage = 0;
                    phase ^= 1;
                }
            }
        }
    } else if (warp >= 8 && a.r.rows) {
        // ---------------------------------------------------------- gathered rows
        // warp w: the four rows 4 f .., f = w, w + 8, w + 16, w + 24 of this CTA's
        const uint32_t lead = elected();
        const uint64_t pol = l2_normal_policy();
        const uint32_t lead_full = Pair ? cluster_map(&full_bar[0], 0u) : smem_u32(&full_bar[0]);
        const int w = warp - 8;
        int stage = 0;
        uint32_t phase = 0;
        bool ok = true;
        for (long long i = pair; i < tiles && ok; i += pairs) {
            const GroupTile t = group_tile<Pair>(plan, a.r.N, a.ftiles, i);
            const int half = (t.rows + kGmUnit - 1) / kGmUnit * (kGmUnit / kCtas);
            const int fours = loaded_rows(t, half, (int)rank, 4) / 4;
            const int all = loaded_rows(t, half, 0, 4) + (Pair ? loaded_rows(t, half, 1, 4) : 0);
            int mine = 0, src[4][4];
            {
                const int f = w + kGmGatherWarps * ((lane >> 2) & 3);
                if (f < fours)                          // behind the last row: that row again
                    mine = source_row(a.r, t.row + min((int)rank * half + f * 4 + (lane & 3),
                                                       t.rows - 1));
            }
#pragma unroll
            for (int q = 0; q < 16; ++q) src[q / 4][q % 4] = __shfl_sync(kFull, mine, q);
            for (int kb = 0; kb < a.kblocks; ++kb) {
                ok = __all_sync(kFull, mbar_wait_cluster(&empty_bar[stage], phase ^ 1));
                if (!ok) {
                    latch_error(a.r.err, CRC_ETIMEOUT);
                    break;
                }
                uint8_t* sb = smem + stage * kGmStage + kGmA;
                const uint32_t fb = lead_full + (uint32_t)(stage * 8);
                if (leader && w == 0 && lead)
                    mbar_arrive_expect_tx(&full_bar[stage], all * 128);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int f = w + kGmGatherWarps * q;
                    if (f < fours)
                        tma_gather4_of<Pair>(lead, sb + f * 512, &mx, fb, x_column<W8>(a, kb), src[q],
                                             pol);
                }
                // A warp without rows in this tile would hold nothing back, and miss a turn if it
                // came late by a whole one: the stage is not empty again before each has been here.
                arrive_by(&empty_bar[stage], lead);
                if (++stage == kGmStages) {
                    stage = 0;
                    phase ^= 1;
                }
            }
        }
    } else if (warp == 1) {
        // ---------------------------------------------------------- MMA
        if (leader) {
            const uint32_t lead = elected();
            int stage = 0, acc = 0, failed = 0;
            uint32_t phase = 0, acc_phase = 0;
            for (long long i = pair; i < tiles && !failed; i += pairs) {
                const GroupTile t = group_tile<Pair>(plan, a.r.N, a.ftiles, i);
                if (!__all_sync(kFull, mbar_wait_cluster(&tempty_bar[acc], acc_phase ^ 1))) {
                    latch_error(a.r.err, CRC_ETIMEOUT);
                    break;
                }
                tc_fence_after();
                const int cols = (t.rows + kGmUnit - 1) / kGmUnit * kGmUnit;
                const uint32_t idesc = W8 ? idesc_e4m3_f32_mn(128 * kCtas, cols)
                                          : idesc_bf16_f32(128 * kCtas, cols) | (TW ? kIdescMnA : 0);
                const uint32_t d_tmem = tmem_base + (uint32_t)(acc * 256);
                for (int kb = 0; kb < a.kblocks; ++kb) {
                    if (!__all_sync(kFull, mbar_wait_cluster(&full_bar[stage], phase))) {
                        latch_error(a.r.err, CRC_ETIMEOUT);
                        failed = 1;
                        break;
                    }
                    tc_fence_after();
                    const uint32_t sa = smem_u32(smem + stage * kGmStage), sb = sa + kGmA;
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk)
                        umma_by<W8, Pair>(d_tmem,
                                         TW ? sw128_mnmajor_desc(sa + kk * 2048, 8192)
                                            : sw128_kmajor_desc(sa + kk * 32),
                                         sw128_kmajor_desc(sb + kk * 32), idesc, (kb | kk) != 0,
                                         lead);
                    commit_of<Pair>(&empty_bar[stage], lead);
                    if (++stage == kGmStages) {
                        stage = 0;
                        phase ^= 1;
                    }
                }
                if (failed) break;
                commit_of<Pair>(&tfull_bar[acc], lead);
                acc ^= 1;
                if (acc == 0) acc_phase ^= 1;
            }
            if (lead) {
                if constexpr (Pair)
                    umma_commit_pair_local(drain_bar);
                else
                    umma_commit(drain_bar);
                if (!mbar_wait(drain_bar, 0)) latch_error(a.r.err, CRC_ETIMEOUT);
            }
        }
    } else if (warp >= 4 && warp < 8) {
        // ---------------------------------------------------------- epilogue
        const int quarter = warp & 3;
        const uint32_t tempty_lead = Pair ? cluster_map(&tempty_bar[0], 0u) : 0u;
        constexpr int kCols = GLU ? 64 : 128;           // columns of y of this CTA
        constexpr int kRow = kCols * 2;                 // bytes of a staged row
        int acc = 0, buf = 0;
        uint32_t acc_phase = 0;
        bool ok = true;
        for (long long i = pair; i < tiles && ok; i += pairs) {
            const GroupTile t = group_tile<Pair>(plan, a.r.N, a.ftiles, i);
            const int col0 = (t.ft * kCtas + (int)rank) * kCols;
            // this thread's rows of W: lanes t / 4 + 8 h of the quarter's two halves
            float ws[2][2] = {};
            float* xs = scales + acc * 256;
            if constexpr (W8) {
#pragma unroll
                for (int g = 0; g < 2; ++g)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int col = col0 + quarter * (kCols / 4) + (GLU ? 0 : g * 16) + h * 8 +
                                        lane / 4;
                        if (col < a.out)
                            ws[g][h] = a.ws[(long long)t.e * a.ws_stride +
                                            (GLU && g ? (long long)a.out : 0) + col];
                    }
                // (written two tiles after its last use, with that tile's barriers between)
                for (int r = quarter * 32 + lane; r < 256; r += 128)
                    xs[r] = r < t.rows ? a.xs[source_row(a.r, t.row + r)] : 0.f;
            }
            // one outcome for the four warps, which go on together
            ok = group4_all(mbar_wait_cluster(&tfull_bar[acc], acc_phase), 1);
            if (!ok) {
                latch_error(a.r.err, CRC_ETIMEOUT);
                break;
            }
            tc_fence_after();
            const uint32_t tbase =
                tmem_base + (uint32_t)(acc * 256) + ((uint32_t)(quarter * 32) << 16);
            for (int c0 = 0; c0 < t.rows; c0 += 32) {
                float v[2][16];
                tmem_ld_frag(tbase + (uint32_t)c0, v[0]);
                tmem_ld_frag(tbase + (uint32_t)c0 + (16u << 16), v[1]);
                tmem_ld_wait();
                pin16(v[0]);
                pin16(v[1]);
                if (c0 + 32 >= t.rows) {               // all read: the next tile but one may go on
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) {
                        if (leader)
                            mbar_arrive(&tempty_bar[acc]);
                        else
                            mbar_arrive_remote(tempty_lead + (uint32_t)(acc * 8));
                    }
                }
                if constexpr (W8) {
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        const float x = xs[c0 + k / 4 * 8 + (lane & 3) * 2 + (k & 1)];
                        v[0][k] *= ws[0][(k >> 1) & 1] * x;
                        v[1][k] *= ws[1][(k >> 1) & 1] * x;
                    }
                }
                if constexpr (GLU) {
#pragma unroll
                    for (int k = 0; k < 16; ++k) v[0][k] = gm_silu_up(v[0][k], v[1][k]);
                }
                const uint32_t st = smem_u32(staging) + buf * (32 * 256);
                // matrices of a store: rows 8 i .. of y and 8 columns, twice two of either
                const int r = (lane >> 4) * 8 + (lane & 7), part = (lane >> 3) & 1;
#pragma unroll
                for (int g = 0; g < (GLU ? 1 : 2); ++g)
#pragma unroll
                    for (int p = 0; p < 2; ++p) {       // rows 16 p .. of y
                        uint32_t m[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const int at = 4 * (2 * p + k / 2) + 2 * (k % 2);
                            const __nv_bfloat162 h =
                                __floats2bfloat162_rn(v[g][at], v[g][at + 1]);
                            m[k] = *reinterpret_cast<const uint32_t*>(&h);
                        }
                        const int row = p * 16 + r;
                        const int chunk = quarter * (kCols / 32) + g * 2 + part;
                        store_transposed(st + row * kRow + ((chunk ^ (row & 7)) << 4), m);
                    }
                named_sync(2, 128);
                constexpr int kChunks = kCols / 8;
#pragma unroll
                for (int k = 0; k < 32 * kChunks / 128; ++k) {
                    const int n = k * 128 + quarter * 32 + lane;
                    const int row = n / kChunks, chunk = n % kChunks;
                    const int c = c0 + row, col = col0 + chunk * 8;
                    if (c < t.rows && col < a.out &&
                        CRC_IN_BOUNDS(t.row + c < a.r.E && t.e < a.r.N, a.r.err))
                        *reinterpret_cast<uint4*>(a.y + (long long)(t.row + c) * a.out + col) =
                            *reinterpret_cast<const uint4*>(staging + buf * (32 * 256) +
                                                            row * kRow +
                                                            ((chunk ^ (row & 7)) << 4));
                }
                // (the buffer is written again behind the next piece's barrier)
                buf ^= 1;
            }
            acc ^= 1;
            if (acc == 0) acc_phase ^= 1;
        }
    }

    tc_fence_before();
    __syncthreads();
    // neither CTA leaves (or frees TMEM) while the other may still arrive on its
    // barriers or have MMAs write its TMEM
    if constexpr (Pair) cluster_sync();
    if (warp == 1) {
        tc_fence_after();
        if constexpr (Pair)
            tmem_dealloc_pair(tmem_base, 512);
        else
            tmem_dealloc(tmem_base, 512);
    }
}

}  // namespace crc
