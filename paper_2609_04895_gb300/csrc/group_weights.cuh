// Gradients of the experts' matrices, dW_e = sum over its rows of dy_i x_row(i)^T.
//
// The contraction runs over an expert's rows, so both operands lie across it (MN-major): a
// block is 64 rows of dy and x as they are in memory, 128 columns of dy (the 128 rows of
// tcgen05.mma's A) and 256 of x (its N).  An expert's last rows, when they are not sixteen, come
// four at a time by their numbers, out of range behind the last one, where TMA fills in zeros: no
// product has another expert's rows in it.  (With zeros in one operand alone their infinities would
// not vanish.  Cleared in shared memory instead, the fence behind it, which waits for copies in
// flight, cost 4%.)
//
// What bounds it: an expert has some hundred rows, so a tile's 32768 sums are written after a
// few blocks, 128 KB in fp32; the writes of dW are most of its bytes.  Tiles leave through
// shared memory by TMA.  An expert without rows has zeros.  4096 tokens x 8 (128 experts of
// 2048 x 768, fp32) take 191 us alone and 204 in a row (111 without the stores), of 146 that the
// bytes take; 613 tokens x 4, gathered (32 experts of 5760 x 2880, bf16), 249 of 160: TMA takes some
// 20 ns for four gathered rows of 64 columns, 198 us in all.  (On CTA pairs, which gather half as
// much, 311 and 207: a tile is a few blocks, and two CTAs wait for each other at each; with x as the
// 128 rows of A, stores of 64-byte rows, 295.)
//
// Work: tiles of (expert, 128 rows, 256 columns of dW), dealt to the CTAs in turn, so that
// those running together share an expert's rows in L2.
#pragma once

#include "group.cuh"

namespace crc {

// Warps 0 dy, 1 MMA, 2 x in order, 4-7 epilogue, 8-15 gathered rows of x.
constexpr int kGwThreads = 512;
constexpr int kGwRows = 64;                // rows of a block
constexpr int kGwM = 128, kGwN = 256;
constexpr int kGwA = kGwRows * kGwM * 2, kGwB = kGwRows * kGwN * 2, kGwStage = kGwA + kGwB;
constexpr int kGwChunk = kGwRows * 128;    // 64 columns of a block
// Rows that one accumulator sums, at most: the tensor cores cut a sum's low bits at each step of 16
// rows, so a sum shrinks by an error that grows with its steps.  More rows are parts of one size,
// the first in one accumulator, the others in turn in the second one, and are added in fp32.
// Error of fp32 dW in the mean square, of itself, for operands of either sign (of one sign): 256 rows
// 2.3e-7, 1024 and more 1.0e-6 (2.2e-6); in two accumulators whatever the rows 8192 had 4.4e-6
// (1.4e-5), 32768 1.9e-5 (8.3e-5).  The second accumulator is drained between parts while the tensor
// cores wait.  Us for 32 experts of 2048 x 768, two accumulators whatever the rows / parts: 1024 rows
// each 91 / 91, 2048 175 / 179, 4096 312 / 325, 8192 587 / 606.  (The last part added on the way out
// took 2% less at 2048 rows, but 3% more for all calls of fewer: 128 registers a thread.)
// bf16 dW is off by half a step of 2^-8 anyway: 16384 rows shrink a sum by 8e-5 of itself at most.
template <bool F32>
constexpr int kGwPart = F32 ? 1024 : 16384;
constexpr int kGwStages = 4;
constexpr int kGwBufs = 1;                 // pieces of 32 rows x 128 bytes of an epilogue warp
constexpr int kGwStaging = 4 * kGwBufs * 4096;

struct GroupGradArgs {
    GroupRows r;
    int mtiles, ntiles;          // of an expert's matrix [n][k]
    int n, k;
};

struct GroupGradSmem {
    static constexpr size_t bytes() {
        return 1024 + (size_t)kGwStages * kGwStage + kGwStaging + 256;
    }
};
static_assert(GroupGradSmem::bytes() + sizeof(GroupPlan) < 232448, "shared memory");

// Rows of a block that has `left` of them, to the next 16.
__device__ __forceinline__ int round16(int left) {
    return left >= kGwRows ? kGwRows : (left + 15) / 16 * 16;
}

// Rows of a part of an expert's `count`, a multiple of kGwRows where there are several parts.
template <bool F32>
__device__ __forceinline__ int part_of(int count) {
    if (count <= kGwPart<F32>) return count;
    const int parts = (count + kGwPart<F32> - 1) / kGwPart<F32>;
    return ((count + parts - 1) / parts + kGwRows - 1) / kGwRows * kGwRows;
}

// Parts: some expert may have more rows than an accumulator sums.  (Without, 249 us for 613
// tokens' gathered bf16 gradient, 254 with.)
template <bool F32, bool Parts>
__global__ void __launch_bounds__(kGwThreads, 1)
    group_weights_grad_kernel(const __grid_constant__ CUtensorMap mdy,
                              const __grid_constant__ CUtensorMap mx,
                              const __grid_constant__ CUtensorMap mdy16,
                              const __grid_constant__ CUtensorMap mx16,
                              const __grid_constant__ CUtensorMap mdy1,
                              const __grid_constant__ CUtensorMap mx1,
                              const __grid_constant__ CUtensorMap mdw, GroupGradArgs a) {
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    __shared__ GroupPlan plan;
    uint8_t* smem = reinterpret_cast<uint8_t*>(
        (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t* staging = smem + kGwStages * kGwStage;
    uint64_t* full_bar = reinterpret_cast<uint64_t*>(staging + kGwStaging);
    uint64_t* empty_bar = full_bar + kGwStages;
    uint64_t* tfull_bar = empty_bar + kGwStages;
    uint64_t* tempty_bar = tfull_bar + 2;
    uint64_t* drain_bar = tempty_bar + 2;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drain_bar + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kGwStages; ++s) {
            mbar_init(&full_bar[s], 2);                // dy and x
            mbar_init(&empty_bar[s], 1 + (a.r.rows ? 8 : 0));
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(&tfull_bar[s], 1);
            mbar_init(&tempty_bar[s], 4);
        }
        mbar_init(drain_bar, 1);
        fence_mbar_init();
        tma_prefetch_desc(&mdy);
        tma_prefetch_desc(&mx);
        tma_prefetch_desc(&mdy16);
        tma_prefetch_desc(&mx16);
        tma_prefetch_desc(&mdy1);
        tma_prefetch_desc(&mx1);
        tma_prefetch_desc(&mdw);
    }
    if (warp == 1) {
        tmem_alloc(tmem_slot, 512);
        tmem_relinquish();
    }
    pdl_begin();
    const int tiles = a.mtiles * a.ntiles;               // of an expert
    make_plan(plan, a.r, [&](int) { return (long long)tiles; });
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    const long long all = (long long)a.r.N * tiles;

    if (warp == 0 || (warp == 2 && !a.r.rows)) {
        // ---------------------------------------------------------- rows of dy, of x
        const uint64_t pol = l2_normal_policy();
        const uint32_t lead = elected();
        const bool is_x = warp == 2;
        int stage = 0, issued = 0;
        uint32_t phase = 0;
        bool ok = true;
        for (long long w = blockIdx.x; w < all && ok; w += gridDim.x) {
            const int e = (int)(w / tiles), tile = (int)(w % tiles);
            const int count = plan.count[e], row0 = plan.begin[e];
            const int col = is_x ? tile % a.ntiles * kGwN : tile / a.ntiles * kGwM;
            for (int r = 0; r < count; r += kGwRows) {
                ok = __all_sync(kFull, mbar_wait(&empty_bar[stage], phase ^ 1));
                if (!ok) {
                    latch_error(a.r.err, CRC_ETIMEOUT);
                    break;
                }
                uint8_t* s = smem + stage * kGwStage + (is_x ? kGwA : 0);
                const int left = min(count - r, kGwRows), some = round16(left);
                if (lead)
                    mbar_arrive_expect_tx(&full_bar[stage], (is_x ? kGwN : kGwM) / 64 * some * 128);
                const uint32_t fb = smem_u32(&full_bar[stage]);
                if (left == kGwRows) {
#pragma unroll
                    for (int c = 0; c < kGwN / 64; ++c)
                        if (is_x || c < kGwM / 64)
                            tma_load_2d_of<false>(lead, s + c * kGwChunk, is_x ? &mx : &mdy, fb,
                                                  col + c * 64, row0 + r, pol);
                } else {
                    int q = 0;
                    for (; q + 16 <= left; q += 16)
#pragma unroll
                        for (int c = 0; c < kGwN / 64; ++c)
                            if (is_x || c < kGwM / 64)
                                tma_load_2d_of<false>(lead, s + c * kGwChunk + q * 128,
                                                      is_x ? &mx16 : &mdy16, fb, col + c * 64,
                                                      row0 + r + q, pol);
                    for (; q < some; q += 4) {
                        int src[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) src[i] = q + i < left ? row0 + r + q + i : -1;
#pragma unroll
                        for (int c = 0; c < kGwN / 64; ++c)
                            if (is_x || c < kGwM / 64)
                                tma_gather4_of<false>(lead, s + c * kGwChunk + q * 128,
                                                      is_x ? &mx1 : &mdy1, fb, col + c * 64, src,
                                                      pol);
                    }
                }
                ++issued;
                if (++stage == kGwStages) {
                    stage = 0;
                    phase ^= 1;
                }
            }
        }
        // Never leave with copies in flight.
        if (lane == 0) {
            int s = stage;
            uint32_t ph = phase;
            for (int k = 0; k < min(issued, kGwStages); ++k) {
                if (--s < 0) {
                    s = kGwStages - 1;
                    ph ^= 1;
                }
                if (!mbar_wait(&full_bar[s], ph)) latch_error(a.r.err, CRC_ETIMEOUT);
            }
        }
    } else if (warp >= 8 && a.r.rows) {
        // ---------------------------------------------------------- gathered rows of x
        // warp w: the rows 8 w .. 8 w + 7 of a block, two fours of 64 columns at a time.  The next
        // block's are looked up while this one waits for its stage.
        const uint32_t lead = elected();
        const uint64_t pol = l2_normal_policy();
        const int at = (warp - 8) * 8;
        int stage = 0;
        uint32_t phase = 0;
        bool ok = true;
        for (long long w = blockIdx.x; w < all && ok; w += gridDim.x) {
            const int e = (int)(w / tiles), tile = (int)(w % tiles);
            const int count = plan.count[e], row0 = plan.begin[e];
            const int col = tile % a.ntiles * kGwN;
            // behind the last row: out of range
            const auto look = [&](int r) {
                const int i = r + at + (lane & 7);
                return i < count ? source_row(a.r, row0 + i) : -1;
            };
            int next = count > 0 ? look(0) : 0;
            for (int r = 0; r < count; r += kGwRows) {
                int src[2][4];
#pragma unroll
                for (int q = 0; q < 8; ++q) src[q / 4][q % 4] = __shfl_sync(kFull, next, q);
                if (r + kGwRows < count) next = look(r + kGwRows);
                ok = __all_sync(kFull, mbar_wait(&empty_bar[stage], phase ^ 1));
                if (!ok) {
                    latch_error(a.r.err, CRC_ETIMEOUT);
                    break;
                }
                const int some = round16(count - r);
                if (warp == 8 && lead)
                    mbar_arrive_expect_tx(&full_bar[stage], kGwN / 64 * some * 128);
                uint8_t* s = smem + stage * kGwStage + kGwA + at * 128;
                if (at < some)
#pragma unroll
                    for (int c = 0; c < kGwN / 64; ++c)
#pragma unroll
                        for (int q = 0; q < 2; ++q)
                            tma_gather4_of<false>(lead, s + c * kGwChunk + q * 512, &mx1, smem_u32(&full_bar[stage]),
                                           col + c * 64, src[q], pol);
                // A warp without rows in this block would hold nothing back, and miss a turn if it
                // came late by a whole one: the stage is not empty again before each has been here.
                arrive_by(&empty_bar[stage], lead);
                if (++stage == kGwStages) {
                    stage = 0;
                    phase ^= 1;
                }
            }
        }
    } else if (warp == 1) {
        // ---------------------------------------------------------- MMA
        constexpr uint32_t kIdesc = idesc_bf16_f32(kGwM, kGwN) | kIdescMnA | kIdescMnB;
        const uint32_t lead = elected();
        int stage = 0, acc = 0;
        uint32_t phase = 0, used = 0;                    // used: bit a, accumulator a's phase
        bool ok = true;
        const auto take = [&](int at) {
            ok = mbar_wait_warp(&tempty_bar[at], (used >> at & 1) ^ 1);
            if (!ok) latch_error(a.r.err, CRC_ETIMEOUT);
            tc_fence_after();
        };
        for (long long w = blockIdx.x; w < all && ok; w += gridDim.x) {
            const int count = plan.count[(int)(w / tiles)];
            if (count == 0) continue;
            take(acc);
            const int part = Parts ? part_of<F32>(count) : count;
            int cur = acc, start = 0;                    // start: the part's first row
            for (int r = 0; r < count && ok; r += kGwRows) {
                if (Parts && r - start == part) {
                    commit_by(&tfull_bar[cur], lead);
                    used ^= 1u << cur;
                    cur = acc ^ 1;
                    start = r;
                    take(cur);
                    if (!ok) break;
                }
                const uint32_t d_tmem = tmem_base + (uint32_t)(cur * 256);
                ok = mbar_wait_warp(&full_bar[stage], phase);
                if (!ok) {
                    latch_error(a.r.err, CRC_ETIMEOUT);
                    break;
                }
                const int some = min(count - r, kGwRows);
                uint8_t* s = smem + stage * kGwStage;
                tc_fence_after();
                const uint32_t sa = smem_u32(s), sb = sa + kGwA;
#pragma unroll
                for (int kk = 0; kk < kGwRows / 16; ++kk)
                    if (kk * 16 < some)
                        umma_by<false, false>(d_tmem, sw128_mnmajor_desc(sa + kk * 2048, kGwChunk),
                                     sw128_mnmajor_desc(sb + kk * 2048, kGwChunk), kIdesc,
                                     r != start || kk != 0, lead);
                commit_by(&empty_bar[stage], lead);
                if (++stage == kGwStages) {
                    stage = 0;
                    phase ^= 1;
                }
            }
            if (!ok) break;
            commit_by(&tfull_bar[cur], lead);
            used ^= 1u << cur;
            if (cur == acc) acc ^= 1;
        }
        if (lead) {
            umma_commit(drain_bar);
            if (!mbar_wait(drain_bar, 0)) latch_error(a.r.err, CRC_ETIMEOUT);
        }
    } else if (warp >= 4 && warp < 8) {
        // ---------------------------------------------------------- epilogue
        const int quarter = warp & 3;
        uint8_t* my_stage = staging + quarter * kGwBufs * 4096;
        constexpr int kCols = F32 ? 32 : 64;             // columns of a 128-byte piece
        int acc = 0, buf = 0;
        uint32_t used = 0;                               // as the MMA warp's
        const auto full = [&](int at) {
            const bool ok = mbar_wait_warp(&tfull_bar[at], used >> at & 1);
            if (!ok) latch_error(a.r.err, CRC_ETIMEOUT);
            tc_fence_after();
            return ok;
        };
        const auto release = [&](int at) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&tempty_bar[at]);
            used ^= 1u << at;
        };
        for (long long w = blockIdx.x; w < all; w += gridDim.x) {
            const int e = (int)(w / tiles), tile = (int)(w % tiles);
            const int row = tile / a.ntiles * kGwM + quarter * 32, col = tile % a.ntiles * kGwN;
            const int count = plan.count[e], part = Parts ? part_of<F32>(count) : count;
            const bool some = count > 0, several = Parts && part < count;
            const uint32_t quarters = (uint32_t)(quarter * 32) << 16;
            const uint32_t tbase = tmem_base + (uint32_t)(acc * 256) + quarters;
            if (some && !full(acc)) break;
            if (several) {
                // every part but the first is added to the first one's accumulator
                const uint32_t tbase1 = tmem_base + (uint32_t)((acc ^ 1) * 256) + quarters;
                bool ok = true;
                for (int r = part; r < count; r += part) {
                    ok = full(acc ^ 1);
                    if (!ok) break;
#pragma unroll 1
                    for (int c = 0; c < kGwN; c += 32) {
                        float v[32], u[32];
                        tmem_ld32(tbase + (uint32_t)c, v);
                        tmem_ld32(tbase1 + (uint32_t)c, u);
                        tmem_ld_wait();
                        pin16(v);
                        pin16(v + 16);
                        pin16(u);
                        pin16(u + 16);
#pragma unroll
                        for (int i = 0; i < 32; ++i) v[i] += u[i];
                        tmem_st32(tbase + (uint32_t)c, v);
                    }
                    tmem_st_wait();
                    release(acc ^ 1);
                }
                if (!ok) break;
            }
#pragma unroll 1
            for (int c = 0; c < kGwN; c += kCols) {
                uint4 q[8];
                if (some) {
                    float v[kCols];
#pragma unroll
                    for (int i = 0; i < kCols; i += 32) tmem_ld32(tbase + (uint32_t)(c + i), v + i);
                    tmem_ld_wait();
#pragma unroll
                    for (int i = 0; i < kCols; i += 16) pin16(v + i);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        uint32_t u[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            if constexpr (F32) {
                                u[i] = __float_as_uint(v[4 * j + i]);
                            } else {
                                const __nv_bfloat162 h =
                                    __floats2bfloat162_rn(v[8 * j + 2 * i], v[8 * j + 2 * i + 1]);
                                u[i] = *reinterpret_cast<const uint32_t*>(&h);
                            }
                        }
                        q[j] = make_uint4(u[0], u[1], u[2], u[3]);
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) q[j] = make_uint4(0, 0, 0, 0);
                }
                uint8_t* sbuf = my_stage + buf * 4096;
                buf = (buf + 1) % kGwBufs;
                if (lane == 0) bulk_wait_read<kGwBufs - 1>();      // the store that used sbuf is done
                __syncwarp();
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    *reinterpret_cast<uint4*>(sbuf + lane * 128 + ((j ^ (lane & 7)) << 4)) = q[j];
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0 && row < a.n && col + c < a.k &&
                    CRC_IN_BOUNDS(e < a.r.N && row >= 0, a.r.err)) {
                    tma_store_3d(&mdw, sbuf, col + c, row, e);
                    bulk_commit();
                }
            }
            if (some) {
                release(acc);
                if (!several) acc ^= 1;
            }
        }
        if (lane == 0) bulk_wait<0>();                   // every store has landed
    }

    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem_base, 512);
    }
}

}  // namespace crc
