// Products of a few rows with matrices in 4 bits: y = W_e x for every choice of an expert
// e, W = scale * code with one bf16 scale for G columns of a row (rows4.cu writes both).
//
// Mathematics.  For a group q of columns, part = sum over it of code * x is formed first,
// exactly as products (4 by 8 significant bits) and in fp32 as a sum, and y += scale_q part
// in fp32, so no weight is rounded.  A code becomes a bf16 number by two bit operations: its
// four bits with the top one turned over, put below the exponent of 128, are 136 + code.  The
// 136 is taken off as a product of its own, -136 x, whose tile starts the group's sum (or is
// added to it) and serves both row tiles of the warp.
//
// What bounds it.  A decoded token reads its experts' codes once, so the bytes do: half a
// byte a weight and 2 / G for the scale.  At 6.8 TB/s an SM has to turn over some 47 weights a
// clock, more than scalar fp32 instructions could (about 3 a weight), so the fragments of
// mma.sync m16n8k16 are filled from the packed words in registers: the eight columns of the
// product are eight choices of the same expert.  (tcgen05 takes its operands from shared
// memory: codes would have to be widened to bf16 and written back there, 4 bytes of
// traffic for each half byte that came in, for a product that the bytes bound anyway.)
//
// A CTA takes 32, 64, 128 or 256 rows (with gate and up: half of them each), its eight warps
// 32 rows and a share of the columns each; a warp's codes and scales come by TMA into a ring
// of its own, 256 columns a time, and the shares are summed in a fixed order at the end.
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
constexpr int kBoxCols = 256;                        // columns of a stage: 128 bytes a row
constexpr int kCodeBytes = 32 * 128;                 // a stage's codes: two tiles of 16 rows
constexpr int kScaleBytes = 2 * 256;                 // and scales, at most 8 groups x 16 rows x 2
constexpr int kStageBytes = kCodeBytes + kScaleBytes;
constexpr int kMaxStages = 4;
constexpr int kMaxChoices = 8192;
constexpr int kMaxTokens = 1024;
constexpr int kMaxExperts = 256;

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
    int n, k, out;               // rows of a tile's matrix, columns, columns of y
    int glu;
    int row_warps;               // 1, 2, 4, 8; the other factor of kWarps splits the columns
    int stages;
    int by_choice;               // grid.y: choices (a choice whose expert came before leaves)
};

__device__ __forceinline__ void mma_bf16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0,
                                         uint32_t b1, const float (&c)[4]) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
        "{%8,%9}, {%10,%11,%12,%13};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(c[0]), "f"(c[1]),
          "f"(c[2]), "f"(c[3]));
}

// Codes i and i + 4 of a word (i by the shift before) as bf16 136 + code.
__device__ __forceinline__ uint32_t widen2(uint32_t w) {
    uint32_t r;
    asm("lop3.b32 %0, %1, 0x000f000f, 0x43084308, 0x6a;" : "=r"(r) : "r"(w));
    return r;
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

constexpr uint32_t kMinus136 = 0xC308C308u;          // two bf16 -136

// One warp's columns of its two row tiles for NT * 8 choices: boxes first, first + step, ...
// acc[tile][nt][4] in the fragments' order.  False if a wait ran out.
template <int G, int NT>
__device__ __forceinline__ bool warp_products(const Matvec4Args& a, const CUtensorMap* mw,
                                              const CUtensorMap* ms, uint8_t* codes,
                                              uint8_t* scales, uint64_t* full, uint32_t& turn,
                                              const uint16_t* const (&xrow)[NT], int slot, int row,
                                              int first, int step, int boxes,
                                              float (&acc)[2][NT][4]) {
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int mine = first < boxes ? (boxes - first + step - 1) / step : 0;
    const int row1 = a.glu ? row : row + 16, half1 = a.glu ? 1 : 0;
    constexpr uint32_t kBytes = kCodeBytes + 2 * 32 * (kBoxCols / G);
    const auto issue = [&](int i, uint32_t use) {
        if (lane == 0) {
            const int s = use % a.stages;
            const int box = first + i * step;
            uint8_t* c = codes + s * kCodeBytes;
            uint8_t* q = scales + s * kScaleBytes;
            const uint64_t pol = l2_evict_first_policy();
            mbar_arrive_expect_tx(&full[s], kBytes);
            tma_load_4d(c, mw, &full[s], box * 128, row, 0, slot, pol);
            tma_load_4d(c + 2048, mw, &full[s], box * 128, row1, half1, slot, pol);
            tma_load_4d(q, ms, &full[s], row, box * (kBoxCols / G), 0, slot, pol);
            tma_load_4d(q + 256, ms, &full[s], row1, box * (kBoxCols / G), half1, slot, pol);
        }
    };
    for (int i = 0; i < a.stages && i < mine; ++i) issue(i, turn + i);
    const uint32_t m136[4] = {kMinus136, kMinus136, kMinus136, kMinus136};
    const float none[4] = {0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < mine; ++i, ++turn) {
        const int s = turn % a.stages;
        const int col0 = (first + i * step) * kBoxCols;
        const int steps = min(8, (a.k - col0) / 32);
        if (!mbar_wait_warp(&full[s], (turn / a.stages) & 1)) {
            latch_error(a.err, CRC_ETIMEOUT);
            return false;
        }
        // tile rows g and g + 8: 128-byte rows, 16-byte pieces at piece ^ (row % 8)
        const uint32_t cw = smem_u32(codes + s * kCodeBytes) + g * 128 + t * 4;
        const uint32_t cs = smem_u32(scales + s * kScaleBytes) + g * 2;
        float part[2][NT][4], base[NT][4];
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            if (c < steps) {
                constexpr int kPer = G / 32;             // steps of a group
                uint32_t b[NT][4];
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    uint4 v = make_uint4(0, 0, 0, 0);
                    if (xrow[j])
                        v = __ldg(reinterpret_cast<const uint4*>(xrow[j] + col0 + c * 32 + t * 8));
                    // columns i and i + 4 of the eight, as the codes of a word lie
                    b[j][0] = __byte_perm(v.x, v.z, 0x5410);
                    b[j][1] = __byte_perm(v.x, v.z, 0x7632);
                    b[j][2] = __byte_perm(v.y, v.w, 0x5410);
                    b[j][3] = __byte_perm(v.y, v.w, 0x7632);
                }
                uint32_t lo[2][4], hi[2][4];
#pragma unroll
                for (int tile = 0; tile < 2; ++tile) {
                    const uint32_t at = cw + tile * 2048 + ((c ^ g) << 4);
                    const uint32_t w0 = lds32(at), w1 = lds32(at + 1024);
                    lo[tile][0] = widen2(w0);
                    lo[tile][1] = widen2(w1);
                    lo[tile][2] = widen2(w0 >> 4);
                    lo[tile][3] = widen2(w1 >> 4);
                    hi[tile][0] = widen2(w0 >> 8);
                    hi[tile][1] = widen2(w1 >> 8);
                    hi[tile][2] = widen2(w0 >> 12);
                    hi[tile][3] = widen2(w1 >> 12);
                }
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    if (c % kPer == 0) {
                        mma_bf16(base[j], m136, b[j][0], b[j][1], none);
                        mma_bf16(base[j], m136, b[j][2], b[j][3], base[j]);
                        mma_bf16(part[0][j], lo[0], b[j][0], b[j][1], base[j]);
                        mma_bf16(part[1][j], lo[1], b[j][0], b[j][1], base[j]);
                    } else {
                        if (c % kPer == 1)
                            mma_bf16(base[j], m136, b[j][0], b[j][1], none);
                        else
                            mma_bf16(base[j], m136, b[j][0], b[j][1], base[j]);
                        mma_bf16(base[j], m136, b[j][2], b[j][3], base[j]);
                        mma_bf16(part[0][j], lo[0], b[j][0], b[j][1], part[0][j]);
                        mma_bf16(part[1][j], lo[1], b[j][0], b[j][1], part[1][j]);
                    }
                    mma_bf16(part[0][j], hi[0], b[j][2], b[j][3], part[0][j]);
                    mma_bf16(part[1][j], hi[1], b[j][2], b[j][3], part[1][j]);
                }
                if (c % kPer == kPer - 1) {
#pragma unroll
                    for (int tile = 0; tile < 2; ++tile) {
                        const uint32_t at = cs + tile * 256 + (c / kPer) * 32;
                        const float s0 = lds_bf16(at), s1 = lds_bf16(at + 16);
#pragma unroll
                        for (int j = 0; j < NT; ++j)
#pragma unroll
                            for (int v = 0; v < 4; ++v) {
                                const float p =
                                    kPer > 1 ? part[tile][j][v] + base[j][v] : part[tile][j][v];
                                acc[tile][j][v] = fmaf(v < 2 ? s0 : s1, p, acc[tile][j][v]);
                            }
                    }
                }
            }
        }
        __syncwarp();                                  // every lane has read the stage
        if (i + a.stages < mine) issue(i + a.stages, turn + a.stages);
    }
    return true;
}

__device__ __forceinline__ float silu_up(float gate, float up) {
    return __fdividef(gate, 1.f + __expf(-gate)) * up;
}

// The products of list[at .. at + NT * 8) choices, and their outputs.
template <int G, int NT>
__device__ __forceinline__ bool choices_products(const Matvec4Args& a, const CUtensorMap* mw,
                                                 const CUtensorMap* ms, uint8_t* codes,
                                                 uint8_t* scales, float* sums, uint64_t* full,
                                                 uint32_t& turn, const uint16_t* list, int count,
                                                 int slot, int tile0) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int splits = kWarps / a.row_warps;
    const int rw = warp / splits, split = warp % splits;
    const int each = a.glu ? 16 : 32;                   // rows of y of a warp
    const uint16_t* xrow[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const int i = j * 8 + g;
        xrow[j] = i < count ? a.x + (long long)(list[i] / a.x_div) * a.ldx : nullptr;
    }
    float acc[2][NT][4] = {};
    const int boxes = (a.k + kBoxCols - 1) / kBoxCols;
    const bool ok = warp_products<G, NT>(a, mw, ms, codes, scales, full, turn, xrow, slot,
                                         (tile0 + rw) * each, split, splits, boxes, acc);
    // sums[warp][choice][32 rows]: what the warps that share the rows found
#pragma unroll
    for (int tile = 0; tile < 2; ++tile)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const int i = j * 8 + 2 * t + (v & 1), r = tile * 16 + g + (v >> 1) * 8;
                sums[(warp * NT * 8 + i) * 33 + r] = acc[tile][j][v];
            }
    __syncthreads();
    const int rows = a.row_warps * each;                // rows of y of this CTA
    for (int o = threadIdx.x; o < rows * count; o += kThreads) {
        const int i = o / rows, r = o % rows;
        const int col = tile0 * each + r;
        if (col >= a.out) continue;
        const int w0 = r / each * splits, rr = r % each;
        float v = 0.f, u = 0.f;
        for (int w = w0; w < w0 + splits; ++w) {
            v += sums[(w * NT * 8 + i) * 33 + rr];
            if (a.glu) u += sums[(w * NT * 8 + i) * 33 + rr + 16];
        }
        if (a.glu) v = silu_up(v, u);
        a.y[(long long)list[i] * a.out + col] = __bfloat16_as_ushort(__float2bfloat16_rn(v));
    }
    __syncthreads();
    return ok;
}

// NT: choices of a pass over the weights, in eights.
template <int G, int NT>
__global__ void __launch_bounds__(kThreads) matvec4_kernel(const __grid_constant__ CUtensorMap mw,
                                                           const __grid_constant__ CUtensorMap ms,
                                                           Matvec4Args a) {
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    __shared__ uint64_t full[kWarps][kMaxStages];
    __shared__ int found;
    uint8_t* smem = reinterpret_cast<uint8_t*>(
        (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const int warp = threadIdx.x >> 5;
    uint8_t* codes = smem + warp * a.stages * kCodeBytes;
    uint8_t* scales = smem + kWarps * a.stages * kCodeBytes + warp * a.stages * kScaleBytes;
    float* sums = reinterpret_cast<float*>(smem + kWarps * a.stages * kStageBytes);
    uint16_t* list = reinterpret_cast<uint16_t*>(sums + kWarps * NT * 8 * 33);
    if (threadIdx.x < kWarps * kMaxStages) mbar_init(&full[0][0] + threadIdx.x, 1);
    if (threadIdx.x == 0) {
        found = 0;
        fence_mbar_init();
        tma_prefetch_desc(&mw);
        tma_prefetch_desc(&ms);
    }
    __syncthreads();
    pdl_begin();
    // the choices of this CTA's expert.  A choice without one (grid.y's last by expert, or
    // its own by choice) has zeros for its product.
    int e = blockIdx.y;
    if (a.by_choice) {
        e = a.topk[blockIdx.y];
        bool again = false;
        for (int c = threadIdx.x; c < (int)blockIdx.y; c += kThreads) again |= a.topk[c] == e;
        if (__syncthreads_or(again)) return;            // an earlier choice of it has a CTA
    }
    if (!a.topk) {
        for (int c = threadIdx.x; c < a.E; c += kThreads) list[c] = (uint16_t)c;
        if (threadIdx.x == 0) found = a.E;
    } else {
        // in any order: a choice's result does not depend on its column of the fragments
        for (int c = threadIdx.x; c < a.E; c += kThreads) {
            const int id = a.topk[c];
            if (id == e || (id >= a.N && e >= a.N)) list[atomicAdd(&found, 1)] = (uint16_t)c;
        }
    }
    __syncthreads();
    const int count = found;
    if (count == 0) return;
    int slot = -1;
    if (e < a.N) slot = a.slot ? a.slot[e] : e;
    const int each = a.glu ? 16 : 32;
    const int tile0 = blockIdx.x * a.row_warps;
    if (slot < 0 || slot >= a.slots) {
        const int rows = a.row_warps * each;
        for (int o = threadIdx.x; o < rows * count; o += kThreads) {
            const int col = tile0 * each + o % rows;
            if (col < a.out) a.y[(long long)list[o / rows] * a.out + col] = 0;
        }
        return;
    }
    uint32_t turn = 0;
    for (int at = 0; at < count; at += NT * 8) {
        const int some = min(count - at, NT * 8);
        bool ok;
        if (NT == 1 || some <= 8)
            ok = choices_products<G, 1>(a, &mw, &ms, codes, scales, sums, full[warp], turn,
                                        list + at, some, slot, tile0);
        else if (NT == 2 || some <= 16)
            ok = choices_products<G, (NT < 2 ? 1 : 2)>(a, &mw, &ms, codes, scales, sums,
                                                       full[warp], turn, list + at, some, slot,
                                                       tile0);
        else
            ok = choices_products<G, NT>(a, &mw, &ms, codes, scales, sums, full[warp], turn,
                                         list + at, some, slot, tile0);
        if (!__syncthreads_and(ok)) return;
    }
}

size_t smem_bytes(int stages, int nt, int E) {
    return 1024 + (size_t)kWarps * stages * kStageBytes + (size_t)kWarps * nt * 8 * 33 * 4 +
           (size_t)E * 2 + 16;
}

template <int G, int NT>
int launch(const CUtensorMap& mw, const CUtensorMap& ms, const Matvec4Args& a, dim3 grid,
           cudaStream_t st) {
    auto kern = matvec4_kernel<G, NT>;
    const size_t most = smem_bytes(kMaxStages, NT, kMaxChoices);
    static PerDevice ready;
    const int up = ready.get(current_device(), [&] {
        return cuda_status(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                (int)most)) == CRC_OK;
    });
    if (!up) return CRC_ECUDA;
    cudaError_t e;
    {
        ProfScope prof(CRC_KERNEL_MATVEC4, st);
        e = launch_dependent(kern, grid, kThreads, smem_bytes(a.stages, NT, a.E), st, 1, mw, ms,
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

// Codes as (k / 2, n, gate / up, slots), a box of 128 bytes x 16 rows; scales as
// (n, k / G, gate / up, slots), 16 rows x the groups of 256 columns.
bool make_maps(CUtensorMap* mw, CUtensorMap* ms, const crc_matvec4_weights& w) {
    auto enc = encode_fn();
    if (!enc) return false;
    const cuuint64_t k2 = w.k / 2, n = w.n, groups = w.k / w.group, slots = w.slots;
    const cuuint64_t parts = w.glu ? 2 : 1;
    const cuuint32_t ones[4] = {1, 1, 1, 1};
    const cuuint64_t dw[4] = {k2, n, parts, slots};
    const cuuint64_t sw[3] = {k2, n * k2, (cuuint64_t)w.codes_stride};
    const cuuint32_t bw[4] = {128, 16, 1, 1};
    const cuuint64_t ds[4] = {n, groups, parts, slots};
    const cuuint64_t ss[3] = {n * 2, n * groups * 2, (cuuint64_t)w.scale_stride};
    const cuuint32_t bs[4] = {16, (cuuint32_t)(kBoxCols / w.group), 1, 1};
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
    if (!topk_dev && (K != 1 || w->expert_slot_dev)) return CRC_EINVAL;
    if (M == 0) return CRC_OK;
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
    a.out = w->n;
    a.glu = w->glu;
    // a grid row for every expert and one for choices without any, or for every choice
    a.by_choice = topk_dev && a.E <= a.N;
    const int groups = !topk_dev ? 1 : a.by_choice ? a.E : a.N + 1;
    const int each = a.glu ? 16 : 32;
    const int tiles = (a.n + each - 1) / each;
    const int boxes = (a.k + kBoxCols - 1) / kBoxCols;
    const int active = !topk_dev ? 1 : a.E < a.N ? a.E : a.N;
    // More rows a CTA when there are enough CTAs without (and no warp without columns)
    a.row_warps = 1;
    while (a.row_warps < kWarps &&
           (kWarps / a.row_warps > boxes ||
            (long long)active * ((tiles + 2 * a.row_warps - 1) / (2 * a.row_warps)) >=
                4ll * sm_count()))
        a.row_warps *= 2;
    const int splits = kWarps / a.row_warps;
    const int each_warp = (boxes + splits - 1) / splits;
    a.stages = each_warp < kMaxStages ? each_warp : kMaxStages;
    const dim3 grid((unsigned)((tiles + a.row_warps - 1) / a.row_warps), (unsigned)groups);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    // Choices of one expert: no more than M (or all of them without a Top-K)
    const bool few = M <= 8;
#define CRC_G(G) (few ? launch<G, 1>(mw, ms, a, grid, st) : launch<G, 4>(mw, ms, a, grid, st))
    return w->group == 32 ? CRC_G(32) : w->group == 64 ? CRC_G(64) : CRC_G(128);
#undef CRC_G
}
