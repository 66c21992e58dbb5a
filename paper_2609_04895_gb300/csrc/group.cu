// Matrix products grouped by expert and their gradients: argument checks, tensor maps, launches.
#include <cudaTypedefs.h>

#include "crc_internal.h"
#include "group_matmul.cuh"
#include "group_weights.cuh"

namespace crc {

PFN_cuTensorMapEncodeTiled_v12000 encode_fn();      // router.cu

namespace {

inline bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

bool encode(CUtensorMap* m, CUtensorMapDataType type, int rank, const void* base,
            const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box) {
    const cuuint32_t ones[5] = {1, 1, 1, 1, 1};
    auto enc = encode_fn();
    return enc && enc(m, type, rank, const_cast<void*>(base), dims, strides, box, ones,
                      CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                      CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                      CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

constexpr int kSingleRows = 48, kGatheredRows = 40, kShortRows = 8;

constexpr CUtensorMapDataType kBf16Map = CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;

// `rows` rows of x in order; 1: four gathered.  k: columns of a row.
bool rows_map(CUtensorMap* m, bool w8, const void* x, int64_t x_rows, int k, int64_t x_stride,
              int rows) {
    const int es = w8 ? 1 : 2;
    const cuuint64_t dims[2] = {(cuuint64_t)k, (cuuint64_t)x_rows};
    const cuuint64_t strides[1] = {(cuuint64_t)x_stride * es};
    const cuuint32_t box[2] = {(cuuint32_t)(128 / es), (cuuint32_t)rows};
    return encode(m, w8 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : kBf16Map, 2, x, dims, strides, box);
}

// An expert's matrix [n][k]: `cols` of k times `rows` of n.
bool matrix_map(CUtensorMap* m, const crc_group_weights& w, int cols, int rows) {
    const bool w8 = w.weight_type == CRC_E4M3;
    const cuuint64_t es = w8 ? 1 : 2;
    const cuuint64_t dims[3] = {(cuuint64_t)w.k, (cuuint64_t)w.n, (cuuint64_t)w.N};
    const cuuint64_t strides[2] = {w.k * es, (cuuint64_t)w.w_stride};
    const cuuint32_t box[3] = {(cuuint32_t)cols, (cuuint32_t)rows, 1};
    return encode(m, w8 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : kBf16Map, 3, w.w_dev, dims, strides,
                  box);
}
// Gate and up [2][n][k] as (k, 16 rows, gate / up, n / 16, experts).
bool glu_map(CUtensorMap* m, const crc_group_weights& w) {
    const bool w8 = w.weight_type == CRC_E4M3;
    const cuuint64_t es = w8 ? 1 : 2, k = w.k, n = w.n;
    const cuuint64_t dims[5] = {k, 16, 2, n / 16, (cuuint64_t)w.N};
    const cuuint64_t strides[4] = {k * es, n * k * es, 16 * k * es, (cuuint64_t)w.w_stride};
    const cuuint32_t box[5] = {(cuuint32_t)(128 / es), 16, 2, 4, 1};
    return encode(m, w8 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : kBf16Map, 5, w.w_dev, dims, strides,
                  box);
}

template <bool W8, bool GLU, bool TW, bool Pair>
int launch_products_on(const CUtensorMap& mw, const CUtensorMap& mx, const CUtensorMap& mx8,
                       GroupArgs& a, cudaStream_t st) {
    auto kern = group_matmul_kernel<W8, GLU, TW, Pair>;
    constexpr size_t smem = GroupSmem::bytes();
    constexpr int kRows = (GLU ? 64 : 128) * (Pair ? 2 : 1);      // columns of y of a tile
    a.ftiles = (a.out + kRows - 1) / kRows;
    static PerDevice resident;                 // CTAs or pairs that fit the GPU at once
    const int fit = resident.get(current_device(), [&] {
        if (cuda_status(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                             (int)smem)))
            return 0;
        if (!Pair) return sm_count() > 0 ? sm_count() : -1;
        cudaLaunchAttribute at[1];
        at[0].id = cudaLaunchAttributeClusterDimension;
        at[0].val.clusterDim.x = 2;
        at[0].val.clusterDim.y = 1;
        at[0].val.clusterDim.z = 1;
        cudaLaunchConfig_t c = {};
        c.gridDim = dim3((unsigned)(sm_count() / 2 * 2));
        c.blockDim = dim3(kGmThreads);
        c.dynamicSmemBytes = smem;
        c.attrs = at;
        c.numAttrs = 1;
        int n = 0;
        if (cuda_status(cudaOccupancyMaxActiveClusters(&n, (const void*)kern, &c))) return 0;
        return n > 0 ? n : -1;
    });
    if (fit < 1) return CRC_ECUDA;
    cudaError_t e;
    {
        ProfScope prof(CRC_KERNEL_GROUP, st);
        e = launch_dependent(kern, dim3((unsigned)(Pair ? 2 * fit : fit)), kGmThreads, smem, st,
                             Pair ? 2 : 1, mw, mx, mx8, a);
    }
    note_launch();
    return cuda_status(e);
}

template <bool W8, bool GLU, bool TW>
int launch_products(const CUtensorMap& mw, const CUtensorMap& mx, const CUtensorMap& mx8,
                    GroupArgs& a, cudaStream_t st) {
    // CTAs by themselves for few rows an expert on average, fewer if they are gathered from long rows
    // (a pair gathers a tile's rows once, two CTAs by themselves twice).  What pairs take more than
    // CTAs by themselves, at 16 / 32 / 48 / 64 / 96 rows an expert in bf16 (in 8 bits), per cent:
    //   in order, 128 experts of 2048 x 768   2 (28) / 2 (23) / -1 (14) / -1 (14) / 2 (12)
    //             32 of 2880 x 2880         10 (12) / 10 (11) / 4 (5) / 4 (3) / -6 (-13)
    //             its gradient's rows           10 / 10 / 4 / 4 / -7
    //   gathered, gate and up, 128 of 768 x 2048   1 (1) / 2 (0) / 4 (3) / -2 (-3)
    //             64 of 1024 x 1024              2 (11) / 2 (11) / -4 (5) / -4 (6)
    //             64 of 1024 x 512 (short rows)   4 (23) / 3 (23) / -3 (13) / -3 (16)
    //             16 of 512 x 256 (short rows)  29 (33) / 25 (28) / 37 (40) / 28 (33)
    // and at 36 and 40 rows gathered 2 to 4, 128 of 1536 x 4096 and of 768 x 2048, 64 of 1024 x 2048.
    const int most = a.r.rows && a.kblocks > kShortRows ? kGatheredRows : kSingleRows;
    const bool single = (long long)a.r.E <= (long long)most * a.r.N;
    return single ? launch_products_on<W8, GLU, TW, false>(mw, mx, mx8, a, st)
                  : launch_products_on<W8, GLU, TW, true>(mw, mx, mx8, a, st);
}

int check_weights(const crc_group_weights* w) {
    if (!w || w->reserved != 0) return CRC_EINVAL;
    if (w->weight_type != CRC_BF16 && w->weight_type != CRC_E4M3) return CRC_EINVAL;
    if (w->N < 1 || w->n < 1 || w->k < 1) return CRC_EINVAL;
    if (w->glu != 0 && w->glu != 1) return CRC_EINVAL;
    const bool w8 = w->weight_type == CRC_E4M3;
    if (w->N > kGroupMaxExperts || w->n % (w->glu ? 16 : 8) || w->k % (w8 ? 16 : 8) ||
        w->n > 65536 || w->k > 65536)
        return CRC_EUNSUPPORTED;
    const int64_t bytes = (int64_t)w->n * w->k * (w->glu ? 2 : 1) * (w8 ? 1 : 2);
    if (w->w_stride % 16 || w->w_stride < bytes) return CRC_EINVAL;
    if (w->w_stride >= (1ll << 40)) return CRC_EUNSUPPORTED;
    if (!w->w_dev || !aligned(w->w_dev, 16)) return CRC_EINVAL;
    if (w8) {
        if (!w->scale_dev || !aligned(w->scale_dev, 4) || w->scale_stride % 4 ||
            w->scale_stride < (int64_t)w->n * 4 * (w->glu ? 2 : 1))
            return CRC_EINVAL;
    } else if (w->scale_dev) {
        return CRC_EINVAL;
    }
    return CRC_OK;
}

// Rows of x with `k` elements of `es` bytes, and how E rows in order take them.
int check_rows(int64_t x_stride, int64_t x_rows, const int32_t* rows, int32_t K, int64_t E, int k,
               int es) {
    if (E < 0 || x_rows < 0 || K < 1) return CRC_EINVAL;
    if (x_stride < k || x_stride * es % 16 != 0) return CRC_EINVAL;
    if (E > (1 << 30) || x_rows > (1 << 30) || x_stride > (1 << 30)) return CRC_EUNSUPPORTED;
    if (E == 0) return CRC_OK;                 // (an array of no rows may have no address)
    if (rows ? !aligned(rows, 4) : (K != 1 || x_rows < E)) return CRC_EINVAL;
    if (x_rows < 1) return CRC_EINVAL;
    return CRC_OK;
}

GroupRows group_rows(const crc_group_weights& w, const int32_t* offsets, const int32_t* rows,
                     int32_t K, int64_t x_rows, int64_t E) {
    GroupRows r = {};
    r.offsets = offsets;
    r.rows = rows;
    r.err = device_error_word();
    r.E = (int)E;
    r.N = w.N;
    r.K = K;
    r.x_rows = (int)x_rows;
    return r;
}

// crc_group_matmul; split: crc_group_matmul_split.
int group_products(const crc_group_weights* w, bool split, const void* x_dev, int64_t x_stride,
                   int64_t x_rows, const float* x_scale_dev, const int32_t* offsets_dev,
                   const int32_t* rows_dev, int32_t K, int64_t E, uint16_t* y_dev, void* stream) {
    int rc = check_weights(w);
    if (rc) return rc;
    const bool w8 = w->weight_type == CRC_E4M3;
    if (split && !w8) return CRC_EINVAL;
    const int columns = split ? 2 * w->k : w->k;
    rc = check_rows(x_stride, x_rows, rows_dev, K, E, columns, w8 ? 1 : 2);
    if (rc) return rc;
    if (w8 ? (E > 0 && !x_scale_dev) || !aligned(x_scale_dev, 4) : x_scale_dev != nullptr)
        return CRC_EINVAL;
    if (E == 0) return CRC_OK;
    if (!x_dev || !aligned(x_dev, 16) || !offsets_dev || !aligned(offsets_dev, 4) || !y_dev ||
        !aligned(y_dev, 16))
        return CRC_EINVAL;
    CUtensorMap mw, mx, mx8;
    if (!(w->glu ? glu_map(&mw, *w) : matrix_map(&mw, *w, w8 ? 128 : 64, 128)) ||
        !rows_map(&mx, w8, x_dev, x_rows, columns, x_stride, rows_dev ? 1 : kGmBoxRows) ||
        !(rows_dev || rows_map(&mx8, w8, x_dev, x_rows, columns, x_stride, kGmLastRows)))
        return CRC_ECUDA;
    if (rows_dev) mx8 = mx;                    // (not used)
    GroupArgs a = {};
    a.r = group_rows(*w, offsets_dev, rows_dev, K, x_rows, E);
    a.y = y_dev;
    a.xs = x_scale_dev;
    a.ws = w->scale_dev;
    a.ws_stride = w->scale_stride / 4;
    a.split = split;
    a.lo = w->k;
    a.kblocks = (w->k + (w8 ? 127 : 63)) / (w8 ? 128 : 64) << a.split;
    a.out = w->n;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (w8)
        return w->glu ? launch_products<true, true, false>(mw, mx, mx8, a, st)
                      : launch_products<true, false, false>(mw, mx, mx8, a, st);
    return w->glu ? launch_products<false, true, false>(mw, mx, mx8, a, st)
                  : launch_products<false, false, false>(mw, mx, mx8, a, st);
}

}  // namespace
}  // namespace crc

using namespace crc;

extern "C" {

int crc_group_matmul(const crc_group_weights* w, const void* x_dev, int64_t x_stride,
                     int64_t x_rows, const float* x_scale_dev, const int32_t* offsets_dev,
                     const int32_t* rows_dev, int32_t K, int64_t E, uint16_t* y_dev,
                     void* stream) {
    return group_products(w, false, x_dev, x_stride, x_rows, x_scale_dev, offsets_dev, rows_dev, K,
                          E, y_dev, stream);
}

int crc_group_matmul_split(const crc_group_weights* w, const uint8_t* x_dev, int64_t x_stride,
                           int64_t x_rows, const float* x_scale_dev, const int32_t* offsets_dev,
                           const int32_t* rows_dev, int32_t K, int64_t E, uint16_t* y_dev,
                           void* stream) {
    return group_products(w, true, x_dev, x_stride, x_rows, x_scale_dev, offsets_dev, rows_dev, K,
                          E, y_dev, stream);
}

int crc_group_matmul_grad(const crc_group_weights* w, const uint16_t* dy_dev,
                          const uint16_t* x_dev, int64_t x_stride, int64_t x_rows,
                          const int32_t* offsets_dev, const int32_t* rows_dev, int32_t K,
                          int64_t E, uint16_t* dx_dev, void* dw_dev, int32_t dw_type,
                          void* stream) {
    // (the matrices are read for dx only)
    crc_group_weights v;
    if (!w) return CRC_EINVAL;
    v = *w;
    if (!dx_dev && !v.w_dev) v.w_dev = reinterpret_cast<const void*>(uintptr_t(16));
    int rc = check_weights(&v);
    if (rc) return rc;
    if (v.weight_type != CRC_BF16 || v.glu) return CRC_EINVAL;
    if (dw_dev && dw_type != CRC_BF16 && dw_type != CRC_F32) return CRC_EINVAL;
    rc = check_rows(x_stride, x_rows, rows_dev, K, E, v.k, 2);
    if (rc) return rc;
    if (!aligned(dx_dev, 16) || !aligned(dw_dev, 16)) return CRC_EINVAL;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (E == 0) {                                    // no rows: every matrix's gradient is 0
        if (!dw_dev) return CRC_OK;
        return cuda_status(cudaMemsetAsync(
            dw_dev, 0, (size_t)v.N * v.n * v.k * (dw_type == CRC_F32 ? 4 : 2), st));
    }
    if (!dx_dev && !dw_dev) return CRC_OK;
    if (!dy_dev || !aligned(dy_dev, 16) || !offsets_dev || !aligned(offsets_dev, 4) ||
        (dw_dev && (!x_dev || !aligned(x_dev, 16))))
        return CRC_EINVAL;
    if (dx_dev) {
        CUtensorMap mw, mdy, mdy8;
        if (!matrix_map(&mw, v, 64, 64) || !rows_map(&mdy, false, dy_dev, E, v.n, v.n, kGmBoxRows) ||
            !rows_map(&mdy8, false, dy_dev, E, v.n, v.n, kGmLastRows))
            return CRC_ECUDA;
        GroupArgs a = {};
        a.r = group_rows(v, offsets_dev, nullptr, 1, E, E);
        a.y = dx_dev;
        a.kblocks = (v.n + 63) / 64;
        a.out = v.k;
        rc = launch_products<false, false, true>(mw, mdy, mdy8, a, st);
        if (rc) return rc;
    }
    if (!dw_dev) return CRC_OK;
    CUtensorMap mdy, mx, mdy16, mx16, mdy1, mx1, mdw;
    const bool f32 = dw_type == CRC_F32;
    const cuuint64_t es = f32 ? 4 : 2;
    const cuuint64_t dims[3] = {(cuuint64_t)v.k, (cuuint64_t)v.n, (cuuint64_t)v.N};
    const cuuint64_t strides[2] = {v.k * es, (cuuint64_t)v.n * v.k * es};
    const cuuint32_t box[3] = {f32 ? 32u : 64u, 32, 1};
    if (!rows_map(&mdy, false, dy_dev, E, v.n, v.n, kGwRows) ||
        !rows_map(&mx, false, x_dev, x_rows, v.k, x_stride, kGwRows) ||
        !rows_map(&mdy16, false, dy_dev, E, v.n, v.n, 16) ||
        !rows_map(&mx16, false, x_dev, x_rows, v.k, x_stride, 16) ||
        !rows_map(&mdy1, false, dy_dev, E, v.n, v.n, 1) ||
        !rows_map(&mx1, false, x_dev, x_rows, v.k, x_stride, 1) ||
        !encode(&mdw, f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : kBf16Map, 3, dw_dev, dims, strides,
                box))
        return CRC_ECUDA;
    GroupGradArgs a = {};
    a.r = group_rows(v, offsets_dev, rows_dev, K, x_rows, E);
    a.mtiles = (v.n + kGwM - 1) / kGwM;
    a.ntiles = (v.k + kGwN - 1) / kGwN;
    a.n = v.n;
    a.k = v.k;
    const size_t smem = GroupGradSmem::bytes();
    const bool parts = E > (f32 ? kGwPart<true> : kGwPart<false>);
    auto kern = f32 ? (parts ? group_weights_grad_kernel<true, true>
                             : group_weights_grad_kernel<true, false>)
                    : (parts ? group_weights_grad_kernel<false, true>
                             : group_weights_grad_kernel<false, false>);
    static PerDevice ready[2][2];
    const int up = ready[f32][parts].get(current_device(), [&] {
        return cuda_status(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                (int)smem)) == CRC_OK;
    });
    if (!up) return CRC_ECUDA;
    cudaError_t e;
    {
        ProfScope prof(CRC_KERNEL_GROUP, st);
        e = launch_dependent(kern, dim3((unsigned)sm_count()), kGwThreads, smem, st, 1, mdy, mx,
                             mdy16, mx16, mdy1, mx1, mdw, a);
    }
    note_launch();
    return cuda_status(e);
}

}  // extern "C"
