// Row operators around the router heads: the root-mean-square norm with the
// residual's addition, its gradient, and the 8-bit form of rows.
//
//   s = x + r,  rstd = (mean s^2 + eps)^(-1/2),  y = s rstd w
//   scale = max |y| / 448,  q = e4m3(y / scale)                  (one scale a row)
//   dx = dres + rstd (v - xhat mean(v xhat)),  v = dy w,  xhat = s rstd
//   dw = sum over rows of dy xhat
//
// All three are bound by memory: a row is read once into registers, its sums
// and maxima are taken across one CTA, and what leaves is written from the
// same registers.  Sums, statistics and dw are fp32; h, s and dx are rounded
// once, to the types of their arrays.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "crc_internal.h"

namespace crc {
namespace {

constexpr float kE4m3Max = 448.0f;
constexpr int kMaxRow = 32768;       // 1024 threads x 4 groups of 8 elements

__device__ __forceinline__ float max_nan(float a, float b) {   // a NaN stays
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// Eight elements of a row <-> eight floats.
template <typename T>
struct Vec8;
template <>
struct Vec8<__nv_bfloat16> {
    uint4 v;
    __device__ __forceinline__ void load(const __nv_bfloat16* p) {
        v = *reinterpret_cast<const uint4*>(p);
    }
    __device__ __forceinline__ void get(float (&f)[8]) const {
        const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(u[i] << 16);
            f[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
        }
    }
};
template <>
struct Vec8<float> {
    float4 a, b;
    __device__ __forceinline__ void load(const float* p) {
        a = *reinterpret_cast<const float4*>(p);
        b = *reinterpret_cast<const float4*>(p + 4);
    }
    __device__ __forceinline__ void get(float (&f)[8]) const {
        f[0] = a.x, f[1] = a.y, f[2] = a.z, f[3] = a.w;
        f[4] = b.x, f[5] = b.y, f[6] = b.z, f[7] = b.w;
    }
};

__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&f)[8]) {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
        u[i] = *reinterpret_cast<const uint32_t*>(&b);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(u[0], u[1], u[2], u[3]);
}
__device__ __forceinline__ void store8(float* p, const float (&f)[8]) {
    reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
}

// Eight values to e4m3, rounded to nearest even, saturating at +-448.
__device__ __forceinline__ uint2 to_e4m3(const float (&f)[8]) {
    uint16_t h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;"
            : "=h"(h[i])
            : "f"(f[2 * i + 1]), "f"(f[2 * i]));
    return make_uint2(h[0] | ((uint32_t)h[1] << 16), h[2] | ((uint32_t)h[3] << 16));
}

// Sum (or NaN-keeping maximum) of v over the CTA, in one fixed order; every
// thread gets it.  `buf`: 32 floats, not in use by an earlier reduction that a
// thread may still be reading.
template <bool MAX>
__device__ __forceinline__ float cta_reduce(float v, float* buf) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const float u = __shfl_xor_sync(0xffffffffu, v, o);
        v = MAX ? max_nan(v, u) : v + u;
    }
    const int warps = blockDim.x >> 5;
    if (warps == 1) return v;
    const int lane = threadIdx.x & 31;
    if (lane == 0) buf[threadIdx.x >> 5] = v;
    __syncthreads();
    v = lane < warps ? buf[lane] : 0.f;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const float u = __shfl_xor_sync(0xffffffffu, v, o);
        v = MAX ? max_nan(v, u) : v + u;
    }
    return v;
}

// The row's scale and q = e4m3(y / scale).  A row of zeros has scale 1; a NaN
// or an infinity in it goes on to the scale.
__device__ __forceinline__ float row_scale(float amax) {
    return amax == 0.f ? 1.f : amax / kE4m3Max;
}
__device__ __forceinline__ uint2 quantize8(float (&y)[8], float scale) {
    if (scale >= 1e-30f) {
        const float inv = 1.f / scale;
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] *= inv;
    } else {                        // 1 / scale may overflow (or scale is a NaN)
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] /= scale;
    }
    return to_e4m3(y);
}

struct NormArgs {
    const void *x, *res;
    const __nv_bfloat16* w;
    void* res_out;
    __nv_bfloat16* h;
    uint8_t* q;
    float *scale, *rstd;
    long long ldx;                  // elements between rows of x (the other arrays are dense)
    int M, d;
    float eps;
};

// One CTA a row; a thread holds VPT groups of eight elements, group g of
// thread i at 8 (i + g blockDim).
template <typename T, int VPT>
__global__ void __launch_bounds__(1024) rms_norm_kernel(NormArgs a) {
    __shared__ float red[2][32];
    const long long row = blockIdx.x;
    const int d = a.d, nvec = d >> 3;
    const T* x = static_cast<const T*>(a.x) + row * a.ldx;
    const T* res = static_cast<const T*>(a.res) + (a.res ? row * d : 0);
    float v[VPT][8];
    Vec8<T> lx[VPT], lr[VPT];
#pragma unroll
    for (int g = 0; g < VPT; ++g) {
        const int i = threadIdx.x + g * blockDim.x;
        if (i < nvec) {
            lx[g].load(x + 8 * i);
            if (a.res) lr[g].load(res + 8 * i);
        }
    }
    float ss = 0.f;
#pragma unroll
    for (int g = 0; g < VPT; ++g) {
        const int i = threadIdx.x + g * blockDim.x;
        if (i >= nvec) continue;
        lx[g].get(v[g]);
        if (a.res) {
            float r[8];
            lr[g].get(r);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[g][j] += r[j];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) ss = fmaf(v[g][j], v[g][j], ss);
        if (a.res_out) store8(static_cast<T*>(a.res_out) + row * d + 8 * i, v[g]);
    }
    ss = cta_reduce<false>(ss, red[0]);
    const float rstd = __frsqrt_rn(ss / (float)d + a.eps);
    if (a.rstd && threadIdx.x == 0) a.rstd[row] = rstd;
    float amax = 0.f;
#pragma unroll
    for (int g = 0; g < VPT; ++g) {
        const int i = threadIdx.x + g * blockDim.x;
        if (i >= nvec) continue;
        Vec8<__nv_bfloat16> lw;
        float w[8];
        lw.load(a.w + 8 * i);
        lw.get(w);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            v[g][j] = v[g][j] * rstd * w[j];
            amax = max_nan(amax, fabsf(v[g][j]));
        }
        if (a.h) store8(a.h + row * d + 8 * i, v[g]);
    }
    if (!a.q) return;
    const float scale = row_scale(cta_reduce<true>(amax, red[1]));
    if (threadIdx.x == 0) a.scale[row] = scale;
#pragma unroll
    for (int g = 0; g < VPT; ++g) {
        const int i = threadIdx.x + g * blockDim.x;
        if (i < nvec) *reinterpret_cast<uint2*>(a.q + row * d + 8 * i) = quantize8(v[g], scale);
    }
}

// q and scale of bf16 rows, one CTA a row.
template <int VPT>
__global__ void __launch_bounds__(1024) quantize_rows_kernel(const __nv_bfloat16* x, long long ldx,
                                                             int d, uint8_t* q, float* scale) {
    __shared__ float red[32];
    const long long row = blockIdx.x;
    const int nvec = d >> 3;
    Vec8<__nv_bfloat16> l[VPT];
#pragma unroll
    for (int g = 0; g < VPT; ++g) {
        const int i = threadIdx.x + g * blockDim.x;
        if (i < nvec) l[g].load(x + row * ldx + 8 * i);
    }
    float amax = 0.f, v[8];
#pragma unroll
    for (int g = 0; g < VPT; ++g) {
        if ((int)(threadIdx.x + g * blockDim.x) >= nvec) continue;
        l[g].get(v);
#pragma unroll
        for (int j = 0; j < 8; ++j) amax = max_nan(amax, fabsf(v[j]));
    }
    const float s = row_scale(cta_reduce<true>(amax, red));
    if (threadIdx.x == 0) scale[row] = s;
#pragma unroll
    for (int g = 0; g < VPT; ++g) {
        const int i = threadIdx.x + g * blockDim.x;
        if (i >= nvec) continue;
        l[g].get(v);
        *reinterpret_cast<uint2*>(q + row * d + 8 * i) = quantize8(v, s);
    }
}

struct NormGradArgs {
    const __nv_bfloat16 *dy, *w;
    const void *s, *dres;
    const float* rstd;
    void* dx;
    float* part;                    // [gridDim.x][d] partial dw
    int M, d;
};

// A CTA takes rows blockIdx.x, + gridDim.x, ...; a thread keeps the dw sums of
// its columns in registers and writes them once, so that no order of CTAs
// changes a sum.
template <typename T, int VPT>
__global__ void __launch_bounds__(1024) rms_norm_grad_kernel(NormGradArgs a) {
    __shared__ float red[2][32];
    const int d = a.d, nvec = d >> 3;
    float dw[VPT][8] = {};
    int flip = 0;
    for (long long row = blockIdx.x; row < a.M; row += gridDim.x, flip ^= 1) {
        Vec8<__nv_bfloat16> ldy[VPT], lw[VPT];
        Vec8<T> ls[VPT], lr[VPT];
#pragma unroll
        for (int g = 0; g < VPT; ++g) {
            const int i = threadIdx.x + g * blockDim.x;
            if (i < nvec) {
                ldy[g].load(a.dy + row * d + 8 * i);
                ls[g].load(static_cast<const T*>(a.s) + row * d + 8 * i);
                if (a.dres) lr[g].load(static_cast<const T*>(a.dres) + row * d + 8 * i);
                lw[g].load(a.w + 8 * i);
            }
        }
        const float rstd = a.rstd[row];
        float dot = 0.f;
#pragma unroll
        for (int g = 0; g < VPT; ++g) {
            if ((int)(threadIdx.x + g * blockDim.x) >= nvec) continue;
            float dy[8], s[8], w[8];
            ldy[g].get(dy);
            ls[g].get(s);
            lw[g].get(w);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float xhat = s[j] * rstd;
                dot = fmaf(dy[j] * w[j], xhat, dot);
                dw[g][j] = fmaf(dy[j], xhat, dw[g][j]);
            }
        }
        const float c = cta_reduce<false>(dot, red[flip]) / (float)d;
#pragma unroll
        for (int g = 0; g < VPT; ++g) {
            const int i = threadIdx.x + g * blockDim.x;
            if (i >= nvec) continue;
            float dy[8], s[8], w[8], r[8] = {};
            ldy[g].get(dy);
            ls[g].get(s);
            lw[g].get(w);
            if (a.dres) lr[g].get(r);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float v = dy[j] * w[j] - s[j] * rstd * c;
                r[j] = fmaf(rstd, v, r[j]);
            }
            store8(static_cast<T*>(a.dx) + row * d + 8 * i, r);
        }
    }
    if (!a.part) return;
#pragma unroll
    for (int g = 0; g < VPT; ++g) {
        const int i = threadIdx.x + g * blockDim.x;
        if (i < nvec) store8(a.part + (size_t)blockIdx.x * d + 8 * i, dw[g]);
    }
}

// dw[c] = sum of the G partial rows: eight row groups a column, then their sum.
__global__ void __launch_bounds__(256) norm_dw_kernel(const float* part, int G, int d, float* dw) {
    __shared__ float sm[8][32];
    const int c = blockIdx.x * 32 + (threadIdx.x & 31), grp = threadIdx.x >> 5;
    float s = 0.f;
    if (c < d)
        for (int g = grp; g < G; g += 8) s += part[(size_t)g * d + c];
    sm[grp][threadIdx.x & 31] = s;
    __syncthreads();
    if (grp == 0 && c < d) {
#pragma unroll
        for (int k = 1; k < 8; ++k) s += sm[k][threadIdx.x];
        dw[c] = s;
    }
}

// Threads and groups a thread for rows of d elements.
struct RowShape {
    int threads, vpt;
};
RowShape row_shape(int d) {
    const int nvec = d / 8;
    int vpt = 1;
    while (vpt < 4 && nvec > 512 * vpt) vpt *= 2;
    const int t = (nvec + vpt - 1) / vpt;
    return {(t + 31) / 32 * 32, vpt};
}

inline bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

// Rows that a gradient call's CTAs share.
int grad_ctas(int M) {
    const long long most = 4ll * sm_count();
    return (int)(M < most ? M : most);
}

int check_rows(int64_t M, int32_t d) {
    if (M < 0 || d < 1) return CRC_EINVAL;
    if (d % 8 != 0 || d > kMaxRow || M > 0x7fffffffll) return CRC_EUNSUPPORTED;
    return CRC_OK;
}

#define CRC_VPT(vpt, K, ...)                                      \
    do {                                                          \
        if ((vpt) == 1) K(1, __VA_ARGS__);                        \
        else if ((vpt) == 2) K(2, __VA_ARGS__);                   \
        else K(4, __VA_ARGS__);                                   \
    } while (0)

}  // namespace
}  // namespace crc

using namespace crc;

extern "C" {

int crc_rms_norm(const void *x_dev, int64_t x_stride, const void* residual_dev,
                 const uint16_t* weight_dev, int32_t stream_type, int64_t M, int32_t d, double eps,
                 void* residual_out_dev, uint16_t* out_dev, uint8_t* out8_dev, float* scale8_dev,
                 float* rstd_dev, void* stream) {
    const int rc = check_rows(M, d);
    if (rc) return rc;
    if (stream_type != CRC_BF16 && stream_type != CRC_F32) return CRC_EINVAL;
    if (!(eps >= 0.0) || !(eps < 1e30)) return CRC_EINVAL;
    if (x_stride < d || x_stride % 8 != 0) return CRC_EINVAL;
    if ((out8_dev == nullptr) != (scale8_dev == nullptr)) return CRC_EINVAL;
    if (M == 0) return CRC_OK;
    if (!x_dev || !weight_dev) return CRC_EINVAL;
    if (!out_dev && !out8_dev && !residual_out_dev && !rstd_dev) return CRC_EINVAL;
    if (!aligned(x_dev, 16) || !aligned(residual_dev, 16) || !aligned(weight_dev, 16) ||
        !aligned(residual_out_dev, 16) || !aligned(out_dev, 16) || !aligned(out8_dev, 8) ||
        !aligned(scale8_dev, 4) || !aligned(rstd_dev, 4))
        return CRC_EINVAL;
    NormArgs a;
    a.x = x_dev;
    a.res = residual_dev;
    a.w = reinterpret_cast<const __nv_bfloat16*>(weight_dev);
    a.res_out = residual_out_dev;
    a.h = reinterpret_cast<__nv_bfloat16*>(out_dev);
    a.q = out8_dev;
    a.scale = scale8_dev;
    a.rstd = rstd_dev;
    a.ldx = x_stride;
    a.M = (int)M;
    a.d = d;
    a.eps = (float)eps;
    const RowShape sh = row_shape(d);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    {
        ProfScope prof(CRC_KERNEL_NORM, st);
#define CRC_K(V, T) rms_norm_kernel<T, V><<<(unsigned)M, sh.threads, 0, st>>>(a)
        if (stream_type == CRC_BF16)
            CRC_VPT(sh.vpt, CRC_K, __nv_bfloat16);
        else
            CRC_VPT(sh.vpt, CRC_K, float);
#undef CRC_K
    }
    note_launch();
    return cuda_status(cudaGetLastError());
}

size_t crc_rms_norm_grad_workspace_bytes(int64_t M, int32_t d) {
    if (check_rows(M, d) != CRC_OK || M < 1) return 0;
    return ((size_t)grad_ctas((int)M) * d * sizeof(float) + 255) / 256 * 256;
}

int crc_rms_norm_grad(const uint16_t* dy_dev, const void* s_dev, const uint16_t* weight_dev,
                      const float* rstd_dev, const void* dres_dev, int32_t stream_type, int64_t M,
                      int32_t d, void* dx_dev, float* dw_dev, void* workspace_dev,
                      size_t workspace_bytes, void* stream) {
    const int rc = check_rows(M, d);
    if (rc) return rc;
    if (stream_type != CRC_BF16 && stream_type != CRC_F32) return CRC_EINVAL;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (dw_dev && !aligned(dw_dev, 4)) return CRC_EINVAL;
    if (M == 0)                                      // no rows: their sum is zero
        return dw_dev ? cuda_status(cudaMemsetAsync(dw_dev, 0, (size_t)d * 4, st)) : CRC_OK;
    if (!dy_dev || !s_dev || !weight_dev || !rstd_dev || !dx_dev) return CRC_EINVAL;
    if (!aligned(dy_dev, 16) || !aligned(s_dev, 16) || !aligned(weight_dev, 16) ||
        !aligned(rstd_dev, 4) || !aligned(dres_dev, 16) || !aligned(dx_dev, 16))
        return CRC_EINVAL;
    if (dw_dev && (!workspace_dev || !aligned(workspace_dev, 256) ||
                   workspace_bytes < crc_rms_norm_grad_workspace_bytes(M, d)))
        return CRC_EINVAL;
    NormGradArgs a;
    a.dy = reinterpret_cast<const __nv_bfloat16*>(dy_dev);
    a.w = reinterpret_cast<const __nv_bfloat16*>(weight_dev);
    a.s = s_dev;
    a.dres = dres_dev;
    a.rstd = rstd_dev;
    a.dx = dx_dev;
    a.part = dw_dev ? static_cast<float*>(workspace_dev) : nullptr;
    a.M = (int)M;
    a.d = d;
    const RowShape sh = row_shape(d);
    const int G = grad_ctas((int)M);
    {
        ProfScope prof(CRC_KERNEL_NORM, st);
#define CRC_K(V, T) rms_norm_grad_kernel<T, V><<<G, sh.threads, 0, st>>>(a)
        if (stream_type == CRC_BF16)
            CRC_VPT(sh.vpt, CRC_K, __nv_bfloat16);
        else
            CRC_VPT(sh.vpt, CRC_K, float);
#undef CRC_K
    }
    note_launch();
    int e = cuda_status(cudaGetLastError());
    if (e || !dw_dev) return e;
    {
        ProfScope prof(CRC_KERNEL_NORM, st);
        norm_dw_kernel<<<(d + 31) / 32, 256, 0, st>>>(a.part, G, d, dw_dev);
    }
    note_launch();
    return cuda_status(cudaGetLastError());
}

int crc_quantize_rows(const uint16_t* x_dev, int64_t x_stride, int64_t M, int32_t d,
                      uint8_t* out8_dev, float* scale8_dev, void* stream) {
    const int rc = check_rows(M, d);
    if (rc) return rc;
    if (x_stride < d || x_stride % 8 != 0) return CRC_EINVAL;
    if (M == 0) return CRC_OK;
    if (!x_dev || !out8_dev || !scale8_dev) return CRC_EINVAL;
    if (!aligned(x_dev, 16) || !aligned(out8_dev, 8) || !aligned(scale8_dev, 4)) return CRC_EINVAL;
    const RowShape sh = row_shape(d);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const __nv_bfloat16* x = reinterpret_cast<const __nv_bfloat16*>(x_dev);
    {
        ProfScope prof(CRC_KERNEL_QUANTIZE, st);
#define CRC_K(V, dummy) \
    quantize_rows_kernel<V><<<(unsigned)M, sh.threads, 0, st>>>(x, x_stride, d, out8_dev, scale8_dev)
        CRC_VPT(sh.vpt, CRC_K, 0);
#undef CRC_K
    }
    note_launch();
    return cuda_status(cudaGetLastError());
}

}  // extern "C"
