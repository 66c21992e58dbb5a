// 4-bit rows with group scales: bringing rows to 4 bits.
//
// A group of G columns shares scale = bf16(max / 7); a code is the quotient by that
// (rounded) scale, to the nearest whole number, two's complement, two a byte with the even
// column in the low half.  Scales lie group by group, the rows of a matrix side by side
// ([k / G][n]), as matvec4.cu's fragments read them.
//
// A warp takes 512 columns of a row at a time, 16 a lane, so a group is 2, 4 or 8 lanes; a
// CTA 32 rows, whose scales leave through shared memory as 64-byte pieces.  Bound by
// memory, 2 bytes read and half a byte written an element, beside the instructions, some eight
// an element: a layer's gate and up (64 experts, 537 MB) take 128 us, 5.3 TB/s (206 when each
// code compared its rest with half a step), one expert's 3.5.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "crc_device.cuh"
#include "crc_internal.h"
#include "pdl.cuh"

namespace crc {
namespace {

constexpr int kQThreads = 256;
constexpr int kQRows = 32, kQCols = 512;
constexpr int kRowsAWarp = kQRows / (kQThreads / 32);

inline bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

struct Quantize4Args {
    const uint16_t* x;
    uint8_t* q;
    uint16_t* scale;
    long long ldx;               // elements between rows
    int n, k;                    // rows and columns of a matrix
};

// 1.5 * 2^23 plus the whole number nearest to v / a, ties to the even one: its low bits are the
// code's.  v inv is within 2^-23 of the quotient's value, and Markstein's correction from there
// rounds it to fp32 as a division would (v - q a is exact, a >= 2^-100).  With 8 significant bits
// each, v / a is a tie exactly or at least 2^-10 away from one, so the rounding to fp32 changes no
// code.
__device__ __forceinline__ uint32_t code_bits(float v, float a, float inv) {
    const float q = v * inv;
    return __float_as_uint(fmaf(fmaf(-q, a, v), inv, q) + 12582912.f);
}
__device__ __forceinline__ float low_half(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high_half(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
// The codes of eight bf16 numbers, two a byte.
__device__ __forceinline__ uint32_t eight_codes(const uint32_t (&w)[4], float a, float inv) {
    uint32_t e[4], o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        e[i] = code_bits(low_half(w[i]), a, inv);
        o[i] = code_bits(high_half(w[i]), a, inv);
    }
    const uint32_t even = __byte_perm(__byte_perm(e[0], e[1], 0x0040),
                                      __byte_perm(e[2], e[3], 0x0040), 0x5410);
    const uint32_t odd = __byte_perm(__byte_perm(o[0], o[1], 0x0040),
                                     __byte_perm(o[2], o[3], 0x0040), 0x5410);
    return (even & 0x0f0f0f0fu) | ((odd << 4) & 0xf0f0f0f0u);
}

template <int G>
__global__ void __launch_bounds__(kQThreads) quantize_rows4_kernel(Quantize4Args a) {
    __shared__ uint16_t sc[kQCols / G][kQRows + 2];
    pdl_begin();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int r0 = blockIdx.x * kQRows, col0 = blockIdx.y * kQCols;
    const long long mat = blockIdx.z;
    const int col = col0 + lane * 16;
    uint4 u[kRowsAWarp][2];
#pragma unroll
    for (int i = 0; i < kRowsAWarp; ++i) {
        const int r = r0 + i * (kQThreads / 32) + warp;
        u[i][0] = u[i][1] = make_uint4(0, 0, 0, 0);
        if (r < a.n && col < a.k) {                 // k is a multiple of 32: both pieces or none
            const uint4* p =
                reinterpret_cast<const uint4*>(a.x + (mat * a.n + r) * a.ldx + col);
            u[i][0] = __ldcs(p);
            u[i][1] = __ldcs(p + 1);
        }
    }
#pragma unroll
    for (int i = 0; i < kRowsAWarp; ++i) {
        const int r = r0 + i * (kQThreads / 32) + warp;
        const uint32_t w[8] = {u[i][0].x, u[i][0].y, u[i][0].z, u[i][0].w,
                               u[i][1].x, u[i][1].y, u[i][1].z, u[i][1].w};
        // the largest magnitude by its bits: NaN above infinity above the rest
        uint32_t top = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            top = __vmaxu2(top, w[j] & 0x7fff7fffu);
        top = max(top & 0xffffu, top >> 16);
#pragma unroll
        for (int o = 1; o < G / 16; o <<= 1) top = max(top, __shfl_xor_sync(kFull, top, o));
        const float amax = __uint_as_float(top << 16);
        __nv_bfloat16 s = __float2bfloat16_rn(__fdiv_rn(amax, 7.f));
        if (__bfloat162float(s) == 0.f) s = __float2bfloat16_rn(1.f);
        const float af = __bfloat162float(s);
        uint32_t lo = 0, hi = 0;
        if (af >= 0x1p-100f && af < 3.e38f) {
            const float inv = __frcp_rn(af);
            lo = eight_codes({w[0], w[1], w[2], w[3]}, af, inv);
            hi = eight_codes({w[4], w[5], w[6], w[7]}, af, inv);
        } else if (af < 1.f) {
            // a tiny scale has a rest that is not exact, or no inverse: the division itself
#pragma unroll 1
            for (int j = 0; j < 8; ++j) {
                const float q0 = rintf(__fdiv_rn(__uint_as_float(w[j] << 16), af));
                const float q1 = rintf(__fdiv_rn(__uint_as_float(w[j] & 0xffff0000u), af));
                const int c0 = (int)fminf(fmaxf(q0, -7.f), 7.f);
                const int c1 = (int)fminf(fmaxf(q1, -7.f), 7.f);
                const uint32_t b = (uint32_t)(c0 & 15) | (uint32_t)(c1 & 15) << 4;
                if (j < 4)
                    lo |= b << (8 * j);
                else
                    hi |= b << (8 * j - 32);
            }
        }
        // (a scale that is infinite or NaN: codes 0, and the group stands for NaN)
        if (r < a.n && col < a.k) {
            *reinterpret_cast<uint2*>(a.q + (mat * a.n + r) * (a.k / 2) + col / 2) =
                make_uint2(lo, hi);
            if (lane % (G / 16) == 0)
                sc[lane / (G / 16)][i * (kQThreads / 32) + warp] = __bfloat16_as_ushort(s);
        }
    }
    __syncthreads();
    const int groups = a.k / G;
    for (int j = threadIdx.x; j < kQCols / G * kQRows; j += kQThreads) {
        const int g = col0 / G + j / kQRows, r = r0 + j % kQRows;
        if (g < groups && r < a.n)
            a.scale[(mat * groups + g) * a.n + r] = sc[j / kQRows][j % kQRows];
    }
}

}  // namespace
}  // namespace crc

using namespace crc;

extern "C" int crc_quantize_rows4(const uint16_t* x_dev, int64_t x_stride, int32_t matrices,
                                  int32_t n, int32_t k, int32_t group, uint8_t* out4_dev,
                                  uint16_t* scale_dev, void* stream) {
    if (matrices < 0 || n < 0 || k < 1) return CRC_EINVAL;
    if ((group != 32 && group != 64 && group != 128) || k % group != 0 || k > 32768)
        return CRC_EUNSUPPORTED;
    if (matrices > 65535 || n > (1 << 28)) return CRC_EUNSUPPORTED;
    if (x_stride < k || x_stride % 8 != 0) return CRC_EINVAL;
    if (matrices == 0 || n == 0) return CRC_OK;
    if (!x_dev || !out4_dev || !scale_dev || !aligned(x_dev, 16) || !aligned(out4_dev, 16) ||
        !aligned(scale_dev, 16))
        return CRC_EINVAL;
    Quantize4Args a;
    a.x = x_dev;
    a.q = out4_dev;
    a.scale = scale_dev;
    a.ldx = x_stride;
    a.n = n;
    a.k = k;
    const dim3 grid((unsigned)((n + kQRows - 1) / kQRows), (unsigned)((k + kQCols - 1) / kQCols),
                    (unsigned)matrices);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e;
    {
        ProfScope prof(CRC_KERNEL_QUANTIZE, st);
        auto kern = group == 32   ? quantize_rows4_kernel<32>
                    : group == 64 ? quantize_rows4_kernel<64>
                                  : quantize_rows4_kernel<128>;
        e = launch_dependent(kern, grid, kQThreads, 0, st, 1, a);
    }
    note_launch();
    return cuda_status(e);
}
