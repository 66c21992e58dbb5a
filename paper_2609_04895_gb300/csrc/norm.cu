// Row operators around the router heads: the root-mean-square norm with the
// residual's addition, its gradient, and the 8-bit form of rows.
//
//   s = x + r,  rstd = (mean s^2 + eps)^(-1/2),  y = s rstd w
//   scale = max |y| / 448,  q = e4m3(y / scale)                  (one scale a row)
//   dx = dres + rstd (v - xhat mean(v xhat)),  v = dy w,  xhat = s rstd
//   dw = sum over rows of dy xhat
//
// All three are bound by memory: a row is read once, its sums and maxima are taken
// across the warps that share it, and what leaves is written from the same registers.
// Sums, statistics and dw are fp32; h, s and dx are rounded once, to the types of their
// arrays.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "crc_device.cuh"
#include "crc_internal.h"
#include "pdl.cuh"
#include "row_team.cuh"

namespace crc {
namespace {

constexpr float kE4m3Max = 448.0f;
constexpr int kMaxRow = 32768;       // 1024 threads x 4 groups of 8 elements

// Two fp32 operations an instruction, each rounded like its scalar form.
__device__ __forceinline__ uint64_t pack2(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpack2(uint64_t v, float& a, float& b) {
    asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v));
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
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

// What eight e4m3 numbers leave of the values they were rounded from: exact in fp32.
__device__ __forceinline__ void take_e4m3(float (&f)[8], const uint2& q) {
    const uint32_t w[2] = {q.x, q.y};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t h;
        asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)(w[i / 2] >> (i % 2 * 16))));
        float a, b;
        asm("{\n\t.reg .b16 x, y;\n\tmov.b32 {x, y}, %2;\n\tcvt.f32.f16 %0, x;\n\tcvt.f32.f16 %1, y;\n\t}"
            : "=f"(a), "=f"(b)
            : "r"(h));
        f[2 * i] -= a;
        f[2 * i + 1] -= b;
    }
}

// The row's scale.  A row of zeros has scale 1, as has one so small that the quotient is
// zero (which would make NaN of the row's zeros); a NaN or an infinity goes on to the scale.
__device__ __forceinline__ float row_scale(float amax) {
    const float s = amax / kE4m3Max;
    return s == 0.f ? 1.f : s;
}
// e4m3(y / scale) of a row's values, the quotient that of a division: v = y inv(scale) is
// off by less than two units of its last place, and Markstein's correction
// v + inv (y - v scale), the remainder in one rounding, takes it to the rounded quotient.
// (Without it, 0.045 % of normal bf16 values fell from the middle of two e4m3 values to
// the other side; with the division itself 184320 x 2880 values took 388 us, so 242.)  The
// remainder has to be exact where it decides: from v = 2^-10 on, below which q is 0, it
// is a multiple of 2^-33 ulp(scale), no less than 2^-149 for scales from 2^-93 on.  All of
// it is taken with the other sign, which leaves the sign of zeros to y.
struct RowDivide {
    float scale;
    bool plain;
    uint64_t neg_inv, same;
    __device__ __forceinline__ explicit RowDivide(float s) : scale(s) {
        plain = s >= 0x1p-80f && s < __int_as_float(0x7f800000);
        const float inv = 1.f / s;
        neg_inv = pack2(-inv, -inv);
        same = pack2(s, s);
    }
    __device__ __forceinline__ uint2 operator()(float (&y)[8]) const {
        if (plain) {
#pragma unroll
            for (int i = 0; i < 8; i += 2)
                asm("{\n\t.reg .b64 p, v;\n\tmov.b64 p, {%0, %1};\n\tmul.rn.f32x2 v, p, %2;\n\t"
                    "fma.rn.f32x2 p, v, %3, p;\n\tfma.rn.f32x2 p, p, %2, v;\n\t"
                    "mov.b64 {%0, %1}, p;\n\t}"
                    : "+f"(y[i]), "+f"(y[i + 1])
                    : "l"(neg_inv), "l"(same));
        } else {                    // 1 / scale may overflow, or scale is not finite
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] /= scale;
        }
        uint2 q = to_e4m3(y);
        if (plain) q.x ^= 0x80808080u, q.y ^= 0x80808080u;
        return q;
    }
};

// Largest magnitude of eight bf16 with m's, two at a time; a NaN stays.
__device__ __forceinline__ __nv_bfloat162 max_abs8(__nv_bfloat162 m, const uint4& v) {
    const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t a = u[i] & 0x7fff7fffu;
        m = __hmax2_nan(m, *reinterpret_cast<const __nv_bfloat162*>(&a));
    }
    return m;
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
    int warps;                      // of a row
    float eps;
};

// A few warps a row, one CTA for one or more rows; a thread holds VPT groups of
// eight elements, group g of thread i at 8 (i + g threads).  Bound by memory, behind two
// reductions a row: 4097 x 2880 fp32 rows with all outputs 29 us, 6.1 TB/s; 8192 x 2048
// bf16 26 us, 5.8 TB/s.
template <typename T, int VPT, int THREADS>
__global__ void __launch_bounds__(THREADS) rms_norm_kernel(NormArgs a) {
    __shared__ float red[2][32];
    pdl_begin();
    const RowTeam team(a.warps);
    const long long row = (long long)blockIdx.x * (blockDim.x / team.threads) + team.id;
    if (row >= a.M) return;
    const int d = a.d, nvec = d >> 3;
    const T* x = static_cast<const T*>(a.x) + row * a.ldx;
    const T* res = static_cast<const T*>(a.res) + (a.res ? row * d : 0);
    float v[VPT][8];
    Vec8<T> lx[VPT], lr[VPT];
#pragma unroll
    for (int g = 0; g < VPT; ++g) {
        const int i = team.thread + g * team.threads;
        if (i < nvec) {
            lx[g].load(x + 8 * i);
            if (a.res) lr[g].load(res + 8 * i);
        }
    }
    float ss = 0.f;
#pragma unroll
    for (int g = 0; g < VPT; ++g) {
        const int i = team.thread + g * team.threads;
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
    ss = row_reduce<false>(ss, red[0], team);
    const float rstd = __frsqrt_rn(ss / (float)d + a.eps);
    if (a.rstd && team.thread == 0) a.rstd[row] = rstd;
    float amax = 0.f;
#pragma unroll
    for (int g = 0; g < VPT; ++g) {
        const int i = team.thread + g * team.threads;
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
    const float scale = row_scale(row_reduce<true>(amax, red[1], team));
    if (team.thread == 0) a.scale[row] = scale;
    const RowDivide divide(scale);
#pragma unroll
    for (int g = 0; g < VPT; ++g) {
        const int i = team.thread + g * team.threads;
        if (i < nvec) *reinterpret_cast<uint2*>(a.q + row * d + 8 * i) = divide(v[g]);
    }
}

// q and scale of bf16 rows, the same division of a row.  CTAs stay and take row after
// row, the next on its way while a row is reduced: there is so little to do for a
// row that a CTA for every two of 2880 elements took 324 us where this took 235, and takes
// 242 with the quotient of a division (184320 rows, 6.6 TB/s).
// Split: a row in two pieces, d elements of hi and d of lo, hi = e4m3(x / s) and lo = e4m3(x / s -
// hi) with a power of two s.  hi has four significant bits of x's eight and the rest no more than
// four, so lo is exact where it is not below e4m3's smallest steps (2^-9).
template <bool Split, int VPT, int THREADS>
__global__ void __launch_bounds__(THREADS)
    quantize_rows_kernel(const __nv_bfloat16* x, long long ldx, int M, int d, int warps, uint8_t* q,
                         float* scale) {
    __shared__ float red[2][32];
    pdl_begin();
    const RowTeam team(warps);
    const int rows = blockDim.x / team.threads, nvec = d >> 3;
    const long long step = (long long)gridDim.x * rows;
    long long row = (long long)blockIdx.x * rows + team.id;
    Vec8<__nv_bfloat16> cur[VPT], nxt[VPT];
    auto load = [&](Vec8<__nv_bfloat16>(&l)[VPT], long long r) {
        if (r >= M) return;
#pragma unroll
        for (int g = 0; g < VPT; ++g) {
            const int i = team.thread + g * team.threads;
            if (i < nvec) l[g].load(x + r * ldx + 8 * i);
        }
    };
    auto take = [&](Vec8<__nv_bfloat16>(&l)[VPT], float* buf) {       // the row held by l
        __nv_bfloat162 m = __floats2bfloat162_rn(0.f, 0.f);
#pragma unroll
        for (int g = 0; g < VPT; ++g)
            if (team.thread + g * team.threads < nvec) m = max_abs8(m, l[g].v);
        const float amax = max_nan(__low2float(m), __high2float(m));
        const float most = row_reduce<true>(amax, buf, team);
        const float s = Split ? split_scale(most) : row_scale(most);
        if (team.thread == 0) scale[row] = s;
        if constexpr (Split) {
            const float inv = 1.f / s;                  // s is 2^-126 .. 2^120
#pragma unroll
            for (int g = 0; g < VPT; ++g) {
                const int i = team.thread + g * team.threads;
                if (i >= nvec) continue;
                float v[8];
                l[g].get(v);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] *= inv;
                uint2* to = reinterpret_cast<uint2*>(q + row * 2 * d + 8 * i);
                const uint2 hi = to_e4m3(v);
                take_e4m3(v, hi);
                to[0] = hi;
                to[nvec] = to_e4m3(v);
            }
            return;
        }
        const RowDivide divide(s);
#pragma unroll
        for (int g = 0; g < VPT; ++g) {
            const int i = team.thread + g * team.threads;
            if (i >= nvec) continue;
            float v[8];
            l[g].get(v);
            *reinterpret_cast<uint2*>(q + row * d + 8 * i) = divide(v);
        }
    };
    // Two rows a turn: a copy from one's registers to the other's would wait for the row
    // on its way (293 us).
    load(cur, row);
    while (row < M) {
        load(nxt, row + step);
        take(cur, red[0]);
        row += step;
        if (row >= M) break;
        load(cur, row + step);
        take(nxt, red[1]);
        row += step;
    }
}

constexpr int kMaxGradStages = 8;
constexpr int kMaxGradTeams = 8;
constexpr int kGradRing = 216 * 1024;          // at most, of an SM

// `bytes` contiguous bytes (a multiple of 16, both ends 16-byte aligned) to shared
// memory, completing on bar.
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes,
                                          uint64_t* bar) {
    asm volatile(
        "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
            smem_u32(dst)),
        "l"(reinterpret_cast<uint64_t>(src)), "r"(bytes), "r"(smem_u32(bar))
        : "memory");
}

struct NormGradArgs {
    const __nv_bfloat16 *dy, *w;
    const void *s, *dres;
    const float* rstd;
    void* dx;
    float* part;                    // [gridDim.x][d] partial dw
    uint32_t* err;
    int M, d;
    int warps;                      // of a row
    int stages, stage_bytes;        // of a team's ring
};

// Teams of warps, one or more a CTA, take row after row.  A thread keeps the dw sums of
// its columns in registers; at the end a CTA adds its teams' up and writes one row of
// partial sums, so that no order of CTAs changes a sum.  CTAs of 256 threads, four an SM:
// one of 1024 has a quarter of the partial sums and took 30.0 us where these take 26.5
// (8000 x 2048 bf16); short rows share one (8000 x 512: 14.1 us with a CTA a row, 10.1 so).
//
// The rows come through a ring in shared memory, whole rows by asynchronous bulk
// copies: the bytes on the way then cost no registers.  (With the next row in registers
// two CTAs of 256 threads fit an SM: 8000 x 2048 bf16 took 29 us without dw.)  A stage
// is filled again one row after its own: by then every thread has used all that it
// read of it.  RING false: rows too wide for two stages, read straight to registers.
template <typename T, int VPT, int THREADS, bool RING, bool TEAMS>
__global__ void __launch_bounds__(THREADS, VPT == 1 ? 2 : 1) rms_norm_grad_kernel(NormGradArgs a) {
    extern __shared__ __align__(128) uint8_t smem[];
    pdl_begin();
    __shared__ float red[2][32];
    __shared__ __align__(8) uint64_t bars[TEAMS ? kMaxGradTeams : 1][kMaxGradStages];
    __shared__ uint32_t lost[2][TEAMS ? kMaxGradTeams : 1];    // row_tell's, by turns
    const RowTeam team = TEAMS ? RowTeam(a.warps) : RowTeam();
    const int d = a.d, nvec = d >> 3, teams = TEAMS ? blockDim.x / team.threads : 1;
    const long long first = (long long)blockIdx.x * teams + team.id, step = (long long)gridDim.x * teams;
    uint8_t* ring = smem + (size_t)team.id * a.stages * a.stage_bytes;
    uint64_t* full = bars[team.id];
    const uint32_t dy_bytes = 2u * d, s_bytes = (uint32_t)sizeof(T) * d;
    const uint32_t row_bytes = dy_bytes + s_bytes + (a.dres ? s_bytes : 0u);
    auto fill = [&](int stage, long long row) {            // one thread
        uint8_t* at = ring + (size_t)stage * a.stage_bytes;
        mbar_arrive_expect_tx(&full[stage], row_bytes);
        bulk_load(at, a.dy + row * d, dy_bytes, &full[stage]);
        bulk_load(at + dy_bytes, static_cast<const T*>(a.s) + row * d, s_bytes, &full[stage]);
        if (a.dres)
            bulk_load(at + dy_bytes + s_bytes, static_cast<const T*>(a.dres) + row * d, s_bytes,
                      &full[stage]);
    };
    if constexpr (RING) {
        if (team.thread == 0) {
            lost[0][team.id] = lost[1][team.id] = 0u;
            for (int i = 0; i < a.stages; ++i) mbar_init(&full[i], 1);
            fence_mbar_init();
            long long row = first;
            for (int i = 0; i < a.stages && row < a.M; ++i, row += step) fill(i, row);
        }
    }
    uint64_t dw[VPT][4] = {};          // pairs of neighbouring columns
    Vec8<__nv_bfloat16> lw[VPT];
#pragma unroll
    for (int g = 0; g < VPT; ++g) {
        const int i = team.thread + g * team.threads;
        if (i < nvec) lw[g].load(a.w + 8 * i);
    }
    if constexpr (RING) __syncthreads();
    const float inv_d = 1.f / (float)d;
    int flip = 0, stage = 0;
    uint32_t phase = 0;
    bool arrived = true;
    for (long long row = first; row < a.M; row += step, flip ^= 1) {
        const float rstd = a.rstd[row];
        const __nv_bfloat16* dyp = a.dy + row * d;
        const T* sp = static_cast<const T*>(a.s) + row * d;
        const T* rp = static_cast<const T*>(a.dres) + (a.dres ? row * d : 0);
        if constexpr (RING) {
            arrived = row_tell(mbar_wait(&full[stage], phase), &lost[flip][team.id]);
            const uint8_t* at = ring + (size_t)stage * a.stage_bytes;
            dyp = reinterpret_cast<const __nv_bfloat16*>(at);
            sp = reinterpret_cast<const T*>(at + dy_bytes);
            rp = reinterpret_cast<const T*>(at + dy_bytes + s_bytes);
        }
        Vec8<__nv_bfloat16> ldy[VPT];
        Vec8<T> ls[VPT], lr[VPT];
#pragma unroll
        for (int g = 0; g < VPT; ++g) {
            const int i = team.thread + g * team.threads;
            if (i >= nvec) continue;
            ldy[g].load(dyp + 8 * i);
            ls[g].load(sp + 8 * i);
            if (a.dres) lr[g].load(rp + 8 * i);
        }
        const uint64_t r2 = pack2(rstd, rstd);
        uint64_t dot2 = 0;
#pragma unroll
        for (int g = 0; g < VPT; ++g) {
            if (team.thread + g * team.threads >= nvec) continue;
            float dy[8], s[8], w[8];
            ldy[g].get(dy);
            ls[g].get(s);
            lw[g].get(w);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint64_t y2 = pack2(dy[2 * j], dy[2 * j + 1]);
                const uint64_t xhat = mul2(pack2(s[2 * j], s[2 * j + 1]), r2);
                dot2 = fma2(mul2(y2, pack2(w[2 * j], w[2 * j + 1])), xhat, dot2);
                dw[g][j] = fma2(y2, xhat, dw[g][j]);
            }
        }
        float dot, dot_odd;
        unpack2(dot2, dot, dot_odd);
        dot += dot_odd;
        const float c = row_reduce<false>(dot, red[flip], team) * inv_d;
        const uint64_t k2 = pack2(-rstd * c, -rstd * c);
        if constexpr (RING) {
            arrived = row_all(arrived, &lost[flip][team.id], team);
            if (!arrived) {
                // all of the team leave here, none with a copy on its way: rows up to
                // stages - 2 ahead are asked for, one more at the first
                const int asked = a.stages - (row != first);
                for (int i = 0; i < asked && row + i * step < a.M; ++i) {
                    (void)mbar_wait(&full[stage], phase);
                    if (++stage == a.stages) {
                        stage = 0;
                        phase ^= 1;
                    }
                }
                break;
            }
            // every thread of the team is past the row before this one
            const int before = (stage ? stage : a.stages) - 1;
            const long long next = row + (a.stages - 1) * step;
            if (team.thread == 0 && row != first && next < a.M) fill(before, next);
            if (++stage == a.stages) {
                stage = 0;
                phase ^= 1;
            }
        }
#pragma unroll
        for (int g = 0; g < VPT; ++g) {
            const int i = team.thread + g * team.threads;
            if (i >= nvec) continue;
            float dy[8], s[8], w[8], r[8] = {};
            ldy[g].get(dy);
            ls[g].get(s);
            lw[g].get(w);
            if (a.dres) lr[g].get(r);
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                // dres + rstd (dy w - s rstd c)
                const uint64_t v = fma2(pack2(s[j], s[j + 1]), k2,
                                        mul2(pack2(dy[j], dy[j + 1]), pack2(w[j], w[j + 1])));
                unpack2(fma2(r2, v, pack2(r[j], r[j + 1])), r[j], r[j + 1]);
            }
            store8(static_cast<T*>(a.dx) + row * d + 8 * i, r);
        }
    }
    if (!arrived) latch_error(a.err, CRC_ETIMEOUT);
    if (!a.part) return;
    // the teams' sums, in order, through the ring's memory; one team writes its own
    float* sums = reinterpret_cast<float*>(smem);
    if (teams > 1) __syncthreads();    // every row is through the ring
#pragma unroll
    for (int g = 0; g < VPT; ++g) {
        const int i = team.thread + g * team.threads;
        if (i >= nvec) continue;
        float f[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) unpack2(dw[g][j], f[2 * j], f[2 * j + 1]);
        store8(teams > 1 ? sums + (size_t)team.id * d + 8 * i : a.part + (size_t)blockIdx.x * d + 8 * i,
               f);
    }
    if (teams == 1) return;
    __syncthreads();
    for (int i = 4 * threadIdx.x; i < d; i += 4 * blockDim.x) {
        float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int r = 0; r < teams; ++r) {
            const float4 v = *reinterpret_cast<const float4*>(sums + (size_t)r * d + i);
            t.x += v.x, t.y += v.y, t.z += v.z, t.w += v.w;
        }
        *reinterpret_cast<float4*>(a.part + (size_t)blockIdx.x * d + i) = t;
    }
}

// dw[c] = sum of the G partial rows: 32 row groups a column, then their sum.
__global__ void __launch_bounds__(1024) norm_dw_kernel(const float* part, int G, int d, float* dw) {
    __shared__ float sm[32][33];
    pdl_begin();                      // the partial rows are written
    const int lane = threadIdx.x & 31, grp = threadIdx.x >> 5;
    const int c = blockIdx.x * 32 + lane;
    float s = 0.f;
    if (c < d) {
#pragma unroll 8
        for (int g = grp; g < G; g += 32) s += __ldcg(part + (size_t)g * d + c);
    }
    sm[grp][lane] = s;
    __syncthreads();
    s = sm[lane][grp];                 // column grp of this block
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (lane == 0 && blockIdx.x * 32 + grp < d) dw[blockIdx.x * 32 + grp] = s;
}

// How a call's rows are divided: warps and groups of eight a thread for a row,
// rows a CTA.
struct RowShape {
    int warps, vpt, rows;
    int threads() const { return 32 * warps * rows; }
    unsigned grid(long long M) const { return (unsigned)((M + rows - 1) / rows); }
};
RowShape row_shape(int d, long long M, int most) {
    const int nvec = d / 8;
    // Few rows: one group a thread, the shortest way through a row.  Many: up to
    // `most`, which leaves fewer threads to a reduction and more loads to each.
    int vpt = M <= 4 * sm_count() ? 1 : most;
    if (nvec > 512 * vpt) vpt = nvec > 1024 ? 4 : 2;
    while (vpt > 1 && nvec <= 32 * (vpt - 1)) --vpt;
    const int warps = (nvec + 32 * vpt - 1) / (32 * vpt);
    return {warps, vpt, warps < 8 ? 8 / warps : 1};
}
// A gradient's rows, through rings of three or more (stages 0: none); 8000 x 2048 bf16,
// us without dw, four teams an SM: three stages 23.5, two 27.
struct GradShape : RowShape {
    int stages, stage_bytes;
    int smem() const { return rows * stages * stage_bytes; }
};
GradShape grad_shape(int d, int elem, bool dres) {
    const int nvec = d / 8;
    GradShape g;
    g.vpt = nvec <= 512 ? 1 : nvec <= 1024 ? 2 : 4;
    g.warps = (nvec + 32 * g.vpt - 1) / (32 * g.vpt);
    g.stage_bytes = (d * (2 + elem * (dres ? 2 : 1)) + 127) / 128 * 128;
    g.rows = 1;
    g.rows = g.warps < 8 ? 8 / g.warps : 1;                      // teams
    const int cta = g.rows * g.stage_bytes;                      // bytes of a stage of all teams
    g.stages = 36 * 1024 / cta;
    g.stages = g.stages < 3 ? 3 : g.stages < kMaxGradStages ? g.stages : kMaxGradStages;
    if (g.stages * cta > kGradRing / 2) {                        // two CTAs an SM, or one
        g.stages = kGradRing / 2 / cta;
        if (g.stages < 2) g.stages = kGradRing / cta;
        if (g.stages < 2) g.stages = 0;
        if (g.stages > 4) g.stages = 4;
    }
    return g;
}

inline bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

// The most CTAs of a gradient call (the rows of its workspace); as many of them run
// as stay resident.
int grad_ctas(int M) {
    const long long most = 4ll * sm_count();
    return (int)(M < most ? M : most);
}

int check_rows(int64_t M, int32_t d) {
    if (M < 0 || d < 1) return CRC_EINVAL;
    if (d % 8 != 0 || d > kMaxRow || M > 0x7fffffffll) return CRC_EUNSUPPORTED;
    return CRC_OK;
}

// K(groups a thread, most threads a CTA): rows of up to 512 threads leave a thread
// 128 registers, the widest rows 64.
#define CRC_SHAPE(sh, K, ...)                                            \
    do {                                                                 \
        if ((sh).threads() > 512) {                                      \
            if ((sh).vpt <= 2) K(2, 1024, __VA_ARGS__);                  \
            else K(4, 1024, __VA_ARGS__);                                \
        } else if ((sh).vpt == 1) K(1, 512, __VA_ARGS__);                \
        else if ((sh).vpt == 2) K(2, 512, __VA_ARGS__);                  \
        else if ((sh).vpt == 3) K(3, 512, __VA_ARGS__);                  \
        else K(4, 512, __VA_ARGS__);                                     \
    } while (0)

template <typename T, int VPT, int THREADS, bool RING, bool TEAMS = false>
int launch_grad_t(const GradShape& sh, int& G, const NormGradArgs& a, cudaStream_t stream) {
    auto kern = rms_norm_grad_kernel<T, VPT, THREADS, RING, TEAMS>;
    const int smem = RING ? sh.smem() : 0;
    static PerDevice ready;
    const int up = ready.get(current_device(), [&] {
        return cuda_status(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                RING ? kGradRing : 0)) == CRC_OK;
    });
    if (!up) return CRC_ECUDA;
    const long long ctas = sh.grid(a.M);
    if (ctas < G) G = (int)ctas;
    if (G > sm_count()) {
        int fit = 0;
        if (const int rc = cuda_status(
                cudaOccupancyMaxActiveBlocksPerMultiprocessor(&fit, kern, sh.threads(), smem)))
            return rc;
        if (fit < 1) return CRC_ECUDA;
        const long long most = (long long)fit * sm_count();
        G = (int)(G < most ? G : most);
    }
    cudaError_t e;
    {
        ProfScope prof(CRC_KERNEL_NORM, stream);
        e = launch_dependent(kern, dim3((unsigned)G), sh.threads(), smem, stream, 1, a);
    }
    note_launch();
    return cuda_status(e);
}
template <typename T>
int launch_grad(const GradShape& sh, int& G, const NormGradArgs& a, cudaStream_t stream) {
    if (!sh.stages)
        return sh.threads() > 512 ? launch_grad_t<T, 4, 1024, false>(sh, G, a, stream)
                                  : launch_grad_t<T, 4, 512, false>(sh, G, a, stream);
    if (sh.vpt == 1)
        return sh.rows > 1 ? launch_grad_t<T, 1, 512, true, true>(sh, G, a, stream)
                           : launch_grad_t<T, 1, 512, true>(sh, G, a, stream);
    if (sh.vpt == 2) return launch_grad_t<T, 2, 512, true>(sh, G, a, stream);
    return sh.threads() > 512 ? launch_grad_t<T, 4, 1024, true>(sh, G, a, stream)
                              : launch_grad_t<T, 4, 512, true>(sh, G, a, stream);
}

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
    // us with 1, 2, 4 groups a thread: 4097 x 2880 fp32 29.3, 29.8, 31.5 (the two inputs
    // of four groups are 64 registers); 8192 x 2048 bf16 35.2, 27.2, 26.1
    const RowShape sh = row_shape(d, M, stream_type == CRC_F32 ? 1 : 4);
    a.M = (int)M;
    a.d = d;
    a.warps = sh.warps;
    a.eps = (float)eps;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e;
    {
        ProfScope prof(CRC_KERNEL_NORM, st);
#define CRC_K(V, B, T) \
    e = launch_dependent(rms_norm_kernel<T, V, B>, dim3(sh.grid(M)), sh.threads(), 0, st, 1, a)
        if (stream_type == CRC_BF16)
            CRC_SHAPE(sh, CRC_K, __nv_bfloat16);
        else
            CRC_SHAPE(sh, CRC_K, float);
#undef CRC_K
    }
    note_launch();
    return cuda_status(e);
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
    const GradShape sh = grad_shape(d, stream_type == CRC_BF16 ? 2 : 4, dres_dev != nullptr);
    int G = grad_ctas((int)M);
    a.err = device_error_word();
    a.warps = sh.warps;
    a.stages = sh.stages;
    a.stage_bytes = sh.stage_bytes;
    const int rg = stream_type == CRC_BF16 ? launch_grad<__nv_bfloat16>(sh, G, a, st)
                                           : launch_grad<float>(sh, G, a, st);
    if (rg) return rg;
    if (!dw_dev) return CRC_OK;
    cudaError_t e;
    {
        ProfScope prof(CRC_KERNEL_NORM, st);
        e = launch_dependent(norm_dw_kernel, dim3((unsigned)((d + 31) / 32)), 1024, 0, st, 1,
                             (const float*)a.part, G, d, dw_dev);
    }
    note_launch();
    return cuda_status(e);
}

static int launch_quantize(bool split, const uint16_t* x_dev, int64_t x_stride, int64_t M,
                           int32_t d, uint8_t* out8_dev, float* scale8_dev, void* stream) {
    const int rc = check_rows(M, d);
    if (rc) return rc;
    if (x_stride < d || x_stride % 8 != 0) return CRC_EINVAL;
    if (M == 0) return CRC_OK;
    if (!x_dev || !out8_dev || !scale8_dev) return CRC_EINVAL;
    if (!aligned(x_dev, 16) || !aligned(out8_dev, 8) || !aligned(scale8_dev, 4)) return CRC_EINVAL;
    // Three or four groups a thread, by which leaves fewer lanes idle.  us with 2, 3, 4:
    // 184320 x 2880 336, 243, 265; 65536 x 1024 37, 39, 33; 20000 x 6144 3: 57, 4: 62;
    // 20000 x 8192 88, 93, 79; 30000 x 6000 97, 87, 91.
    const int nvec = d / 8;
    const auto idle = [nvec](int g) { return (nvec + 32 * g - 1) / (32 * g) * (32 * g) - nvec; };
    const RowShape sh = row_shape(d, M, idle(4) < idle(3) ? 4 : 3);
    // CTAs for 2048 threads an SM.  Of three or four groups (64 registers a thread) 1024 are
    // resident, and the rest begin where others end; with the resident ones alone
    // 184320 x 2880 took 244 us in place of 243, 65536 x 2048 (in threes) 85 in place of 75.
    const long long most = (long long)sm_count() * (2048 / sh.threads());
    const unsigned grid = (unsigned)(sh.grid(M) < most ? sh.grid(M) : most);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const __nv_bfloat16* x = reinterpret_cast<const __nv_bfloat16*>(x_dev);
    cudaError_t e;
    {
        ProfScope prof(CRC_KERNEL_QUANTIZE, st);
#define CRC_K(V, B, S)                                                                          \
    e = launch_dependent(quantize_rows_kernel<S, V, B>, dim3(grid), sh.threads(), 0, st, 1, x,   \
                         (long long)x_stride, (int)M, (int)d, sh.warps, out8_dev, scale8_dev)
        if (split)
            CRC_SHAPE(sh, CRC_K, true);
        else
            CRC_SHAPE(sh, CRC_K, false);
#undef CRC_K
    }
    note_launch();
    return cuda_status(e);
}

int crc_quantize_rows(const uint16_t* x_dev, int64_t x_stride, int64_t M, int32_t d,
                      uint8_t* out8_dev, float* scale8_dev, void* stream) {
    return launch_quantize(false, x_dev, x_stride, M, d, out8_dev, scale8_dev, stream);
}

int crc_split_rows(const uint16_t* x_dev, int64_t x_stride, int64_t M, int32_t d,
                   uint8_t* out8_dev, float* scale8_dev, void* stream) {
    return launch_quantize(true, x_dev, x_stride, M, d, out8_dev, scale8_dev, stream);
}

}  // extern "C"
