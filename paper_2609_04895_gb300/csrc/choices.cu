// Choices of a prompt or a training batch: their order by expert, and the sum over a
// token's choices with its gradient.
//
// Order.  A choice's place is the number of choices of smaller experts plus the number of
// earlier choices of its own expert: a counting sort, stable, with no atomics on places.
// A chunk of choices belongs to one CTA of 32 warps; a warp ranks 32 choices at a time by
// the lanes with the same expert and keeps its own counts, a scan over the warps and over
// the experts gives every warp its first place.  Up to kOneChunk choices it is one kernel
// of one CTA; above, a kernel counts every chunk and a second one places them, after each
// CTA has summed the counts of the chunks.  Bound by the latency of its launches and of
// the passes in them, not by its 9 bytes a choice.
//
// Sum and gradient.  One pass over the rows, 16 bytes a thread and choice, eight choices'
// loads in flight; the choices are summed in fp32 in rank order.  Bound by memory.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "crc_device.cuh"
#include "crc_internal.h"
#include "pdl.cuh"

namespace crc {
namespace {

constexpr int kOrderThreads = 1024;
constexpr int kWarps = kOrderThreads / 32;
constexpr int kSteps = 4;                                   // choices a lane and sub-chunk
constexpr int kSub = kOrderThreads * kSteps;                // choices of a sub-chunk
constexpr int kOneChunk = 2 * kSub;
constexpr int kMaxChunks = 128;
constexpr int kMaxExperts = 256;
constexpr int kBins = kMaxExperts + 1;                      // the last: no expert

inline bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

struct OrderArgs {
    const uint8_t* topk;
    int32_t* offsets;
    int32_t* rows;
    int32_t* place;
    int32_t* counts;        // [N + 1][chunks], NULL: one chunk
    int E, N, chunk, chunks;
};

__device__ __forceinline__ int bin_of(const OrderArgs& a, int c) {
    const int e = a.topk[c];
    return e < a.N ? e : a.N;
}

// counts[bin][chunk]
__global__ void __launch_bounds__(kOrderThreads) count_choices_kernel(OrderArgs a) {
    __shared__ int hist[kBins];
    for (int b = threadIdx.x; b <= a.N; b += kOrderThreads) hist[b] = 0;
    __syncthreads();
    pdl_begin();
    const int c0 = blockIdx.x * a.chunk;
    const int c1 = min(a.E, c0 + a.chunk);
    for (int c = c0 + threadIdx.x; c < c1; c += kOrderThreads) atomicAdd(&hist[bin_of(a, c)], 1);
    __syncthreads();
    for (int b = threadIdx.x; b <= a.N; b += kOrderThreads)
        a.counts[b * a.chunks + blockIdx.x] = hist[b];
}

__global__ void __launch_bounds__(kOrderThreads) order_choices_kernel(OrderArgs a) {
    __shared__ int start[kBins + 31], before[kBins];
    __shared__ int count[kWarps][kBins];        // a warp's choices of each expert, then its first place
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int bins = a.N + 1;
    for (int b = threadIdx.x; b < kBins + 31; b += kOrderThreads) start[b] = 0;
    __syncthreads();
    pdl_begin();
    const int c0 = blockIdx.x * a.chunk;
    const int c1 = min(a.E, c0 + a.chunk);
    // totals of every expert, and those of the chunks before this one
    if (a.counts) {
        for (int b = warp; b < bins; b += kWarps) {
            int all = 0, mine = 0;
#pragma unroll
            for (int i = 0; i < kMaxChunks / 32; ++i) {
                const int k = i * 32 + lane;
                const int v = k < a.chunks ? a.counts[b * a.chunks + k] : 0;
                all += v;
                if (k < (int)blockIdx.x) mine += v;
            }
            all = __reduce_add_sync(kFull, all);
            mine = __reduce_add_sync(kFull, mine);
            if (lane == 0) {
                start[b] = all;
                before[b] = mine;
            }
        }
    } else {
        for (int c = c0 + threadIdx.x; c < c1; c += kOrderThreads) atomicAdd(&start[bin_of(a, c)], 1);
        for (int b = threadIdx.x; b < bins; b += kOrderThreads) before[b] = 0;
    }
    __syncthreads();
    // exclusive sum over the experts: nine a lane
    if (warp == 0) {
        constexpr int kEach = (kBins + 31) / 32;
        int v[kEach], sum = 0;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            v[i] = sum;
            sum += start[lane * kEach + i];
        }
        int incl = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int u = __shfl_up_sync(kFull, incl, o);
            if (lane >= o) incl += u;
        }
        __syncwarp();
#pragma unroll
        for (int i = 0; i < kEach; ++i) start[lane * kEach + i] = incl - sum + v[i];
    }
    __syncthreads();
    if (blockIdx.x == 0)
        for (int b = threadIdx.x; b < bins; b += kOrderThreads) a.offsets[b] = start[b];
    __syncthreads();
    for (int b = threadIdx.x; b < bins; b += kOrderThreads) start[b] += before[b];

    for (int s0 = c0; s0 < c1; s0 += kSub) {
        for (int b = lane; b < bins; b += 32) count[warp][b] = 0;
        __syncwarp();
        int bin[kSteps], rank[kSteps];
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const int c = s0 + warp * (32 * kSteps) + i * 32 + lane;
            bin[i] = c < c1 ? bin_of(a, c) : -1;
        }
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const unsigned same = __match_any_sync(kFull, bin[i]);
            const unsigned below = same & ((1u << lane) - 1);
            if (bin[i] >= 0) rank[i] = count[warp][bin[i]] + __popc(below);
            __syncwarp();
            if (bin[i] >= 0 && below == 0) count[warp][bin[i]] += __popc(same);
            __syncwarp();
        }
        __syncthreads();
        // each expert's counts over the warps: its first place in every warp
        for (int b = warp; b < bins; b += kWarps) {
            const int v = count[lane][b];
            int incl = v;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int u = __shfl_up_sync(kFull, incl, o);
                if (lane >= o) incl += u;
            }
            const int first = start[b];
            count[lane][b] = first + incl - v;
            __syncwarp();
            if (lane == 31) start[b] = first + incl;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            if (bin[i] < 0) continue;
            const int c = s0 + warp * (32 * kSteps) + i * 32 + lane;
            const int at = count[warp][bin[i]] + rank[i];
            const bool real = bin[i] < a.N;
            if (CRC_IN_BOUNDS(at >= 0 && at < a.E, (uint32_t*)nullptr)) a.rows[at] = real ? c : -1;
            if (a.place) a.place[c] = real ? at : -1;
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------
// the sum over a token's choices
// ---------------------------------------------------------------------------
constexpr int kBatch = 8;                    // choices whose loads are in flight together
constexpr int kSumThreads = 256;

struct SumArgs {
    const uint16_t* y;           // [rows][d]
    const uint16_t* dout;        // gradient: [M][d]
    const int32_t* place;        // [M][K] or NULL
    const float* gates;          // [M][K] or NULL
    uint16_t* out;               // [M][d], the gradient: dy [rows][d]
    float* dgates;               // gradient: [M][K] or NULL
    long long rows;
    int M, K, d, team;           // team: threads of a token, a multiple of 32
};

__device__ __forceinline__ void widen(const uint4& u, float (&f)[8]) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ uint4 narrow(const float (&f)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// The row of choice j of token m, -1 if it has none.
__device__ __forceinline__ long long row_of(const SumArgs& a, int m, int j) {
    const long long c = (long long)m * a.K + j;
    const long long r = a.place ? a.place[c] : c;
    return r >= 0 && r < a.rows ? r : -1;
}

__global__ void __launch_bounds__(kSumThreads) sum_choices_kernel(SumArgs a) {
    pdl_begin();
    const int t = threadIdx.x % a.team;
    const int m = blockIdx.x * (blockDim.x / a.team) + threadIdx.x / a.team;
    if (m >= a.M) return;
    for (int v = t; v < a.d / 8; v += a.team) {
        float sum[8] = {};
        for (int j0 = 0; j0 < a.K; j0 += kBatch) {
            uint4 u[kBatch];
            float g[kBatch];
            bool on[kBatch];
#pragma unroll
            for (int j = 0; j < kBatch; ++j) {
                const long long r = j0 + j < a.K ? row_of(a, m, j0 + j) : -1;
                on[j] = r >= 0;
                g[j] = on[j] && a.gates ? a.gates[(long long)m * a.K + j0 + j] : 1.f;
                if (on[j]) u[j] = __ldcs(reinterpret_cast<const uint4*>(a.y + r * a.d) + v);
            }
#pragma unroll
            for (int j = 0; j < kBatch; ++j) {
                if (!on[j]) continue;
                float f[8];
                widen(u[j], f);
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[i] = fmaf(g[j], f[i], sum[i]);
            }
        }
        *(reinterpret_cast<uint4*>(a.out + (long long)m * a.d) + v) = narrow(sum);
    }
}

// dy[place] = gate dout, dgates = <dout, y[place]>: a token's threads share its rows, and
// the dot products of eight choices are summed over the lanes and then the warps.
__global__ void __launch_bounds__(kSumThreads) sum_choices_grad_kernel(SumArgs a) {
    __shared__ float part[kSumThreads / 32][kBatch];
    pdl_begin();
    const int t = threadIdx.x % a.team;
    const int m = blockIdx.x * (blockDim.x / a.team) + threadIdx.x / a.team;
    const bool real = m < a.M;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int j0 = 0; j0 < a.K; j0 += kBatch) {
        long long r[kBatch];
        float g[kBatch], dot[kBatch];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            r[j] = real && j0 + j < a.K ? row_of(a, m, j0 + j) : -1;
            g[j] = r[j] >= 0 && a.gates ? a.gates[(long long)m * a.K + j0 + j] : 1.f;
            dot[j] = 0.f;
        }
        if (real)
            for (int v = t; v < a.d / 8; v += a.team) {
                float f[8];
                widen(*(reinterpret_cast<const uint4*>(a.dout + (long long)m * a.d) + v), f);
                uint4 u[kBatch];
                if (a.dgates)
#pragma unroll
                    for (int j = 0; j < kBatch; ++j)
                        if (r[j] >= 0)
                            u[j] = __ldcs(reinterpret_cast<const uint4*>(a.y + r[j] * a.d) + v);
#pragma unroll
                for (int j = 0; j < kBatch; ++j) {
                    if (r[j] < 0) continue;
                    if (a.dgates) {
                        float y[8];
                        widen(u[j], y);
#pragma unroll
                        for (int i = 0; i < 8; ++i) dot[j] = fmaf(f[i], y[i], dot[j]);
                    }
                    if (a.out) {
                        float w[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) w[i] = g[j] * f[i];
                        *(reinterpret_cast<uint4*>(a.out + r[j] * a.d) + v) = narrow(w);
                    }
                }
            }
        if (!a.dgates) continue;
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
#pragma unroll
            for (int o = 16; o; o >>= 1) dot[j] += __shfl_xor_sync(kFull, dot[j], o);
            if (lane == 0) part[warp][j] = dot[j];
        }
        __syncthreads();
        if (real && t < kBatch && j0 + t < a.K) {
            float s = 0.f;
            for (int w = 0; w < a.team / 32; ++w) s += part[warp + w][t];
            a.dgates[(long long)m * a.K + j0 + t] = s;
        }
        __syncthreads();
    }
}

int order_chunk(long long E) {
    const long long each = (E + kMaxChunks - 1) / kMaxChunks;
    return (int)((each + kSub - 1) / kSub * kSub);
}

int check_order(int32_t M, int32_t K, int32_t N) {
    if (M < 0 || K < 1 || N < 1) return CRC_EINVAL;
    if (N > kMaxExperts || K > 32 || (int64_t)M * K > (1 << 30)) return CRC_EUNSUPPORTED;
    return CRC_OK;
}

int check_sum(int64_t rows, int32_t M, int32_t K, int32_t d, const void* place) {
    if (rows < 0 || M < 0 || K < 1 || d < 1) return CRC_EINVAL;
    if (d % 8 != 0 || d > 32768 || K > 32 || rows > (1 << 30) || (int64_t)M * K > (1 << 30))
        return CRC_EUNSUPPORTED;
    if (!place && rows < (int64_t)M * K) return CRC_EINVAL;
    return CRC_OK;
}

// Threads of a token: as few as leave no 16-byte piece more than the other threads have.
void sum_shape(SumArgs& a, unsigned* grid, unsigned* threads) {
    const int vec = a.d / 8;
    const int turns = (vec + kSumThreads - 1) / kSumThreads;
    a.team = ((vec + turns - 1) / turns + 31) / 32 * 32;
    const int tokens = kSumThreads / a.team;
    *threads = tokens * a.team;
    *grid = (unsigned)((a.M + tokens - 1) / tokens);
}

}  // namespace
}  // namespace crc

using namespace crc;

extern "C" {

size_t crc_group_choices_workspace_bytes(int32_t M, int32_t K, int32_t N) {
    if (check_order(M, K, N) != CRC_OK) return 0;
    const long long E = (long long)M * K;
    if (E <= kOneChunk) return 0;
    return (size_t)(N + 1) * kMaxChunks * sizeof(int32_t);
}

int crc_group_choices(const uint8_t* topk_dev, int32_t M, int32_t K, int32_t N,
                      int32_t* offsets_dev, int32_t* rows_dev, int32_t* place_dev,
                      void* workspace_dev, size_t workspace_bytes, void* stream) {
    const int rc = check_order(M, K, N);
    if (rc) return rc;
    if (!offsets_dev || !aligned(offsets_dev, 4)) return CRC_EINVAL;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int E = M * K;
    if (E == 0)                                      // no choices: every expert's first place is 0
        return cuda_status(cudaMemsetAsync(offsets_dev, 0, (size_t)(N + 1) * 4, st));
    if (!topk_dev || !rows_dev || !aligned(rows_dev, 4) || !aligned(place_dev, 4))
        return CRC_EINVAL;
    const size_t need = crc_group_choices_workspace_bytes(M, K, N);
    if (need && (!workspace_dev || !aligned(workspace_dev, 256) || workspace_bytes < need))
        return CRC_EINVAL;
    OrderArgs a;
    a.topk = topk_dev;
    a.offsets = offsets_dev;
    a.rows = rows_dev;
    a.place = place_dev;
    a.counts = need ? static_cast<int32_t*>(workspace_dev) : nullptr;
    a.E = E;
    a.N = N;
    a.chunk = need ? order_chunk(E) : E;
    a.chunks = need ? (E + a.chunk - 1) / a.chunk : 1;
    cudaError_t e;
    if (need) {
        {
            ProfScope prof(CRC_KERNEL_CHOICES, st);
            e = launch_dependent(count_choices_kernel, dim3((unsigned)a.chunks), kOrderThreads, 0,
                                 st, 1, a);
        }
        note_launch();
        if (e != cudaSuccess) return cuda_status(e);
    }
    {
        ProfScope prof(CRC_KERNEL_CHOICES, st);
        e = launch_dependent(order_choices_kernel, dim3((unsigned)a.chunks), kOrderThreads, 0, st,
                             1, a);
    }
    note_launch();
    return cuda_status(e);
}

int crc_sum_choices(const uint16_t* y_dev, int64_t y_rows, const int32_t* place_dev,
                    const float* gates_dev, int32_t M, int32_t K, int32_t d, uint16_t* out_dev,
                    void* stream) {
    const int rc = check_sum(y_rows, M, K, d, place_dev);
    if (rc) return rc;
    if (M == 0) return CRC_OK;
    if ((y_rows > 0 && !y_dev) || !out_dev || !aligned(y_dev, 16) || !aligned(out_dev, 16) ||
        !aligned(place_dev, 4) || !aligned(gates_dev, 4))
        return CRC_EINVAL;
    SumArgs a = {};
    a.y = y_dev;
    a.place = place_dev;
    a.gates = gates_dev;
    a.out = out_dev;
    a.rows = y_rows;
    a.M = M;
    a.K = K;
    a.d = d;
    unsigned grid, threads;
    sum_shape(a, &grid, &threads);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e;
    {
        ProfScope prof(CRC_KERNEL_SUM, st);
        e = launch_dependent(sum_choices_kernel, dim3(grid), threads, 0, st, 1, a);
    }
    note_launch();
    return cuda_status(e);
}

int crc_sum_choices_grad(const uint16_t* dout_dev, const uint16_t* y_dev, int64_t y_rows,
                         const int32_t* place_dev, const float* gates_dev, int32_t M, int32_t K,
                         int32_t d, uint16_t* dy_dev, float* dgates_dev, void* stream) {
    const int rc = check_sum(y_rows, M, K, d, place_dev);
    if (rc) return rc;
    if (dgates_dev && !y_dev && y_rows > 0) return CRC_EINVAL;
    if (M == 0 || (!dy_dev && !dgates_dev)) return CRC_OK;
    if (!dout_dev || !aligned(dout_dev, 16) || !aligned(y_dev, 16) || !aligned(dy_dev, 16) ||
        !aligned(place_dev, 4) || !aligned(gates_dev, 4) || !aligned(dgates_dev, 4))
        return CRC_EINVAL;
    SumArgs a = {};
    a.y = y_dev;
    a.dout = dout_dev;
    a.place = place_dev;
    a.gates = gates_dev;
    a.out = dy_dev;
    a.dgates = dgates_dev;
    a.rows = y_rows;
    a.M = M;
    a.K = K;
    a.d = d;
    unsigned grid, threads;
    sum_shape(a, &grid, &threads);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e;
    {
        ProfScope prof(CRC_KERNEL_SUM, st);
        e = launch_dependent(sum_choices_grad_kernel, dim3(grid), threads, 0, st, 1, a);
    }
    note_launch();
    return cuda_status(e);
}

}  // extern "C"
