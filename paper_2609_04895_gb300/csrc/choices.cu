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
// the passes in them, not by its 9 bytes a choice: 148 choices take 2.7 us, 8192 6.1, 262144
// (32768 tokens, 128 experts) 10.6.
//
// Sum and gradient.  One pass over the rows, 16 bytes a thread and choice, as many choices'
// loads in flight as fit the registers; the choices are summed in fp32 in rank order.  Bound by
// memory: 4096 tokens x 8 of d = 2048 25.4 us, 6.0 TB/s; the gradient, with the gates', 50 us, 5.8
// TB/s; small batches by their launch (1.5 to 2.5 us).
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "crc_device.cuh"
#include "crc_internal.h"
#include "pdl.cuh"

namespace crc {
namespace {

constexpr int kOrderThreads = 1024;
constexpr int kWarps = kOrderThreads / 32;
constexpr int kSteps = 8;                                   // choices of a lane at a time
constexpr int kSub = kOrderThreads * kSteps;                // choices of a CTA at a time
// Up to kOneChunk choices one CTA does it all, above that chunks of kMinChunk or more: most of a
// CTA's time are its scattered 4-byte stores.  Us, one CTA / chunks: 2048 choices 4.8 / 5.7, 4725
// 7.7 / 5.8, 8192 11.3 / 6.1; chunks of 1024 / 2048: 16000 choices 6.5 / 7.5.
constexpr int kOneChunk = 2048;
constexpr int kMaxChunks = 128, kMinChunk = 1024;
constexpr int kMaxExperts = 256;
constexpr int kBins = kMaxExperts + 1;                      // the last: no expert
constexpr int kBinBits = 9;

inline bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

struct OrderArgs {
    const uint8_t* topk;
    int32_t* offsets;
    int32_t* rows;
    int32_t* place;
    int32_t* counts;        // [chunks][N + 1], NULL: one chunk
    uint32_t* err;
    int E, N, chunk, chunks;
};

__device__ __forceinline__ int bin_of(const OrderArgs& a, int c) {
    const int e = a.topk[c];
    return e < a.N ? e : a.N;
}

// counts[chunk][bin]
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
        a.counts[blockIdx.x * (a.N + 1) + b] = hist[b];
}

// The bins' exclusive sum, in place: start[0 .. kBins + 30], zeros behind the last.  One warp.
__device__ __forceinline__ void scan_bins(int* start) {
    constexpr int kEach = (kBins + 31) / 32;
    const int lane = threadIdx.x & 31;
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

// The lanes whose bin is this one's, by a ballot for each bit.  (4 to 9% less for a call than by
// __match_any_sync.)
__device__ __forceinline__ unsigned same_bin(int bin, int bits) {
    unsigned same = __ballot_sync(kFull, bin >= 0);
    if (bin < 0) same = ~same;
#pragma unroll
    for (int b = 0; b < kBinBits; ++b) {
        if (b >= bits) break;
        const bool one = bin >> b & 1;
        const unsigned ones = __ballot_sync(kFull, one);
        same &= one ? ones : ~ones;
    }
    return same;
}

__global__ void __launch_bounds__(kOrderThreads) order_choices_kernel(OrderArgs a) {
    __shared__ int start[kBins + 31];           // each expert's first place, of this CTA's in turn
    __shared__ int total[kBins + 31];           // and its choices
    __shared__ int count[kWarps][kBins];        // a warp's choices of each, then those before it
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int bins = a.N + 1, bits = 32 - __clz(a.N);
    for (int b = threadIdx.x; b < kBins + 31; b += kOrderThreads) start[b] = total[b] = 0;
    pdl_begin();
    const int c0 = blockIdx.x * a.chunk;
    const int c1 = min(a.E, c0 + a.chunk);
    const int steps = (min(a.chunk, kSub) + kOrderThreads - 1) / kOrderThreads;
    const auto choice = [&](int s0, int i) { return s0 + (warp * steps + i) * 32 + lane; };
    int bin[kSteps], rank[kSteps];
    const auto load = [&](int s0) {
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const int c = choice(s0, i);
            bin[i] = i < steps && c < c1 ? bin_of(a, c) : -1;
        }
    };
    load(c0);
    if (a.counts) {
        // every expert's choices, and those of the chunks before this one: a thread a part of
        // the chunks for one expert
        const int wide = (bins + 31) / 32 * 32, parts = kOrderThreads / wide;
        const int part = threadIdx.x / wide, b = threadIdx.x % wide;
        int all = 0, mine = 0;
        if (part < parts && b < bins)
#pragma unroll 8
            for (int k = part; k < a.chunks; k += parts) {
                const int v = a.counts[k * bins + b];
                all += v;
                if (k < (int)blockIdx.x) mine += v;
            }
        int* scratch = &count[0][0];
        scratch[threadIdx.x] = all;
        scratch[kOrderThreads + threadIdx.x] = mine;
        __syncthreads();
        all = mine = 0;
        if ((int)threadIdx.x < bins) {
            for (int p = 0; p < parts; ++p) {
                all += scratch[p * wide + threadIdx.x];
                mine += scratch[kOrderThreads + p * wide + threadIdx.x];
            }
            start[threadIdx.x] = all;
        }
        __syncthreads();
        if (warp == 0) scan_bins(start);
        __syncthreads();
        if ((int)threadIdx.x < bins) {
            if (blockIdx.x == 0) a.offsets[threadIdx.x] = start[threadIdx.x];
            start[threadIdx.x] += mine;
        }
    }
    for (int s0 = c0; s0 < c1; s0 += kSub) {
        if (s0 > c0) load(s0);
        for (int b = lane; b < bins; b += 32) count[warp][b] = 0;
        __syncwarp();
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            if (i >= steps) break;
            const unsigned same = same_bin(bin[i], bits);
            const unsigned below = same & ((1u << lane) - 1);
            if (bin[i] >= 0) rank[i] = count[warp][bin[i]] + __popc(below);
            __syncwarp();
            if (bin[i] >= 0 && below == 0) count[warp][bin[i]] += __popc(same);
            __syncwarp();
        }
        __syncthreads();
        // each expert's choices in the warps before
        for (int b = warp; b < bins; b += kWarps) {
            const int v = count[lane][b];
            int incl = v;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int u = __shfl_up_sync(kFull, incl, o);
                if (lane >= o) incl += u;
            }
            count[lane][b] = incl - v;
            if (lane == 31) total[b] = incl;
        }
        __syncthreads();
        if (!a.counts) {                        // one chunk: these are all choices
            if ((int)threadIdx.x < bins) start[threadIdx.x] = total[threadIdx.x];
            __syncthreads();
            if (warp == 0) scan_bins(start);
            __syncthreads();
            if ((int)threadIdx.x < bins) a.offsets[threadIdx.x] = start[threadIdx.x];
        }
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            if (bin[i] < 0) continue;
            const int c = choice(s0, i);
            const int at = start[bin[i]] + count[warp][bin[i]] + rank[i];
            const bool real = bin[i] < a.N;
            if (CRC_IN_BOUNDS(at >= 0 && at < a.E, a.err)) a.rows[at] = real ? c : -1;
            if (a.place) a.place[c] = real ? at : -1;
        }
        __syncthreads();
        if ((int)threadIdx.x < bins) start[threadIdx.x] += total[threadIdx.x];
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------
// the sum over a token's choices
// ---------------------------------------------------------------------------
constexpr int kSumThreads = 256;
constexpr int kManyTokens = 30000;
constexpr long long kManyElements = 48ll << 20;

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

// kBatch: choices of a token whose loads are in flight together.  A CTA takes kTurns tokens for
// each team of threads; their rows and gates are looked up once, into shared memory (from global
// memory in each thread 4096 tokens x 8 of d = 2048 took 27.7 us, 25.4 so).
constexpr int kCtaChoices = 256;
template <int kBatch, int kTurns>
__global__ void __launch_bounds__(kSumThreads) sum_choices_kernel(SumArgs a) {
    __shared__ int rows[kCtaChoices];
    __shared__ float gates[kCtaChoices];
    pdl_begin();
    const int teams = blockDim.x / a.team;
    const int t = threadIdx.x % a.team, team = threadIdx.x / a.team;
    const int m0 = blockIdx.x * teams * kTurns;
    const int choices = min(teams * kTurns, a.M - m0) * a.K;
    for (int i = threadIdx.x; i < choices; i += blockDim.x) {
        const long long r = row_of(a, m0, i);
        rows[i] = (int)r;
        gates[i] = a.gates ? a.gates[(long long)m0 * a.K + i] : 1.f;
    }
    __syncthreads();
#pragma unroll 1
    for (int turn = 0; turn < kTurns; ++turn) {
        const int at = turn * teams + team, m = m0 + at;
        if (m >= a.M) return;
        const int* r = rows + at * a.K;
        const float* g = gates + at * a.K;
        for (int v = t; v < a.d / 8; v += a.team) {
            float sum[8] = {};
            for (int j0 = 0; j0 < a.K; j0 += kBatch) {
                uint4 u[kBatch];
#pragma unroll
                for (int j = 0; j < kBatch; ++j) {
                    u[j] = make_uint4(0, 0, 0, 0);
                    if (j0 + j < a.K && r[j0 + j] >= 0)
                        u[j] = __ldcs(reinterpret_cast<const uint4*>(
                                          a.y + (long long)r[j0 + j] * a.d) + v);
                }
#pragma unroll
                for (int j = 0; j < kBatch; ++j) {
                    if (j0 + j >= a.K || r[j0 + j] < 0) continue;
                    float f[8];
                    widen(u[j], f);
#pragma unroll
                    for (int i = 0; i < 8; ++i) sum[i] = fmaf(g[j0 + j], f[i], sum[i]);
                }
            }
            *(reinterpret_cast<uint4*>(a.out + (long long)m * a.d) + v) = narrow(sum);
        }
    }
}

// dy[place] = gate dout, dgates = <dout, y[place]>: a token's threads share its rows, and
// the dot products are summed over the lanes and then the warps.
// kBatch: choices of a token whose loads are in flight together; kTok: tokens of a team.
template <int kBatch, int kTok>
__global__ void __launch_bounds__(kSumThreads) sum_choices_grad_kernel(SumArgs a) {
    constexpr int kDots = kTok * kBatch;
    __shared__ float part[kSumThreads / 32][kDots];
    pdl_begin();
    const int t = threadIdx.x % a.team;
    const int m = (blockIdx.x * (blockDim.x / a.team) + threadIdx.x / a.team) * kTok;
    const bool real = m < a.M;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int j0 = 0; j0 < a.K; j0 += kBatch) {
        long long r[kTok][kBatch];
        float g[kTok][kBatch], dot[kTok][kBatch];
#pragma unroll
        for (int k = 0; k < kTok; ++k)
#pragma unroll
            for (int j = 0; j < kBatch; ++j) {
                const bool has = m + k < a.M && j0 + j < a.K;
                r[k][j] = has ? row_of(a, m + k, j0 + j) : -1;
                g[k][j] = r[k][j] >= 0 && a.gates
                              ? a.gates[(long long)(m + k) * a.K + j0 + j]
                              : 1.f;
                dot[k][j] = 0.f;
            }
        if (real)
            for (int v = t; v < a.d / 8; v += a.team) {
                uint4 d[kTok], u[kTok][kBatch];
#pragma unroll
                for (int k = 0; k < kTok; ++k)
                    if (m + k < a.M)
                        d[k] = *(reinterpret_cast<const uint4*>(a.dout + (long long)(m + k) * a.d) +
                                 v);
                if (a.dgates)
#pragma unroll
                    for (int k = 0; k < kTok; ++k)
#pragma unroll
                        for (int j = 0; j < kBatch; ++j)
                            if (r[k][j] >= 0)
                                u[k][j] = __ldcs(
                                    reinterpret_cast<const uint4*>(a.y + r[k][j] * a.d) + v);
#pragma unroll
                for (int k = 0; k < kTok; ++k) {
                    if (m + k >= a.M) break;
                    float f[8];
                    widen(d[k], f);
#pragma unroll
                    for (int j = 0; j < kBatch; ++j) {
                        if (r[k][j] < 0) continue;
                        if (a.dgates) {
                            float y[8];
                            widen(u[k][j], y);
#pragma unroll
                            for (int i = 0; i < 8; ++i) dot[k][j] = fmaf(f[i], y[i], dot[k][j]);
                        }
                        if (a.out) {
                            float w[8];
#pragma unroll
                            for (int i = 0; i < 8; ++i) w[i] = g[k][j] * f[i];
                            *(reinterpret_cast<uint4*>(a.out + r[k][j] * a.d) + v) = narrow(w);
                        }
                    }
                }
            }
        if (!a.dgates) continue;
#pragma unroll
        for (int q = 0; q < kDots; ++q) {
            float s = dot[q / kBatch][q % kBatch];
#pragma unroll
            for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(kFull, s, o);
            if (lane == 0) part[warp][q] = s;
        }
        __syncthreads();
        const int k = t / kBatch, j = j0 + t % kBatch;
        if (t < kDots && m + k < a.M && j < a.K) {
            float s = 0.f;
            for (int w = 0; w < a.team / 32; ++w) s += part[warp + w][t];
            a.dgates[(long long)(m + k) * a.K + j] = s;
        }
        __syncthreads();
    }
}

// Threads of a token: as few as leave no 16-byte piece more than the other threads have.
int team_of(int d) {
    const int vec = d / 8;
    const int turns = (vec + kSumThreads - 1) / kSumThreads;
    return ((vec + turns - 1) / turns + 31) / 32 * 32;
}

template <int kBatch, int kTurns>
cudaError_t launch_sum_of(SumArgs& a, cudaStream_t st) {
    a.team = team_of(a.d);
    const int teams = kSumThreads / a.team, tokens = teams * kTurns;
    return launch_dependent(sum_choices_kernel<kBatch, kTurns>,
                            dim3((unsigned)((a.M + tokens - 1) / tokens)), teams * a.team, 0, st, 1,
                            a);
}
cudaError_t launch_sum(SumArgs& a, cudaStream_t st) {
    // One choice and many tokens: several tokens a team.  Us, one / eight: d = 256, 32000 tokens 5.9 /
    // 7.4, 64000 11.8 / 12.9; d = 816, 16000 11.6 / 12.6, 32000 23.0 / 22.6, 64000 55.6 / 48.0; d =
    // 2048, 16000 24.9 / 25.4, 32000 57.3 / 50.5, 64000 112 / 95; d = 4096, 16000 47.7 / 52.9, 32000
    // 92.6 / 94.1, 64000 183 / 179.
    if (a.K == 1)
        return a.M >= kManyTokens && (long long)a.M * a.d >= kManyElements
                   ? launch_sum_of<1, 8>(a, st)
                   : launch_sum_of<1, 1>(a, st);
    if (a.K == 2) return launch_sum_of<2, 1>(a, st);
    if (a.K <= 4) return launch_sum_of<4, 1>(a, st);
    return launch_sum_of<8, 1>(a, st);
}

template <int kBatch, int kTok>
cudaError_t launch_grad_of(SumArgs& a, cudaStream_t st) {
    a.team = team_of(a.d);
    const int teams = kSumThreads / a.team, tokens = teams * kTok;
    return launch_dependent(sum_choices_grad_kernel<kBatch, kTok>,
                            dim3((unsigned)((a.M + tokens - 1) / tokens)), teams * a.team, 0, st, 1,
                            a);
}
cudaError_t launch_grad(SumArgs& a, cudaStream_t st) {
    // One or two choices: several tokens' loads together.  Us, one / several tokens: 14400
    // tokens of d = 816, K = 1, 22.6 / 21.5; 4000 of d = 1280, K = 2, 14.3 / 13.4.
    if (a.K == 1) return launch_grad_of<1, 4>(a, st);
    if (a.K == 2) return launch_grad_of<2, 2>(a, st);
    return launch_grad_of<4, 1>(a, st);
}

int order_chunk(long long E) {
    const long long each = (E + kMaxChunks - 1) / kMaxChunks;
    const long long chunk = (each + kOrderThreads - 1) / kOrderThreads * kOrderThreads;
    return (int)(chunk < kMinChunk ? kMinChunk : chunk);
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
    a.err = device_error_word();
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
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e;
    {
        ProfScope prof(CRC_KERNEL_SUM, st);
        e = launch_sum(a, st);
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
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e;
    {
        ProfScope prof(CRC_KERNEL_SUM, st);
        e = launch_grad(a, st);
    }
    note_launch();
    return cuda_status(e);
}

}  // extern "C"
