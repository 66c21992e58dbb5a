// The mixture-of-experts layer for a few tokens: entry points, workspace and
// the experts' kernels.
#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>

#include "crc_internal.h"
#include "moe_route.cuh"

namespace crc {
namespace {

constexpr int kMoeMaxTokens = 1024;
constexpr int kMoeMaxEntries = 8192;      // M K
constexpr int kCtrlWords = 64;

inline bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
inline size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }

struct MoeLayout {
    size_t ctrl, ids, gates, xscale, h, y, total;
};

MoeLayout moe_layout(const crc_moe& m, int M) {
    const size_t E = (size_t)M * m.K;
    MoeLayout l;
    l.ctrl = 0;
    l.ids = up256(kCtrlWords * 4);
    l.gates = l.ids + up256(E);
    l.xscale = l.gates + up256(E * 4);
    l.h = l.xscale + up256((size_t)M * 4);
    l.y = l.h + up256(E * m.f * 2);
    l.total = l.y + up256(E * m.d * 4);
    return l;
}

int check_moe(const crc_moe* m) {
    if (!m || m->reserved != 0) return CRC_EINVAL;
    if (m->N < 1 || m->K < 1 || m->d < 1 || m->f < 1 || m->slots < 1) return CRC_EINVAL;
    if (m->weight_type != CRC_BF16 && m->weight_type != CRC_E4M3) return CRC_EINVAL;
    if (m->renormalize != 0 && m->renormalize != 1) return CRC_EINVAL;
    const bool w8 = m->weight_type == CRC_E4M3;
    if (m->N % 16 != 0 || m->N > kMoeMaxN || m->K > m->N || m->K > 32) return CRC_EUNSUPPORTED;
    if (m->d % (w8 ? 16 : 8) != 0 || m->f % 16 != 0 || m->d > 32768 || m->f > 32768)
        return CRC_EUNSUPPORTED;
    if (!m->gate_up_dev || !m->down_dev || !aligned(m->gate_up_dev, 16) ||
        !aligned(m->down_dev, 16) || !aligned(m->router_dev, 16) ||
        !aligned(m->expert_slot_dev, 4))
        return CRC_EINVAL;
    const int64_t es = w8 ? 1 : 2;
    const int64_t third = (int64_t)m->f * m->d * es;
    if (m->gate_up_stride % 16 || m->down_stride % 16 || m->gate_up_stride < 2 * third ||
        m->down_stride < third)
        return CRC_EINVAL;
    if (m->gate_up_stride >= (1ll << 40) || m->down_stride >= (1ll << 40)) return CRC_EUNSUPPORTED;
    if (w8) {
        if (!m->gate_up_scale_dev || !m->down_scale_dev || !aligned(m->gate_up_scale_dev, 4) ||
            !aligned(m->down_scale_dev, 4) || m->gate_up_scale_stride % 4 ||
            m->down_scale_stride % 4 || m->gate_up_scale_stride < 8ll * m->f ||
            m->down_scale_stride < 4ll * m->d)
            return CRC_EINVAL;
    } else if (m->gate_up_scale_dev || m->down_scale_dev) {
        return CRC_EINVAL;
    }
    return CRC_OK;
}

struct MoeArgs {
    crc_moe m;
    const uint16_t* x;
    const uint8_t* x8;
    const float* xs8;
    long long ldx;
    int M;
    const uint8_t* ids;
    const float* gates;
    __nv_bfloat16* h;                // [M K][f]
    float* y;                        // [M K][d]
    uint16_t* out;
};

__device__ __forceinline__ int slot_of(const crc_moe& m, int e) {
    const int s = m.expert_slot_dev ? m.expert_slot_dev[e] : e;
    return s >= 0 && s < m.slots ? s : -1;
}
__device__ __forceinline__ float e4m3(uint8_t v) {
    __nv_fp8_e4m3 q;
    q.__x = v;
    return (float)q;
}
__device__ __forceinline__ float weight_at(const void* row, int i, bool w8) {
    return w8 ? e4m3(static_cast<const uint8_t*>(row)[i])
              : __bfloat162float(static_cast<const __nv_bfloat16*>(row)[i]);
}

// h = silu(gate x) * up x: a warp a (choice, element of f).
__global__ void moe_gate_up_kernel(MoeArgs a) {
    pdl_wait();
    const crc_moe& m = a.m;
    const int lane = threadIdx.x & 31;
    const long long i = (long long)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
    if (i >= (long long)a.M * m.K * m.f) return;
    const int entry = (int)(i / m.f), j = (int)(i % m.f), tok = entry / m.K;
    const int s = slot_of(m, a.ids[entry]);
    if (s < 0) return;
    const bool w8 = m.weight_type == CRC_E4M3;
    const size_t row = (size_t)m.d * (w8 ? 1 : 2);
    const uint8_t* wg = static_cast<const uint8_t*>(m.gate_up_dev) + s * m.gate_up_stride + j * row;
    const uint8_t* wu = wg + (size_t)m.f * row;
    float g = 0.f, u = 0.f;
    for (int k = lane; k < m.d; k += 32) {
        const float x = a.x8 ? e4m3(a.x8[(size_t)tok * m.d + k])
                             : __uint_as_float((uint32_t)a.x[tok * a.ldx + k] << 16);
        g = fmaf(x, weight_at(wg, k, w8), g);
        u = fmaf(x, weight_at(wu, k, w8), u);
    }
    g = warp_sum(g);
    u = warp_sum(u);
    if (a.x8) {
        g *= a.xs8[tok];
        u *= a.xs8[tok];
    }
    if (w8) {
        const float* sc = reinterpret_cast<const float*>(
            reinterpret_cast<const uint8_t*>(m.gate_up_scale_dev) + s * m.gate_up_scale_stride);
        g *= sc[j];
        u *= sc[m.f + j];
    }
    if (lane == 0) a.h[(size_t)entry * m.f + j] = __float2bfloat16_rn(g / (1.f + expf(-g)) * u);
}

// out = sum_k gate_k down_k h_k: a warp a (token, element of d).
__global__ void moe_down_kernel(MoeArgs a) {
    const crc_moe& m = a.m;
    const int lane = threadIdx.x & 31;
    const long long i = (long long)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
    if (i >= (long long)a.M * m.d) return;
    const int tok = (int)(i / m.d), c = (int)(i % m.d);
    const bool w8 = m.weight_type == CRC_E4M3;
    float out = 0.f;
    for (int k = 0; k < m.K; ++k) {
        const int entry = tok * m.K + k;
        const int s = slot_of(m, a.ids[entry]);
        if (s < 0) continue;
        const uint8_t* w = static_cast<const uint8_t*>(m.down_dev) + s * m.down_stride +
                           (size_t)c * m.f * (w8 ? 1 : 2);
        float y = 0.f;
        for (int j = lane; j < m.f; j += 32)
            y = fmaf(__bfloat162float(a.h[(size_t)entry * m.f + j]), weight_at(w, j, w8), y);
        y = warp_sum(y);
        if (w8)
            y *= reinterpret_cast<const float*>(
                reinterpret_cast<const uint8_t*>(m.down_scale_dev) + s * m.down_scale_stride)[c];
        out = fmaf(a.gates[entry], y, out);
    }
    if (lane == 0) reinterpret_cast<__nv_bfloat16*>(a.out)[(size_t)tok * m.d + c] =
                       __float2bfloat16_rn(out);
}

int launch_route(const MoeRouteArgs& r, cudaStream_t stream) {
    cudaLaunchConfig_t c = {};
    c.blockDim = dim3(kRouteThreads);
    c.stream = stream;
    cudaError_t e;
    ProfScope prof(CRC_KERNEL_MOE_ROUTE, stream);
    if (r.scores) {
        c.gridDim = dim3((unsigned)((r.M + 7) / 8));
        e = cudaLaunchKernelEx(&c, moe_topk_kernel, r);
    } else {
        cudaLaunchAttribute at[1];
        at[0].id = cudaLaunchAttributeClusterDimension;
        at[0].val.clusterDim.x = kRouteCtas;
        at[0].val.clusterDim.y = 1;
        at[0].val.clusterDim.z = 1;
        c.attrs = at;
        c.numAttrs = 1;
        c.gridDim = dim3((unsigned)((r.M + kRouteTokens - 1) / kRouteTokens * kRouteCtas));
        e = cudaLaunchKernelEx(&c, moe_route_kernel, r);
    }
    note_launch();
    return cuda_status(e);
}

}  // namespace
}  // namespace crc

using namespace crc;

extern "C" {

size_t crc_moe_workspace_bytes(const crc_moe* m, int32_t M) {
    if (check_moe(m) != CRC_OK || M < 1 || M > kMoeMaxTokens || M * m->K > kMoeMaxEntries)
        return 0;
    return moe_layout(*m, M).total;
}

int crc_moe_layer(const crc_moe* m, const uint16_t* x_dev, int64_t x_stride, const uint8_t* x8_dev,
                  const float* x8_scale_dev, const float* scores_dev, int64_t scores_stride,
                  int32_t M, uint16_t* out_dev, uint8_t* topk_dev, float* gates_dev,
                  void* workspace_dev, size_t workspace_bytes, void* stream) {
    int rc = check_moe(m);
    if (rc) return rc;
    if (M < 0) return CRC_EINVAL;
    if ((x8_dev == nullptr) != (x8_scale_dev == nullptr)) return CRC_EINVAL;
    if (x8_dev && m->weight_type != CRC_E4M3) return CRC_EINVAL;
    if (M == 0) return CRC_OK;
    if (M > kMoeMaxTokens || M * m->K > kMoeMaxEntries) return CRC_EUNSUPPORTED;
    if (!x_dev && !(x8_dev && scores_dev)) return CRC_EINVAL;
    if (x_dev && (x_stride < m->d || x_stride % 8 != 0)) return CRC_EINVAL;
    if (scores_dev ? scores_stride < m->N : !m->router_dev) return CRC_EINVAL;
    if (!out_dev || !aligned(x_dev, 16) || !aligned(x8_dev, 16) || !aligned(x8_scale_dev, 4) ||
        !aligned(scores_dev, 4) || !aligned(out_dev, 16) || !aligned(gates_dev, 4))
        return CRC_EINVAL;
    if (!m->expert_slot_dev && m->N > m->slots) return CRC_EINVAL;
    const MoeLayout l = moe_layout(*m, M);
    if (!workspace_dev || !aligned(workspace_dev, 256) || workspace_bytes < l.total)
        return CRC_EINVAL;
    uint8_t* ws = static_cast<uint8_t*>(workspace_dev);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    MoeRouteArgs r = {};
    r.x = x_dev;
    r.w = m->router_dev;
    r.scores = scores_dev;
    r.ldx = x_stride;
    r.lds = scores_stride;
    r.M = M;
    r.N = m->N;
    r.K = m->K;
    r.d = m->d;
    r.renorm = m->renormalize;
    r.ids = ws + l.ids;
    r.gates = reinterpret_cast<float*>(ws + l.gates);
    r.ids_out = topk_dev;
    r.gates_out = gates_dev;
    r.xscale = m->weight_type == CRC_E4M3 && !x8_dev ? reinterpret_cast<float*>(ws + l.xscale)
                                                     : nullptr;
    r.ctrl = reinterpret_cast<uint32_t*>(ws + l.ctrl);
    r.ctrl_words = kCtrlWords;
    if ((rc = launch_route(r, st))) return rc;
    MoeArgs a;
    a.m = *m;
    a.x = x_dev;
    a.x8 = x8_dev;
    a.xs8 = x8_scale_dev;
    a.ldx = x_stride;
    a.M = M;
    a.ids = r.ids;
    a.gates = r.gates;
    a.h = reinterpret_cast<__nv_bfloat16*>(ws + l.h);
    a.y = reinterpret_cast<float*>(ws + l.y);
    a.out = out_dev;
    {
        ProfScope prof(CRC_KERNEL_MOE, st);
        moe_gate_up_kernel<<<(unsigned)(((long long)M * m->K * m->f + 7) / 8), 256, 0, st>>>(a);
        moe_down_kernel<<<(unsigned)(((long long)M * m->d + 7) / 8), 256, 0, st>>>(a);
    }
    note_launch();
    note_launch();
    return cuda_status(cudaGetLastError());
}

}  // extern "C"
