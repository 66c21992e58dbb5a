// The mixture-of-experts layer for a few tokens: entry points, workspace and
// the experts' kernels.
#include <cudaTypedefs.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "crc_internal.h"
#include "moe_experts.cuh"
#include "moe_route.cuh"

namespace crc {

PFN_cuTensorMapEncodeTiled_v12000 encode_fn();      // router.cu

namespace {

constexpr int kMoeMaxTokens = 1024;
constexpr int kMoeMaxEntries = 8192;      // M K

inline bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
inline size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }

// Rows of a tile, by an expert's mean share of the choices, with room for a few more so
// that few experts need a second pass over their weights, or the tokens if that is fewer.
// Narrow tiles leave room for more row blocks in flight.  us with 16 / 32 / 64 rows, 8-bit
// weights: mean 6.25 (d = 2048, f = 768) 116 / 118 / 128, 7.5 (d = 4096, f = 1536)
// 396 / 381 / 387, 18.75 (d = 2048, f = 1024) 120 / 95 / 101, 25 (d = f = 2880)
// 238 / 162 / 169; bf16: 6.25 187 / 188 / 189, 7.5 699 / 705 / 710, 18.75 150 / 133 / 136, 25
// 319 / 261 / 257, 31 (d = 2048, f = 768) 232 / 243 / 231.
int row_tile(int M, int K, int N) {
    const int E = M * K;
    if (E <= 128 * 16 && (M <= 16 || E <= 6 * N)) return 16;
    if (E <= 128 * 32 && (M <= 32 || E <= 26 * N)) return 32;
    return 64;
}

struct MoeLayout {
    size_t ctrl, hmax, logits, ids, gates, xscale, h, y, xq, hq, total;     // hmax right behind ctrl
};

MoeLayout moe_layout(const crc_moe& m, int M) {
    const size_t E = (size_t)M * m.K;
    MoeLayout l;
    l.ctrl = 0;
    l.hmax = kCtrlWords * 4;
    l.logits = up256(l.hmax + E * 4);
    l.ids = l.logits + (few_choices(M, m.K) ? up256((size_t)M * m.N * 4) : 0);
    l.gates = l.ids + up256(E);
    l.xscale = l.gates + up256(E * 4);
    l.h = l.xscale + up256((size_t)M * 4);
    l.y = l.h + up256(E * m.f * 4);
    l.xq = l.y + up256(E * m.d * 4);
    const bool pieces = m.weight_type == CRC_E4M3 && row_tile(M, m.K, m.N) > 16;
    l.hq = l.xq + (pieces ? up256((size_t)M * 2 * m.d) : 0);
    l.total = l.hq + (pieces ? up256(E * 2 * m.f) : 0);
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

// Tensor maps of the weights.  gate and up as (d, 16 rows, gate / up, f / 16,
// slots), a box of one 128-byte row x 16 x 2 x 4: four groups of 16 gate rows
// and the 16 up rows of the same elements.  down as (f, d, slots), 128 rows a box.
bool make_expert_maps(CUtensorMap* m13, CUtensorMap* m2, const crc_moe& m) {
    auto enc = encode_fn();
    if (!enc) return false;
    const bool w8 = m.weight_type == CRC_E4M3;
    const cuuint64_t es = w8 ? 1 : 2, d = m.d, f = m.f, slots = m.slots;
    const cuuint32_t bk = w8 ? 128 : 64;
    const CUtensorMapDataType type =
        w8 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
    const cuuint32_t ones[5] = {1, 1, 1, 1, 1};
    const cuuint64_t dims13[5] = {d, 16, 2, f / 16, slots};
    const cuuint64_t str13[4] = {d * es, f * d * es, 16 * d * es, (cuuint64_t)m.gate_up_stride};
    const cuuint32_t box13[5] = {bk, 16, 2, 4, 1};
    const cuuint64_t dims2[3] = {f, d, slots};
    const cuuint64_t str2[2] = {f * es, (cuuint64_t)m.down_stride};
    const cuuint32_t box2[3] = {bk, 128, 1};
    return enc(m13, type, 5, const_cast<void*>(m.gate_up_dev), dims13, str13, box13, ones,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
               CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS &&
           enc(m2, type, 3, const_cast<void*>(m.down_dev), dims2, str2, box2, ones,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
               CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <bool W8, int NT>
int launch_experts(const crc_moe& m, const MoeArgs& a, cudaStream_t stream) {
    using Cfg = MoeCfg<W8, NT>;
    auto kern = moe_experts_kernel<W8, NT>;
    static PerDevice ready;
    const int up = ready.get(current_device(), [&] {
        return cuda_status(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                Cfg::SMEM)) == CRC_OK;
    });
    if (!up) return CRC_ECUDA;
    CUtensorMap m13, m2;
    if (!make_expert_maps(&m13, &m2, m)) return CRC_ECUDA;
    // no more CTAs than items there can be
    const long long experts = (long long)a.M * a.K < a.N ? (long long)a.M * a.K : a.N;
    const long long items =
        (experts + (long long)a.M * a.K / NT) * (a.ft + a.dt + 1) +
        (long long)a.M * (a.d / 16) / kSplitUnits + 1;
    cudaError_t e;
    {
        ProfScope prof(CRC_KERNEL_MOE, stream);
        e = launch_dependent(kern, dim3((unsigned)(items < sm_count() ? items : sm_count())),
                             kMoeThreads, Cfg::SMEM, stream, 1, m13, m2, a);
    }
    note_launch();
    return cuda_status(e);
}

int launch_route(const MoeRouteArgs& r, cudaStream_t stream) {
    cudaError_t e;
    {
        ProfScope prof(CRC_KERNEL_MOE_ROUTE, stream);
        if (r.logits)
            e = launch_dependent(moe_logits_kernel, dim3((unsigned)((r.N + 7) / 8), (unsigned)r.M),
                                 kRouteThreads, 0, stream, 1, r);
        else if (r.scores)
            e = launch_dependent(moe_topk_kernel, dim3((unsigned)((r.M + 7) / 8)), kRouteThreads, 0,
                                 stream, 1, r);
        else
            e = launch_dependent(
                moe_route_kernel,
                dim3((unsigned)((r.M + kRouteTokens - 1) / kRouteTokens * kRouteCtas)),
                kRouteThreads, 0, stream, kRouteCtas, r);
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
    r.logits = few_choices(M, m->K) && !scores_dev ? reinterpret_cast<float*>(ws + l.logits) : nullptr;
    r.ids = ws + l.ids;
    r.gates = reinterpret_cast<float*>(ws + l.gates);
    r.ids_out = topk_dev;
    r.gates_out = gates_dev;
    r.xscale = m->weight_type == CRC_E4M3 && !x8_dev ? reinterpret_cast<float*>(ws + l.xscale)
                                                     : nullptr;
    r.ctrl = reinterpret_cast<uint32_t*>(ws + l.ctrl);
    const bool w8 = m->weight_type == CRC_E4M3;
    r.ctrl_words = kCtrlWords + (w8 ? M * m->K : 0);
    MoeArgs a = {};
    a.x = x8_dev ? x8_dev : reinterpret_cast<const uint8_t*>(x_dev);
    a.x_bytes = x8_dev ? m->d : 2 * x_stride;
    a.xs = x8_dev ? x8_scale_dev : r.xscale;
    a.x_split = w8 && !x8_dev;
    a.ids = r.ids;
    a.gates = r.gates;
    a.logits = r.logits;
    a.ids_out = topk_dev;
    a.gates_out = gates_dev;
    a.renorm = m->renormalize;
    a.expert_slot = m->expert_slot_dev;
    a.s13 = m->gate_up_scale_dev;
    a.s2 = m->down_scale_dev;
    a.s13_stride = m->gate_up_scale_stride / 4;
    a.s2_stride = m->down_scale_stride / 4;
    a.h = reinterpret_cast<float*>(ws + l.h);
    a.y = reinterpret_cast<float*>(ws + l.y);
    a.xq = ws + l.xq;
    a.hq = ws + l.hq;
    a.hmax = reinterpret_cast<uint32_t*>(ws + l.hmax);
    a.ctrl = r.ctrl;
    a.err = device_error_word();
    a.out = reinterpret_cast<__nv_bfloat16*>(out_dev);
    a.M = M;
    a.N = m->N;
    a.K = m->K;
    a.d = m->d;
    a.f = m->f;
    a.slots = m->slots;
    const int bk = w8 ? 256 : 128;           // elements of 256 bytes
    a.kb1 = (m->d + bk - 1) / bk;
    a.kb2 = (m->f + bk - 1) / bk;
    a.ft = (m->f + 63) / 64;
    a.dt = (m->d + 127) / 128;
    if ((rc = launch_route(r, st))) return rc;
    const int nt = row_tile(M, m->K, m->N);
    if (w8)
        return nt == 16   ? launch_experts<true, 16>(*m, a, st)
               : nt == 32 ? launch_experts<true, 32>(*m, a, st)
                          : launch_experts<true, 64>(*m, a, st);
    return nt == 16   ? launch_experts<false, 16>(*m, a, st)
           : nt == 32 ? launch_experts<false, 32>(*m, a, st)
                      : launch_experts<false, 64>(*m, a, st);
}

}  // extern "C"
