"""Host-only checks of the operators around the router heads: argument checks of
crc_rms_norm, crc_rms_norm_grad, crc_quantize_rows and crc_moe_layer (nothing is
launched here)."""
import ctypes

import pytest

EINVAL, EUNSUPPORTED = 1, 2


@pytest.fixture(scope="module")
def C():
    from paper_2609_04895_gb300 import build
    build.build()
    from paper_2609_04895_gb300 import crc
    crc.load()
    return crc


def test_struct_layout(C):
    assert ctypes.sizeof(C.crc_moe) == 32 + 10 * 8
    assert ctypes.sizeof(C.crc_kernel_times) == 2 * 8 * len(C.KERNEL_KINDS)


def norm(C, x=256, ldx=64, res=None, w=512, kind=1, M=4, d=64, eps=1e-6, ro=None, out=1024,
         out8=None, sc=None, rstd=None):
    return C.load().crc_rms_norm(x, ldx, res, w, kind, M, d, eps, ro, out, out8, sc, rstd, None)


@pytest.mark.parametrize("bad,code", [
    (dict(d=0), EINVAL), (dict(M=-1), EINVAL), (dict(d=60, ldx=64), EUNSUPPORTED),
    (dict(d=32776, ldx=32776), EUNSUPPORTED), (dict(M=1 << 31), EUNSUPPORTED),
    (dict(kind=3), EINVAL), (dict(kind=0), EINVAL), (dict(eps=-1.0), EINVAL),
    (dict(eps=float("nan")), EINVAL), (dict(ldx=56), EINVAL), (dict(ldx=68), EINVAL),
    (dict(out8=4096), EINVAL), (dict(sc=4096), EINVAL), (dict(x=None), EINVAL),
    (dict(w=None), EINVAL), (dict(out=None), EINVAL), (dict(x=264), EINVAL),
    (dict(res=8), EINVAL), (dict(out=1032), EINVAL), (dict(out8=4, sc=4096), EINVAL),
    (dict(rstd=2), EINVAL), (dict(ro=8), EINVAL),
])
def test_norm_arguments(C, bad, code):
    assert norm(C, **bad) == code
    assert norm(C, M=0) == 0


def grad(C, dy=256, s=512, w=1024, rstd=2048, dres=None, kind=1, M=4, d=64, dx=4096, dw=None,
         ws=None, wsb=0):
    return C.load().crc_rms_norm_grad(dy, s, w, rstd, dres, kind, M, d, dx, dw, ws, wsb, None)


@pytest.mark.parametrize("bad,code", [
    (dict(d=4), EUNSUPPORTED), (dict(kind=3), EINVAL), (dict(M=-1), EINVAL),
    (dict(dy=None), EINVAL), (dict(s=None), EINVAL), (dict(w=None), EINVAL),
    (dict(rstd=None), EINVAL), (dict(dx=None), EINVAL), (dict(dx=8), EINVAL),
    (dict(dres=8), EINVAL), (dict(dw=8192), EINVAL), (dict(dw=2), EINVAL),
    (dict(dw=8192, ws=128, wsb=1 << 20), EINVAL), (dict(dw=8192, ws=256, wsb=16), EINVAL),
])
def test_norm_gradient_arguments(C, bad, code):
    assert grad(C, **bad) == code
    assert grad(C, M=0) == 0
    assert C.crc_rms_norm_grad_workspace_bytes(0, 64) == 0
    assert C.crc_rms_norm_grad_workspace_bytes(4, 60) == 0
    assert C.crc_rms_norm_grad_workspace_bytes(4, 64) >= 4


@pytest.mark.parametrize("bad,code", [
    (dict(d=12), EUNSUPPORTED), (dict(ldx=8), EINVAL), (dict(ldx=17), EINVAL),
    (dict(x=None), EINVAL), (dict(q=None), EINVAL), (dict(sc=None), EINVAL), (dict(x=8), EINVAL),
    (dict(q=4), EINVAL), (dict(M=-1), EINVAL),
])
def test_quantize_arguments(C, bad, code):
    call = lambda x=256, ldx=16, M=2, d=16, q=512, sc=1024: C.load().crc_quantize_rows(  # noqa: E731
        x, ldx, M, d, q, sc, None)
    assert call(**bad) == code
    assert call(M=0) == 0


def moe(C, **over):
    m = C.crc_moe(N=16, K=2, d=64, f=32, slots=16, weight_type=1, renormalize=1, reserved=0,
                  gate_up_dev=256, down_dev=512, gate_up_stride=2 * 64 * 32 * 2,
                  down_stride=64 * 32 * 2, router_dev=1024)
    for k, v in over.items():
        setattr(m, k, v)
    return m


W8 = dict(weight_type=3, gate_up_scale_dev=256, down_scale_dev=256, gate_up_scale_stride=256,
          down_scale_stride=256)


@pytest.mark.parametrize("bad,code", [
    (dict(reserved=1), EINVAL), (dict(N=0), EINVAL), (dict(N=24), EUNSUPPORTED),
    (dict(N=144), EUNSUPPORTED), (dict(K=0), EINVAL), (dict(K=17), EUNSUPPORTED),
    (dict(N=64, slots=64, K=33), EUNSUPPORTED), (dict(d=60), EUNSUPPORTED), (dict(f=24), EUNSUPPORTED),
    (dict(f=8), EUNSUPPORTED), (dict(slots=0), EINVAL), (dict(weight_type=2), EINVAL),
    (dict(renormalize=2), EINVAL), (dict(gate_up_dev=None), EINVAL), (dict(down_dev=8), EINVAL),
    (dict(gate_up_stride=8192 - 16), EINVAL), (dict(down_stride=4096 + 8), EINVAL),
    (dict(gate_up_stride=1 << 40), EUNSUPPORTED), (dict(router_dev=8), EINVAL),
    (dict(expert_slot_dev=2), EINVAL), (dict(gate_up_scale_dev=256), EINVAL),
    (dict(weight_type=3), EINVAL), (dict(W8, d=72), EUNSUPPORTED),
    (dict(W8, gate_up_scale_stride=252), EINVAL), (dict(W8, down_scale_stride=252), EINVAL),
    (dict(W8, down_scale_dev=2), EINVAL),
])
def test_moe_description(C, bad, code):
    m = moe(C, **bad)
    assert C.crc_moe_workspace_bytes(m, 4) == 0
    assert C.load().crc_moe_layer(ctypes.byref(m), 256, 64, None, None, None, 0, 4, 4096, None,
                                  None, 256, 1 << 30, None) == code


def test_moe_arguments(C):
    m = moe(C)
    n = C.crc_moe_workspace_bytes(m, 4)
    assert n > 0 and C.crc_moe_workspace_bytes(m, 0) == 0
    assert C.crc_moe_workspace_bytes(m, 1025) == 0
    assert C.crc_moe_workspace_bytes(moe(C, K=16), 513) == 0
    assert C.crc_moe_workspace_bytes(moe(C, **W8), 4) > 0

    def call(m=m, x=256, ldx=64, x8=None, xs=None, scores=None, lds=0, M=4, out=4096, topk=None,
             gates=None, ws=256, wsb=n):
        return C.load().crc_moe_layer(ctypes.byref(m), x, ldx, x8, xs, scores, lds, M, out, topk,
                                      gates, ws, wsb, None)

    assert C.load().crc_moe_layer(None, 256, 64, None, None, None, 0, 4, 4096, None, None, 256, n,
                                  None) == EINVAL
    assert call(M=0) == 0
    assert call(M=-1) == EINVAL
    assert call(M=1025) == EUNSUPPORTED
    assert call(m=moe(C, K=16), M=513) == EUNSUPPORTED
    assert call(x=None) == EINVAL and call(x=8) == EINVAL
    assert call(ldx=56) == EINVAL and call(ldx=68) == EINVAL
    assert call(out=None) == EINVAL and call(out=8) == EINVAL
    assert call(ws=None) == EINVAL and call(ws=128) == EINVAL and call(wsb=n - 1) == EINVAL
    assert call(x8=256, xs=256) == EINVAL                        # 16-bit weights
    assert call(m=moe(C, **W8), x8=256) == EINVAL                # rows without their scales
    assert call(scores=256, lds=15) == EINVAL
    assert call(scores=2, lds=16) == EINVAL
    assert call(gates=2) == EINVAL
    assert call(m=moe(C, router_dev=None)) == EINVAL
    assert call(m=moe(C, slots=8)) == EINVAL                     # 16 experts, 8 slots, no map
