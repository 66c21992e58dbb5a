"""Calls with no choices: they do nothing (a gradient sets dw to zero), whatever Top-K is."""
import ctypes

import pytest

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def P():
    from paper_2609_04895_gb300 import build
    build.build()
    import paper_2609_04895_gb300 as P
    P.crc.load()
    return P


@pytest.mark.parametrize("K", [1, 2, 8])
def test_no_rows_have_no_address(P, K):
    """An empty tensor's address is NULL: of rows too, which K > 1 wants for E > 0."""
    w = P.crc.crc_group_weights(N=4, n=32, k=64, glu=0, weight_type=1, reserved=0, w_dev=256,
                                w_stride=32 * 64 * 2, scale_dev=None, scale_stride=0)
    lib = P.crc.load()
    assert lib.crc_group_matmul(ctypes.byref(w), None, 64, 0, None, 512, None, K, 0, None, None) == 0
    assert lib.crc_group_matmul_grad(ctypes.byref(w), None, None, 64, 0, 512, None, K, 0, None, None,
                                     2, None) == 0
    assert lib.crc_group_matmul(ctypes.byref(w), 256, 64, 0, None, 512, None, K, 8, 1024, None) == 1


@pytest.mark.gpu
@pytest.mark.parametrize("K", [1, 4])
def test_a_prompt_of_no_tokens(P, K):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    g = torch.Generator(device="cuda").manual_seed(1)
    new = lambda *s: torch.randn(s, device="cuda", generator=g).bfloat16()  # noqa: E731
    w13, w2 = new(16, 2, 48, 64), new(16, 64, 48)
    x, topk = new(0, 64), torch.empty((0, K), dtype=torch.uint8, device="cuda")
    gates = torch.empty((0, K), device="cuda")
    assert P.MoeLayer(w13, w2, K=K).prompt(x, topk, gates).shape == (0, 64)
    (q13, s13), (q2, s2) = P.quantize_rows(w13), P.quantize_rows(w2)
    lay = P.MoeLayer(q13, q2, K=K, gate_up_scale=s13, down_scale=s2)
    assert lay.prompt(x, topk, gates).shape == (0, 64)
    off, rows, place = P.group_choices(topk, 16)
    dw = torch.ones((16, 96, 64), device="cuda")
    dx, _ = P.group_matmul_grad(new(0, 96), x, w13.flatten(1, 2), off, rows=rows, K=K, dw=dw)
    assert dx.shape == (0, 64) and (dw == 0).all()
    dy, dg = P.sum_choices_grad(x, place, gates=gates, y=dx)
    assert dy.shape == (0, 64) and dg.shape == (0, K)
    assert P.crc.crc_device_error() == 0
