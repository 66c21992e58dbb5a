"""The norm's gradient, 8-bit rows and the norm where a team of warps takes row after row:
every form of the kernels (groups a thread, teams a CTA, rings of two to eight rows and
none), with more rows than are resident at once."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U16, U32 = 2.0 ** -8, 2.0 ** -24      # unit roundoff of bf16 (8 significant bits) and fp32
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
RND = {"bf16": U16, "f32": U32}


@pytest.fixture(scope="module")
def P():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_04895_gb300 import build
    build.build()
    import paper_2609_04895_gb300 as P
    P.crc.load()
    return P


def randn(g, *shape, scale=1.0, dtype=torch.bfloat16):
    return (torch.randn(shape, device="cuda", generator=g) * scale).to(dtype)


# rows, d: eight, four and two teams a CTA; one of 8 to 16 warps with one, two and four
# groups a thread; more than 512 threads; rows too wide for a ring
GRAD = [(40009, 200), (20011, 264), (20011, 512), (8003, 1000), (6007, 2048), (4001, 2880),
        (3001, 4096), (2003, 4104), (2003, 6144), (1801, 8192), (1601, 8200), (1601, 12288),
        (1301, 16384), (1301, 16392), (901, 20480), (701, 32768)]


@pytest.mark.parametrize("M,d", GRAD)
@pytest.mark.parametrize("stream", ["bf16", "f32"])
@pytest.mark.parametrize("dres", [True, False])
def test_gradient_of_many_rows(P, M, d, stream, dres):
    g = torch.Generator(device="cuda").manual_seed(M + d)
    s, w = randn(g, M, d, scale=3.0, dtype=DT[stream]), randn(g, d)
    dy = randn(g, M, d)
    dr = randn(g, M, d, dtype=DT[stream]) if dres else None
    rstd = torch.empty(M, device="cuda")
    P.rms_norm(s, w, 1e-5, rstd=rstd)
    dx, dw = P.rms_norm_grad(dy, s, w, rstd, dres=dr)
    again, dw_again = P.rms_norm_grad(dy, s, w, rstd, dres=dr)
    assert torch.equal(again, dx) and torch.equal(dw_again, dw)
    alone, _ = P.rms_norm_grad(dy, s, w, rstd, dres=dr, want_dw=False)
    assert torch.equal(alone, dx)
    # in place, on the residual's gradient and on s
    if dres:
        a = dr.clone()
        assert torch.equal(P.rms_norm_grad(dy, s, w, rstd, dres=a, dx=a)[0], dx)
    a = s.clone()
    assert torch.equal(P.rms_norm_grad(dy, a, w, rstd, dres=dr, dx=a)[0], dx)
    tol = (math.sqrt(d) + 16) * U32
    want_dw = torch.zeros(d, dtype=torch.float64, device="cuda")
    wmag = torch.zeros_like(want_dw)
    for i in range(0, M, 2048):
        at = slice(i, min(i + 2048, M))
        t, y = s[at].double(), dy[at].double()
        r = (t.square().mean(1, keepdim=True) + 1e-5) ** -0.5
        xh, v = t * r, y * w.double()
        res = dr[at].double() if dres else torch.zeros_like(t)
        want = res + r * (v - xh * (v * xh).mean(1, keepdim=True))
        # magnitudes that the fp32 sums and products round
        mag = r * (v.abs() + xh.abs() * (v * xh).abs().mean(1, keepdim=True)) + res.abs()
        off = (dx[at].double() - want).abs()
        assert (off <= RND[stream] * want.abs() + 2 * tol * mag).all()
        want_dw += (y * xh).sum(0)
        wmag += (y * xh).abs().sum(0)
    assert ((dw.double() - want_dw).abs() <= (math.sqrt(M) + math.sqrt(d) + 16) * U32 * wmag).all()
    assert P.crc.crc_device_error() == 0


@pytest.mark.parametrize("M,d", [(40001, 64), (40001, 264), (30001, 512), (20001, 768), (8003, 2880),
                                 (5003, 4104), (3001, 8192), (2501, 12288), (1501, 16384),
                                 (1501, 16392), (1001, 32768)])
def test_eight_bit_rows_of_many_rows(P, M, d):
    g = torch.Generator(device="cuda").manual_seed(M + d)
    # neighbouring rows of different size: a scale or a value of another row is seen
    x = randn(g, M, d)
    x *= torch.exp2((torch.arange(M, device="cuda") % 13 - 6).float())[:, None].bfloat16()
    x[M // 2] = 0
    q, sc = P.quantize_rows(x)
    want = (x.abs().amax(1).double() / 448.0).float()
    want[M // 2] = 1.0
    assert torch.equal(sc, want)
    q64 = (x.float() / sc[:, None]).to(torch.float8_e4m3fn)
    assert torch.equal(q.view(torch.uint8), q64.view(torch.uint8))


@pytest.mark.parametrize("M,d", [(20011, 264), (5001, 1000), (3001, 4104), (2001, 8192), (1501, 16384),
                                 (1501, 16392), (701, 32768)])
@pytest.mark.parametrize("stream", ["bf16", "f32"])
def test_norm_of_many_rows(P, M, d, stream):
    g = torch.Generator(device="cuda").manual_seed(M + d)
    x, res, w = (randn(g, M, d, dtype=DT[stream]), randn(g, M, d, scale=3.0, dtype=DT[stream]),
                 randn(g, d))
    h, ro = torch.empty((M, d), dtype=torch.bfloat16, device="cuda"), torch.empty_like(x)
    P.rms_norm(x, w, 1e-5, residual=res, residual_out=ro, out=h)
    s = x.double() + res.double()
    assert ((ro.double() - s).abs() <= (RND[stream] + U32) * s.abs()).all()
    y = s * (s.square().mean(1, keepdim=True) + 1e-5) ** -0.5 * w.double()
    tol = (math.sqrt(d) + 12) * U32
    assert ((h.double() - y).abs() <= (U16 + tol) * y.abs()).all()
