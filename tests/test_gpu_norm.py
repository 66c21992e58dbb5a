"""Root-mean-square norm with the residual's addition, its gradient, and rows in
8 bits, against their definitions in 64 bits and against differences."""
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


ROWS = [(1, 8), (1, 2048), (3, 200), (7, 1000), (2, 2880), (301, 264), (1000, 2880), (5, 4096),
        (2, 8192), (3, 16392), (2, 32768), (5000, 64)]


def near_e4m3(q, scale, y):
    """q is y / scale rounded to e4m3: within half a step (and the last bit of the
    quotient), saturating; the step is 2^-9 below 2^-6."""
    v = y / scale[:, None]
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
    return (q.double() - v).abs() <= 0.5 * step + 1e-5 * v.abs()


@pytest.mark.parametrize("M,d", ROWS)
@pytest.mark.parametrize("stream", ["bf16", "f32"])
@pytest.mark.parametrize("residual", [True, False])
def test_norm(P, M, d, stream, residual):
    g = torch.Generator(device="cuda").manual_seed(M + d)
    x, w = randn(g, M, d, dtype=DT[stream]), randn(g, d)
    res = randn(g, M, d, scale=3.0, dtype=DT[stream]) if residual else None
    h = torch.empty((M, d), dtype=torch.bfloat16, device="cuda")
    ro = torch.empty_like(x)
    q = torch.empty((M, d), dtype=torch.float8_e4m3fn, device="cuda")
    sc, rstd = torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    got = P.rms_norm(x, w, 1e-5, residual=res, residual_out=ro, out=h, out8=q, scale8=sc,
                     rstd=rstd)
    assert got is h
    s = x.double() + (res.double() if residual else 0.0)
    # the sum of two values is rounded to fp32 in any case
    assert ((ro.double() - s).abs() <= (RND[stream] + U32) * s.abs()).all()
    r = (s.square().mean(1) + 1e-5) ** -0.5
    # fp32 sums of positive terms over at most 1024 x 32 partial sums
    tol = (math.sqrt(d) + 8) * U32
    assert ((rstd.double() - r).abs() <= tol * r).all()
    y = s * r[:, None] * w.double()
    assert ((h.double() - y).abs() <= (U16 + tol + 4 * U32) * y.abs()).all()
    a = y.abs().amax(1) / 448.0
    assert ((sc.double() - a).abs() <= (tol + 8 * U32) * a).all()
    assert near_e4m3(q, sc.double(), y).all()
    # any one output alone gives the same bits
    assert torch.equal(P.rms_norm(x, w, 1e-5, residual=res), h)
    q2, sc2 = torch.empty_like(q), torch.empty_like(sc)
    assert P.rms_norm(x, w, 1e-5, residual=res, out8=q2, scale8=sc2) is None
    assert torch.equal(q2.view(torch.uint8), q.view(torch.uint8)) and torch.equal(sc2, sc)


def test_norm_in_place_and_strided(P):
    g = torch.Generator(device="cuda").manual_seed(1)
    big = randn(g, 9, 4, 256)
    x, w, res = big[:, 2], randn(g, 256), randn(g, 9, 256)
    ref_s = torch.empty_like(res)
    ref = P.rms_norm(x.contiguous(), w, residual=res, residual_out=ref_s)
    kept = big.clone()
    stream = res.clone()
    out = P.rms_norm(x, w, residual=stream, residual_out=stream)       # the residual in place
    assert torch.equal(out, ref) and torch.equal(stream, ref_s) and torch.equal(big, kept)
    y = x.contiguous()
    out = P.rms_norm(y, w, residual=res, residual_out=y)               # x in place
    assert torch.equal(out, ref) and torch.equal(y, ref_s)


def test_rows_of_zeros_and_not_finite_rows(P):
    g = torch.Generator(device="cuda").manual_seed(2)
    x, w = randn(g, 6, 512), randn(g, 512)
    clean = P.rms_norm(x, w)
    x[1] = 0
    x[2, 3] = float("nan")
    x[4, 500] = float("inf")
    q = torch.empty((6, 512), dtype=torch.float8_e4m3fn, device="cuda")
    sc = torch.empty(6, device="cuda")
    h = torch.empty_like(x)
    P.rms_norm(x, w, out=h, out8=q, scale8=sc)
    assert torch.equal(h[[0, 3, 5]], clean[[0, 3, 5]])
    assert (h[1] == 0).all() and (q[1].float() == 0).all() and sc[1] == 1.0
    assert torch.isnan(h[2].float()).all() and torch.isnan(sc[2])
    assert torch.isnan(q[2].float()).all()
    assert torch.isnan(h[4, 500].float()) and (h[4, :500] == 0).all()  # rstd = 0
    # eps = 0 on a row of zeros: 0 times infinity
    assert torch.isnan(P.rms_norm(x[1:2], w, 0.0).float()).all()


@pytest.mark.parametrize("M,d", [(1, 8), (1, 2048), (5, 200), (33, 2880), (1000, 264), (2000, 2048),
                                 (3, 32768), (610, 1000)])
@pytest.mark.parametrize("stream", ["bf16", "f32"])
@pytest.mark.parametrize("dres", [True, False])
def test_gradient(P, M, d, stream, dres):
    g = torch.Generator(device="cuda").manual_seed(M + d)
    s, w = randn(g, M, d, scale=3.0, dtype=DT[stream]), randn(g, d)
    dy = randn(g, M, d)
    dr = randn(g, M, d, dtype=DT[stream]) if dres else None
    rstd = torch.empty(M, device="cuda")
    P.rms_norm(s, w, 1e-5, rstd=rstd)
    dx, dw = P.rms_norm_grad(dy, s, w, rstd, dres=dr)
    t = s.double().requires_grad_(True)
    wd = w.double().requires_grad_(True)
    r = (t.square().mean(1, keepdim=True) + 1e-5) ** -0.5
    gx, gw = torch.autograd.grad(((t * r * wd) * dy.double()).sum(), (t, wd))
    gx = gx + (dr.double() if dres else 0.0)
    # magnitudes that the fp32 sums and products round
    rd = r.detach()
    v = (dy.double() * w.double()).abs()
    xh = s.double().abs() * rd
    mag = rd * (v + xh * (v * xh).mean(1, keepdim=True)) + (dr.double().abs() if dres else 0.0)
    tol = (math.sqrt(d) + 16) * U32
    assert ((dx.double() - gx).abs() <= RND[stream] * gx.abs() + 2 * tol * mag).all()
    wmag = (dy.double().abs() * xh).sum(0)
    assert ((dw.double() - gw).abs() <= (math.sqrt(M) + math.sqrt(d) + 16) * U32 * wmag).all()
    # without dw: the same dx; again: the same bits
    dx2, none = P.rms_norm_grad(dy, s, w, rstd, dres=dr, want_dw=False)
    assert none is None and torch.equal(dx2, dx)
    dx3, dw3 = P.rms_norm_grad(dy, s, w, rstd, dres=dr)
    assert torch.equal(dx3, dx) and torch.equal(dw3, dw)


def test_gradient_against_differences(P):
    """(f(s + e u) - f(s - e u)) / 2e of the fp32 forward pass's own definition, in
    64 bits, along random directions, against <dx, u> and <dw, u>."""
    g = torch.Generator(device="cuda").manual_seed(5)
    M, d = 4, 264
    s, w, dy = randn(g, M, d, dtype=torch.float32), randn(g, d), randn(g, M, d)
    rstd = torch.empty(M, device="cuda")
    P.rms_norm(s, w, 1e-5, rstd=rstd)
    dx, dw = P.rms_norm_grad(dy, s, w, rstd)

    def f(s, w):
        return (s * (s.square().mean(1, keepdim=True) + 1e-5) ** -0.5 * w * dy.double()).sum()

    e = 1e-5
    for i in range(5):
        u = torch.randn(M, d, device="cuda", generator=g).double()
        k = torch.randn(d, device="cuda", generator=g).double()
        s0, w0 = s.double(), w.double()
        num = (f(s0 + e * u, w0) - f(s0 - e * u, w0)) / (2 * e)
        ana = (dx.double() * u).sum()
        assert abs(num - ana) <= 1e-5 * (dx.double() * u).abs().sum()
        num = (f(s0, w0 + e * k) - f(s0, w0 - e * k)) / (2 * e)
        ana = (dw.double() * k).sum()
        assert abs(num - ana) <= 1e-5 * (dw.double() * k).abs().sum()


def test_gradient_in_place_and_without_rows(P):
    g = torch.Generator(device="cuda").manual_seed(6)
    s, w, dy, dr = (randn(g, 40, 256), randn(g, 256), randn(g, 40, 256), randn(g, 40, 256))
    rstd = torch.empty(40, device="cuda")
    P.rms_norm(s, w, rstd=rstd)
    dx, dw = P.rms_norm_grad(dy, s, w, rstd, dres=dr)
    a = dr.clone()
    P.rms_norm_grad(dy, s, w, rstd, dres=a, dx=a)
    assert torch.equal(a, dx)
    b = s.clone()
    P.rms_norm_grad(dy, b, w, rstd, dres=dr, dx=b)
    assert torch.equal(b, dx)
    _, dw0 = P.rms_norm_grad(dy[:0], s[:0], w, rstd[:0], dw=torch.ones_like(dw))
    assert (dw0 == 0).all()


@pytest.mark.parametrize("M,d", ROWS)
def test_quantize_rows(P, M, d):
    g = torch.Generator(device="cuda").manual_seed(M * d)
    x = randn(g, M, d, scale=d ** -0.5)
    x[M // 2] *= 0 if M > 1 else 1
    q, sc = P.quantize_rows(x)
    a = x.double().abs().amax(1) / 448.0
    a[a == 0] = 1.0
    assert ((sc.double() - a).abs() <= 2 * U32 * a).all()
    assert near_e4m3(q, sc.double(), x.double()).all()
    assert torch.isfinite(q.float()).all()


def test_quantize_shapes_strides_and_extremes(P):
    g = torch.Generator(device="cuda").manual_seed(9)
    x = randn(g, 6, 2, 48, 64)
    q, sc = P.quantize_rows(x)
    assert q.shape == x.shape and sc.shape == x.shape[:-1]
    y = x.reshape(-1, 64)[::3]
    q2, sc2 = P.quantize_rows(y)
    assert torch.equal(q2.view(torch.uint8), q.view(torch.uint8).reshape(-1, 64)[::3])
    assert torch.equal(sc2, sc.reshape(-1)[::3])
    z = torch.zeros((5, 64), dtype=torch.bfloat16, device="cuda")
    z[0, 0], z[1, 1], z[2, 2] = 1e-38, 3e38, float("nan")
    z[3, 3], z[3, 4] = float("-inf"), 2.0
    q, sc = P.quantize_rows(z)
    assert abs(float(q[0, 0].float())) == 448.0 and float(q[1, 1].float()) == 448.0
    assert float(q[0, 1].float()) == 0.0
    assert torch.isnan(sc[2]) and torch.isnan(q[2].float()).all()
    assert torch.isinf(sc[3]) and torch.isnan(q[3, 3].float()) and q[3, 4].float() == 0
    assert sc[4] == 1.0 and (q[4].float() == 0).all()


def test_refusals_of_the_binding(P):
    x = torch.zeros((4, 64), dtype=torch.bfloat16, device="cuda")
    w = torch.zeros(64, dtype=torch.bfloat16, device="cuda")
    for bad in (lambda: P.rms_norm(x.half(), w), lambda: P.rms_norm(x, w.float()),
                lambda: P.rms_norm(x, w[:32]), lambda: P.rms_norm(x.t(), w),
                lambda: P.rms_norm(x, w, residual=x.float()), lambda: P.rms_norm(x.cpu(), w),
                lambda: P.quantize_rows(x.float()),
                lambda: P.rms_norm_grad(x, x, w, torch.zeros(3, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    y = torch.zeros((4, 60), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(P.CrcError):
        P.rms_norm(y, w[:60].contiguous())
