"""The gradient of the sum over choices along directions that add its elements up."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U16, U32 = 2.0 ** -8, 2.0 ** -24


@pytest.fixture(scope="module")
def P():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_04895_gb300 import build
    build.build()
    import paper_2609_04895_gb300 as P
    P.crc.load()
    return P


@pytest.mark.parametrize("M,K,d", [(40, 4, 256), (301, 8, 264), (90, 1, 2880), (33, 2, 4096)])
def test_differences_along_the_gradient(P, M, K, d):
    """f = <dout, sum(y, gates)> changes by the sum of |dy| |u| along u = sign(dy) gate |normal|, so
    that a scaled, missing or exchanged gate shows: each element of dy is off by half a bf16 step, and
    the sum of |dy u| is the change itself."""
    g = torch.Generator(device="cuda").manual_seed(M)
    R = M * K + 5
    place = torch.randperm(R, device="cuda", generator=g)[:M * K].to(torch.int32).view(M, K)
    place[torch.rand((M, K), device="cuda", generator=g) < 0.2] = -1
    y = torch.randn((R, d), device="cuda", generator=g).bfloat16()
    dout = torch.randn((M, d), device="cuda", generator=g).bfloat16()
    gates = torch.rand((M, K), device="cuda", generator=g)
    dy, dg = P.sum_choices_grad(dout, place, gates=gates, y=y,
                                dy=torch.zeros((R, d), dtype=torch.bfloat16, device="cuda"))

    def f(y, gates):
        ok = (place >= 0)[..., None]
        rows = torch.where(ok, y[place.clamp(min=0).long()], 0.0)
        return (dout.double() * (rows * gates[..., None]).sum(1)).sum()
    y0, g0, h = y.double(), gates.double(), 1e-3
    uy = torch.zeros((R, d), dtype=torch.float64, device="cuda")
    m, j = torch.nonzero(place >= 0, as_tuple=True)
    uy[place[m, j].long()] = dout.double()[m].sign() * g0[m, j][:, None]
    uy *= torch.randn((R, d), device="cuda", generator=g, dtype=torch.float64).abs()
    by_y = (f(y0 + h * uy, g0) - f(y0 - h * uy, g0)) / (2 * h)
    got = (dy.double() * uy).sum()
    assert by_y > 0 and abs(by_y - got) <= 1e-9 * by_y + (U16 + U32) * by_y
    # what this notices: no gates, another choice's, 1% too much
    for wrong in (torch.ones_like(g0), g0.flatten().roll(1).view(M, K), 1.01 * g0):
        off = (dout.double()[m] * wrong[m, j][:, None] * uy[place[m, j].long()]).sum()
        assert abs(by_y - off) > 2 * (U16 + U32) * by_y
    # the gates' direction: the sign of each choice's own product
    ug = torch.zeros((M, K), dtype=torch.float64, device="cuda")
    prod = dout.double()[m] * y0[place[m, j].long()]
    ug[m, j] = prod.sum(-1).sign()
    by_g = (f(y0, g0 + h * ug) - f(y0, g0 - h * ug)) / (2 * h)
    got = (dg.double() * ug).sum()
    # every dot product is off by at most d steps of its terms
    assert by_g > 0 and abs(by_g - got) <= 1e-9 * by_g + d * U32 * prod.abs().sum()
    assert (dg[place < 0] == 0).all()
