"""Rows in 8 bits, bit for bit: q = e4m3(x / scale) with the division rounded to fp32
once, as the header states it."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_04895_gb300 import build
    build.build()
    import paper_2609_04895_gb300 as P
    P.crc.load()
    return P


def bits(q):
    return q.view(torch.uint8)


@pytest.mark.parametrize("M,d", [(4000, 2048), (20000, 2880), (30000, 264), (3, 32768)])
@pytest.mark.parametrize("exponent", [0, -40, -76, -84, -100, -120, 100])
def test_the_quotient_is_rounded_as_a_division(P, M, d, exponent):
    """Quotients that fall on the middle of two e4m3 values are common (a bf16 row
    whose largest value is 448 times a power of two, among others): a product with the
    rounded reciprocal takes some of them to the other side."""
    g = torch.Generator(device="cuda").manual_seed(M + d)
    x = (torch.randn((M, d), device="cuda", generator=g) * 2.0 ** exponent).bfloat16()
    q, sc = P.quantize_rows(x)
    assert torch.equal(sc, (x.abs().amax(1).double() / 448.0).float())
    want = (x.float() / sc[:, None]).to(torch.float8_e4m3fn)
    assert torch.equal(bits(q), bits(want))


def test_every_bf16_against_scales_of_many_rows(P):
    """All bf16 values up to a row's largest, for 300 largest values of every mantissa."""
    v = torch.arange(0x7f80, dtype=torch.int32, device="cuda").to(torch.int16).view(torch.bfloat16)
    v = v[v.float() <= 2.0 ** 20]
    v = torch.cat([v, -v])[:len(v) // 4 * 8]
    tops = torch.exp2(torch.linspace(-110.0, 20.0, 300, device="cuda")).bfloat16()
    for i in range(0, 300, 50):
        top = tops[i:i + 50, None]
        x = torch.where(v.abs()[None] <= top, v[None], torch.zeros_like(top))
        x[:, :1] = top
        x = x[:, torch.arange(32768, device="cuda") % x.shape[1]].contiguous()
        x[:, :1] = top
        q, sc = P.quantize_rows(x)
        assert torch.equal(sc, (top[:, 0].double() / 448.0).float())
        assert torch.equal(bits(q), bits((x.float() / sc[:, None]).to(torch.float8_e4m3fn)))


def test_a_row_too_small_for_a_scale_is_zero(P):
    """max |y| / 448 is zero in fp32 below 3.2e-43: the zeros of such a row stay zeros."""
    d = 256
    x = torch.zeros((3, d), device="cuda")
    x[0, ::3], x[1, 5], x[2] = 1e-3, -1e-3, 1.0
    w = torch.ones(d, dtype=torch.int16, device="cuda").view(torch.bfloat16)       # 9.2e-41
    q = torch.empty((3, d), dtype=torch.float8_e4m3fn, device="cuda")
    sc, h = torch.empty(3, device="cuda"), torch.empty((3, d), dtype=torch.bfloat16, device="cuda")
    P.rms_norm(x, w, 1.0, out=h, out8=q, scale8=sc)
    assert (sc[:2] == 1.0).all() and (q[:2].float() == 0).all()
    assert 0.0 < float(sc[2]) < 1e-42 and (q[2].float() > 400).all()
