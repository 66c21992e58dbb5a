"""The C entries under their own names, with addresses, against the functions on tensors."""
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


M, N, K, n, k = 40, 8, 2, 48, 64


@pytest.fixture(scope="module")
def a(P):
    g = torch.Generator(device="cuda").manual_seed(1)
    new = lambda *s: torch.randn(s, device="cuda", generator=g).bfloat16()  # noqa: E731
    a = dict(x=new(M, k), w=new(N, n, k), dy=new(M * K, n), dout=new(M, n),
             gates=torch.rand((M, K), device="cuda", generator=g),
             topk=torch.randint(0, N, (M, K), device="cuda", generator=g).to(torch.uint8))
    a["offsets"], a["rows"], a["place"] = P.group_choices(a["topk"], N)
    a["y"] = P.group_matmul(a["x"], a["w"], a["offsets"], rows=a["rows"], K=K)
    return a


def of(P, w, scale=None):
    return P.crc.crc_group_weights(N=N, n=n, k=k, glu=0, weight_type=1 if scale is None else 3,
                                   reserved=0, w_dev=w.data_ptr(), w_stride=w[0].nbytes,
                                   scale_dev=None if scale is None else scale.data_ptr(),
                                   scale_stride=0 if scale is None else 4 * n)


def p(*ts):
    return [None if t is None else t.data_ptr() for t in ts]


def test_group_choices(P, a):
    out = [torch.full_like(a[name], -7) for name in ("offsets", "rows", "place")]
    P.crc.crc_group_choices(*p(a["topk"]), M, K, N, *p(*out), None, 0)
    assert all(torch.equal(o, a[name]) for o, name in zip(out, ("offsets", "rows", "place")))


def test_group_matmul_and_its_gradient(P, a):
    y = torch.empty_like(a["y"])
    P.crc.crc_group_matmul(of(P, a["w"]), *p(a["x"]), k, M, None, *p(a["offsets"], a["rows"]), K, M * K,
                           *p(y))
    assert torch.equal(y, a["y"])
    dx = torch.empty((M * K, k), dtype=torch.bfloat16, device="cuda")
    dw = torch.empty((N, n, k), device="cuda")
    P.crc.crc_group_matmul_grad(of(P, a["w"]), *p(a["dy"], a["x"]), k, M, *p(a["offsets"], a["rows"]),
                                K, M * K, *p(dx, dw), P.crc.F32)
    want = P.group_matmul_grad(a["dy"], a["x"], a["w"], a["offsets"], rows=a["rows"], K=K)
    assert torch.equal(dx, want[0]) and torch.equal(dw, want[1])


def test_split_rows(P, a):
    x8, xs = P.split_rows(a["x"])
    got8, gots = torch.zeros_like(x8), torch.zeros_like(xs)
    P.crc.crc_split_rows(*p(a["x"]), k, M, k, *p(got8, gots))
    assert torch.equal(got8.view(torch.uint8), x8.view(torch.uint8)) and torch.equal(gots, xs)
    w8, ws = P.quantize_rows(a["w"])
    y = torch.empty_like(a["y"])
    P.crc.crc_group_matmul_split(of(P, w8, ws), *p(x8), 2 * k, M, *p(xs, a["offsets"], a["rows"]), K,
                                 M * K, *p(y))
    assert torch.equal(y, P.group_matmul(x8, w8, a["offsets"], rows=a["rows"], K=K, x_scale=xs,
                                         w_scale=ws))


def test_sum_choices_and_its_gradient(P, a):
    out = torch.empty((M, n), dtype=torch.bfloat16, device="cuda")
    P.crc.crc_sum_choices(*p(a["y"]), M * K, *p(a["place"], a["gates"]), M, K, n, *p(out))
    assert torch.equal(out, P.sum_choices(a["y"], a["place"], gates=a["gates"]))
    dy, dg = torch.empty_like(a["y"]), torch.empty_like(a["gates"])
    P.crc.crc_sum_choices_grad(*p(a["dout"], a["y"]), M * K, *p(a["place"], a["gates"]), M, K, n,
                               *p(dy, dg))
    want = P.sum_choices_grad(a["dout"], a["place"], gates=a["gates"], y=a["y"])
    assert torch.equal(dy, want[0]) and torch.equal(dg, want[1])


def test_4_bit_rows_and_products(P, a):
    q, s = P.quantize_rows4(a["w"], 32)
    gq, gs = torch.zeros_like(q), torch.zeros_like(s)
    P.crc.crc_quantize_rows4(*p(a["w"]), k, N, n, k, 32, *p(gq, gs))
    assert torch.equal(gq, q) and torch.equal(gs, s)
    w = P.crc.crc_matvec4_weights(N=N, n=n, k=k, slots=N, glu=0, group=32, reserved=0,
                                  codes_dev=q.data_ptr(), scale_dev=s.data_ptr(),
                                  codes_stride=q[0].nbytes, scale_stride=s[0].nbytes,
                                  expert_slot_dev=None)
    y = torch.empty((M, K, n), dtype=torch.bfloat16, device="cuda")
    P.crc.crc_matvec4(w, *p(a["x"]), k, 0, *p(a["topk"]), M, K, *p(y))
    assert torch.equal(y, P.matvec4(a["x"], q, s, topk=a["topk"]))


def test_refusals_name_the_entry(P, a):
    with pytest.raises(P.CrcError, match="crc_group_matmul_split"):
        P.crc.crc_group_matmul_split(of(P, a["w"]), *p(a["x"]), 2 * k, M, None, *p(a["offsets"]), None, 1,
                                     8, *p(a["y"]))
    with pytest.raises(P.CrcError, match="crc_matvec4"):
        P.crc.crc_matvec4(P.crc.crc_matvec4_weights(), None, k, 0, None, M, K, None)
