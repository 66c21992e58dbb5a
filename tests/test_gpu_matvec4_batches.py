"""4-bit products of the same choices in calls of few and many: the number of warps that share
a row's columns changes with the call, the definition's bounds hold for each."""
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


def weights(P, g, slots, n, k, G, glu):
    w = torch.randn((slots, *((2, n) if glu else (n,)), k), device="cuda", generator=g)
    q, a = P.quantize_rows4((w * k ** -0.5).bfloat16(), G)
    v = torch.stack((q & 15, q >> 4), -1).flatten(-2).to(torch.int8)
    v = torch.where(v > 7, v - 16, v).double().unflatten(-1, (-1, G)) * a.double().mT[..., None]
    return q, a, v.flatten(-2)


@pytest.mark.parametrize("k,G", [(512, 32), (2048, 64), (2880, 32), (4096, 128)])
@pytest.mark.parametrize("glu", [False, True])
def test_a_choice_alone_and_among_others(P, k, G, glu):
    """1 to 1000 rows of two experts, and rows without choices: 1, 2, 4 and 8 warps a tile, and a
    pass of 8 choices or of 16."""
    n, N = 200, 16
    g = torch.Generator(device="cuda").manual_seed(k)
    q, a, v = weights(P, g, N, n, k, G, glu)
    x = torch.randn((1000, k), device="cuda", generator=g).bfloat16()
    topk = torch.randint(0, N, (1000, 2), device="cuda", generator=g).to(torch.uint8)
    xd = x[:1].double()
    w = v[topk[0].long()]                                # [2](2)[n][k]
    p = torch.einsum("...nk,k->...n", w, xd[0])
    s = 2 * k * U32 * torch.einsum("...nk,k->...n", w.abs(), xd[0].abs())
    if glu:
        sg = p[:, 0] / (1 + torch.exp(-p[:, 0]))
        want = sg * p[:, 1]
        bound = ((U16 + 64 * U32) * want.abs() + 1.1 * s[:, 0] * (p[:, 1].abs() + s[:, 1])
                 + sg.abs() * s[:, 1])
    else:
        want, bound = p, U16 * p.abs() + s
    for M in (1, 2, 3, 7, 8, 20, 63, 64, 200, 1000):
        y = P.matvec4(x[:M], q, a, topk=topk[:M])
        assert ((y[0].double() - want).abs() <= bound).all()
        assert torch.equal(y, P.matvec4(x[:M], q, a, topk=topk[:M]))
        if not glu:                                      # one expert by its slot alone
            one = P.matvec4(x[:M], q[topk[0, 0].item():], a[topk[0, 0].item():])
            assert ((one[0, 0].double() - want[0]).abs() <= bound[0]).all()
    assert P.crc.crc_device_error() == 0
