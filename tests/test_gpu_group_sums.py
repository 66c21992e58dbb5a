"""How far the matrices' gradients may be off when an expert has many rows: the error of a
tensor core's accumulator grows with the rows that it sums, that of a call does not."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24


@pytest.fixture(scope="module")
def P():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_04895_gb300 import build
    build.build()
    import paper_2609_04895_gb300 as P
    P.crc.load()
    return P


def offsets_of(counts):
    o = torch.zeros(len(counts) + 1, dtype=torch.int64)
    o[1:] = torch.tensor(counts).cumsum(0)
    return o.to(torch.int32).cuda()


def definition(dy, x, offsets, src):
    at = offsets.tolist()
    out = torch.zeros((len(at) - 1, dy.shape[1], x.shape[1]), dtype=torch.float64, device="cuda")
    for e in range(len(at) - 1):
        for r in range(at[e], at[e + 1], 8192):
            s = slice(r, min(at[e + 1], r + 8192))
            out[e] += dy[s].double().t() @ x[src[s].long()].double()
    return out


# rows of the experts: of a part, of two, of three and more, whose last may be short
COUNTS = [[1024], [1025, 3, 2049], [4103, 0, 5], [2048, 4096, 4097], [32768, 700], [8191, 0, 0, 6145]]


@pytest.mark.parametrize("counts", COUNTS)
@pytest.mark.parametrize("gather", [False, True])
def test_fp32_gradients_do_not_lose_bits_with_the_rows(P, counts, gather):
    """An accumulator cuts its sum at each step of 16 rows, by 0.72 2^-24 of it on average (half
    a unit in the last place, over the mantissas).  Operands of either sign: after t of T steps the
    sum is sqrt(t / T) of the last one in the mean square, and if all cuts pointed one way they would
    make 0.72 2^-24 2/3 T, for the 64 steps of 1024 rows 31 2^-24.  The sums of the parts are added
    in fp32."""
    n, k = 264, 136
    g = torch.Generator(device="cuda").manual_seed(sum(counts))
    E = sum(counts)
    dy = torch.randn((E, n), device="cuda", generator=g).bfloat16()
    x = torch.randn((E, k), device="cuda", generator=g).bfloat16()
    src = torch.randperm(E, device="cuda", generator=g) if gather else torch.arange(E, device="cuda")
    off = offsets_of(counts)
    w = torch.zeros((len(counts), n, k), dtype=torch.bfloat16, device="cuda")
    _, dw = P.group_matmul_grad(dy, x, w, off, rows=src.to(torch.int32) if gather else None,
                                want_dx=False)
    want = definition(dy, x, off, src)
    for e, c in enumerate(counts):
        if c == 0:
            assert (dw[e] == 0).all()
            continue
        err = ((dw[e].double() - want[e]).norm() / want[e].norm()).item()
        parts = (c + 1023) // 1024
        assert err <= (31 + parts ** 0.5) * U32, (c, err)
    assert P.crc.crc_device_error() == 0
    # the same bits again, and for an expert by itself
    _, again = P.group_matmul_grad(dy, x, w, off, rows=src.to(torch.int32) if gather else None,
                                   want_dx=False)
    assert torch.equal(dw, again)
    last = E - counts[-1]
    if counts[-1]:
        _, alone = P.group_matmul_grad(dy[last:], x[src[last:]].contiguous(), w[-1:],
                                       offsets_of(counts[-1:]), want_dx=False)
        assert torch.equal(alone[0], dw[-1])


def test_bf16_gradients_of_many_rows_are_not_shrunk(P):
    """Sums of one sign, which cuts shrink the most: 16384 rows an accumulator are 1024 steps, each
    of which may cut four times where the sum is large (the products come in fours), 0.72 2^-24 of
    half of the last sum on average: 9e-5.  Roundings to bf16 (1.7e-3 in the mean square) leave
    2.6e-5 in the mean of 4096; four times that is room enough."""
    R, n = 65536 + 40, 64
    g = torch.Generator(device="cuda").manual_seed(1)
    spread = torch.exp(torch.rand(n, device="cuda", generator=g) * 3)   # all mantissas
    dy = (torch.randn((R, n), device="cuda", generator=g).abs() * spread).bfloat16()
    x = (torch.randn((R, n), device="cuda", generator=g).abs() * spread.flip(0)).bfloat16()
    off = offsets_of([R])
    dw = torch.empty((1, n, n), dtype=torch.bfloat16, device="cuda")
    P.group_matmul_grad(dy, x, dw, off, want_dx=False, dw=dw)
    want = definition(dy, x, off, torch.arange(R, device="cuda"))
    shrunk = ((dw.double() - want) / want).mean().item()
    assert abs(shrunk) <= 9e-5 + 4 * 2.6e-5, shrunk
