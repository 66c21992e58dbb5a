"""Grouped products on either side of the rules that choose CTAs by themselves or pairs, and
with few gathered rows, against their definitions in 64 bits."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U16, U32 = 2.0 ** -8, 2.0 ** -24      # unit roundoff of bf16 (8 significant bits) and fp32


@pytest.fixture(scope="module")
def P():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_04895_gb300 import build
    build.build()
    import paper_2609_04895_gb300 as P
    P.crc.load()
    return P


def randn(g, *shape, scale=1.0):
    return (torch.randn(shape, device="cuda", generator=g) * scale).bfloat16()


def offsets_of(counts):
    o = torch.zeros(len(counts) + 1, dtype=torch.int64)
    o[1:] = torch.tensor(counts).cumsum(0)
    return o.to(torch.int32).cuda()


def silu(x):
    return x / (1 + torch.exp(-x))


def plain(x, w, offsets, src, glu):
    """y and its bound for sorted rows, x and w in 64 bits: sums of k products in fp32 by units that
    may cut instead of round (a step and not half of one each), two scales, the rounding to bf16."""
    k = w.shape[-1]
    y = torch.zeros((src.numel(), w.shape[-2]), dtype=torch.float64, device="cuda")
    b = torch.zeros_like(y)
    at = offsets.tolist()
    for e in range(len(at) - 1):
        s = slice(at[e], at[e + 1])
        xe = x[src[s].long()]
        parts = [(xe @ m.t(), 2 * k * U32 * (xe.abs() @ m.abs().t())) for m in (w[e] if glu else (w[e],))]
        if not glu:
            y[s], d = parts[0]
            b[s] = (U16 + 3 * U32) * y[s].abs() + d
            continue
        (gt, dg), (u, du) = parts
        y[s] = silu(gt) * u
        # silu's slope is below 1.1; the fast exponential and division are off by some 25 steps
        b[s] = (U16 + 67 * U32) * y[s].abs() + 1.1 * dg * (u.abs() + du) + silu(gt).abs() * du
    return y, b


def around(mean, N):
    """Rows of N experts with that mean, uneven, one of them without."""
    c = [mean + (-1) ** i * (i % mean) for i in range(N)]
    c[1], c[2] = 0, c[2] + c[1]
    c[-1] += mean * N - sum(c)
    return c


# rows an expert, on average: 40 gathered from more than 8 pieces of 128 bytes, else 48
@pytest.mark.parametrize("mean", [1, 8, 17, 39, 40, 41, 47, 48, 49])
@pytest.mark.parametrize("k", [64, 640, 2048])
@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("glu", [False, True])
@pytest.mark.parametrize("w8", [False, True])
def test_products_on_both_sides_of_the_rules(P, mean, k, gather, glu, w8):
    n, N = 272, 6
    k = 2 * k if w8 else k                              # as many pieces
    counts = [1] * N if mean == 1 else around(mean, N)
    assert sum(counts) == mean * N and min(counts) >= 0
    g = torch.Generator(device="cuda").manual_seed(mean + k)
    E, K = sum(counts), 3 if gather else 1
    w = randn(g, N, *((2, n) if glu else (n,)), k, scale=k ** -0.5)
    x = randn(g, max(1, E // 2) if gather else E, k)
    rows, src = None, torch.arange(E, device="cuda")
    if gather:
        rows = torch.randint(0, x.shape[0] * K, (E,), device="cuda", generator=g).to(torch.int32)
        src = rows // K
    xs = ws = None
    xd, wd = x.double(), w.double()
    if w8:
        (x, xs), (w, ws) = P.quantize_rows(x), P.quantize_rows(w)
        xd, wd = x.double() * xs.double()[:, None], w.double() * ws.double()[..., None]
    off = offsets_of(counts)
    y = P.group_matmul(x, w, off, rows=rows, K=K, x_scale=xs, w_scale=ws)
    want, b = plain(xd, wd, off, src, glu)
    assert ((y.double() - want).abs() <= b).all()
    assert P.crc.crc_device_error() == 0


@pytest.mark.parametrize("N,k,n,counts", [
    (128, 2048, 256, [1]), (128, 2048, 256, [9, 1, 2]), (32, 256, 512, [1]), (4, 1024, 2048, [3]),
    (2, 640, 512, [1, 130]), (8, 4096, 128, [16, 1]),
])
def test_few_gathered_rows(P, N, k, n, counts):
    """Some of the warps that gather have no rows in a tile: products and gradients."""
    g = torch.Generator(device="cuda").manual_seed(N + k)
    counts = (counts * N)[:N]
    E = sum(counts)
    x, w, dy = randn(g, E, k), randn(g, N, n, k, scale=k ** -0.5), randn(g, E, n)
    rows = torch.randperm(E, device="cuda", generator=g).to(torch.int32)
    off = offsets_of(counts)
    y = P.group_matmul(x, w, off, rows=rows, K=1)
    want, b = plain(x.double(), w.double(), off, rows, False)
    assert ((y.double() - want).abs() <= b).all()
    dx, dw = P.group_matmul_grad(dy, x, w, off, rows=rows, K=1)
    at = off.tolist()
    for e in range(N):
        s = slice(at[e], at[e + 1])
        d, xe, we = dy[s].double(), x[rows[s].long()].double(), w[e].double()
        want = d @ we
        assert ((dx[s].double() - want).abs()
                <= U16 * want.abs() + 2 * n * U32 * (d.abs() @ we.abs())).all()
        want = d.t() @ xe
        assert ((dw[e].double() - want).abs()
                <= 2 * max(1, counts[e]) * U32 * (d.abs().t() @ xe.abs())).all()
    assert P.crc.crc_device_error() == 0
