"""The MoE layer's precision between its products: the product of silu and up enters the
second product in two pieces, bf16 (16 significant bits) or e4m3 (2^-9 of an element,
2^-21 of its row's largest).  One piece would fail both tests here."""
import math

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


class Layer:
    def __init__(self, P, N, K, d, f, M, kind):
        g = torch.Generator(device="cuda").manual_seed(N + M + f)
        new = lambda *s, k=1.0: (torch.randn(s, device="cuda", generator=g) * k).bfloat16()  # noqa: E731
        self.x, router = new(M, d), new(N, d, k=d ** -0.5)
        w13, w2 = new(N, 2, f, d, k=2 * d ** -0.5), new(N, d, f, k=f ** -0.5)
        s13 = s2 = self.x8 = self.xs = None
        self.w8 = kind != "bf16"
        if self.w8:
            (w13, s13), (w2, s2) = P.quantize_rows(w13), P.quantize_rows(w2)
        if kind == "w8x8":
            self.x8, self.xs = P.quantize_rows(self.x)
        self.layer = P.MoeLayer(w13, w2, K=K, router=router, gate_up_scale=s13, down_scale=s2)
        self.topk = torch.empty((M, K), dtype=torch.uint8, device="cuda")
        self.out = self.layer(self.x, x8=self.x8, x_scale=self.xs, topk=self.topk)
        self.w13, self.w2, self.router = w13.double(), w2.double(), router.double()
        if self.w8:
            self.w13 *= s13.double()[..., None]
            self.w2 *= s2.double()[..., None]

    def exact(self, change=None):
        """out in 64 bits and a bound of its errors before the last rounding; change(h):
        what the second product takes in place of h."""
        x = self.x.double() if self.x8 is None else self.x8.double() * self.xs.double()[:, None]
        d, f = self.w13.shape[-1], self.w2.shape[-1]
        ids = self.topk.long()
        g = torch.softmax(self.x.double() @ self.router.t(), -1).gather(1, ids)
        g = g / g.sum(1, keepdim=True)
        out, err = torch.zeros_like(x), torch.zeros_like(x)
        # fp32 sums: the random walk's estimate with room, and scales
        cd, cf = (8 * math.sqrt(d) + 2) * U32, (8 * math.sqrt(f) + 2) * U32
        for e in torch.unique(ids).tolist():
            m, k = torch.nonzero(ids == e, as_tuple=True)
            w13, w2 = self.w13[e], self.w2[e]
            xa = x[m].abs()
            xe = 2.0 ** -21 * xa.amax(1, keepdim=True) * (self.w8 and self.x8 is None)
            a, b = x[m] @ w13[0].t(), x[m] @ w13[1].t()
            ea = cd * (xa @ w13[0].abs().t()) + xe * w13[0].abs().sum(1)
            eb = cd * (xa @ w13[1].abs().t()) + xe * w13[1].abs().sum(1)
            silu = a * torch.sigmoid(a)
            h = silu * b
            # __expf is 2 + 1.173 |a| units of the last place off, __fdividef two
            fast = (2 + 1.2 * a.abs() + 2 + 8) * 2 * U32 * h.abs()
            eh = 1.1 * ea * b.abs() + silu.abs() * eb + ea * eb + fast
            top = (h.abs() + eh).amax(1, keepdim=True)
            eh = eh + (2.0 ** -9 * h.abs() + 2.0 ** -21 * top if self.w8 else U16 ** 2 * h.abs())
            ge = g[m, k][:, None]
            out.index_add_(0, m, ge * ((change(h) if change else h) @ w2.t()))
            # gates 1e-5 off
            err.index_add_(0, m, ge * (eh @ w2.abs().t() + (cf + 1e-5) * (h.abs() @ w2.abs().t())))
        return out, err


SIZES = [(16, 2, 1024, 768, 1), (32, 4, 1024, 768, 12), (32, 4, 512, 1024, 40), (16, 2, 512, 2880, 200),
         (64, 4, 1024, 512, 300)]


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("kind", ["bf16", "w8", "w8x8"])
def test_elements_within_the_pieces_bound(P, size, kind):
    c = Layer(P, *size, kind)
    want, err = c.exact()
    off = (c.out.double() - want).abs()
    assert (off <= err + U16 * (want.abs() + err)).all()


def excess(out, want):
    """What out's mean squared error has beyond that of rounding the exact values to
    bf16, as a share of their mean square, and the estimate's own spread (4 sigma)."""
    own = (want.bfloat16().double() - want).square().mean()
    scale = want.square().mean()
    spread = 4 * math.sqrt(2 / want.numel()) * own / scale
    return float(((out.double() - want).square().mean() - own) / scale), float(spread)


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("kind", ["bf16", "w8", "w8x8"])
def test_mean_error_is_that_of_two_pieces(P, size, kind):
    """Independent errors of h's elements, each delta of the element, put delta of it
    into the output's root mean square.  Two bf16 pieces: below 2^-12 with all fp32
    sums.  e4m3: at most 2^-9 of an element, as good as uniform, 2^-9 / sqrt 3."""
    c = Layer(P, *size, kind)
    want, _ = c.exact()
    limit = (2.0 ** -9 / math.sqrt(3) if c.w8 else 2.0 ** -12) ** 2
    got, spread = excess(c.out, want)
    assert got <= limit + spread
    # the same in 64 bits with h in one bf16 piece is seen
    one, _ = c.exact(lambda h: h.to(torch.bfloat16).double())
    got, spread = excess(one.bfloat16(), want)
    assert got > limit + spread
