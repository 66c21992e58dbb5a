"""Rows in two 8-bit pieces, their products with 8-bit matrices, and prompts of a layer with 8-bit
experts, which keep what the layer's own call keeps."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U16, U32 = 2.0 ** -8, 2.0 ** -24      # unit roundoff of bf16 (8 significant bits) and fp32
E4 = torch.float8_e4m3fn


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


def pieces(x):
    """(out8, scale) by the definition, on the host."""
    x = x.double().cpu()
    most = x.abs().amax(-1)
    e = torch.frexp(most)[1] - 8                        # most / 2^e in [128, 256)
    scale = torch.ldexp(torch.ones_like(most), e.clamp(min=-126))
    scale = torch.where(most > 0, scale, 2.0 ** -126)
    v = (x / scale[:, None]).float()                    # 8 bits: exact
    hi = v.to(E4)
    lo = (v - hi.float()).to(E4)
    return torch.stack((hi, lo), 1), scale.float()


def check_split(P, x, **kw):
    q, s = P.split_rows(x, **kw)
    wq, ws = pieces(x)
    assert torch.equal(s.cpu(), ws)
    # (as values: a zero's sign does not matter)
    assert torch.equal(q.float().cpu(), wq.float())
    err = (q.double().sum(1) * s.double()[:, None] - x.double()).abs()
    most = x.double().abs().amax(-1, keepdim=True)
    # a value in [2^e, 2^(e + 1)) is a multiple of 2^(e - 7), and lo of 2^-9, its smallest step: exact
    # from e = -2 on, which is 2^-9 of a largest value of 128 and less of a larger one
    assert (err[x.double().abs() >= 2.0 ** -9 * most] == 0).all()
    assert (err <= 2.0 ** -17 * most).all()
    return q, s


@pytest.mark.parametrize("M,d", [(1, 8), (3, 264), (33, 768), (70, 2880), (5, 4096), (9, 8192),
                                 (2, 32768), (4097, 16), (3, 24)])
@pytest.mark.parametrize("exponent", [0, -60, -110, 100])
def test_split_rows(P, M, d, exponent):
    g = torch.Generator(device="cuda").manual_seed(M + d)
    x = torch.randn((M, d), device="cuda", generator=g, dtype=torch.float64)
    # values of all sizes within a row
    x = x * torch.exp2(-16 * torch.rand((M, d), device="cuda", generator=g, dtype=torch.float64))
    check_split(P, (x * 2.0 ** exponent).bfloat16())


def test_split_rows_of_special_values(P):
    x = torch.zeros((5, 64), dtype=torch.bfloat16, device="cuda")
    x[1, 5], x[2, 7], x[3, 0], x[4, 1] = float("inf"), float("nan"), 3.38e38, -2.0 ** -133
    q, s = P.split_rows(x)
    assert s[1].isnan() and s[2].isnan()
    assert (q[0].float() == 0).all() and s[0] == 2.0 ** -126
    keep = [0, 3]
    wq, ws = pieces(x[keep])
    assert torch.equal(s[keep].cpu(), ws) and torch.equal(q[keep].float().cpu(), wq.float())
    assert s[4] == 2.0 ** -126 and q[4, 0, 1].float() == -2.0 ** -7


def test_split_rows_strided_given_none_and_on_a_stream(P):
    big = randn(torch.Generator(device="cuda").manual_seed(1), 50, 512)
    q, s = check_split(P, big[:, 64:320])
    out, sc = torch.empty_like(q), torch.empty_like(s)
    got = P.split_rows(big[:, 64:320], out8=out, scale=sc)
    assert got[0] is out and torch.equal(out.view(torch.uint8), q.view(torch.uint8))
    assert P.split_rows(big[:0])[0].shape == (0, 2, 512)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = P.split_rows(big[:, 64:320], stream=side)
    side.synchronize()
    assert torch.equal(got[0].view(torch.uint8), q.view(torch.uint8)) and torch.equal(got[1], s)


# --------------------------------------------------------------------------- #
def silu(x):
    return x / (1 + torch.exp(-x))


def plain(x, w, offsets, src, glu):
    """y and its bound for sorted rows; x, w in 64 bits.  (Two products a column.)"""
    k = w.shape[-1]
    y = torch.zeros((src.numel(), w.shape[-2]), dtype=torch.float64, device="cuda")
    b = torch.zeros_like(y)
    at = offsets.tolist()
    for e in range(len(at) - 1):
        s = slice(at[e], at[e + 1])
        xe = x[src[s].long()]
        # hi is within 17/16 of |x| and lo within 1/16: their products sum to 9/8 of |x w| at most
        parts = [(xe @ m.t(), 1.125 * xe.abs() @ m.abs().t()) for m in (w[e] if glu else (w[e],))]
        if not glu:
            y[s] = parts[0][0]
            b[s] = (U16 + 3 * U32) * y[s].abs() + 2 * 2 * k * U32 * parts[0][1]
            continue
        (g, dg), (u, du) = ((v, (2 * 2 * k + 3) * U32 * d) for v, d in parts)
        y[s] = silu(g) * u
        b[s] = (U16 + 64 * U32) * y[s].abs() + 1.1 * dg * (u.abs() + du) + silu(g).abs() * du
    return y, b


# n, k, rows of the experts: CTAs by themselves and pairs, columns that end inside a piece
SHAPES = [(16, 16, [1, 0, 2]), (48, 80, [17, 0, 15, 33]), (512, 320, [1, 2, 0, 300]),
          (272, 144, [255, 256, 257, 0]), (128, 2048, [9, 1, 0, 16]), (256, 1152, [40, 70, 130, 3])]


@pytest.mark.parametrize("n,k,counts", SHAPES)
@pytest.mark.parametrize("glu", [False, True])
@pytest.mark.parametrize("gather", [False, True])
def test_products_of_split_rows(P, n, k, counts, glu, gather):
    g = torch.Generator(device="cuda").manual_seed(n + k)
    N, E, K = len(counts), sum(counts), 3 if gather else 1
    off = torch.tensor([sum(counts[:i]) for i in range(N + 1)], dtype=torch.int32, device="cuda")
    w, ws = P.quantize_rows(randn(g, N, *((2, n) if glu else (n,)), k, scale=k ** -0.5))
    x = randn(g, max(1, E // 2) if gather else E, k)
    x8, xs = P.split_rows(x)
    rows, src = None, torch.arange(E, device="cuda")
    if gather:
        rows = torch.randint(0, x.shape[0] * K, (E,), device="cuda", generator=g).to(torch.int32)
        src = rows // K
    y = P.group_matmul(x8, w, off, rows=rows, K=K, x_scale=xs, w_scale=ws)
    xd = x8.double().sum(1) * xs.double()[:, None]
    want, b = plain(xd, w.double() * ws.double()[..., None], off, src, glu)
    assert ((y.double() - want).abs() <= b).all()
    assert P.crc.crc_device_error() == 0


def test_an_experts_split_rows_do_not_see_anothers(P):
    g = torch.Generator(device="cuda").manual_seed(3)
    w, ws = P.quantize_rows(randn(g, 3, 64, 80))
    off = torch.tensor([0, 21, 56, 65], dtype=torch.int32, device="cuda")
    x = randn(g, 65, 80)

    def y():
        x8, xs = P.split_rows(x)
        return P.group_matmul(x8, w, off, x_scale=xs, w_scale=ws)
    clean = y()
    x[30], x[40] = float("nan"), float("inf")
    got = y()
    keep = [i for i in range(65) if i not in (30, 40)]
    assert torch.equal(got[keep], clean[keep]) and got[[30, 40]].isnan().all()


# --------------------------------------------------------------------------- #
def layer_of(P, M, N, K, d, f):
    g = torch.Generator(device="cuda").manual_seed(2)
    (g13, s13), (g2, s2) = (P.quantize_rows(randn(g, N, 2, f, d, scale=d ** -0.5)),
                            P.quantize_rows(randn(g, N, d, f, scale=f ** -0.5)))
    x = randn(g, M, d)
    lay = P.MoeLayer(g13, g2, K=K, N=N, gate_up_scale=s13, down_scale=s2)
    scores = torch.softmax(torch.randn((M, N), device="cuda", generator=g) * 2, -1)
    topk = torch.empty((M, K), dtype=torch.uint8, device="cuda")
    gates = torch.empty((M, K), device="cuda")
    out = lay(x, scores=scores, topk=topk, gates=gates)
    w13, w2 = g13.double() * s13.double()[..., None], g2.double() * s2.double()[..., None]
    want = torch.zeros((M, d), dtype=torch.float64, device="cuda")
    for e in range(N):
        m, j = torch.nonzero(topk == e, as_tuple=True)
        if m.numel():
            h = silu(x[m].double() @ w13[e, 0].t()) * (x[m].double() @ w13[e, 1].t())
            want.index_add_(0, m, gates[m, j].double()[:, None] * (h @ w2[e].t()))
    return lay, x, topk, gates, out.double(), want


@pytest.mark.parametrize("M,N,K,d,f", [(1024, 32, 4, 512, 256), (300, 16, 2, 2880, 96),
                                       (1, 32, 4, 256, 512)])
def test_a_prompt_of_8_bit_experts_keeps_what_a_decode_step_keeps(P, M, N, K, d, f):
    """h, y and out are rounded to bf16, some 2^-9 / sqrt(3) of themselves each in the mean square,
    and x and h go in pieces that hold bf16; a decode step's h is off by 6e-4 and its out by one
    rounding.  (One e4m3 piece is off by 2^-4 / sqrt(12) of an element or so: 1.8e-2.)"""
    lay, x, topk, gates, decode, want = layer_of(P, M, N, K, d, f)
    out = lay.prompt(x, topk, gates).double()
    r = 2.0 ** -9 / 3 ** 0.5
    assert (out - want).norm() <= 3 * r * want.norm()
    assert (out - decode).norm() <= (4 * r + 6e-4) * want.norm()
    assert P.crc.crc_device_error() == 0


def test_a_prompt_in_one_piece(P):
    """pieces=1: the products of quantize_rows, bit for bit."""
    lay, x, topk, gates, _, want = layer_of(P, 200, 32, 4, 512, 256)
    g13, g2, _, _, s13, s2 = lay.tensors
    off, rows, place = P.group_choices(topk, 32)
    x8, xs = P.quantize_rows(x)
    h8, hs = P.quantize_rows(P.group_matmul(x8, g13, off, rows=rows, K=4, x_scale=xs, w_scale=s13))
    y = P.group_matmul(h8, g2, off, x_scale=hs, w_scale=s2)
    out = lay.prompt(x, topk, gates, pieces=1)
    assert torch.equal(out, P.sum_choices(y, place, gates=gates))
    assert (out.double() - want).norm() > 10 * (lay.prompt(x, topk, gates).double() - want).norm()


def test_a_prompt_of_8_bit_experts_captured_padded_and_on_a_stream(P):
    lay, x, topk, gates, _, _ = layer_of(P, 300, 16, 2, 512, 96)
    out = torch.empty_like(x)
    lay.prompt(x, topk, gates, out=out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lay.prompt(x, topk, gates, out=out)
    side = torch.cuda.Stream()
    for turn in range(3):
        x.copy_(torch.randn_like(x))
        topk.copy_(topk.roll(turn + 1, 0))
        topk[280:] = 255                                # padded tokens
        graph.replay()
        want = lay.prompt(x, topk, gates)
        assert torch.equal(out, want) and (out[280:] == 0).all()
        side.wait_stream(torch.cuda.current_stream())
        got = lay.prompt(x, topk, gates, stream=side)
        side.synchronize()
        assert torch.equal(got, want)
    assert lay.prompt(x[:0], topk[:0], gates[:0]).shape == (0, 512)
    assert P.crc.crc_device_error() == 0
