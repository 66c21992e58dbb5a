"""Products grouped by expert and their gradients against their definitions in 64 bits and
against differences; the layer that they make with the choices' order and sum."""
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


def randn(g, *shape, scale=1.0, dtype=torch.bfloat16):
    return (torch.randn(shape, device="cuda", generator=g) * scale).to(dtype)


def offsets_of(counts, first=0):
    o = torch.zeros(len(counts) + 1, dtype=torch.int64)
    o[1:] = torch.tensor(counts).cumsum(0)
    return (o + first).to(torch.int32).cuda()


# n, k, rows of the experts
SHAPES = [
    (256, 128, [16]), (8, 8, [1, 0, 2]), (16, 16, [0, 0, 3, 1]), (48, 72, [17, 0, 15, 33]),
    (512, 320, [1, 2, 0, 300]), (264, 200, [255, 256, 257, 0]), (1024, 512, [31, 129, 0, 64, 513]),
    (80, 2880, [5, 40]), (528, 64, [0, 1000, 7]), (128, 136, [100] * 12),
    (64, 72, [1025, 2500, 0, 30, 1024]),
]


def bounds(y, prods, terms):
    """Sums of `terms` products in fp32 (in any order, by units that may cut instead of
    round: a step and not half of one each) and the rounding to bf16."""
    return U16 * y.abs() + 2 * terms * U32 * prods


def silu(x):
    return x / (1 + torch.exp(-x))


def plain(x, w, offsets, src, glu):
    """y and its bound for sorted rows; x, w in 64 bits."""
    E, n, k = src.numel(), w.shape[-2], w.shape[-1]
    y = torch.zeros((E, n), dtype=torch.float64, device="cuda")
    b = torch.zeros_like(y)
    at = offsets.tolist()
    for e in range(len(at) - 1):
        s = slice(at[e], at[e + 1])
        xe = x[src[s].long()]
        if not glu:
            y[s] = xe @ w[e].t()
            b[s] = bounds(y[s], xe.abs() @ w[e].abs().t(), k)
            continue
        g, u = xe @ w[e][0].t(), xe @ w[e][1].t()
        dg, du = (2 * k * U32 * (xe.abs() @ w[e][i].abs().t()) for i in (0, 1))
        y[s] = silu(g) * u
        # silu's slope is below 1.1; the fast exponential and division are off by some 25 steps
        b[s] = (U16 + 64 * U32) * y[s].abs() + 1.1 * dg * (u.abs() + du) + silu(g).abs() * du
    return y, b


def inputs(counts, n, k, glu, gather, w8, P, seed, first=0, tail=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    N, E = len(counts), sum(counts) + first + tail
    w = randn(g, N, *((2, n) if glu else (n,)), k, scale=k ** -0.5)
    K = 3 if gather else 1
    x = randn(g, max(1, (E + 2) // 2) if gather else E, k)
    rows = None
    src = torch.arange(E, device="cuda")
    if gather:                                          # any token's choices, in any order
        rows = torch.randint(0, x.shape[0] * K, (E,), device="cuda", generator=g).to(torch.int32)
        src = rows // K
    xs = ws = None
    if w8:
        (x, xs), (w, ws) = P.quantize_rows(x), P.quantize_rows(w)
    return dict(x=x, w=w, offsets=offsets_of(counts, first), rows=rows, K=K, x_scale=xs,
                w_scale=ws), src


def values(t, scale):
    t = t.double()
    return t if scale is None else t * scale.double()[..., None]


@pytest.mark.parametrize("n,k,counts", SHAPES)
@pytest.mark.parametrize("glu", [False, True])
@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("w8", [False, True])
def test_products(P, n, k, counts, glu, gather, w8):
    if w8:
        k = (k + 15) // 16 * 16
    if glu:
        n = (n + 15) // 16 * 16
    a, src = inputs(counts, n, k, glu, gather, w8, P, n + k)
    y = P.group_matmul(**a)
    want, b = plain(values(a["x"], a["x_scale"]), values(a["w"], a["w_scale"]), a["offsets"], src,
                    glu)
    # (e4m3: two scales more)
    assert ((y.double() - want).abs() <= b + 3 * U32 * want.abs()).all()
    assert P.crc.crc_device_error() == 0


@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("glu", [False, True])
def test_rows_outside_the_offsets_stay(P, gather, glu):
    """Rows before the first offset and behind the last are as they were."""
    a, src = inputs([20, 0, 37], 160, 96, glu, gather, False, P, 5, first=9, tail=30)
    y = torch.full((src.numel(), 160), 7.0, dtype=torch.bfloat16, device="cuda")
    if gather:
        a["rows"][66:] = -1                             # as group_choices leaves them
    P.group_matmul(**a, y=y)
    assert (y[:9] == 7).all() and (y[66:] == 7).all()
    want, b = plain(a["x"].double(), a["w"].double(), a["offsets"], src, glu)
    assert ((y.double() - want).abs() <= b)[9:66].all()
    assert P.crc.crc_device_error() == 0


@pytest.mark.parametrize("glu", [False, True])
def test_strided_rows_and_experts(P, glu):
    n, k = 96, 72
    g = torch.Generator(device="cuda").manual_seed(8)
    big = randn(g, 70, k + 24)
    parts = 2 if glu else 1
    slots = randn(g, 3, 3 * n * k, scale=k ** -0.5)
    w = (slots.as_strided((3, 2, n, k), (3 * n * k, n * k, k, 1)) if glu
         else slots.as_strided((3, n, k), (3 * n * k, k, 1)))
    off = offsets_of([20, 19, 31])
    y = P.group_matmul(big[:, :k], w, off)
    assert torch.equal(y, P.group_matmul(big[:, :k].contiguous(), w.contiguous(), off))
    assert parts and y.shape == (70, n)


def test_one_row_of_x(P):
    """A single token's choices: x has one row, whatever its stride says."""
    g = torch.Generator(device="cuda").manual_seed(2)
    x, w = randn(g, 1, 64), randn(g, 8, 24, 64)
    off = offsets_of([1, 0, 0, 1, 0, 2, 0, 0])
    y = P.group_matmul(x, w, off, rows=torch.arange(4, dtype=torch.int32, device="cuda"), K=4)
    want, b = plain(x.double(), w.double(), off, torch.zeros(4, device="cuda"), False)
    assert ((y.double() - want).abs() <= b).all()


def test_an_experts_rows_do_not_see_anothers(P):
    """NaN and infinities in one expert's rows and matrix stay with it, tile by tile."""
    counts = [21, 35, 300, 9]
    a, src = inputs(counts, 136, 88, False, False, False, P, 3)
    clean = P.group_matmul(**a)
    a["x"][21:56] = float("nan")
    a["w"][1] = float("inf")
    y = P.group_matmul(**a)
    assert torch.equal(y[:21], clean[:21]) and torch.equal(y[56:], clean[56:])
    assert y[21:56].isnan().all()


def test_results_do_not_depend_on_the_batch(P):
    """An expert's rows give the same bits alone and in a batch."""
    a, _ = inputs([3, 400, 37], 512, 1024, True, False, False, P, 4)
    y = P.group_matmul(**a)
    alone = P.group_matmul(a["x"][403:].contiguous(), a["w"][2:], offsets_of([37]))
    assert torch.equal(y[403:], alone)


# --------------------------------------------------------------------------- #
def plain_grad(dy, x, w, offsets, src):
    at = offsets.tolist()
    dx = torch.zeros((dy.shape[0], w.shape[2]), dtype=torch.float64, device="cuda")
    dw = torch.zeros(w.shape, dtype=torch.float64, device="cuda")
    bx, bw = torch.zeros_like(dx), torch.zeros_like(dw)
    for e in range(len(at) - 1):
        s = slice(at[e], at[e + 1])
        d, xe = dy[s], x[src[s].long()]
        dx[s], bx[s] = d @ w[e], d.abs() @ w[e].abs()
        dw[e], bw[e] = d.t() @ xe, 2 * max(1, xe.shape[0]) * U32 * (d.abs().t() @ xe.abs())
    return dx, bounds(dx, bx, w.shape[1]), dw, bw


@pytest.mark.parametrize("n,k,counts", SHAPES)
@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("dw_type", ["f32", "bf16"])
def test_gradients(P, n, k, counts, gather, dw_type):
    a, src = inputs(counts, n, k, False, gather, False, P, n + k + 1)
    dy = randn(torch.Generator(device="cuda").manual_seed(n), src.numel(), n)
    dw = torch.full(a["w"].shape, 7.0, device="cuda",
                    dtype={"f32": torch.float32, "bf16": torch.bfloat16}[dw_type])
    dx, got = P.group_matmul_grad(dy, a["x"], a["w"], a["offsets"], rows=a["rows"], K=a["K"],
                                  dw=dw)
    assert got is dw
    wx, bx, ww, bw = plain_grad(dy.double(), a["x"].double(), a["w"].double(), a["offsets"], src)
    assert ((dx.double() - wx).abs() <= bx).all()
    assert ((dw.double() - ww).abs() <= bw + (U16 if dw_type == "bf16" else 0) * ww.abs()).all()
    for e, c in enumerate(counts):
        assert c or (dw[e] == 0).all()
    assert P.crc.crc_device_error() == 0


def test_gradients_by_themselves_and_with_made_outputs(P):
    a, src = inputs([20, 0, 50], 64, 48, False, True, False, P, 1)
    dy = randn(torch.Generator(device="cuda").manual_seed(1), 70, 64)
    by = dict(rows=a["rows"], K=a["K"])
    dx, dw = P.group_matmul_grad(dy, a["x"], a["w"], a["offsets"], **by)
    assert dw.dtype == torch.float32
    x1, none = P.group_matmul_grad(dy, a["x"], a["w"], a["offsets"], want_dw=False, **by)
    assert none is None and torch.equal(x1, dx)
    none, w1 = P.group_matmul_grad(dy, a["x"], a["w"], a["offsets"], want_dx=False, **by)
    assert none is None and torch.equal(w1, dw)


@pytest.mark.parametrize("gather", [False, True])
def test_a_matrix_gradient_does_not_see_the_next_experts_rows(P, gather):
    """The last rows of an expert share a block with the next one's, which may hold anything."""
    counts = [5, 16, 17, 64, 65, 1]
    a, src = inputs(counts, 72, 136, False, False, False, P, 6)
    dy = randn(torch.Generator(device="cuda").manual_seed(6), src.numel(), 72)
    rows = src.to(torch.int32) if gather else None
    _, clean = P.group_matmul_grad(dy, a["x"], a["w"], a["offsets"], rows=rows, want_dx=False)
    at = a["offsets"].tolist()
    for e in (1, 3, 5):
        for bad in (float("nan"), float("inf")):
            x, d = a["x"].clone(), dy.clone()
            x[at[e]:at[e + 1]] = bad
            d[at[e]:at[e + 1]] = -bad
            _, dw = P.group_matmul_grad(d, x, a["w"], a["offsets"], rows=rows, want_dx=False)
            for o in range(len(counts)):
                assert (dw[o].isnan() | dw[o].isinf()).all() if o == e else torch.equal(dw[o], clean[o])


def test_rows_outside_the_offsets_have_no_part_in_the_gradients(P):
    a, src = inputs([20, 0, 37], 64, 96, False, False, False, P, 5, first=9, tail=30)
    dy = randn(torch.Generator(device="cuda").manual_seed(2), src.numel(), 64)
    dx = torch.full((src.numel(), 96), 7.0, dtype=torch.bfloat16, device="cuda")
    x = a["x"].clone()
    x[:9], x[66:] = float("nan"), float("inf")
    _, dw = P.group_matmul_grad(dy, x, a["w"], a["offsets"], dx=dx)
    wx, bx, ww, bw = plain_grad(dy.double(), a["x"].double(), a["w"].double(), a["offsets"], src)
    assert (dx[:9] == 7).all() and (dx[66:] == 7).all()
    assert ((dx.double() - wx).abs() <= bx)[9:66].all() and ((dw.double() - ww).abs() <= bw).all()


def test_gradients_against_differences(P):
    """<dy, y> along random directions of x and of the matrices, in 64 bits."""
    a, src = inputs([20, 0, 50, 7], 64, 48, False, True, False, P, 11)
    g = torch.Generator(device="cuda").manual_seed(11)
    dy = randn(g, 77, 64)
    dx, dw = P.group_matmul_grad(dy, a["x"], a["w"], a["offsets"], rows=a["rows"], K=a["K"])

    def f(x, w):
        return (dy.double() * plain(x, w, a["offsets"], src, False)[0]).sum()
    x0, w0, h = a["x"].double(), a["w"].double(), 1e-3
    ux = torch.randn(x0.shape, device="cuda", generator=g, dtype=torch.float64)
    uw = torch.randn(w0.shape, device="cuda", generator=g, dtype=torch.float64)
    by_x = (f(x0 + h * ux, w0) - f(x0 - h * ux, w0)) / (2 * h)
    by_w = (f(x0, w0 + h * uw) - f(x0, w0 - h * uw)) / (2 * h)
    _, bx, _, bw = plain_grad(dy.double(), x0, w0, a["offsets"], src)
    # a choice's row of dx counts for its token; each element within its bound
    u = ux[src.long()]
    assert abs(by_x - (dx.double() * u).sum()) <= 1e-9 + (bx * u.abs()).sum()
    assert abs(by_w - (dw.double() * uw).sum()) <= 1e-9 + (bw * uw.abs()).sum()


# --------------------------------------------------------------------------- #
def test_bad_offsets_and_rows_are_reported(P):
    """What is not offsets has no rows; a row outside x reads row 0.  Both latch an error."""
    a, src = inputs([20, 10, 37], 64, 96, False, True, False, P, 5)
    y = torch.full((67, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    for bad in ([0, 30, 20, 67], [0, 20, 30, 68], [-1, 20, 30, 67]):
        off = torch.tensor(bad, dtype=torch.int32, device="cuda")
        P.group_matmul(a["x"], a["w"], off, rows=a["rows"], K=3, y=y.fill_(7.0))
        assert P.crc.crc_device_error() == P.crc.CRC_EDEVICE
        P.group_matmul_grad(y, a["x"], a["w"], off, rows=a["rows"], K=3)
        assert P.crc.crc_device_error() == P.crc.CRC_EDEVICE
    for bad in (-1, a["x"].shape[0] * 3, 2 ** 31 - 1):
        rows = a["rows"].clone()
        rows[25] = bad
        P.group_matmul(a["x"], a["w"], a["offsets"], rows=rows, K=3, y=y)
        assert P.crc.crc_device_error() == P.crc.CRC_EDEVICE
        rows[25] = 0
        assert torch.equal(y, P.group_matmul(a["x"], a["w"], a["offsets"], rows=rows, K=3))
    assert P.crc.crc_device_error() == 0


def test_no_rows(P):
    w = randn(torch.Generator(device="cuda").manual_seed(1), 3, 64, 48)
    off = torch.zeros(4, dtype=torch.int32, device="cuda")
    x = torch.empty((0, 48), dtype=torch.bfloat16, device="cuda")
    assert P.group_matmul(x, w, off).shape == (0, 64)
    dx, dw = P.group_matmul_grad(torch.empty((0, 64), dtype=torch.bfloat16, device="cuda"), x, w,
                                 off, dw=torch.ones((3, 64, 48), device="cuda"))
    assert dx.shape == (0, 48) and (dw == 0).all()
    # rows, but none of an expert
    x = randn(torch.Generator(device="cuda").manual_seed(1), 5, 48)
    y = torch.full((5, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    assert (P.group_matmul(x, w, off, y=y) == 7).all()
    _, dw = P.group_matmul_grad(y, x, w, off)
    assert (dw == 0).all()


@pytest.mark.parametrize("N", [1, 256])
def test_numbers_of_experts(P, N):
    g = torch.Generator(device="cuda").manual_seed(N)
    counts = torch.randint(0, 4, (N,), generator=torch.Generator().manual_seed(N)).tolist()
    counts[-1] = 3
    a, src = inputs(counts, 40, 64, False, False, False, P, N)
    y = P.group_matmul(**a)
    want, b = plain(a["x"].double(), a["w"].double(), a["offsets"], src, False)
    assert ((y.double() - want).abs() <= b).all()
    dy = randn(g, src.numel(), 40)
    dx, dw = P.group_matmul_grad(dy, a["x"], a["w"], a["offsets"])
    wx, bx, ww, bw = plain_grad(dy.double(), a["x"].double(), a["w"].double(), a["offsets"], src)
    assert ((dx.double() - wx).abs() <= bx).all() and ((dw.double() - ww).abs() <= bw).all()


# --------------------------------------------------------------------------- #
# the operators together
# --------------------------------------------------------------------------- #
def layer_inputs(M, N, K, d, f, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    z = torch.randn((M, N), device="cuda", generator=g)
    top = z.topk(K, dim=-1)
    return dict(x=randn(g, M, d), gate_up=randn(g, N, 2, f, d, scale=d ** -0.5),
                down=randn(g, N, d, f, scale=f ** -0.5), topk=top.indices.to(torch.uint8),
                gates=torch.softmax(top.values, -1))


def layer(P, a, N, K, **st):
    off, rows, place = P.group_choices(a["topk"], N, **st)
    h = P.group_matmul(a["x"], a["gate_up"], off, rows=rows, K=K, **st)
    y = P.group_matmul(h, a["down"], off, **st)
    return P.sum_choices(y, place, gates=a["gates"], **st)


@pytest.mark.parametrize("M,N,K,d,f", [(1, 16, 2, 256, 512), (700, 32, 4, 2880, 96),
                                       (3000, 128, 8, 512, 128)])
def test_layer(P, M, N, K, d, f):
    a = layer_inputs(M, N, K, d, f, M)
    pad = M // 5                                        # padded tokens at the end
    a["topk"][M - pad:] = 255
    out = layer(P, a, N, K)
    want = torch.zeros((M, d), dtype=torch.float64, device="cuda")
    slack = torch.zeros_like(want)
    x = a["x"].double()
    for e in range(N):
        m, j = torch.nonzero(a["topk"] == e, as_tuple=True)
        if not m.numel():
            continue
        w, v = a["gate_up"][e].double(), a["down"][e].double()
        h = silu(x[m] @ w[0].t()) * (x[m] @ w[1].t())
        y = h @ v.t()
        g = a["gates"][m, j].double()[:, None]
        want.index_add_(0, m, g * y)
        # h is rounded to bf16 and so is y (twice U16 leaves room for the fp32 sums here)
        slack.index_add_(0, m, 2 * U16 * g * (h.abs() @ v.abs().t() + y.abs()))
    assert ((out.double() - want).abs() <= slack + U16 * want.abs()).all()
    assert (out[M - pad:] == 0).all() and P.crc.crc_device_error() == 0


def test_layer_agrees_with_the_decode_layer(P):
    """The same experts, choices and gates as MoeLayer, which keeps h in 16 bits."""
    M, N, K, d, f = 200, 32, 4, 512, 256
    a = layer_inputs(M, N, K, d, f, 2)
    scores = torch.softmax(torch.randn((M, N), device="cuda") * 2, -1)
    topk = torch.empty((M, K), dtype=torch.uint8, device="cuda")
    gates = torch.empty((M, K), device="cuda")
    want = P.MoeLayer(a["gate_up"], a["down"], K=K, N=N)(a["x"], scores=scores, topk=topk,
                                                        gates=gates)
    a["topk"], a["gates"] = topk, gates
    out = layer(P, a, N, K)
    e = (out.double() - want.double()).norm() / want.double().norm()
    # three roundings of some 2^-9 / sqrt(3) each in the mean square (h, y, out) and one (out)
    assert e <= 4 * 2.0 ** -9 / 3 ** 0.5


@pytest.mark.parametrize("w8", [False, True])
def test_a_decode_layers_prompt(P, w8):
    """MoeLayer.prompt against the same layer's call for as many tokens as that takes, and more
    tokens than it takes; a slot's matrices one after the other."""
    M, N, K, d, f = 1024, 32, 4, 512, 256
    a = layer_inputs(M, N, K, d, f, 2)
    g13, g2, s13, s2 = a["gate_up"], a["down"], None, None
    if w8:
        (g13, s13), (g2, s2) = P.quantize_rows(g13), P.quantize_rows(g2)
    slots = torch.zeros((N, 3 * f * d), dtype=g13.dtype, device="cuda")
    slots[:, :2 * f * d], slots[:, 2 * f * d:] = g13.flatten(1), g2.flatten(1)
    lay = P.MoeLayer(*P.expert_views(slots, f, d), K=K, N=N, gate_up_scale=s13, down_scale=s2)
    scores = torch.softmax(torch.randn((M, N), device="cuda") * 2, -1)
    topk = torch.empty((M, K), dtype=torch.uint8, device="cuda")
    gates = torch.empty((M, K), device="cuda")
    want = lay(a["x"], scores=scores, topk=topk, gates=gates).double()
    out = lay.prompt(a["x"], topk, gates)
    # bf16: three roundings of some 2^-9 / sqrt(3) each in the mean square (h, y, out) and one;
    # 8 bits: x and h have four significant bits, an error of at most 2^-4 of each element
    # (2^-4 / sqrt(3) in the mean square), where the call keeps eight and more
    e = (out.double() - want).norm() / want.norm()
    assert e <= (3 * 2.0 ** -4 / 3 ** 0.5 if w8 else 4 * 2.0 ** -9 / 3 ** 0.5)
    many = lay.prompt(a["x"].repeat(3, 1), topk.repeat(3, 1), gates.repeat(3, 1))
    assert many.shape == (3 * M, d) and torch.equal(many[M:2 * M], out)
    slot = torch.arange(N, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        P.MoeLayer(*P.expert_views(slots, f, d), K=K, expert_slot=slot, gate_up_scale=s13,
                   down_scale=s2).prompt(a["x"], topk, gates)


def test_layer_captured_twice_and_on_other_streams(P):
    """Two graphs of the layer replayed at once on their streams, with new data each time."""
    N, K = 64, 4
    ins = [layer_inputs(M, N, K, 512, 256, M) for M in (300, 2000)]
    graphs, outs = [], []
    for a in ins:
        layer(P, a, N, K)
        torch.cuda.synchronize()
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            outs.append(layer(P, a, N, K))
        graphs.append(gr)
    streams = [torch.cuda.Stream() for _ in ins]
    for turn in range(3):
        for a in ins:
            a["x"].copy_(torch.randn_like(a["x"]))
            a["topk"].copy_(a["topk"].roll(turn + 1, 0))
        torch.cuda.synchronize()
        for gr, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                gr.replay()
        torch.cuda.synchronize()
        for a, o in zip(ins, outs):
            assert torch.equal(o, layer(P, a, N, K))
    for a, st in zip(ins, streams):                     # eager, on a stream by name
        st.wait_stream(torch.cuda.current_stream())
        o = layer(P, a, N, K, stream=st)
        st.synchronize()
        assert torch.equal(o, layer(P, a, N, K))
    assert P.crc.crc_device_error() == 0


def test_training_step_of_the_layer(P):
    """Gradients of x, of the matrices and of the gates through the four operators, against
    those that autograd takes in 64 bits."""
    M, N, K, d, f = 90, 16, 2, 64, 48
    a = layer_inputs(M, N, K, d, f, 9)
    g = torch.Generator(device="cuda").manual_seed(9)
    dout = randn(g, M, d)
    off, rows, place = P.group_choices(a["topk"], N)
    wgu = a["gate_up"].flatten(1, 2)
    gu = P.group_matmul(a["x"], wgu, off, rows=rows, K=K)
    gate, up = gu.float().chunk(2, -1)
    sg = torch.sigmoid(gate)
    h = (gate * sg * up).bfloat16()
    y = P.group_matmul(h, a["down"], off)
    dy, dgates = P.sum_choices_grad(dout, place, gates=a["gates"], y=y)
    dh, dw2 = P.group_matmul_grad(dy, h, a["down"], off)
    dgu = torch.cat([dh.float() * up * sg * (1 + gate * (1 - sg)), dh.float() * gate * sg], -1)
    dxc, dw1 = P.group_matmul_grad(dgu.bfloat16(), a["x"], wgu, off, rows=rows, K=K)
    dx = P.sum_choices(dxc, place)

    leaves = [t.double().requires_grad_() for t in (a["x"], a["gate_up"], a["down"], a["gates"])]
    x, w13, w2, gates = leaves
    idx = a["topk"].long()
    v = torch.einsum("md,mkpfd->mkpf", x, w13[idx])
    out = (torch.einsum("mkf,mkdf->mkd", silu(v[:, :, 0]) * v[:, :, 1], w2[idx])
           * gates[..., None]).sum(1)
    want = torch.autograd.grad(out, leaves, dout.double())
    for got, w, name in ((dx, want[0], "x"), (dw1.view(N, 2, f, d), want[1], "gate_up"),
                         (dw2, want[2], "down"), (dgates, want[3], "gates")):
        # at most seven roundings to bf16 on the way (gate and up, h, y, dy, dh, their gradient,
        # the choice's row, the sum), each 2^-8 of its value at most, in sums of either sign
        e = (got.double() - w).norm() / w.norm()
        assert e <= 7 * U16, name


@pytest.mark.parametrize("N,k,n,counts", [
    (128, 2048, 256, [1]), (128, 2048, 256, [9, 1, 2]), (32, 256, 512, [1]), (4, 1024, 2048, [3]),
    (2, 640, 512, [1, 130]), (8, 4096, 128, [16, 1]),
])
def test_few_gathered_rows_again_and_again(P, N, k, n, counts):
    """Some of the warps that gather have no rows; none of them misses a turn of the ring."""
    g = torch.Generator(device="cuda").manual_seed(N + k)
    counts = (counts * N)[:N]
    E = sum(counts)
    x, w = randn(g, E, k), randn(g, N, n, k)
    rows = torch.randperm(E, device="cuda", generator=g).to(torch.int32)
    off = offsets_of(counts)
    dy = randn(g, E, n)
    first = P.group_matmul(x, w, off, rows=rows, K=1)
    _, dw = P.group_matmul_grad(dy, x, w, off, rows=rows, K=1, want_dx=False)
    again, dwa = torch.empty_like(first), torch.empty_like(dw)
    for _ in range(1000):
        P.group_matmul(x, w, off, rows=rows, K=1, y=again)
        P.group_matmul_grad(dy, x, w, off, rows=rows, K=1, want_dx=False, dw=dwa)
    assert P.crc.crc_device_error() == 0
    assert torch.equal(first, again) and torch.equal(dw, dwa)
