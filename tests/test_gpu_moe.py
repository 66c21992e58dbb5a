"""The mixture-of-experts layer for a few tokens (crc_moe_layer) against its
definition in 64 bits, at the sizes, types and masks where it can go wrong."""
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
    assert P.crc.crc_device_error() == 0
    return P


def randn(g, *shape, scale=1.0, dtype=torch.bfloat16):
    return (torch.randn(shape, device="cuda", generator=g) * scale).to(dtype)


def bits8(w):
    a = w.float().abs().amax(-1) / 448.0
    a = torch.where(a > 0, a, torch.ones_like(a))
    return (w.float() / a[..., None]).to(torch.float8_e4m3fn), a


class Case:
    """Weights and inputs of one layer, and the layer handle."""

    def __init__(self, P, N, K, d, f, M, w8=False, x8=False, slots=None, image=False,
                 renorm=True, seed=0, x_rows=1):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.N, self.K, self.d, self.f, self.M, self.renorm = N, K, d, f, M, renorm
        self.x = randn(g, M * x_rows, d)[::x_rows]
        self.router = randn(g, N, d, scale=d ** -0.5)
        S = slots or N
        w13 = randn(g, S, 2, f, d, scale=d ** -0.5)
        w2 = randn(g, S, d, f, scale=f ** -0.5)
        self.s13 = self.s2 = None
        if w8:
            w13, self.s13 = bits8(w13)
            w2, self.s2 = bits8(w2)
        if image:                         # gate | up | down in slots with room between them
            n = 3 * f * d
            buf = torch.zeros((S, n + 64), dtype=w13.dtype, device="cuda")
            a, b = P.expert_views(buf, f, d)
            a.copy_(w13)
            b.copy_(w2)
            w13, w2 = a, b
        self.w13, self.w2 = w13, w2
        self.slot = None
        if slots:
            self.slot = torch.full((N,), -1, dtype=torch.int32, device="cuda")
            at = torch.randperm(S, device="cuda", generator=g).to(torch.int32)
            self.slot[torch.randperm(N, device="cuda", generator=g)[:S]] = at[:min(S, N)]
        self.x8 = self.xs = None
        if x8:
            self.x8, self.xs = bits8(self.x)
        self.layer = P.MoeLayer(w13, w2, K=K, router=self.router, expert_slot=self.slot,
                                gate_up_scale=self.s13, down_scale=self.s2, renormalize=renorm)

    def run(self, **kw):
        topk = torch.full((self.M, self.K), 255, dtype=torch.uint8, device="cuda")
        gates = torch.full((self.M, self.K), -7.0, device="cuda")
        args = dict(x8=self.x8, x_scale=self.xs, topk=topk, gates=gates)
        args.update(kw)
        out = self.layer(args.pop("x", self.x), **args)
        return out, topk, gates


def check_routing(c, topk, gates, z=None):
    """S and g against 64 bits; a token whose K-th and next score are closer than
    1e-5 may take either, so only clear ranks are compared."""
    z = c.x.double() @ c.router.double().t() if z is None else z
    order = torch.sort(z, dim=-1, descending=True, stable=True)
    want, v = order.indices[:, :c.K], order.values
    ids = topk.long()
    assert (ids < c.N).all()
    assert (torch.sort(ids, dim=-1).values.diff(dim=-1) > 0).all()       # distinct
    near = torch.zeros(z.shape, dtype=torch.bool, device=z.device)
    close = v.diff(dim=-1).abs() < 1e-5
    near[:, :-1] |= close
    near[:, 1:] |= close
    near = near[:, :c.K]
    assert ((ids == want) | near).all()
    return torch.softmax(z, -1)


def reference(c, topk, p):
    """out in 64 bits for the choices topk, and the bound that the arithmetic has:
    fp32 dot products (8 sqrt(n) u32 of the sum of magnitudes, the random-walk
    estimate with room), h rounded to bf16, out rounded once; hi/lo pieces of 8-bit
    products hold an operand to 2^-21 of its row's largest."""
    K, ids = c.K, topk.long()
    g = torch.gather(p, 1, ids)
    if c.renorm:
        g = g / g.sum(1, keepdim=True)
    x = c.x.double() if c.x8 is None else c.x8.double() * c.xs.double()[:, None]
    w8 = c.s13 is not None
    out = torch.zeros((c.M, c.d), dtype=torch.float64, device="cuda")
    err = torch.zeros_like(out)
    cd, cf = 8 * math.sqrt(c.d) * U32 + 2 * U32, 8 * math.sqrt(c.f) * U32 + 2 * U32
    for e in torch.unique(ids).tolist():
        s = e if c.slot is None else int(c.slot[e])
        if s < 0:
            continue
        m, k = torch.nonzero(ids == e, as_tuple=True)
        w13, w2 = c.w13[s].double(), c.w2[s].double()
        if w8:
            w13 = w13 * c.s13[s].double()[..., None]
            w2 = w2 * c.s2[s].double()[:, None]
        xa = x[m].abs()
        if w8 and c.x8 is None:
            xe = 2.0 ** -21 * xa.amax(1, keepdim=True)
        else:
            xe = torch.zeros_like(xa[:, :1])
        a, b = x[m] @ w13[0].t(), x[m] @ w13[1].t()
        ea = cd * (xa @ w13[0].abs().t()) + xe * w13[0].abs().sum(1)
        eb = cd * (xa @ w13[1].abs().t()) + xe * w13[1].abs().sum(1)
        sig = torch.sigmoid(a)
        h = a * sig * b
        eh = 1.1 * ea * b.abs() + (a * sig).abs() * eb + ea * eb + (U16 + 8 * U32) * h.abs()
        if w8:
            eh = eh + 2.0 ** -21 * (h.abs() + eh).amax(1, keepdim=True)
        ge = g[m, k][:, None]
        out.index_add_(0, m, ge * (h @ w2.t()))
        err.index_add_(0, m, ge * (eh @ w2.abs().t() + (cf + 1e-5) * (h.abs() @ w2.abs().t())))
    return out, err + U16 * (out.abs() + err), g


def check(c, out, topk, gates, z=None, probs=False):
    p = check_routing(c, topk, gates, z)
    if probs:
        p = z
    want, bound, g = reference(c, topk, p)
    assert torch.isfinite(out).all()
    assert ((gates.double() - g).abs() <= 1e-5 * g + 1e-30).all()
    off = (out.double() - want).abs()
    assert (off <= bound).all(), f"worst {float((off / bound.clamp_min(1e-300)).max()):.3g} of bound"
    return want


SIZES = [
    # N, K, d, f, M
    (16, 1, 16, 16, 1),
    (16, 2, 256, 512, 1),
    (16, 2, 256, 512, 4),
    (16, 16, 64, 48, 9),            # every expert for every token
    (32, 4, 2880, 288, 5),          # partial K blocks both ways
    (48, 5, 144, 80, 17),
    (64, 6, 2048, 1024, 16),
    (128, 8, 2048, 768, 1),
    (128, 8, 2048, 768, 33),
    (128, 32, 256, 128, 20),
    (16, 2, 512, 256, 200),         # many rows an expert
    (32, 4, 320, 2880, 131),
    (128, 8, 128, 64, 1024),        # the most tokens and entries
]


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("kind", ["bf16", "w8", "w8x8"])
def test_layer_matches_its_definition(P, size, kind):
    N, K, d, f, M = size
    c = Case(P, N, K, d, f, M, w8=kind != "bf16", x8=kind == "w8x8", seed=N + M,
             renorm=(N + K) % 3 != 0)
    check(c, *c.run())
    assert P.crc.crc_device_error() == 0


@pytest.mark.parametrize("size", [
    (32, 2, 64, 48, 16),            # as many choices as one warp has lanes
    (32, 1, 64, 48, 16),
    (32, 1, 64, 48, 17),            # more tokens than warps
    (32, 1, 64, 48, 32),
    (32, 4, 64, 48, 9),             # one choice more than lanes and some
    (128, 32, 128, 64, 1),
    (96, 3, 4104, 80, 3),           # more than one batch of loads a row
    (112, 7, 328, 64, 40),
    (64, 6, 448, 208, 100),         # tiles of 32 rows
], ids=str)
@pytest.mark.parametrize("kind", ["bf16", "w8", "w8x8"])
def test_sizes_around_the_rules(P, size, kind):
    N, K, d, f, M = size
    if kind != "bf16":
        d = d // 16 * 16
    c = Case(P, N, K, d, f, M, w8=kind != "bf16", x8=kind == "w8x8", seed=7 * N + M)
    check(c, *c.run())
    # the same tokens from given probabilities
    pr = torch.softmax(c.x.float() @ c.router.float().t(), -1)
    check(c, *c.run(scores=pr), z=pr.double(), probs=True)
    assert P.crc.crc_device_error() == 0


@pytest.mark.parametrize("kind", ["bf16", "w8", "w8x8"])
@pytest.mark.parametrize("M", [40, 100, 300])
def test_every_token_takes_the_same_experts(P, kind, M):
    """Many row tiles an expert, whatever the tile that the mean calls for."""
    c = Case(P, 64, 3, 256, 96, M, w8=kind != "bf16", seed=M)
    common = torch.randn(256, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    c.x = (c.x.float() * 0.25 + common).to(torch.bfloat16)
    c.router[:3] += (common * 0.1).to(torch.bfloat16)
    if kind == "w8x8":
        c.x8, c.xs = bits8(c.x)
    out, topk, gates = c.run()
    assert (topk.long().sort(-1).values == torch.arange(3, device="cuda")).all()
    check(c, out, topk, gates)


@pytest.mark.parametrize("kind", ["bf16", "w8", "w8x8"])
@pytest.mark.parametrize("M", [1, 3])
def test_few_choices_without_a_slot(P, kind, M):
    c = Case(P, 64, 8, 256, 96, M, w8=kind != "bf16", x8=kind == "w8x8", slots=16, seed=M)
    check(c, *c.run())
    c.slot.fill_(-1)
    out = torch.full((M, 256), float("nan"), dtype=torch.bfloat16, device="cuda")
    _, topk, gates = c.run(out=out)
    assert (out == 0).all()
    check_routing(c, topk, gates)


def test_smallest_hidden_size(P):
    c = Case(P, 16, 2, 8, 16, 3)
    check(c, *c.run())


def test_d_that_is_no_multiple_of_sixteen(P):
    c = Case(P, 16, 3, 200, 32, 7)
    check(c, *c.run())


@pytest.mark.parametrize("kind", ["bf16", "w8"])
def test_strided_rows_and_slots_of_a_cache(P, kind):
    """x as one layer of hidden [M][L][d]; experts as images in cache slots."""
    c = Case(P, 64, 4, 256, 96, 13, w8=kind == "w8", slots=80, image=True, x_rows=5)
    assert c.x.stride(0) == 5 * 256
    check(c, *c.run())


@pytest.mark.parametrize("kind", ["bf16", "w8", "w8x8"])
def test_experts_without_a_slot_add_nothing(P, kind):
    c = Case(P, 64, 8, 256, 96, 37, w8=kind != "bf16", x8=kind == "w8x8", slots=9)
    out, topk, gates = c.run()
    check(c, out, topk, gates)
    # none resident, and values outside the slots: zero, whatever was there before
    for v in (-1, 9, 2 ** 31 - 1, -2 ** 31):
        c.slot.fill_(v)
        out = torch.full((c.M, c.d), float("nan"), dtype=torch.bfloat16, device="cuda")
        c.run(out=out)
        assert (out == 0).all()
    # a map written between calls counts from the next call
    c.slot.copy_(torch.arange(64, dtype=torch.int32, device="cuda") % 9)
    check(c, *c.run())


def test_scores_of_the_router_heads(P):
    """S from given probabilities is the framework's own Top-K."""
    L, N, K, d, M = 3, 64, 6, 256, 21
    p = P.crc.problem(L, N, K, d, 16, 0, M, 0)
    W = P.synth_weights(L, N, d, seed=3)
    h, _ = P.synth_hidden(M, 1, L, d, seed=4)
    probs = P.route_scores(p, h, W)
    st, tr = P.State(p), P.Trace.alloc(p, 1)
    P.cache_scan(p, probs, st, tr)
    for l in range(L):
        c = Case(P, N, K, d, 96, M, seed=l, renorm=l != 1)
        c.x, c.router = h[:, 0, l], W[l, :N]
        pr = probs[:, 0, l, 0]
        assert pr.stride(0) == L * 3 * N
        out, topk, gates = c.run(x=c.x, scores=pr)
        assert torch.equal(topk, tr.topk[:, 0, l])
        check(c, out, topk, gates, z=pr.double(), probs=True)


def test_scores_and_8_bit_rows_need_no_bf16_rows(P):
    c = Case(P, 32, 4, 256, 96, 21, w8=True, x8=True)
    pr = torch.softmax(c.x.float() @ c.router.float().t(), -1)
    check(c, *c.run(x=None, scores=pr), z=pr.double(), probs=True)


def test_ties_go_to_the_lowest_index(P):
    c = Case(P, 128, 8, 64, 32, 6)
    c.router[::2] = c.router[1]                      # 64 experts with one row
    out, topk, gates = c.run()
    z = (c.x.float() @ c.router.float().t()).cpu()
    for m in range(c.M):
        ids = topk[m].tolist()
        tied = [e for e in ids if e % 2 == 0 or e == 1]
        assert tied == sorted(tied)
        assert tied == [e for e in range(128) if e % 2 == 0 or e == 1][:len(tied)]
        # the rest are the experts above the tied score
        assert all(z[m, e] >= z[m, 0] - 1e-5 for e in ids)


def test_large_and_small_rows(P):
    """Rows far from unit size: the 8-bit pieces have a scale a row."""
    for kind in ("bf16", "w8", "w8x8"):
        c = Case(P, 16, 2, 256, 64, 12, w8=kind != "bf16", x8=kind == "w8x8", seed=5)
        s = torch.tensor([2.0 ** k for k in (-40, -20, -8, -3, 0, 0, 1, 2, 3, 4, 5, 6)],
                         device="cuda")[:, None]
        c.x = (c.x.float() * s).to(torch.bfloat16)
        c.x[5, :] = 0
        c.x[5, 3] = 1.0                               # one large element among zeros
        c.x[4, ::2] *= 2.0 ** -12                     # small elements beside large ones
        if c.x8 is not None:
            c.x8, c.xs = bits8(c.x)
        check(c, *c.run())


def test_rows_of_zeros_and_not_finite_rows_stay_alone(P):
    for kind in ("bf16", "w8"):
        c = Case(P, 16, 2, 256, 64, 24, w8=kind == "w8", seed=6)
        clean, _, _ = c.run()
        clean = clean.clone()
        c.x[3] = 0
        c.x[7, 5] = float("nan")
        c.x[11, 250] = float("inf")
        out, topk, gates = c.run()
        rest = [m for m in range(24) if m not in (3, 7, 11)]
        assert torch.equal(out[rest], clean[rest])
        assert (out[3] == 0).all()
        assert (topk[3].long() == torch.arange(2, device="cuda")).all()
        assert not torch.isfinite(out[7].float()).any()
        assert not torch.isfinite(out[11].float()).any()
        assert (topk < 16).all()


@pytest.mark.parametrize("kind", ["bf16", "w8", "w8x8"])
def test_same_bits_every_time_and_on_another_stream(P, kind):
    c = Case(P, 128, 8, 512, 256, 50, w8=kind != "bf16", x8=kind == "w8x8")
    ref = [t.clone() for t in c.run()]
    ws = torch.empty(c.layer.workspace_bytes(c.M), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    for i in range(20):
        ws.fill_(255 if i % 2 else 0)                # nothing in it is taken for granted
        torch.cuda.synchronize()
        if i < 10:
            got = c.run(workspace=ws)
        else:
            with torch.cuda.stream(side):
                got = c.run(workspace=ws)
        torch.cuda.synchronize()
        for a, b in zip(ref, got):
            assert torch.equal(a, b)


@pytest.mark.parametrize("M,w8", [(2, False), (9, False), (9, True), (70, True)])
def test_captured_in_a_graph(P, M, w8):
    c = Case(P, 64, 4, 256, 128, M, w8=w8)
    ref, _, _ = c.run()
    ref = ref.clone()
    ws = torch.empty(c.layer.workspace_bytes(c.M), dtype=torch.uint8, device="cuda")
    out = torch.zeros_like(ref)
    c.run(out=out, workspace=ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.layer(c.x, out=out, workspace=ws)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, ref)


def test_no_tokens(P):
    c = Case(P, 16, 2, 64, 32, 4)
    out = torch.full((0, 64), 1.0, dtype=torch.bfloat16, device="cuda")
    n = P.crc.crc_launch_count()
    P.crc.crc_moe_layer(c.layer.c, c.x.data_ptr(), 64, None, None, None, 0, 0, out.data_ptr(),
                        None, None, None, 0)
    assert P.crc.crc_launch_count() == n


def test_refusals_of_the_binding(P):
    c = Case(P, 16, 2, 64, 32, 4)
    with pytest.raises(ValueError):
        P.MoeLayer(c.w13.float(), c.w2.float(), K=2, router=c.router)
    with pytest.raises(ValueError):
        P.MoeLayer(c.w13, c.w2.transpose(1, 2), K=2, router=c.router)
    with pytest.raises(ValueError):
        P.MoeLayer(c.w13, c.w2, K=2, router=c.router, gate_up_scale=torch.ones(16, 2, 32).cuda())
    with pytest.raises(ValueError):
        P.MoeLayer(c.w13[:8], c.w2[:8], K=2, router=c.router)
    with pytest.raises(P.CrcError):
        P.MoeLayer(c.w13, c.w2, K=17, router=c.router)
    with pytest.raises(ValueError):
        c.layer(c.x.float())
    with pytest.raises(ValueError):
        c.layer(c.x[:, :32])
    with pytest.raises(ValueError):
        c.layer(c.x, out=torch.empty((4, 64), device="cuda"))
    with pytest.raises(ValueError):
        c.layer(c.x.cpu())
    with pytest.raises(P.CrcError):
        c.layer(c.x, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("M", [1, 7, 40])
@pytest.mark.parametrize("kind", ["bf16", "w8x8"])
def test_a_chain_of_calls_needs_no_waits_between_them(P, kind, M):
    """Norm, layer and slot map one after the other on one stream, in place and in one
    workspace, with nothing between them, equal the same with a wait after each call."""
    w8 = kind != "bf16"
    layers = [Case(P, 64, 4, 512, 128, M, w8=w8, slots=80, seed=i) for i in range(3)]
    weight = torch.ones(512, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(max(c.layer.workspace_bytes(M) for c in layers), dtype=torch.uint8,
                     device="cuda")
    maps = [torch.stack([c.slot.roll(k) for k in range(64)]) for c in layers]

    def run(wait):
        g = torch.Generator(device="cuda").manual_seed(9)
        stream = randn(g, M, 512)
        x = randn(g, M, 512)
        h, q = torch.empty_like(x), torch.empty((M, 512), dtype=torch.float8_e4m3fn, device="cuda")
        sc = torch.empty(M, device="cuda")
        seen = []
        for t in range(20):
            for i, c in enumerate(layers):
                c.slot.copy_(maps[i][(3 * t + i) % 64])
                wait()
                P.rms_norm(x, weight, residual=stream, residual_out=stream, out=h,
                           out8=q if w8 else None, scale8=sc if w8 else None)
                wait()
                c.layer(h, out=x, x8=q if w8 else None, x_scale=sc if w8 else None, workspace=ws)
                wait()
            seen.append(x.clone())
        return torch.stack(seen), stream.clone()

    slow = run(torch.cuda.synchronize)
    for _ in range(3):
        fast = run(lambda: None)
        assert torch.equal(fast[0], slow[0]) and torch.equal(fast[1], slow[1])
    assert torch.isfinite(slow[0].float()).all()


def test_calls_on_two_streams_at_once(P):
    """Layers that run at the same time, each with a workspace, wait for nothing of each
    other's."""
    cases = [Case(P, 64, 4, 1024, 512, 33, seed=1), Case(P, 64, 4, 1024, 512, 5, w8=True, seed=2),
             Case(P, 128, 8, 512, 256, 200, w8=True, seed=3)]
    ref = [c.run()[0].clone() for c in cases]
    ws = [torch.empty(c.layer.workspace_bytes(c.M), dtype=torch.uint8, device="cuda") for c in cases]
    outs = [torch.empty_like(r) for r in ref]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(30):
        for c, w, o, st in zip(cases, ws, outs, streams):
            c.layer(c.x, out=o, workspace=w, stream=st)
    torch.cuda.synchronize()
    for o, r in zip(outs, ref):
        assert torch.equal(o, r)
    assert P.crc.crc_device_error() == 0
