"""Calls on a stream that is not the current one: what the binding makes for them
(workspaces, outputs) belongs to that stream."""
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


class Recorder:
    """The library, but for the calls `names`: their arguments are kept, nothing runs."""

    def __init__(self, lib, names):
        self._lib, self._names, self.calls = lib, names, []

    def __getattr__(self, name):
        if name in self._names:
            return lambda *a: self.calls.append((name, a)) or 0
        return getattr(self._lib, name)


def layer_of(P, seed=0, w8=False, N=64, K=4, d=1024, f=512):
    g = torch.Generator(device="cuda").manual_seed(seed)
    new = lambda *s, k=1.0: (torch.randn(s, device="cuda", generator=g) * k).bfloat16()  # noqa: E731
    w13, w2, router = new(N, 2, f, d, k=d ** -0.5), new(N, d, f, k=f ** -0.5), new(N, d, k=d ** -0.5)
    s13 = s2 = None
    if w8:
        (w13, s13), (w2, s2) = P.quantize_rows(w13), P.quantize_rows(w2)
    return P.MoeLayer(w13, w2, K=K, router=router, gate_up_scale=s13, down_scale=s2), new(33, d)


def calls_of(P):
    """name -> (call(stream), positions of the addresses the binding makes for it)."""
    layer, x = layer_of(P)
    s, dy, w = (torch.zeros((64, 1024), dtype=torch.bfloat16, device="cuda") for _ in range(3))
    rstd = torch.ones(64, device="cuda")
    p = P.crc.problem(2, 16, 2, 256, 4, 1, 2, 0)
    probs = torch.softmax(torch.randn((2, 8, 2, 3, 16), device="cuda"), -1)
    hidden = torch.zeros((2, 8, 2, 256), dtype=torch.bfloat16, device="cuda")
    w_cat = torch.zeros((2, 48, 256), dtype=torch.bfloat16, device="cuda")
    return {
        "crc_moe_layer": (lambda st: layer(x, stream=st), (8, 11)),
        "crc_rms_norm": (lambda st: P.rms_norm(s, w[0], stream=st), (9,)),
        "crc_rms_norm_grad": (lambda st: P.rms_norm_grad(dy, s, w[0], rstd, stream=st), (8, 9, 10)),
        "crc_quantize_rows": (lambda st: P.quantize_rows(s, stream=st), (4, 5)),
        "crc_cache_loss": (lambda st: P.cache_loss(p, probs, 4, 0.05, stream=st), (8, 9, 10, 11)),
        "crc_route_scores": (lambda st: P.route_scores(p, hidden, w_cat, stream=st), (5,)),
    }


@pytest.mark.parametrize("name", ["crc_moe_layer", "crc_rms_norm", "crc_rms_norm_grad",
                                  "crc_quantize_rows", "crc_cache_loss", "crc_route_scores"])
@pytest.mark.parametrize("as_int", [False, True])
def test_memory_of_a_call_is_its_streams(P, monkeypatch, name, as_int):
    """While the calls' kernels may run, no block of one call is handed to a call on
    another stream, or to the current stream.  (Nothing is launched here.)"""
    call, places = calls_of(P)[name]
    torch.cuda.synchronize()
    rec = Recorder(P.crc.load(), {name})
    monkeypatch.setattr(P.crc, "_lib", rec)
    streams = [torch.cuda.Stream() for _ in range(2)]
    call(None)
    for st in streams:
        call(st.cuda_stream if as_int else st)
    assert [n for n, _ in rec.calls] == [name] * 3
    own, first, second = ([a[i] for i in places] for _, a in rec.calls)
    assert all(own) and all(first) and all(second)
    assert not set(own) & set(first) and not set(own) & set(second) and not set(first) & set(second)
    assert rec.calls[1][1][-1] == streams[0].cuda_stream
    # freed blocks of the two calls are not the current stream's
    sizes = [256 << k for k in range(16)]
    held = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(8)]
    taken = {t.data_ptr() for t in held}
    assert not taken & (set(first) | set(second))


def test_the_current_stream_by_name_and_the_default_stream(P):
    layer, x = layer_of(P)
    ref = layer(x)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        a, b = layer(x, stream=side), layer(x, stream=side.cuda_stream)
        c = layer(x, stream=0)
    torch.cuda.synchronize()
    for t in (a, b, c):
        assert torch.equal(t, ref)


def test_calls_on_several_streams_without_workspaces(P):
    """Layers and gradients at the same time, each call with a workspace of the binding's
    making, and allocations of the current stream in between."""
    layers = [layer_of(P, 1), layer_of(P, 2, True), layer_of(P, 3, True, 128, 8, 512, 256)]
    g = torch.Generator(device="cuda").manual_seed(4)
    s, dy, w = (torch.randn((3000, 512), device="cuda", generator=g).bfloat16() for _ in range(3))
    rstd = torch.empty(3000, device="cuda")
    P.rms_norm(s, w[0], rstd=rstd)
    ref = [layer(x) for layer, x in layers] + list(P.rms_norm_grad(dy, s, w[0], rstd))
    sizes = [layer.workspace_bytes(33) for layer, _ in layers] + [1 << 20, 1 << 22]
    streams = [torch.cuda.Stream() for _ in range(4)]
    torch.cuda.synchronize()
    outs = []
    for _ in range(30):
        got = [layer(x, stream=st) for (layer, x), st in zip(layers, streams)]
        got += P.rms_norm_grad(dy, s, w[0], rstd, stream=streams[3])
        outs.append(got)
        for n in sizes:
            torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    for got in outs:
        for a, b in zip(got, ref):
            assert torch.equal(a, b)
    assert P.crc.crc_device_error() == 0


@pytest.mark.parametrize("as_int", [False, True])
def test_a_state_and_its_calls_on_a_named_stream(P, as_int):
    """State, synthetic inputs, router heads, scan, step and losses on a stream that is
    not the current one, nothing passed in but the stream, equal those on the current one."""
    p = P.crc.problem(2, 32, 4, 256, 8, 1, 3, 0)

    def run(stream):
        w = P.synth_weights(2, 32, 256, seed=1, stream=stream)
        h, _ = P.synth_hidden(3, 16, 2, 256, seed=2, stream=stream)
        probs = P.route_scores(p, h, w, stream=stream)
        a, b = P.State(p, stream=stream), P.State(p, stream=stream)
        P.cache_scan(p, probs, a, stream=stream)
        P.route_and_cache(p, h, w, b, stream=stream)
        loss, means, grad = P.cache_loss(p, probs, 8, 0.05, stream=stream)
        # blocks that the calls gave back, asked for again by the current stream
        held = [torch.full((1 << k,), 255, dtype=torch.uint8, device="cuda") for k in range(8, 22)]
        torch.cuda.synchronize()
        del held
        return [probs, loss, means, grad], a.read(stream), b.read(stream)

    side = torch.cuda.Stream()
    ref, a0, b0 = run(None)
    got, a1, b1 = run(side.cuda_stream if as_int else side)
    for x, y in zip(got, ref):
        assert torch.equal(x, y)
    for x, y in ((a1, a0), (b1, b0)):
        assert x["error"] == 0 and x["misses"] == y["misses"] and x["proactive"] == y["proactive"]
