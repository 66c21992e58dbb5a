"""Rows in 4 bits, code for code, and products with 4-bit matrices against 64 bits."""
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


def plain_rows4(x, G):
    """Codes (before packing) and scales by the definition, on the host in 64 bits."""
    v = x.double().cpu().unflatten(-1, (-1, G))
    a = (v.abs().amax(-1) / 7).to(torch.bfloat16)
    a = torch.where(a == 0, torch.ones_like(a), a)
    q = torch.round(v / a.double()[..., None])
    q = torch.where(torch.isfinite(a)[..., None], q, torch.zeros_like(q))
    return q.clamp(-7, 7).flatten(-2).to(torch.int64), a.transpose(-1, -2).contiguous()


def unpack(q):
    q = q.cpu().to(torch.int64)
    lo, hi = q & 15, q >> 4
    v = torch.stack((lo, hi), -1).flatten(-2)
    return torch.where(v > 7, v - 16, v)


def check_rows4(P, x, G, **kw):
    q, a = P.quantize_rows4(x, G, **kw)
    wq, wa = plain_rows4(x, G)
    assert torch.equal(a.cpu().view(torch.int16), wa.view(torch.int16))
    assert torch.equal(unpack(q), wq)
    return q, a


@pytest.mark.parametrize("lead,n,k", [((), 1, 128), ((), 33, 384), ((3,), 40, 512), ((2, 2), 8, 640),
                                      ((), 31, 2944), ((5, 1), 70, 1024)])
@pytest.mark.parametrize("G", [32, 64, 128])
@pytest.mark.parametrize("exponent", [0, -70, -99, -103, -128, 100])
def test_rows4(P, lead, n, k, G, exponent):
    g = torch.Generator(device="cuda").manual_seed(n + k)
    x = torch.randn((*lead, n, k), device="cuda", generator=g, dtype=torch.float64)
    check_rows4(P, (x * 2.0 ** exponent).bfloat16(), G)


@pytest.mark.parametrize("G", [32, 64, 128])
@pytest.mark.parametrize("exponent", [0, -60, -98, -101, -126])
def test_quotients_in_the_middle_go_to_the_even_code(P, G, exponent):
    """Halves of the scale times odd numbers, for all 128 mantissas of a scale."""
    g = torch.Generator(device="cuda").manual_seed(G)
    a = (torch.arange(128, 256, device="cuda").double() * 2.0 ** (exponent - 7))
    odd = torch.randint(-6, 6, (128, 8 * G), device="cuda", generator=g) + 0.5
    x = a[:, None] * odd
    x[:, ::G] = 7 * a[:, None]                          # gives each group that scale, or one near
    check_rows4(P, x.bfloat16(), G)


def test_rows4_of_special_values(P):
    x = torch.zeros((6, 128), dtype=torch.bfloat16, device="cuda")
    x[1, 5] = float("inf")
    x[2, 70] = float("nan")
    x[3] = 2.0 ** -133                                  # the smallest number: its scale is zero
    x[4, 3], x[4, 64:] = -3.3e38, 1e-30
    x[5, ::2] = -0.0
    q, a = P.quantize_rows4(x, 32)
    wq, wa = plain_rows4(torch.where(torch.isfinite(x), x, torch.zeros_like(x)), 32)
    a, s = a.cpu(), unpack(q)
    assert a[0, 1] == float("inf") and a[2, 2].isnan() and (s[1] == 0).all() and (s[2] == 0).all()
    for r in (0, 3, 4, 5):
        assert torch.equal(a[:, r], wa[:, r]) and torch.equal(s[r], wq[r])
    assert (a[:, 3] == 1).all() and (s[3] == 0).all()


def test_rows4_of_strided_rows(P):
    big = torch.randn((50, 512), device="cuda").bfloat16()
    q, a = check_rows4(P, big[:, 64:320], 64)
    out, sc = torch.empty_like(q), torch.empty_like(a)
    got = P.quantize_rows4(big[:, 64:320], 64, out4=out, scale=sc)
    assert got[0] is out and torch.equal(out, q) and torch.equal(sc, a)
    assert P.quantize_rows4(big[:0], 64)[0].shape == (0, 256)


# --------------------------------------------------------------------------- #
def weights4(P, g, slots, n, k, G, glu):
    w = torch.randn((slots, *((2, n) if glu else (n,)), k), device="cuda", generator=g)
    q, a = P.quantize_rows4((w * k ** -0.5).bfloat16(), G)
    v = unpack(q).cuda().double().unflatten(-1, (-1, G)) * a.double().mT[..., None]
    return q, a, v.flatten(-2)


def plain4(x, v, topk, slot, glu):
    """y [M][K][n] and its bound; x [M][K][k] in 64 bits, v [slots](2)[n][k]."""
    M, K = topk.shape
    n, k = v.shape[-2:]
    y = torch.zeros((M, K, n), dtype=torch.float64, device="cuda")
    b = torch.zeros_like(y)
    for m in range(M):
        for j in range(K):
            e = int(topk[m, j])
            s = int(slot[e]) if e < slot.numel() else -1
            if not 0 <= s < v.shape[0]:
                continue
            w = v[s]
            if not glu:
                y[m, j] = w @ x[m, j]
                b[m, j] = U16 * y[m, j].abs() + 2 * k * U32 * (w.abs() @ x[m, j].abs())
                continue
            g, u = w[0] @ x[m, j], w[1] @ x[m, j]
            dg, du = (2 * k * U32 * (w[i].abs() @ x[m, j].abs()) for i in (0, 1))
            sg = g / (1 + torch.exp(-g))
            y[m, j] = sg * u
            b[m, j] = ((U16 + 64 * U32) * y[m, j].abs() + 1.1 * dg * (u.abs() + du)
                       + sg.abs() * du)
    return y, b


# N, slots, n, k, M, K
CASES = [(16, 16, 32, 128, 1, 1), (16, 16, 8, 128, 1, 4), (32, 8, 40, 384, 2, 4),
         (16, 16, 256, 512, 9, 2), (4, 4, 72, 640, 33, 2), (1, 1, 136, 2048, 40, 1),
         (128, 32, 768, 2048, 1, 8), (3, 3, 24, 1152, 70, 3), (256, 256, 16, 256, 30, 6)]


@pytest.mark.parametrize("N,slots,n,k,M,K", CASES)
@pytest.mark.parametrize("G", [32, 64, 128])
@pytest.mark.parametrize("glu", [False, True])
@pytest.mark.parametrize("per_choice", [False, True])
def test_matvec4(P, N, slots, n, k, M, K, G, glu, per_choice):
    g = torch.Generator(device="cuda").manual_seed(N + n + k + M)
    q, a, v = weights4(P, g, slots, n, k, G, glu)
    # any ids, the same one more than once in a token, some without an expert or a slot
    topk = torch.randint(0, min(256, N + 1), (M, K), device="cuda", generator=g).to(torch.uint8)
    if M * K == 1:
        topk.zero_()
    slot = torch.full((N,), -1, dtype=torch.int32, device="cuda")
    some = torch.randperm(N, device="cuda", generator=g)[:slots]
    slot[some] = torch.randperm(slots, device="cuda", generator=g)[:some.numel()].to(torch.int32)
    x = torch.randn((M, K, k) if per_choice else (M, k), device="cuda", generator=g).bfloat16()
    y = torch.full((M, K, n), 7.0, dtype=torch.bfloat16, device="cuda")
    got = P.matvec4(x, q, a, topk=topk, expert_slot=slot, y=y)
    assert got is y
    xd = x.double() if per_choice else x.double()[:, None].expand(M, K, k)
    want, b = plain4(xd, v, topk.cpu(), slot.cpu(), glu)
    assert ((y.double() - want).abs() <= b).all()
    assert P.crc.crc_device_error() == 0


@pytest.mark.parametrize("glu", [False, True])
def test_matvec4_of_many_rows(P, glu):
    """Hundreds of rows for one expert, the most choices of a call, and the same result for
    a choice whatever is beside it."""
    g = torch.Generator(device="cuda").manual_seed(1)
    q, a, v = weights4(P, g, 2, 48, 256, 64, glu)
    x = torch.randn((1024, 256), device="cuda", generator=g).bfloat16()
    topk = torch.zeros((1024, 8), dtype=torch.uint8, device="cuda")
    topk[:, 3] = 1
    y = P.matvec4(x, q, a, topk=topk)
    for r in (0, 500, 1023):
        alone = P.matvec4(x[r:r + 1], q, a, topk=topk[r:r + 1])
        assert torch.equal(y[r], alone[0])
        want, b = plain4(x[r:r + 1].double()[:, None].expand(1, 8, 256), v, topk[r:r + 1].cpu(),
                         torch.arange(2), glu)
        assert ((y[r:r + 1].double() - want).abs() <= b).all()
    assert torch.equal(y[:, :3], y[:, 4:7])


@pytest.mark.parametrize("M,K,N", [(900, 8, 16), (1024, 1, 255), (37, 32, 3)])
def test_all_choices_without_a_slot_are_zero(P, M, K, N):
    """Hundreds of ids without an expert or a slot, between others."""
    g = torch.Generator(device="cuda").manual_seed(M)
    q, a, v = weights4(P, g, 2, 264, 128, 32, False)
    x = torch.randn((M, 128), device="cuda", generator=g).bfloat16()
    topk = torch.randint(0, 256, (M, K), device="cuda", generator=g).to(torch.uint8)
    slot = torch.full((N,), -1, dtype=torch.int32, device="cuda")
    slot[0], slot[N - 1], slot[1] = 1, 0, 2
    for turn in range(3):
        y = torch.full((M, K, 264), 7.0, dtype=torch.bfloat16, device="cuda")
        P.matvec4(x, q, a, topk=topk, expert_slot=slot, y=y)
        has = (topk == 0) | (topk == N - 1)
        assert (y[~has] == 0).all()
        want = torch.einsum("mnk,mk->mn", v[(topk[has] == 0).long()],
                            x.double()[torch.nonzero(has)[:, 0]])
        bound = U16 * want.abs() + 2 * 128 * U32 * torch.einsum(
            "mnk,mk->mn", v[(topk[has] == 0).long()].abs(), x.double()[torch.nonzero(has)[:, 0]].abs())
        assert ((y[has].double() - want).abs() <= bound).all()


def test_matvec4_without_choices(P):
    """All rows take the one matrix: a dense layer in 4 bits."""
    g = torch.Generator(device="cuda").manual_seed(1)
    q, a, v = weights4(P, g, 1, 200, 384, 128, False)
    x = torch.randn((5, 384), device="cuda", generator=g).bfloat16()
    y = P.matvec4(x, q, a)
    want, b = plain4(x.double()[:, None], v, torch.zeros((5, 1), dtype=torch.int64),
                     torch.zeros(1, dtype=torch.int64), False)
    assert y.shape == (5, 1, 200) and ((y.double() - want).abs() <= b).all()


def test_matvec4_of_strided_slots_and_rows(P):
    """Codes and scales one after the other in each slot, as a transfer would copy them."""
    g = torch.Generator(device="cuda").manual_seed(4)
    n, k, G, S = 64, 256, 64, 6
    q, a, _ = weights4(P, g, S, n, k, G, True)
    cb, sb = q[0].numel(), a[0].numel() * 2
    slots = torch.zeros((S, cb + sb + 64), dtype=torch.uint8, device="cuda")
    slots[:, :cb] = q.view(S, -1)
    slots[:, cb:cb + sb] = a.view(S, -1).view(torch.uint8)
    codes = slots.as_strided(q.shape, (slots.stride(0), *q.stride()[1:]))
    half = slots.view(torch.bfloat16)
    scale = half.as_strided(a.shape, (half.stride(0), *a.stride()[1:]), cb // 2)
    x = torch.randn((3, k + 40), device="cuda", generator=g).bfloat16()[:, :k]
    topk = torch.randint(0, S, (3, 4), device="cuda", generator=g).to(torch.uint8)
    assert torch.equal(P.matvec4(x, codes, scale, topk=topk),
                       P.matvec4(x.contiguous(), q, a, topk=topk))


def test_a_choice_does_not_see_anothers_row(P):
    g = torch.Generator(device="cuda").manual_seed(4)
    q, a, _ = weights4(P, g, 1, 64, 512, 32, False)
    x = torch.randn((11, 512), device="cuda", generator=g).bfloat16()
    clean = P.matvec4(x, q, a)
    x[0], x[7] = float("nan"), float("inf")
    y = P.matvec4(x, q, a)
    keep = [i for i in range(11) if i not in (0, 7)]
    assert torch.equal(y[keep], clean[keep]) and y[0].isnan().all()


def test_matvec4_of_large_and_small_values(P):
    """x near both ends of bf16, and what is not x's in the last columns' box."""
    g = torch.Generator(device="cuda").manual_seed(5)
    q, a, v = weights4(P, g, 2, 16, 288, 32, False)
    topk = torch.tensor([[0], [1], [0]], dtype=torch.uint8, device="cuda")
    base = torch.randn((3, 288), device="cuda", generator=g, dtype=torch.float64)
    for e in (-110, 120):
        x = (base * 2.0 ** e).bfloat16()
        y = P.matvec4(x, q, a, topk=topk)
        want, b = plain4(x.double()[:, None], v, topk.cpu(), torch.arange(2), False)
        assert ((y.double() - want).abs() <= b).all()


def test_matvec4_captured_and_on_a_named_stream(P):
    g = torch.Generator(device="cuda").manual_seed(6)
    q, a, _ = weights4(P, g, 32, 96, 512, 128, True)
    x = torch.randn((3, 512), device="cuda", generator=g).bfloat16()
    topk = torch.randint(0, 32, (3, 4), device="cuda", generator=g).to(torch.uint8)
    slot = torch.randperm(32, device="cuda").to(torch.int32)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y = P.matvec4(x, q, a, topk=topk, expert_slot=slot, stream=side)
    side.synchronize()
    assert torch.equal(y, P.matvec4(x, q, a, topk=topk, expert_slot=slot))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = P.matvec4(x, q, a, topk=topk, expert_slot=slot)
    for turn in range(3):
        x.copy_(torch.randn((3, 512), device="cuda"))
        topk.copy_(torch.randint(0, 33, (3, 4), device="cuda").to(torch.uint8))
        slot.copy_(slot.roll(turn + 1))
        graph.replay()
        assert torch.equal(out, P.matvec4(x, q, a, topk=topk, expert_slot=slot))


def test_no_rows(P):
    q, a, _ = weights4(P, torch.Generator(device="cuda").manual_seed(6), 2, 16, 128, 32, False)
    x = torch.empty((0, 128), dtype=torch.bfloat16, device="cuda")
    topk = torch.empty((0, 2), dtype=torch.uint8, device="cuda")
    assert P.matvec4(x, q, a, topk=topk).shape == (0, 2, 16)


def test_two_products_of_a_decoded_token(P):
    """Gate and up, then down, then the sum over the choices: an expert layer from 4-bit slots,
    against the same on the values that the codes stand for."""
    g = torch.Generator(device="cuda").manual_seed(7)
    N, K, d, f, M = 32, 4, 512, 256, 3
    q1, a1, v1 = weights4(P, g, N, f, d, 32, True)
    q2, a2, v2 = weights4(P, g, N, d, f, 64, False)
    x = torch.randn((M, d), device="cuda", generator=g).bfloat16()
    top = torch.randn((M, N), device="cuda", generator=g).topk(K, -1)
    topk, gates = top.indices.to(torch.uint8), torch.softmax(top.values, -1)
    place = torch.arange(M * K, dtype=torch.int32, device="cuda").view(M, K)
    h = P.matvec4(x, q1, a1, topk=topk)
    y = P.matvec4(h, q2, a2, topk=topk)
    out = P.sum_choices(y.view(M * K, d), place, gates=gates)
    v = torch.einsum("md,mkpfd->mkpf", x.double(), v1[topk.long()])
    hd = v[:, :, 0] / (1 + torch.exp(-v[:, :, 0])) * v[:, :, 1]
    yd = torch.einsum("mkf,mkdf->mkd", hd, v2[topk.long()])
    want = (yd * gates.double()[..., None]).sum(1)
    # h and y are rounded to bf16, then out (twice U16 leaves room for the fp32 sums)
    slack = torch.einsum("mkf,mkdf->mkd", hd.abs(), v2[topk.long()].abs()) + yd.abs()
    slack = 2 * U16 * (slack * gates.double()[..., None]).sum(1)
    assert ((out.double() - want).abs() <= slack + U16 * want.abs()).all()
