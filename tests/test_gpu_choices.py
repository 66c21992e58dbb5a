"""Choices in the order of their experts, and the sum over a token's choices with its
gradient, against their definitions."""
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


def ordered(topk, N):
    """offsets, rows and place from a stable sort on the host."""
    flat = topk.flatten().to(torch.int64).cpu()
    key = torch.where(flat < N, flat, N)
    order = torch.sort(key, stable=True).indices
    n = int((flat < N).sum())
    rows = torch.full_like(flat, -1)
    rows[:n] = order[:n]
    place = torch.full_like(flat, -1)
    place[order[:n]] = torch.arange(n)
    offsets = torch.zeros(N + 1, dtype=torch.int64)
    offsets[1:] = torch.bincount(key, minlength=N + 1)[:N].cumsum(0)
    return [t.to(torch.int32) for t in (offsets, rows, place.view(topk.shape))]


def check_order(P, topk, N, **kw):
    got = P.group_choices(topk, N, **kw)
    for g, w, name in zip(got, ordered(topk, N), ("offsets", "rows", "place")):
        assert torch.equal(g.cpu(), w), name


# one CTA, its last size and the first of two launches; more than a CTA ranks at a time
SIZES = [(1, 1), (1, 32), (31, 1), (33, 1), (37, 4), (2048, 1), (2049, 1), (1023, 3), (1024, 4), (1025, 4), (4096, 1),
         (4097, 1), (2049, 2), (9001, 7), (32768, 8), (160001, 7)]


@pytest.mark.parametrize("M,K", SIZES)
@pytest.mark.parametrize("N", [1, 16, 31, 128, 255, 256])
def test_order(P, M, K, N):
    g = torch.Generator(device="cuda").manual_seed(M * K + N)
    # some ids without an expert where there are such
    topk = torch.randint(0, min(256, N + max(1, N // 8)), (M, K), device="cuda", generator=g)
    check_order(P, topk.to(torch.uint8), N)


@pytest.mark.parametrize("M,K", [(500, 4), (5000, 4)])
def test_order_of_one_sided_choices(P, M, K):
    """All choices of one expert, of none, padded tokens at the end, and the same id in
    every place of a token."""
    for fill in (0, 7, 15, 16, 255):
        check_order(P, torch.full((M, K), fill, dtype=torch.uint8, device="cuda"), 16)
    topk = torch.randint(0, 16, (M, K), device="cuda").to(torch.uint8)
    topk[M // 2:] = 255
    check_order(P, topk, 16)
    check_order(P, topk[:, :1].expand(M, K).contiguous(), 16)


def test_order_in_more_than_a_million_choices(P):
    """Above 128 x 8192 choices a CTA ranks its chunk in several turns."""
    topk = torch.randint(0, 130, (300001, 4), device="cuda").to(torch.uint8)
    check_order(P, topk, 128)


def test_order_of_no_tokens(P):
    offsets, rows, place = P.group_choices(torch.empty((0, 4), dtype=torch.uint8, device="cuda"), 5)
    assert offsets.tolist() == [0] * 6 and rows.numel() == 0 and place.shape == (0, 4)


def test_order_captured_and_on_a_named_stream(P):
    topk = torch.randint(0, 64, (20000, 6), device="cuda").to(torch.uint8)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = P.group_choices(topk, 64, stream=side)
    side.synchronize()
    for g, w in zip(got, ordered(topk, 64)):
        assert torch.equal(g.cpu(), w)
    out = P.group_choices(topk, 64)                     # warm: buffers of the captured call
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.group_choices(topk, 64, offsets=out[0], rows=out[1], place=out[2])
    for seed in range(3):
        topk.copy_(torch.randint(0, 70, topk.shape, device="cuda").to(torch.uint8))
        graph.replay()
        for g, w in zip(out, ordered(topk, 64)):
            assert torch.equal(g.cpu(), w)


# --------------------------------------------------------------------------- #
def randn(g, *shape, scale=1.0, dtype=torch.bfloat16):
    return (torch.randn(shape, device="cuda", generator=g) * scale).to(dtype)


SUMS = [(1, 1, 8), (3, 32, 16), (7, 9, 264), (301, 4, 2880), (64, 8, 2048), (1001, 2, 1000),
        (6500, 1, 88), (13, 5, 32768), (2, 17, 2056), (4, 6, 4096), (13001, 1, 264), (12000, 1, 8)]


def sum_inputs(M, K, d, seed, holes):
    g = torch.Generator(device="cuda").manual_seed(seed)
    R = M * K + 5                                       # more rows than choices
    place = torch.randperm(R, device="cuda", generator=g)[:M * K].to(torch.int32).view(M, K)
    if holes:                                           # choices without a row
        lost = torch.rand((M, K), device="cuda", generator=g) < 0.3
        place[lost] = torch.tensor([-1, R, -2 ** 31, 2 ** 31 - 1], dtype=torch.int32,
                                   device="cuda")[torch.arange(int(lost.sum())) % 4]
    return g, R, place


def picked(y, place):
    """y[place] in 64 bits, zeros for a place outside it."""
    ok = (place >= 0) & (place < y.shape[0])
    return torch.where(ok[..., None], y.double()[place.clamp(0, y.shape[0] - 1).long()], 0.0), ok


@pytest.mark.parametrize("M,K,d", SUMS)
@pytest.mark.parametrize("gated", [True, False])
@pytest.mark.parametrize("holes", [True, False])
def test_sum(P, M, K, d, gated, holes):
    g, R, place = sum_inputs(M, K, d, M + K + d, holes)
    y = randn(g, R, d)
    gates = torch.rand((M, K), device="cuda", generator=g) if gated else None
    out = P.sum_choices(y, place, gates=gates)
    terms, _ = picked(y, place)
    if gated:
        terms = terms * gates.double()[..., None]
    want = terms.sum(1)
    # K products and sums in fp32, each off by half a step, and the output's rounding
    bound = (K + 1) * U32 * terms.abs().sum(1) + U16 * want.abs()
    assert ((out.double() - want).abs() <= bound).all()


def test_sum_without_places_takes_the_rows_in_turn(P):
    """The C call with no place array: choice c is row c."""
    y = randn(torch.Generator(device="cuda").manual_seed(1), 12, 64)
    out = torch.empty((3, 64), dtype=torch.bfloat16, device="cuda")
    P.crc.crc_sum_choices(y.data_ptr(), 12, None, None, 3, 4, 64, out.data_ptr())
    want = y.double().view(3, 4, 64).sum(1)
    assert ((out.double() - want).abs() <= 5 * U32 * y.double().abs().view(3, 4, 64).sum(1)
            + U16 * want.abs()).all()


def test_values_that_no_choice_takes_stay_out(P):
    """NaN and infinities in rows that no choice has do not reach the sum."""
    y = torch.full((9, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
    y[3], y[5] = 1.0, 2.0
    y[0] = float("inf")
    place = torch.tensor([[3, -1, 5], [-1, -1, -1]], dtype=torch.int32, device="cuda")
    gates = torch.tensor([[0.5, float("nan"), 0.25], [1.0, 1.0, float("inf")]], device="cuda")
    out = P.sum_choices(y, place, gates=gates)
    assert (out[0] == 1.0).all() and (out[1] == 0.0).all()


@pytest.mark.parametrize("M,K,d", SUMS)
@pytest.mark.parametrize("gated,dgates", [(True, True), (True, False), (False, False),
                                          (False, True)])
@pytest.mark.parametrize("holes", [True, False])
def test_sum_gradient(P, M, K, d, gated, dgates, holes):
    g, R, place = sum_inputs(M, K, d, M + K + d + 1, holes)
    y, dout = randn(g, R, d), randn(g, M, d)
    gates = torch.rand((M, K), device="cuda", generator=g) if gated else None
    dy = torch.full((R, d), 7.0, dtype=torch.bfloat16, device="cuda")
    got_dy, got_dg = P.sum_choices_grad(dout, place, gates=gates, y=y if dgates else None, dy=dy,
                                        y_rows=R)
    assert got_dy is dy and (got_dg is not None) == dgates
    terms, ok = picked(y, place)
    w = gates.double() if gated else torch.ones((M, K), dtype=torch.float64, device="cuda")
    rows = place[ok].long()
    want = (dout.double()[:, None] * w[..., None])[ok]
    # one product in fp32 and its rounding
    assert ((dy.double()[rows] - want).abs() <= (U16 + U32) * want.abs()).all()
    rest = torch.ones(R, dtype=torch.bool, device="cuda")
    rest[rows] = False
    assert (dy[rest] == 7.0).all()                      # rows that no choice has
    if dgates:
        prod = dout.double()[:, None] * terms
        want = prod.sum(-1)
        # sums over at most d / 8 / 32 turns of 8 in a lane, 5 exchanges and 8 warps
        assert ((got_dg.double() - want).abs()
                <= (d / 32 + 16 + 13) * U32 * prod.abs().sum(-1)).all()


def test_sum_gradient_against_differences(P):
    """<dout, sum(y, g)> along random directions of y and of the gates, in 64 bits."""
    M, K, d = 40, 4, 256
    g, R, place = sum_inputs(M, K, d, 3, True)
    y, dout = randn(g, R, d), randn(g, M, d)
    gates = torch.rand((M, K), device="cuda", generator=g)
    dy = torch.zeros((R, d), dtype=torch.bfloat16, device="cuda")
    dy, dg = P.sum_choices_grad(dout, place, gates=gates, y=y, dy=dy)

    def f(y, gates):
        ok = (place >= 0) & (place < R)
        rows = torch.where(ok[..., None], y[place.clamp(0, R - 1).long()], 0.0)
        return (dout.double() * (rows * gates[..., None]).sum(1)).sum()
    uy = torch.randn((R, d), device="cuda", generator=g, dtype=torch.float64)
    ug = torch.randn((M, K), device="cuda", generator=g, dtype=torch.float64)
    h = 1e-3
    y0, g0 = y.double(), gates.double()
    by_y = (f(y0 + h * uy, g0) - f(y0 - h * uy, g0)) / (2 * h)
    by_g = (f(y0, g0 + h * ug) - f(y0, g0 - h * ug)) / (2 * h)
    # every element of dy is off by half a bf16 step, of dg by d fp32 ones; f is linear in each
    # argument, so its differences are exact but for 64-bit roundings over h
    assert abs(by_y - (dy.double() * uy).sum()) <= 1e-9 + (U16 + U32) * (dy.double() * uy).abs().sum()
    terms, _ = picked(y, place)
    slack = ((dout.double()[:, None] * terms).abs().sum(-1) * ug.abs()).sum() * d * U32
    assert abs(by_g - (dg.double() * ug).sum()) <= 1e-9 + slack


def test_no_tokens_write_nothing(P):
    y = torch.ones((4, 64), dtype=torch.bfloat16, device="cuda")
    none = torch.empty((0, 2), dtype=torch.int32, device="cuda")
    assert P.sum_choices(y, none).shape == (0, 64)
    dy, dg = P.sum_choices_grad(torch.empty((0, 64), dtype=torch.bfloat16, device="cuda"), none,
                                y=y, dy=y)
    assert (dy == 1).all() and dg.shape == (0, 2)
