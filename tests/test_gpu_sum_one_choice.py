"""Sums of one choice a token: one token a team, and several for many wide ones."""
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


# on both sides of 30000 tokens and of 48 x 2^20 elements; teams of one to eight warps, ragged
@pytest.mark.parametrize("M,d", [(29999, 1680), (30000, 1672), (30000, 1680), (30007, 2048),
                                 (50001, 1008), (50331, 992), (200003, 256), (393217, 128),
                                 (400001, 8)])
@pytest.mark.parametrize("gated", [True, False])
def test_one_choice(P, M, d, gated):
    g = torch.Generator(device="cuda").manual_seed(M)
    y = torch.randn((M + 3, d), device="cuda", generator=g, dtype=torch.bfloat16)
    place = torch.randperm(M + 3, device="cuda", generator=g)[:M].to(torch.int32)[:, None]
    place = place.contiguous()
    place[torch.rand((M, 1), device="cuda", generator=g) < 0.1] = -1
    gates = torch.rand((M, 1), device="cuda", generator=g) if gated else None
    out = torch.full((M, d), 7.0, dtype=torch.bfloat16, device="cuda")
    P.sum_choices(y, place, gates=gates, out=out)
    # one product in fp32 and a rounding to bf16; without gates the value itself
    for r in range(0, M, 65536):
        p = place[r:r + 65536, 0]
        want = torch.where((p >= 0)[:, None], y[p.clamp(min=0).long()].double(), 0.0)
        if gated:
            want *= gates[r:r + 65536].double()
        bound = (U16 + U32) * want.abs() if gated else 0 * want
        assert ((out[r:r + 65536].double() - want).abs() <= bound).all()
