"""What MoeLayer.prompt refuses, before anything is launched, on stand-ins for CUDA tensors."""
import pytest

torch = pytest.importorskip("torch")

B, F, U = torch.bfloat16, torch.float32, torch.uint8


class OnGpu:
    """A CPU tensor that says it lies on CUDA device `dev`."""

    def __init__(self, t, dev=0):
        self._t, self._dev = t, dev

    is_cuda = True
    device = property(lambda self: torch.device("cuda", self._dev))

    def get_device(self):
        return self._dev

    def __getattr__(self, name):
        return getattr(self._t, name)


class NoLaunches:
    """The library, but for what launches."""

    def __init__(self, lib):
        self._lib = lib

    def __getattr__(self, name):
        assert name in ("crc_moe_workspace_bytes", "crc_strerror"), name
        return getattr(self._lib, name)


def new(*shape, dtype=B, dev=0):
    return OnGpu(torch.zeros(shape).to(dtype), dev)


@pytest.fixture
def layer(monkeypatch):
    from paper_2609_04895_gb300 import build
    build.build()
    import paper_2609_04895_gb300 as P
    monkeypatch.setattr(P.crc, "_lib", NoLaunches(P.crc.load()))
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda dev: 0, raising=False)
    return P.MoeLayer(new(16, 2, 32, 64), new(16, 64, 32), K=2)


GOOD = dict(x=new(6, 64), topk=new(6, 2, dtype=U), gates=new(6, 2, dtype=F), out=new(6, 64))


@pytest.mark.parametrize("bad", [
    dict(topk=new(5, 2, dtype=U)),          # of fewer tokens than x: a result of five rows
    dict(topk=new(7, 2, dtype=U)),          # of more: rows outside x
    dict(topk=new(12, dtype=U)), dict(topk=new(6, 2, dtype=torch.int64)),
    dict(topk=new(6, 2, dtype=U, dev=1)), dict(x=new(6, 56)), dict(x=new(6, 64, dtype=F)),
    dict(x=new(64)), dict(x=new(6, 64, dev=1)), dict(gates=new(6, 3, dtype=F)),
    dict(gates=new(5, 2, dtype=F)), dict(gates=new(6, 2)), dict(out=new(5, 64)),
    dict(out=new(6, 64, dtype=F)), dict(out=new(6, 64, dev=1)), dict(pieces=0), dict(pieces=3),
])
def test_prompt_refuses_what_does_not_fit(layer, bad):
    with pytest.raises(ValueError):
        layer.prompt(**dict(GOOD, **bad))


def test_prompt_refuses_a_slot_map(layer):
    import paper_2609_04895_gb300 as P
    mapped = P.MoeLayer(*layer.tensors[:2], K=2, N=16, expert_slot=new(16, dtype=torch.int32))
    with pytest.raises(ValueError):
        mapped.prompt(**GOOD)
