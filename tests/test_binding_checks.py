"""Checks that the binding makes before the library is called, on stand-ins for CUDA
tensors (no GPU, nothing is launched)."""
import pytest

torch = pytest.importorskip("torch")


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


class Recorder:
    """The library, but for calls that launch: their arguments are kept."""

    def __init__(self, lib):
        self._lib, self.calls = lib, []

    def __getattr__(self, name):
        if name in ("crc_rms_norm", "crc_rms_norm_grad", "crc_quantize_rows", "crc_moe_layer"):
            return lambda *a: self.calls.append(a) or 0
        return getattr(self._lib, name)


@pytest.fixture
def P(monkeypatch):
    from paper_2609_04895_gb300 import build
    build.build()
    import paper_2609_04895_gb300 as P
    rec = Recorder(P.crc.load())
    monkeypatch.setattr(P.crc, "_lib", rec)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda dev: 0, raising=False)
    P.calls = rec.calls
    return P


def new(*shape, dtype=torch.bfloat16, dev=0):
    return OnGpu(torch.zeros(shape, dtype=dtype), dev)


def layer_of(P, **over):
    a = dict(gate_up=new(16, 2, 32, 64), down=new(16, 64, 32), K=2, router=new(16, 64))
    a.update(over)
    return P.MoeLayer(**a)


def call(layer, x=None, M=4, **over):
    a = dict(out=new(M, 64), workspace=new(1 << 20, dtype=torch.uint8))
    a.update(over)
    return layer(new(M, 64) if x is None else x, **a)


def scores_stride(P):
    return P.calls[-1][6]


def test_scores_keep_their_row_stride(P):
    """A row stride below N (rows that are one row, or that overlap) goes to the library,
    which refuses it; it was raised to N, past the end of the memory."""
    layer = layer_of(P)
    call(layer, scores=OnGpu(torch.zeros(4, 48)[:, :16]))
    assert scores_stride(P) == 48
    call(layer, x=new(1, 64), M=1, scores=OnGpu(torch.zeros(1, 16)))
    assert scores_stride(P) == 16
    call(layer, scores=OnGpu(torch.zeros(1, 16).expand(4, 16)))
    assert scores_stride(P) == 0
    call(layer, scores=OnGpu(torch.zeros(64).as_strided((4, 16), (8, 1))))
    assert scores_stride(P) == 8
    import ctypes
    for stride in (0, 8, 15):
        assert P.crc._lib._lib.crc_moe_layer(ctypes.byref(layer.c), 256, 64, None, None, 256, stride, 4,
                                             4096, None, None, 256, 1 << 30, None) == 1
