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
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
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


def row_calls(P):
    """name -> (call(**changed arguments), its tensor arguments)."""
    f32, f8 = torch.float32, torch.float8_e4m3fn
    M, d = 4, 64
    norm = dict(x=new(M, d), weight=new(d), residual=new(M, d), residual_out=new(M, d),
                out=new(M, d), out8=new(M, d, dtype=f8), scale8=new(M, dtype=f32),
                rstd=new(M, dtype=f32))
    grad = dict(dy=new(M, d), s=new(M, d), weight=new(d), rstd=new(M, dtype=f32), dres=new(M, d),
                dx=new(M, d), dw=new(d, dtype=f32), workspace=new(1 << 16, dtype=torch.uint8))
    quantize = dict(x=new(M, d), out8=new(M, d, dtype=f8), scale=new(M, dtype=f32))
    w8 = dict(gate_up=new(16, 2, 32, 64, dtype=f8), down=new(16, 64, 32, dtype=f8),
              gate_up_scale=new(16, 2, 32, dtype=f32), down_scale=new(16, 64, dtype=f32))
    layer = layer_of(P, **w8)
    moe = dict(x=new(M, d), out=new(M, d), x8=new(M, d, dtype=f8), x_scale=new(M, dtype=f32),
               scores=new(M, 16, dtype=f32), topk=new(M, 2, dtype=torch.uint8),
               gates=new(M, 2, dtype=f32), workspace=new(1 << 20, dtype=torch.uint8))
    made = dict(w8, router=new(16, 64), expert_slot=new(16, dtype=torch.int32))
    return {"rms_norm": (P.rms_norm, norm), "rms_norm_grad": (P.rms_norm_grad, grad),
            "quantize_rows": (P.quantize_rows, quantize), "layer": (layer, moe),
            "MoeLayer": (lambda **a: P.MoeLayer(K=2, **a), made)}


NAMES = ["rms_norm", "rms_norm_grad", "quantize_rows", "layer", "MoeLayer"]


@pytest.mark.parametrize("name", NAMES)
def test_every_tensor_lies_on_one_device(P, name):
    """The launch goes to the current device: a tensor of another GPU, or of the host, is
    refused, whichever argument it is."""
    call_it, args = row_calls(P)[name]
    call_it(**args)
    n = len(P.calls)
    for arg, t in args.items():
        with pytest.raises(ValueError):
            call_it(**dict(args, **{arg: OnGpu(t._t, 1)}))
        with pytest.raises(ValueError):
            call_it(**dict(args, **{arg: t._t}))
    assert len(P.calls) == n


@pytest.mark.parametrize("name", NAMES[:4])
def test_tensors_of_a_device_that_is_not_current(P, name, monkeypatch):
    call_it, args = row_calls(P)[name]
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1)
    n = len(P.calls)
    with pytest.raises(ValueError):
        call_it(**args)
    if name != "layer":
        call_it(**{k: OnGpu(t._t, 1) for k, t in args.items()})
        assert len(P.calls) == n + 1
    else:                                     # its experts lie on device 0
        with pytest.raises(ValueError):
            call_it(**{k: OnGpu(t._t, 1) for k, t in args.items()})


@pytest.mark.parametrize("name", ["rms_norm_grad", "layer"])
def test_a_workspace_is_as_long_as_it_says(P, name):
    """The bytes of an expanded tensor are not all there."""
    call_it, args = row_calls(P)[name]
    for t in (torch.zeros(1, dtype=torch.uint8).expand(1 << 20),
              torch.zeros(1 << 21, dtype=torch.uint8)[::2]):
        with pytest.raises(ValueError):
            call_it(**dict(args, workspace=OnGpu(t)))
    call_it(**dict(args, workspace=OnGpu(torch.zeros((512, 512)))))
    assert 1 << 20 in P.calls[-1]
