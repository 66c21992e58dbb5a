"""Host-only checks of rows in two 8-bit pieces: what the C entries and the binding refuse
(nothing is launched here)."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

EINVAL, EUNSUPPORTED = 1, 2
B, F, I, E4 = torch.bfloat16, torch.float32, torch.int32, torch.float8_e4m3fn


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
    def __init__(self, lib):
        self._lib, self.calls = lib, []

    def __getattr__(self, name):
        if name in ("crc_split_rows", "crc_group_matmul_split", "crc_group_matmul"):
            return lambda *a: self.calls.append((name, a)) or 0
        return getattr(self._lib, name)


@pytest.fixture(scope="module")
def C():
    from paper_2609_04895_gb300 import build
    build.build()
    from paper_2609_04895_gb300 import crc
    crc.load()
    return crc


@pytest.fixture
def P(monkeypatch, C):
    import paper_2609_04895_gb300 as P
    rec = Recorder(C.load())
    monkeypatch.setattr(C, "_lib", rec)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda dev: 0, raising=False)
    P.calls = rec.calls
    return P


def new(*shape, dtype=B, dev=0):
    return OnGpu(torch.zeros(shape).to(dtype), dev)


def split(C, x=256, ldx=64, M=4, d=64, q=512, s=1024):
    return C.load().crc_split_rows(x, ldx, M, d, q, s, None)


@pytest.mark.parametrize("bad,code", [
    (dict(M=-1), EINVAL), (dict(d=0), EINVAL), (dict(d=60), EUNSUPPORTED),
    (dict(d=32776, ldx=32776), EUNSUPPORTED), (dict(ldx=56), EINVAL), (dict(ldx=68), EINVAL),
    (dict(x=None), EINVAL), (dict(q=None), EINVAL), (dict(s=None), EINVAL), (dict(x=264), EINVAL),
    (dict(q=516), EINVAL), (dict(s=1026), EINVAL), (dict(M=1 << 31), EUNSUPPORTED),
])
def test_split_arguments(C, bad, code):
    assert split(C, **bad) == code
    assert split(C, M=0) == 0


def weights(C, **over):
    a = dict(N=4, n=32, k=64, glu=0, weight_type=3, reserved=0, w_dev=256, w_stride=32 * 64,
             scale_dev=4, scale_stride=128)
    a.update(over)
    return C.crc_group_weights(**a)


def matmul(C, w=None, x=256, ldx=128, rows_x=8, xs=4, off=512, rows=None, K=1, E=8, y=1024):
    return C.load().crc_group_matmul_split(ctypes.byref(w or weights(C)), x, ldx, rows_x, xs, off,
                                           rows, K, E, y, None)


@pytest.mark.parametrize("bad,code", [
    (dict(ldx=64), EINVAL), (dict(ldx=120), EINVAL), (dict(ldx=136), EINVAL), (dict(xs=None), EINVAL),
    (dict(xs=2), EINVAL), (dict(x=None), EINVAL), (dict(x=264), EINVAL), (dict(rows_x=7), EINVAL),
    (dict(K=2), EINVAL), (dict(E=-1), EINVAL), (dict(off=None), EINVAL), (dict(y=1032), EINVAL),
])
def test_product_arguments(C, bad, code):
    assert matmul(C, **bad) == code
    assert matmul(C, E=0) == 0


def test_pieces_belong_to_8_bit_matrices(C):
    w = weights(C, weight_type=1, w_stride=32 * 64 * 2, scale_dev=None)
    assert matmul(C, w, xs=None) == EINVAL
    assert matmul(C, weights(C, reserved=1)) == EINVAL


def test_the_binding(P):
    x, xs = new(6, 2, 64, dtype=E4), new(6, dtype=F)
    w, ws, off, y = new(4, 32, 64, dtype=E4), new(4, 32, dtype=F), new(5, dtype=I), new(6, 32)
    P.group_matmul(x, w, off, x_scale=xs, w_scale=ws, y=y)
    name, args = P.calls[-1]
    assert name == "crc_group_matmul_split" and args[2:4] == (128, 6)
    P.group_matmul(new(6, 64, dtype=E4), w, off, x_scale=xs, w_scale=ws, y=y)
    assert P.calls[-1][0] == "crc_group_matmul"
    P.split_rows(new(6, 64), out8=x, scale=xs)
    assert P.calls[-1][0] == "crc_split_rows" and P.calls[-1][1][1:4] == (64, 6, 64)
    n = len(P.calls)
    odd = OnGpu(torch.zeros((6, 2, 128)).to(E4)[..., ::2])
    for bad in (new(6, 2, 64), new(6, 1, 64, dtype=E4), new(6, 2, 48, dtype=E4), odd,
                new(6, 2, 64, dtype=E4, dev=1), new(1, 6, 2, 64, dtype=E4)):
        with pytest.raises(ValueError):
            P.group_matmul(bad, w, off, x_scale=xs, w_scale=ws, y=y)
    with pytest.raises(ValueError):                      # bf16 matrices
        P.group_matmul(x, new(4, 32, 64), off, x_scale=xs, y=y)
    for kw in (dict(x=new(6, 64, dtype=F)), dict(x=new(64)), dict(x=new(6, 64, dev=1)),
               dict(out8=new(6, 64, dtype=E4)), dict(out8=new(6, 2, 64)), dict(scale=new(5, dtype=F)),
               dict(scale=new(6))):
        with pytest.raises(ValueError):
            P.split_rows(**dict(dict(x=new(6, 64), out8=x, scale=xs), **kw))
    assert len(P.calls) == n
