"""Host-only checks of the operators for prompts, training batches and 4-bit experts: what
their C entries refuse and what the binding refuses before them (nothing is launched here)."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

EINVAL, EUNSUPPORTED = 1, 2


@pytest.fixture(scope="module")
def C():
    from paper_2609_04895_gb300 import build
    build.build()
    from paper_2609_04895_gb300 import crc
    crc.load()
    return crc


def test_struct_layout(C):
    assert ctypes.sizeof(C.crc_group_weights) == 24 + 4 * 8
    assert ctypes.sizeof(C.crc_matvec4_weights) == 24 + 6 * 8
    assert len(C.KERNEL_KINDS) == 16


def choices(C, topk=16, M=4, K=2, N=16, off=256, rows=512, place=1024, ws=None, wsb=0):
    return C.load().crc_group_choices(topk, M, K, N, off, rows, place, ws, wsb, None)


@pytest.mark.parametrize("bad,code", [
    (dict(M=-1), EINVAL), (dict(K=0), EINVAL), (dict(N=0), EINVAL), (dict(N=257), EUNSUPPORTED),
    (dict(K=33), EUNSUPPORTED), (dict(M=1 << 30, K=2), EUNSUPPORTED), (dict(topk=None), EINVAL),
    (dict(off=None), EINVAL), (dict(rows=None), EINVAL), (dict(off=2), EINVAL),
    (dict(rows=514), EINVAL), (dict(place=1026), EINVAL), (dict(M=4096), EINVAL),
    (dict(M=4096, ws=128, wsb=1 << 20), EINVAL), (dict(M=4096, ws=256, wsb=64), EINVAL),
])
def test_choices_arguments(C, bad, code):
    assert choices(C, **bad) == code


def test_choices_workspace(C):
    need = C.crc_group_choices_workspace_bytes
    assert need(256, 8, 128) == 0 and need(257, 8, 128) >= 129 * 4
    assert need(-1, 8, 128) == 0 and need(4096, 8, 257) == 0
    assert need(1 << 25, 32, 256) < 1 << 20              # it does not grow with the choices


def weights(C, **over):
    a = dict(N=4, n=32, k=64, glu=0, weight_type=1, reserved=0, w_dev=256, w_stride=32 * 64 * 2,
             scale_dev=None, scale_stride=0)
    a.update(over)
    return C.crc_group_weights(**a)


W8 = dict(weight_type=3, w_stride=32 * 64, scale_dev=4, scale_stride=128)


def matmul(C, w=None, x=256, ldx=64, rows_x=8, xs=None, off=512, rows=None, K=1, E=8, y=1024):
    return C.load().crc_group_matmul(ctypes.byref(w or weights(C)), x, ldx, rows_x, xs, off, rows,
                                     K, E, y, None)


BAD_WEIGHTS = [
    (dict(N=0), EINVAL), (dict(N=257), EUNSUPPORTED), (dict(n=36), EUNSUPPORTED),
    (dict(k=60), EUNSUPPORTED), (dict(glu=2), EINVAL), (dict(glu=1, n=24), EUNSUPPORTED),
    (dict(weight_type=2), EINVAL), (dict(reserved=1), EINVAL), (dict(w_dev=None), EINVAL),
    (dict(w_dev=8), EINVAL), (dict(w_stride=32 * 64 * 2 - 16), EINVAL), (dict(scale_dev=4), EINVAL),
    (dict(w_stride=32 * 64 * 2 + 8), EINVAL), (dict(n=65544), EUNSUPPORTED),
    (dict(w_stride=1 << 40), EUNSUPPORTED), (dict(glu=1), EINVAL),
]


@pytest.mark.parametrize("bad,code", BAD_WEIGHTS + [
    (dict(W8, scale_dev=None), EINVAL), (dict(W8, scale_dev=2), EINVAL),
    (dict(W8, scale_stride=126), EINVAL), (dict(W8, scale_stride=124), EINVAL),
    (dict(W8, k=56), EUNSUPPORTED),
])
def test_weights(C, bad, code):
    assert matmul(C, weights(C, **bad)) == code
    assert matmul(C, weights(C), E=0) == 0


@pytest.mark.parametrize("bad,code", [
    (dict(x=None), EINVAL), (dict(x=264), EINVAL), (dict(ldx=56), EINVAL), (dict(ldx=68), EINVAL),
    (dict(E=-1), EINVAL), (dict(rows_x=7), EINVAL), (dict(K=2), EINVAL), (dict(K=0, rows=4), EINVAL),
    (dict(rows=6), EINVAL), (dict(off=None), EINVAL), (dict(off=514), EINVAL), (dict(y=None), EINVAL),
    (dict(y=1032), EINVAL), (dict(xs=4), EINVAL), (dict(E=(1 << 30) + 1, rows=4), EUNSUPPORTED),
    (dict(rows=4, rows_x=0, K=2), EINVAL), (dict(rows_x=1 << 31), EUNSUPPORTED),
])
def test_matmul_arguments(C, bad, code):
    assert matmul(C, **bad) == code


def test_matmul_of_8_bit_rows(C):
    w = weights(C, **W8)
    assert matmul(C, w) == EINVAL                        # no scales of the rows
    assert matmul(C, w, xs=2) == EINVAL
    assert matmul(C, w, xs=4, ldx=72) == EINVAL          # rows 16 bytes apart
    assert matmul(C, None, xs=None, E=0) == 0
    assert C.load().crc_group_matmul(None, 256, 64, 8, None, 512, None, 1, 8, 1024, None) == EINVAL


def grad(C, w=None, dy=256, x=512, ldx=64, rows_x=8, off=1024, rows=None, K=1, E=8, dx=2048,
         dw=4096, kind=2):
    return C.load().crc_group_matmul_grad(ctypes.byref(w or weights(C)), dy, x, ldx, rows_x, off,
                                          rows, K, E, dx, dw, kind, None)


@pytest.mark.parametrize("bad,code", [
    (dict(dy=None), EINVAL), (dict(dy=8), EINVAL), (dict(x=None), EINVAL), (dict(x=520), EINVAL),
    (dict(dx=2056), EINVAL), (dict(dw=4104), EINVAL), (dict(kind=3), EINVAL), (dict(kind=0), EINVAL),
    (dict(off=None), EINVAL), (dict(ldx=56), EINVAL), (dict(rows_x=4), EINVAL), (dict(E=-1), EINVAL),
    (dict(K=3), EINVAL),
])
def test_gradient_arguments(C, bad, code):
    assert grad(C, **bad) == code
    assert grad(C, dx=None, dw=None) == 0 and grad(C, E=0, dw=None, dy=None, x=None) == 0


def test_gradient_weights(C):
    for bad, code in BAD_WEIGHTS:
        assert grad(C, weights(C, **bad)) == code
    assert grad(C, weights(C, **W8)) == EINVAL
    assert grad(C, weights(C, w_dev=None), dx=None, dw=None) == 0   # read for dx only
    assert C.load().crc_group_matmul_grad(None, 256, 512, 64, 8, 1024, None, 1, 8, 2048, 4096, 2,
                                          None) == EINVAL


def total(C, y=256, n=8, place=512, gates=None, M=4, K=2, d=64, out=1024):
    return C.load().crc_sum_choices(y, n, place, gates, M, K, d, out, None)


def total_grad(C, dout=128, y=256, n=8, place=512, gates=None, M=4, K=2, d=64, dy=1024, dg=2048):
    return C.load().crc_sum_choices_grad(dout, y, n, place, gates, M, K, d, dy, dg, None)


SUM = [(dict(M=-1), EINVAL), (dict(K=0), EINVAL), (dict(K=33), EUNSUPPORTED), (dict(d=0), EINVAL),
       (dict(d=60), EUNSUPPORTED), (dict(d=32776), EUNSUPPORTED), (dict(n=-1), EINVAL),
       (dict(place=None, n=7), EINVAL), (dict(place=514), EINVAL), (dict(gates=2), EINVAL),
       (dict(y=8), EINVAL), (dict(n=(1 << 30) + 1), EUNSUPPORTED)]


@pytest.mark.parametrize("bad,code", SUM + [(dict(y=None), EINVAL), (dict(out=None), EINVAL),
                                            (dict(out=1032), EINVAL)])
def test_sum_arguments(C, bad, code):
    assert total(C, **bad) == code
    assert total(C, M=0) == 0


@pytest.mark.parametrize("bad,code", SUM + [(dict(y=None), EINVAL), (dict(dout=None), EINVAL),
                                            (dict(dout=8), EINVAL), (dict(dy=1032), EINVAL),
                                            (dict(dg=2), EINVAL)])
def test_sum_gradient_arguments(C, bad, code):
    assert total_grad(C, **bad) == code
    assert total_grad(C, M=0) == 0 and total_grad(C, dy=None, dg=None) == 0


def rows4(C, x=256, ldx=64, m=2, n=8, k=64, G=32, q=512, sc=1024):
    return C.load().crc_quantize_rows4(x, ldx, m, n, k, G, q, sc, None)


@pytest.mark.parametrize("bad,code", [
    (dict(m=-1), EINVAL), (dict(n=-1), EINVAL), (dict(k=0), EINVAL), (dict(G=16), EUNSUPPORTED),
    (dict(G=128), EUNSUPPORTED), (dict(k=32800, ldx=32800), EUNSUPPORTED), (dict(ldx=56), EINVAL),
    (dict(ldx=68), EINVAL), (dict(x=None), EINVAL), (dict(q=None), EINVAL), (dict(sc=None), EINVAL),
    (dict(x=264), EINVAL), (dict(q=520), EINVAL), (dict(sc=1032), EINVAL), (dict(m=65536), EUNSUPPORTED),
])
def test_rows4_arguments(C, bad, code):
    assert rows4(C, **bad) == code
    assert rows4(C, m=0) == 0 and rows4(C, n=0) == 0


def weights4(C, **over):
    a = dict(N=4, n=32, k=64, slots=4, glu=0, group=32, reserved=0, codes_dev=256, scale_dev=512,
             codes_stride=32 * 32, scale_stride=32 * 2 * 2, expert_slot_dev=None)
    a.update(over)
    return C.crc_matvec4_weights(**a)


def vec4(C, w=None, x=256, ldx=64, each=0, topk=16, M=4, K=2, y=1024):
    return C.load().crc_matvec4(ctypes.byref(w or weights4(C)), x, ldx, each, topk, M, K, y, None)


@pytest.mark.parametrize("bad,code", [
    (dict(N=0), EINVAL), (dict(N=257, slots=300), EUNSUPPORTED), (dict(n=36), EUNSUPPORTED),
    (dict(k=48), EUNSUPPORTED), (dict(group=16), EUNSUPPORTED), (dict(group=128), EUNSUPPORTED),
    (dict(glu=2), EINVAL), (dict(reserved=1), EINVAL), (dict(codes_dev=None), EINVAL),
    (dict(scale_dev=None), EINVAL), (dict(codes_dev=8), EINVAL), (dict(scale_dev=8), EINVAL),
    (dict(codes_stride=1008), EINVAL), (dict(codes_stride=1032), EINVAL), (dict(glu=1), EINVAL),
    (dict(scale_stride=112), EINVAL), (dict(scale_stride=136), EINVAL), (dict(slots=3), EINVAL),
    (dict(expert_slot_dev=2), EINVAL), (dict(slots=0), EINVAL), (dict(k=32800), EUNSUPPORTED),
])
def test_matvec4_weights(C, bad, code):
    assert vec4(C, weights4(C, **bad)) == code
    assert C.load().crc_matvec4(None, 256, 64, 0, 16, 4, 2, 1024, None) == EINVAL


@pytest.mark.parametrize("bad,code", [
    (dict(M=-1), EINVAL), (dict(K=0), EINVAL), (dict(K=33), EUNSUPPORTED), (dict(each=2), EINVAL),
    (dict(M=1025, K=1), EUNSUPPORTED), (dict(M=1024, K=9), EUNSUPPORTED), (dict(ldx=56), EINVAL),
    (dict(ldx=68), EINVAL), (dict(x=None), EINVAL), (dict(x=264), EINVAL), (dict(y=None), EINVAL),
    (dict(y=1032), EINVAL), (dict(topk=None), EINVAL),
])
def test_matvec4_arguments(C, bad, code):
    assert vec4(C, **bad) == code
    assert vec4(C, M=0) == 0


def test_matvec4_without_choices_takes_no_slots(C):
    assert vec4(C, weights4(C, expert_slot_dev=4), topk=None, K=1) == EINVAL


# --------------------------------------------------------------------------- #
# the binding, on stand-ins for CUDA tensors
# --------------------------------------------------------------------------- #
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

    def reshape(self, *s):
        return OnGpu(self._t.reshape(*s), self._dev)


NAMES = ("crc_group_choices", "crc_group_matmul", "crc_group_matmul_grad", "crc_sum_choices",
         "crc_sum_choices_grad", "crc_quantize_rows4", "crc_matvec4")


class Recorder:
    def __init__(self, lib):
        self._lib, self.calls = lib, []

    def __getattr__(self, name):
        if name in NAMES:
            return lambda *a: self.calls.append((name, a)) or 0
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


B, F, I, U = torch.bfloat16, torch.float32, torch.int32, torch.uint8
E4 = torch.float8_e4m3fn


def new(*shape, dtype=B, dev=0):
    return OnGpu(torch.zeros(shape).to(dtype), dev)


CALLS = {
    "group_choices": (dict(topk=new(6, 2, dtype=U), N=4, offsets=new(5, dtype=I),
                           rows=new(12, dtype=I), place=new(6, 2, dtype=I)),
                      dict(topk=new(12, dtype=U), offsets=new(4, dtype=I), rows=new(12, dtype=F),
                           place=new(12, dtype=I))),
    "group_matmul": (dict(x=new(6, 64), w=new(4, 32, 64), offsets=new(5, dtype=I), y=new(6, 32)),
                     dict(x=new(6, 56), w=new(4, 32, 64, dtype=F), offsets=new(4, dtype=I),
                          y=new(6, 64), x_scale=new(6, dtype=F), w_scale=new(4, 32, dtype=F),
                          rows=new(5, dtype=F))),
    "group_matmul_grad": (dict(dy=new(6, 32), x=new(6, 64), w=new(4, 32, 64),
                               offsets=new(5, dtype=I), dx=new(6, 64), dw=new(4, 32, 64, dtype=F)),
                          dict(dy=new(5, 32), x=new(6, 56), w=new(4, 2, 32, 64),
                               offsets=new(5, dtype=F), dx=new(6, 32), dw=new(4, 64, 32, dtype=F))),
    "sum_choices": (dict(y=new(12, 64), place=new(6, 2, dtype=I), out=new(6, 64),
                         gates=new(6, 2, dtype=F)),
                    dict(y=new(12, 64, dtype=F), place=new(6, 2, dtype=torch.int64),
                         out=new(6, 32), gates=new(6, 3, dtype=F))),
    "sum_choices_grad": (dict(dout=new(6, 64), place=new(6, 2, dtype=I), y=new(12, 64),
                              dy=new(12, 64), dgates=new(6, 2, dtype=F), gates=new(6, 2, dtype=F)),
                         dict(dout=new(6, 64, dtype=F), place=new(5, 2, dtype=I), y=new(12, 32),
                              dy=new(11, 64), dgates=new(6, 2), gates=new(2, 6, dtype=F))),
    "quantize_rows4": (dict(x=new(3, 8, 64), group=32, out4=new(3, 8, 32, dtype=U),
                            scale=new(3, 2, 8)),
                       dict(x=new(64), out4=new(3, 8, 64, dtype=U), scale=new(3, 8, 2))),
    "matvec4": (dict(x=new(5, 64), codes=new(4, 8, 32, dtype=U), scale=new(4, 2, 8),
                     topk=new(5, 2, dtype=U), expert_slot=new(4, dtype=I), y=new(5, 2, 8)),
                dict(x=new(5, 32), codes=new(4, 8, 32), scale=new(4, 2, 16),
                     topk=new(5, 2, dtype=I), expert_slot=new(4, dtype=F), y=new(5, 8))),
}


@pytest.mark.parametrize("name", CALLS)
def test_the_binding_refuses_what_does_not_fit(P, name):
    good, bad = CALLS[name]
    f = getattr(P, name)
    f(**good)
    assert P.calls[-1][0] == "crc_" + name
    n = len(P.calls)
    for k, v in bad.items():
        with pytest.raises(ValueError):
            f(**dict(good, **{k: v}))
    for k, v in good.items():                            # another device, or not contiguous
        if isinstance(v, OnGpu):
            with pytest.raises(ValueError):
                f(**dict(good, **{k: OnGpu(v._t, 1)}))
            t = v._t
            if t.dim() > 1 and k != "place":
                odd = torch.zeros((*t.shape[:-1], 2 * t.shape[-1])).to(t.dtype)[..., ::2]
                with pytest.raises(ValueError):
                    f(**dict(good, **{k: OnGpu(odd)}))
    assert len(P.calls) == n


def test_8_bit_arguments_belong_together(P):
    x, w, off = new(6, 64, dtype=E4), new(4, 32, 64, dtype=E4), new(5, dtype=I)
    xs, ws, y = new(6, dtype=F), new(4, 32, dtype=F), new(6, 32)
    P.group_matmul(x, w, off, x_scale=xs, w_scale=ws, y=y)
    for kw in (dict(x_scale=xs), dict(w_scale=ws), dict(),
               dict(x_scale=new(5, dtype=F), w_scale=ws), dict(x_scale=xs, w_scale=new(4, 31, dtype=F))):
        with pytest.raises(ValueError):
            P.group_matmul(x, w, off, y=y, **kw)
    with pytest.raises(ValueError):
        P.group_matmul(new(6, 64), w, off, w_scale=ws, x_scale=xs, y=y)


def test_strides_and_slots_reach_the_library(P):
    big = OnGpu(torch.zeros((6, 96), dtype=B)[:, :64])
    slots = torch.zeros((4, 3 * 32 * 64), dtype=B)
    w = OnGpu(slots.as_strided((4, 32, 64), (3 * 32 * 64, 64, 1)))
    P.group_matmul(big, w, new(5, dtype=I), y=new(6, 32))
    args = P.calls[-1][1]
    w = P.crc.crc_group_weights.from_buffer_copy(args[0])
    assert args[2] == 96 and w.w_stride == 3 * 32 * 64 * 2
    assert (w.N, w.n, w.k, w.glu, w.weight_type, w.scale_dev) == (4, 32, 64, 0, 1, None)
    P.matvec4(OnGpu(torch.zeros((5, 96), dtype=B)[:, :64]), new(4, 2, 8, 32, dtype=U),
              new(4, 2, 2, 8), topk=new(5, 2, dtype=U), expert_slot=new(9, dtype=I), y=new(5, 2, 8))
    args = P.calls[-1][1]
    c = P.crc.crc_matvec4_weights.from_buffer_copy(args[0])
    assert c.expert_slot_dev and c.codes_stride == 2 * 8 * 32 and c.scale_stride == 2 * 2 * 8 * 2
    assert (c.N, c.slots, c.glu, c.group, args[2], args[3]) == (9, 4, 1, 32, 96, 0)
    P.matvec4(new(5, 2, 64), new(4, 8, 32, dtype=U), new(4, 2, 8), topk=new(5, 2, dtype=U),
              y=new(5, 2, 8))
    assert P.calls[-1][1][3] == 1                        # a row for each choice


def test_unsupported_groups_are_refused(P):
    for kw in (dict(group=16), dict(group=128)):
        with pytest.raises(P.CrcError):
            P.quantize_rows4(new(8, 64), out4=new(8, 32, dtype=U), scale=new(2, 8), **kw)


def test_strides_that_say_nothing(P):
    """One expert, one slot, one group: their strides do not matter."""
    w = OnGpu(torch.zeros((32, 64), dtype=B).as_strided((1, 32, 64), (8, 64, 1)))
    P.group_matmul(new(6, 64), w, new(2, dtype=I), y=new(6, 32))
    assert P.crc.crc_group_weights.from_buffer_copy(P.calls[-1][1][0]).w_stride == 32 * 64 * 2
    codes = OnGpu(torch.zeros((8, 32), dtype=U).as_strided((1, 8, 32), (8, 32, 1)))
    scale = OnGpu(torch.zeros((8,), dtype=B).as_strided((1, 1, 8), (1, 3, 1)))
    P.matvec4(new(5, 64), codes, scale, y=new(5, 1, 8))
    c = P.crc.crc_matvec4_weights.from_buffer_copy(P.calls[-1][1][0])
    assert (c.codes_stride, c.scale_stride, c.group) == (8 * 32, 8 * 2, 64)
