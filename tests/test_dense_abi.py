"""Orthogonalised updates, 8-bit rows and their inner product on the CPU: every
invalid argument becomes its status code before any GPU work, and the
workspace queries answer without a GPU."""
import ctypes
import gc
import weakref

import pytest
import torch

import paper_1408_5093_amd as cc

P = ctypes.c_void_p
INVALID, ALIGN, WORKSPACE, UNSUPPORTED = -1, -2, -3, -4


def _ns(**kw):
    d = cc.ns_desc((2, 20, 30))
    for k, v in kw.items():
        setattr(d, k, v)
    return d


@pytest.mark.parametrize("field,value,code", [
    ("batch", -1, INVALID), ("rows", 0, INVALID), ("cols", 0, INVALID), ("steps", 0, INVALID),
    ("eps", -1.0, INVALID), ("eps", float("nan"), INVALID), ("a", float("inf"), INVALID),
    ("b", float("nan"), INVALID), ("rows", (1 << 20) + 1, UNSUPPORTED),
    ("cols", (1 << 20) + 1, UNSUPPORTED), ("steps", 65, UNSUPPORTED), ("dtype", 2, UNSUPPORTED),
    ("dtype", 9, UNSUPPORTED), ("batch", 65536, UNSUPPORTED),
    ("a", 40.0, UNSUPPORTED),  # singular values grow without bound
])
def test_newton_schulz_descriptor(field, value, code):
    lib = cc.load()
    d = _ns(**{field: value})
    n = ctypes.c_size_t()
    assert lib.caffe_newton_schulz_workspace_size(ctypes.byref(d), ctypes.byref(n)) == code
    assert lib.caffe_newton_schulz(ctypes.byref(d), P(0x1000), P(0x2000), P(0x10000), 1 << 40,
                                   None) == code
    assert lib.caffe_muon_update(ctypes.byref(d), P(0x1000), P(0x2000), P(0x3000), 0.1, 0.9, 0.0,
                                 1.0, 1, P(0x10000), 1 << 40, None) == code
    assert lib.caffe_last_error() != b""


def test_newton_schulz_pointers_and_workspace():
    lib = cc.load()
    d = _ns()
    need = cc.newton_schulz_workspace_size(d)
    assert need > 0

    def call(i=0x1000, o=0x2000, ws=0x10000, n=need):
        return lib.caffe_newton_schulz(ctypes.byref(d), P(i), P(o), P(ws), n, None)

    assert call(i=None) == INVALID and call(o=None) == INVALID
    assert call(i=0x1008) == ALIGN and call(o=0x2004) == ALIGN
    assert call(ws=None) in (INVALID, WORKSPACE) and call(ws=0x10010) == ALIGN
    assert call(n=need - 1) == WORKSPACE
    n = ctypes.c_size_t()
    assert lib.caffe_newton_schulz_workspace_size(None, ctypes.byref(n)) == INVALID
    assert lib.caffe_newton_schulz_workspace_size(ctypes.byref(d), None) == INVALID


def test_muon_update_arguments():
    lib = cc.load()
    d = _ns()
    need = cc.newton_schulz_workspace_size(d)
    nan = float("nan")

    def call(w=0x1000, g=0x2000, v=0x3000, lr=0.1, mu=0.9, wd=0.0, sc=1.0, nest=1, n=need, d=d):
        return lib.caffe_muon_update(ctypes.byref(d), P(w), P(g), P(v), lr, mu, wd, sc, nest,
                                     P(0x10000), n, None)

    for kw in (dict(lr=nan), dict(mu=nan), dict(wd=nan), dict(sc=nan), dict(nest=2),
               dict(w=None), dict(g=None), dict(v=None), dict(w=0x2000), dict(v=0x2000),
               dict(v=0x1000)):
        assert call(**kw) == INVALID, kw
    assert call(w=0x1004) == ALIGN and call(n=need - 1) == WORKSPACE
    assert call(d=_ns(dtype=cc.CAFFE_BF16)) == UNSUPPORTED

    def dev(lr):
        return lib.caffe_muon_update_device_lr(ctypes.byref(d), P(0x1000), P(0x2000), P(0x3000),
                                               P(lr), 0.9, 0.0, 1.0, 1, P(0x10000), 0, None)

    assert dev(None) == INVALID and dev(0x1002) == ALIGN and dev(0x1004) == WORKSPACE


def test_empty_batches_need_no_gpu():
    lib = cc.load()
    d = _ns(batch=0)
    assert lib.caffe_newton_schulz(ctypes.byref(d), None, None, P(0x10000), 1 << 30, None) == 0
    assert lib.caffe_quantize_rows(None, 0, 0, 10, None, None, None) == 0
    d = cc.Ip8Desc(0, 10, 5, 0, cc.CAFFE_F32, cc.CAFFE_F32)
    assert lib.caffe_inner_product_int8(ctypes.byref(d), None, None, None, None, None, None, None,
                                        0, None) == 0


def test_coefficients_that_stay_in_range():
    for coef, steps in (((1.5, -0.5, 0.0), 30), ((3.4445, -4.7750, 2.0315), 10),
                        ((15 / 8, -10 / 8, 3 / 8), 20), ((1.0, 0.0, 0.0), 64)):
        assert cc.newton_schulz_workspace_size(cc.ns_desc((64, 64), steps, coef)) > 0
    for coef, steps in (((2.0, 0.0, 0.0), 20), ((3.0, 5.0, 1.0), 5)):
        with pytest.raises(cc.CaffeError, match="range"):
            cc.newton_schulz_workspace_size(cc.ns_desc((64, 64), steps, coef))


def test_ns_desc_shapes():
    d = cc.ns_desc((384, 192, 3, 3), group=2)
    assert (d.batch, d.rows, d.cols) == (2, 192, 1728)
    d = cc.ns_desc((5, 7, 9))
    assert (d.batch, d.rows, d.cols) == (5, 7, 9)
    for shape, g in (((5,), 1), ((4, 3, 2), 2), ((5, 4), 2), ((5, 4), 0)):
        with pytest.raises(ValueError):
            cc.ns_desc(shape, group=g)


def test_int8_pitch():
    lib = cc.load()
    for cols, pitch in ((1, 128), (128, 128), (129, 256), (9216, 9216), (1 << 17, 1 << 17)):
        assert cc.int8_pitch(cols) == pitch
    for cols in (0, -5, (1 << 17) + 1):
        assert lib.caffe_int8_pitch(cols) == 0
        with pytest.raises(ValueError):
            cc.int8_pitch(cols)


@pytest.mark.parametrize("args,code", [
    ((0x1000, 0, -1, 10, 0x2000, 0x3000), INVALID), ((0x1000, 0, 3, 0, 0x2000, 0x3000), INVALID),
    ((0x1000, 2, 3, 10, 0x2000, 0x3000), UNSUPPORTED),
    ((0x1000, 0, 3, (1 << 17) + 1, 0x2000, 0x3000), UNSUPPORTED),
    ((0x1000, 0, 1 << 31, 10, 0x2000, 0x3000), UNSUPPORTED),
    ((None, 0, 3, 10, 0x2000, 0x3000), INVALID), ((0x1000, 0, 3, 10, None, 0x3000), INVALID),
    ((0x1000, 0, 3, 10, 0x2000, None), INVALID), ((0x1004, 0, 3, 10, 0x2000, 0x3000), ALIGN),
    ((0x1000, 0, 3, 10, 0x2008, 0x3000), ALIGN), ((0x1000, 0, 3, 10, 0x2000, 0x3004), ALIGN),
])
def test_quantize_rows_arguments(args, code):
    x, dt, rows, cols, q, s = args
    assert cc.load().caffe_quantize_rows(P(x), dt, rows, cols, P(q), P(s), None) == code


def _ip8(**kw):
    d = cc.Ip8Desc(3, 100, 7, 0, cc.CAFFE_F32, cc.CAFFE_F32)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


@pytest.mark.parametrize("field,value,code", [
    ("N", -1, INVALID), ("C", 0, INVALID), ("K", 0, INVALID), ("relu", 2, INVALID),
    ("bottom_type", 2, UNSUPPORTED), ("top_type", 16, UNSUPPORTED),
    ("C", (1 << 17) + 1, UNSUPPORTED), ("N", 1 << 30, UNSUPPORTED),
    ("N", (1 << 26) + 1, UNSUPPORTED), ("K", (1 << 26) + 1, UNSUPPORTED), ("N", 1 << 16, UNSUPPORTED),
])
def test_inner_product_int8_descriptor(field, value, code):
    lib = cc.load()
    d = _ip8(**{field: value})
    if field == "N" and value > 0:
        d.K = 1 << 20
    n = ctypes.c_size_t()
    assert lib.caffe_inner_product_int8_workspace_size(ctypes.byref(d), ctypes.byref(n)) == code
    assert lib.caffe_inner_product_int8(ctypes.byref(d), P(0x1000), None, P(0x2000), P(0x3000),
                                        None, P(0x4000), P(0x10000), 1 << 40, None) == code


def test_inner_product_int8_pointers():
    lib = cc.load()

    def call(d=None, x=0x1000, xs=None, w=0x2000, t=0x3000, b=None, top=0x4000, ws=0x10000, n=1 << 20):
        return lib.caffe_inner_product_int8(ctypes.byref(d or _ip8()), P(x), P(xs), P(w), P(t),
                                            P(b), P(top), P(ws), n, None)

    for kw in (dict(x=None), dict(w=None), dict(t=None), dict(top=None), dict(xs=0x5000),
               dict(d=_ip8(bottom_type=cc.CAFFE_INT8_ROWS))):
        assert call(**kw) == INVALID, kw
    for kw in (dict(x=0x1004), dict(w=0x2008), dict(t=0x3004), dict(b=0x5004), dict(top=0x4008),
               dict(ws=0x10080)):
        assert call(**kw) == ALIGN, kw
    assert call(n=3 * 128 + 11) == WORKSPACE
    n = ctypes.c_size_t()
    d = _ip8(bottom_type=cc.CAFFE_INT8_ROWS)
    assert lib.caffe_inner_product_int8_workspace_size(ctypes.byref(d), ctypes.byref(n)) == 0
    assert n.value == 0


def test_host_tensors_and_shapes_are_refused():
    x = torch.zeros(4, 8)
    for f in (lambda: cc.newton_schulz(x), lambda: cc.muon_update(x, x.clone(), x.clone(), 0.1),
              lambda: cc.quantize_rows(x), lambda: cc.newton_schulz(x.double()),
              lambda: cc.quantize_rows(x.half()),
              lambda: cc.inner_product_int8(x, torch.zeros(3, 128, dtype=torch.int8),
                                            torch.zeros(3))):
        with pytest.raises(ValueError):
            f()


def test_streams_of_another_device_are_refused():
    class Other:
        device_index, cuda_stream = 1, 0x1000

    x = torch.zeros(4, 8)
    q, t = torch.zeros(3, 128, dtype=torch.int8), torch.zeros(3)
    for f in (lambda s: cc.newton_schulz(x, stream=s), lambda s: cc.quantize_rows(x, stream=s),
              lambda s: cc.muon_update(x, x.clone(), x.clone(), 0.1, stream=s),
              lambda s: cc.inner_product_int8(x, q, t, stream=s)):
        with pytest.raises(ValueError, match="stream"):
            f(Other())


def test_blobs_that_overlap_in_part():
    """2 x 20 x 30 floats are 4800 bytes (0x12C0)."""
    lib = cc.load()
    d = _ns()
    need = cc.newton_schulz_workspace_size(d)
    for i, o in ((0x8000, 0x8010), (0x8010, 0x8000), (0x8000, 0x92B0), (0x92B0, 0x8000)):
        assert lib.caffe_newton_schulz(ctypes.byref(d), P(i), P(o), P(0x10000), need,
                                       None) == INVALID, (i, o)
    far = 0x80000
    for w, g, v in ((0x8000, 0x92B0, far), (0x8000, far, 0x8010), (far, 0x92B0, 0x8000)):
        assert lib.caffe_muon_update(ctypes.byref(d), P(w), P(g), P(v), 0.1, 0.9, 0.0, 1.0, 1,
                                     P(0x10000), need, None) == INVALID, (w, g, v)


def test_range_of_coefficients_with_a_vanishing_third():
    """t (90 - 90 t)^2 has its largest value, 1200, inside [0, 1]: refused however
    small the coefficient of t^2 is."""
    for c in (0.0, 1e-17, -1e-17, 1e-30, 1e-9):
        with pytest.raises(cc.CaffeError, match="range"):
            cc.newton_schulz_workspace_size(cc.ns_desc((64, 64), 1, (90.0, -90.0, c)))
    # 5 c t^2 + 3 b t + a with b = 0: its root is a range's end or outside
    for coef in ((1.0, 0.0, -1.0), (0.5, 0.0, 0.25), (0.0, 1.0, 0.0), (0.0, 0.0, 1.0)):
        assert cc.newton_schulz_workspace_size(cc.ns_desc((64, 64), 3, coef)) > 0


class _Buffer:
    """A device buffer that notes the streams it is recorded on."""

    def __init__(self, n):
        self.n, self.streams = n, []

    def numel(self):
        return self.n

    def get_device(self):
        return 0

    def record_stream(self, s):
        self.streams.append(s)


@pytest.fixture
def fake_device(monkeypatch):
    """(state, buffers): state holds the current raw stream and whether it captures."""
    state, made = dict(raw=1, capturing=False), []

    def empty(n, **kw):
        made.append(_Buffer(n))
        return made[-1]

    monkeypatch.setattr(torch, "empty", empty)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda i: state["raw"])
    monkeypatch.setattr(torch.cuda, "current_stream", lambda i=None: state["raw"])
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: state["capturing"])
    return state, made


def test_workspace_is_recorded_on_the_streams_that_take_it(fake_device):
    """A buffer that a larger one replaces was recorded on every stream but its own
    that got it, once each: its memory waits for them."""
    state, made = fake_device
    ws = cc.Workspace()
    for raw, n in ((1, 10), (2, 10), (1, 5), (2, 10), (3, 7), (2, 100), (1, 100), (1, 1000)):
        state["raw"] = raw
        assert ws.get(n).numel() >= n
    assert ws.get(0) is None
    assert [b.n for b in made] == [10, 100, 1000]
    assert [b.streams for b in made] == [[2, 3], [1], []]


def test_workspace_keeps_what_a_graph_writes(fake_device):
    """A buffer that a capture took outlives its replacement, others do not."""
    state, made = fake_device
    ws = cc.Workspace()
    ws.get(10)
    ws.get(20)  # (the 10 bytes are dropped)
    state["capturing"] = True
    ws.get(15)
    state["capturing"] = False
    ws.get(20), ws.get(30), ws.get(40)
    state["capturing"] = True
    ws.get(50)  # made under capture
    state["capturing"] = False
    ws.get(60), ws.get(70)
    refs = [weakref.ref(b) for b in made]
    made.clear()
    gc.collect()
    assert [r().n for r in refs if r() is not None] == [20, 50, 70] and ws.buf.n == 70


def test_8_bit_rows_that_overlap_their_input():
    """3 x 100 floats are 1200 (0x4B0) bytes, their rows 384 (0x180), the scales 12."""
    lib = cc.load()

    def rows(x, q, s):
        return lib.caffe_quantize_rows(P(x), 0, 3, 100, P(q), P(s), None)

    far = 0x80000
    for x, q, s in ((0x8000, 0x8000, far), (0x8000, 0x84A0, far), (0x8170, 0x8000, far),
                    (0x8000, far, 0x8000), (0x8000, far, 0x84A0), (0x8000, far, far),
                    (0x8000, far, far + 0x170)):
        assert rows(x, q, s) == INVALID, (hex(x), hex(q), hex(s))
        assert b"overlap" in lib.caffe_last_error()


def test_top_that_overlaps_an_input():
    """N = 3, C = 100, K = 7: 1200 bytes of bottom (384 in 8 bits, 12 of scales), 896 of
    weights, 28 of their scales and of bias, 84 of top."""
    lib = cc.load()
    far = [0x100000 * i for i in range(1, 8)]

    def call(bottom_type=cc.CAFFE_F32, **kw):
        a = dict(zip(("x", "w", "t", "b", "top", "ws", "xs"), far))
        a.update(kw)
        if bottom_type != cc.CAFFE_INT8_ROWS:
            a["xs"] = None
        d = _ip8(bottom_type=bottom_type)
        return lib.caffe_inner_product_int8(ctypes.byref(d), P(a["x"]), P(a["xs"]), P(a["w"]),
                                            P(a["t"]), P(a["b"]), P(a["top"]), P(a["ws"]),
                                            1 << 20, None)

    top = far[4]
    for kind, name, size in ((cc.CAFFE_F32, "x", 1200), (cc.CAFFE_BF16, "x", 600),
                             (cc.CAFFE_INT8_ROWS, "x", 384), (cc.CAFFE_INT8_ROWS, "xs", 12),
                             (cc.CAFFE_F32, "w", 896), (cc.CAFFE_F32, "t", 28),
                             (cc.CAFFE_F32, "b", 28)):
        for at in (top, top + 80, top - (size - 1) // 16 * 16):
            assert call(kind, **{name: at}) == INVALID, (name, at - top)
            assert b"top must not overlap" in lib.caffe_last_error()
