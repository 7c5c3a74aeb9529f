"""Argument errors of the norms and 4-bit layers, found before any device work."""
import ctypes

import pytest

from paper_2501_19090_amd import pifa

FAKE = ctypes.c_void_p(0x1000)  # never dereferenced: validation fails first
INVAL, UNSUP = pifa.PIFA_ERR_INVALID_ARG, pifa.PIFA_ERR_UNSUPPORTED
BF16, F32 = pifa.PIFA_BF16, pifa.PIFA_F32


def test_norm_rejects_bad_args():
    f = pifa.lib().rms_norm_forward
    ok = dict(X=FAKE, R=None, gain=None, eps=1e-5, H=None, Y=FAKE, M=4, d=8, dtype=BF16, stream=None)

    def call(**kw):
        return f(*{**ok, **kw}.values())

    assert call(X=None) == INVAL and call(Y=None) == INVAL and call(M=-1) == INVAL and call(d=0) == INVAL
    assert call(dtype=5) == INVAL and call(H=FAKE) == INVAL  # H and Y may not be one buffer
    for eps in (0.0, -1e-5, float("inf"), float("nan")):
        assert call(eps=eps) == INVAL
    assert call(d=1 << 31) == UNSUP and call(M=1 << 31) == UNSUP
    assert call(M=0) == pifa.PIFA_OK and call(M=0, X=None, Y=None) == pifa.PIFA_OK
    g = pifa.lib().rms_norm_forward_e4m3
    assert g(FAKE, None, None, 1e-5, None, None, FAKE, 4, 8, BF16, None) == INVAL
    assert g(FAKE, None, None, 1e-5, None, FAKE, None, 4, 8, BF16, None) == INVAL
    assert g(None, None, None, 1e-5, None, FAKE, FAKE, 4, 8, F32, None) == INVAL
    assert g(FAKE, None, None, 0.0, None, FAKE, FAKE, 4, 8, F32, None) == INVAL
    assert g(None, None, None, 1e-5, None, None, None, 0, 8, F32, None) == pifa.PIFA_OK


def test_norm_backward_rejects_bad_args():
    f = pifa.lib().rms_norm_backward
    ok = dict(H=FAKE, gain=None, dY=FAKE, dR=None, eps=1e-5, dX=FAKE, dgain=FAKE, M=4, d=8, dtype=BF16, work=None,
              work_bytes=0, stream=None)

    def call(**kw):
        return f(*{**ok, **kw}.values())

    assert call(H=None) == INVAL and call(dY=None) == INVAL and call(M=-1) == INVAL and call(d=0) == INVAL
    assert call(eps=0.0) == INVAL and call(dtype=-1) == INVAL and call(d=1 << 31) == UNSUP
    assert call(dX=None, dgain=None) == pifa.PIFA_OK  # nothing asked
    need = pifa.rms_norm_backward_bytes(4096, 4096)
    assert need > 0 and call(M=4096, d=4096, work=None, work_bytes=need) == INVAL
    assert call(M=4096, d=4096, work=FAKE, work_bytes=need - 1) == INVAL


def test_norm_backward_workspace_holds_partial_sums():
    size = pifa.rms_norm_backward_bytes
    assert size(0, 8) == 0 and size(4, 0) == 0 and size(-1, 8) == 0 and size(1 << 31, 8) == 0
    assert size(1, 4096) == 0  # one row: no partial sums
    for d in (1, 100, 4096, 8192, 40000):
        last = 0
        for M in (1, 2, 16, 17, 300, 4096, 1 << 20):
            n = size(M, d)
            assert n % (4 * d) == 0 and n <= 256 * 4 * d and n >= last
            last = n


def test_q4_rejects_bad_args():
    lib = pifa.lib()
    out = ctypes.c_void_p()
    ref = ctypes.byref(out)
    for d_in, d_out, want in ((0, 4, INVAL), (32, 0, INVAL), (-32, 4, INVAL), (40, 4, UNSUP), (8, 4, UNSUP),
                              ((1 << 21) + 32, 4, UNSUP), (32, 1 << 31, UNSUP)):
        assert lib.q4_layer_create(FAKE, d_in, d_out, BF16, ref) == want
        assert lib.q4_layer_create_mx(FAKE, FAKE, d_in, d_out, ref) == want
    assert lib.q4_layer_create(None, 32, 4, BF16, ref) == INVAL
    assert lib.q4_layer_create(FAKE, 32, 4, 9, ref) == INVAL
    assert lib.q4_layer_create(FAKE, 32, 4, BF16, None) == INVAL
    assert lib.q4_layer_create_mx(None, FAKE, 32, 4, ref) == INVAL
    assert lib.q4_layer_create_mx(FAKE, None, 32, 4, ref) == INVAL
    assert lib.q4_layer_create_mx(FAKE, FAKE, 32, 4, None) == INVAL
    assert out.value is None
    assert lib.q4_layer_forward(None, FAKE, FAKE, 4, None) == INVAL
    assert lib.q4_layer_forward_e4m3(None, FAKE, FAKE, FAKE, 4, None) == INVAL
    assert lib.q4_layer_norm_forward(None, FAKE, None, None, 1e-5, None, FAKE, 4, None) == INVAL
    assert lib.q4_layer_read(None, FAKE, FAKE, None) == INVAL
    assert lib.q4_layer_reserve(None, 4) == INVAL
    assert lib.q4_layer_weight_bytes(None) == 0
    assert lib.q4_layer_destroy(None) == pifa.PIFA_OK


def test_binding_checks_tensors():
    torch = pytest.importorskip("torch")
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    check = pifa._ptr_of
    assert check(None, "R", torch.bfloat16, 1, 0) is None
    assert check(x, "X", torch.bfloat16, 256, -1) == x.data_ptr()
    for bad, dtype, n, dev, err in ((x, torch.float32, 256, -1, TypeError), (x, torch.bfloat16, 257, -1, ValueError),
                                    (x, torch.bfloat16, 256, 0, ValueError), (x.t(), torch.bfloat16, 256, -1, ValueError)):
        with pytest.raises(err):
            check(bad, "X", dtype, n, dev)


def test_sizes_past_a_launch_are_refused():
    """Rows and outputs whose launch would pass 2^32 threads."""
    lib, ref = pifa.lib(), ctypes.byref(ctypes.c_void_p())
    d = (1 << 27) + 1
    assert lib.rms_norm_forward(FAKE, None, None, 1e-5, None, FAKE2, 2, d, BF16, None) == UNSUP
    assert lib.rms_norm_forward_e4m3(FAKE, None, None, 1e-5, None, FAKE2, FAKE, 2, d, BF16, None) == UNSUP
    assert lib.rms_norm_backward(FAKE, None, FAKE, None, 1e-5, FAKE, FAKE, 2, d, BF16, FAKE, 1 << 62, None) == UNSUP
    assert pifa.rms_norm_backward_bytes(2, d) == 0 and pifa.rms_norm_backward_bytes(2, d - 1) == 2 * 4 * (d - 1)
    assert lib.q4_layer_create(FAKE, 32, d, BF16, ref) == UNSUP
    assert lib.q4_layer_create_mx(FAKE, FAKE, 32, d, ref) == UNSUP


FAKE2 = ctypes.c_void_p(0x2000)


def test_rows_of_a_4_bit_call():
    torch = pytest.importorskip("torch")
    rows = pifa._q4_rows
    assert rows(torch.zeros(2, 3, 64), "X", 64, None) == 6 and rows(torch.zeros(64), "X", 64, None) == 1
    assert rows(torch.zeros(0, 64), "X", 64, None) == 0 and rows(torch.zeros(7, 5), "X", 64, 2) == 2
    for shape in ((4, 96), (64, 4), (4, 32), ()):
        with pytest.raises(ValueError):
            rows(torch.zeros(shape), "X", 64, None)


@pytest.fixture
def binding(monkeypatch):
    """The binding on CPU tensors (device -1), with a library that records the calls."""
    torch = pytest.importorskip("torch")
    calls = []

    class Recorder:
        def __getattr__(self, name):
            if name == "rms_norm_backward_bytes":
                return lambda M, d: 4 * d
            return lambda *a: calls.append((name, a)) or pifa.PIFA_OK

    rt = pifa._Torch()
    rt.device, rt.raw_stream = (lambda: -1), (lambda dev: 0)
    monkeypatch.setattr(pifa, "_torch", rt)
    monkeypatch.setattr(pifa, "_lib", Recorder())
    return torch, calls


def _last(calls):
    """(M, d) of the norm call made last."""
    return calls[-1][1][6:8] if calls[-1][0] == "rms_norm_forward" else calls[-1][1][7:9]


def test_inputs_of_another_size_are_refused(binding):
    """A gain of other rows, or an R, dY or dR of other rows with enough values, is
    a mistake; an output may be a larger buffer, of rows as long."""
    torch, calls = binding
    bf = torch.bfloat16
    t = lambda *s: torch.zeros(*s, dtype=bf)
    x, g = t(6, 64), t(64)
    for kw in (dict(R=t(7, 64)), dict(R=t(12, 32)), dict(R=t(3, 128)), dict(H=t(5, 64)), dict(H=t(12, 32)),
               dict(Y=t(3, 128)), dict(Y=t(383))):
        with pytest.raises(ValueError):
            pifa.rms_norm_forward(x, g, 1e-5, **kw)
    for bad in (t(128), t(63), t(2, 64)):
        for call in (lambda: pifa.rms_norm_forward(x, bad, 1e-5), lambda: pifa.rms_norm_forward_e4m3(x, bad, 1e-5),
                     lambda: pifa.rms_norm_backward(x, bad, x, 1e-5), lambda: pifa.rms_norm_forward(x, bad, 1e-5, M=2)):
            with pytest.raises(ValueError):
                call()
    for kw in (dict(R=t(7, 64)), dict(Q=torch.zeros(12, 32).to(torch.float8_e4m3fn)), dict(scale=torch.zeros(5))):
        with pytest.raises(ValueError):
            pifa.rms_norm_forward_e4m3(x, g, 1e-5, **kw)
    for dY, kw in ((t(7, 64), {}), (t(12, 32), {}), (x, dict(dR=t(7, 64))), (x, dict(dX=t(3, 128))),
                   (x, dict(dgain=torch.zeros(63)))):
        with pytest.raises(ValueError):
            pifa.rms_norm_backward(x, g, dY, 1e-5, **kw)
    assert not calls
    # larger outputs, other leading dimensions and flat buffers are rows as well
    pifa.rms_norm_forward(x, g, 1e-5, R=t(2, 3, 64), H=t(9, 64), Y=t(400))
    assert _last(calls) == (6, 64)
    pifa.rms_norm_forward_e4m3(x, g, 1e-5, R=t(384), scale=torch.zeros(8))
    pifa.rms_norm_backward(x, g, t(384), 1e-5, dX=t(8, 64), dgain=torch.zeros(100))
    assert _last(calls) == (6, 64) and len(calls) == 3


def test_rows_of_a_norm_call(binding):
    """d given alone cuts X into rows of d, M given takes the first rows of larger buffers."""
    torch, calls = binding
    t = lambda *s: torch.zeros(*s, dtype=torch.float32)
    pifa.rms_norm_forward(t(384), t(64), 1e-5, d=64)
    assert _last(calls) == (6, 64)
    pifa.rms_norm_forward(t(6, 64), t(32), 1e-5, R=t(384), d=32)
    assert _last(calls) == (12, 32)
    pifa.rms_norm_backward(t(384), None, t(6, 64), 1e-5, d=64)
    assert _last(calls) == (6, 64)
    pifa.rms_norm_forward(t(9, 64), t(64), 1e-5, R=t(5, 64), M=4)
    assert _last(calls) == (4, 64)
    pifa.rms_norm_forward(t(1000), t(64), 1e-5, M=4, d=64)
    assert _last(calls) == (4, 64)
    n = len(calls)
    for X, kw in ((t(100), dict(d=64)), (t(9, 64), dict(M=10)), (t(()), {}), (t(384), dict(d=64, R=t(448)))):
        with pytest.raises(ValueError):
            pifa.rms_norm_forward(X, None, 1e-5, **kw)
    assert len(calls) == n


def test_sizes_of_a_4_bit_call(binding):
    torch, calls = binding
    bf, u8 = torch.bfloat16, torch.uint8
    t = lambda *s: torch.zeros(*s, dtype=bf)
    codes, scales = torch.zeros(24, 32, dtype=u8), torch.zeros(24, 2, dtype=u8)
    for bad in (torch.zeros(25, 2, dtype=u8), torch.zeros(2, 24, dtype=u8), torch.zeros(24, 4, dtype=u8)):
        with pytest.raises(ValueError):
            pifa.q4_layer_create_mx(codes, bad)
    with pytest.raises(ValueError):
        pifa.q4_layer_create(t(24, 64, 2))
    h = pifa._remember(0x5000, d_in=64, d_out=24, dt=pifa.PIFA_BF16, dev=-1)
    try:
        x, y, g = t(6, 64), t(6, 24), t(64)
        q = x.to(torch.float8_e4m3fn)
        for call in (lambda: pifa.q4_layer_forward(h, x, t(3, 48)), lambda: pifa.q4_layer_forward(h, x, t(5, 24)),
                     lambda: pifa.q4_layer_forward_e4m3(h, q, torch.zeros(5), y),
                     lambda: pifa.q4_layer_forward_e4m3(h, q, torch.zeros(6), t(3, 48)),
                     lambda: pifa.q4_layer_norm_forward(h, x, t(128), 1e-5, Y=y),
                     lambda: pifa.q4_layer_norm_forward(h, x, g, 1e-5, R=t(7, 64), Y=y),
                     lambda: pifa.q4_layer_norm_forward(h, x, g, 1e-5, H=t(3, 128), Y=y),
                     lambda: pifa.q4_layer_norm_forward(h, x, g, 1e-5, Y=t(12, 12))):
            with pytest.raises(ValueError):
                call()
        assert not calls
        pifa.q4_layer_forward(h, x, t(9, 24))
        pifa.q4_layer_forward(h, t(9, 64), y, M=6)
        pifa.q4_layer_forward_e4m3(h, q, torch.zeros(9), t(150))  # scales of a larger batch's buffer
        pifa.q4_layer_norm_forward(h, x, g, 1e-5, R=t(384), H=t(7, 64), Y=y)
        assert [c[0] for c in calls] == ["q4_layer_forward"] * 2 + ["q4_layer_forward_e4m3", "q4_layer_norm_forward"]
    finally:
        pifa._forget(h)


def _at(i):
    return ctypes.c_void_p(0x100000 + i)


@pytest.mark.parametrize("dtype,es", [(BF16, 2), (F32, 4)])
def test_norm_outputs_over_inputs_are_refused(dtype, es):
    """An output may be an input, not lie over a part of it or over anything else,
    by as little as a byte at either end."""
    lib, M, d = pifa.lib(), 5, 24
    n, row = M * d * es, d * es
    far = [_at(0x10000 * (i + 1)) for i in range(8)]
    shifts = lambda base, out, size: (_at(0x10000 * (base + 1) - out + 1), _at(0x10000 * (base + 1) + size - 1))

    def forward(X=far[0], R=far[1], gain=far[2], H=far[3], Y=far[4]):
        return lib.rms_norm_forward(X, R, gain, 1e-5, H, Y, M, d, dtype, None)

    for base, size in ((0, n), (1, n), (2, row)):
        for p in shifts(base, n, size):
            assert forward(Y=p) == INVAL and forward(H=p) == INVAL
    assert forward(Y=far[2]) == INVAL and forward(H=far[2]) == INVAL and forward(H=far[4]) == INVAL
    assert forward(H=_at(0x50000 + n - 1)) == INVAL and forward(H=far[0], Y=far[0]) == INVAL

    def e4m3(X=far[0], R=far[1], gain=far[2], H=far[3], Q=far[4], scale=far[5]):
        return lib.rms_norm_forward_e4m3(X, R, gain, 1e-5, H, Q, scale, M, d, dtype, None)

    for base, size in ((0, n), (1, n), (2, row)):
        for p in shifts(base, n, size):
            assert e4m3(H=p) == INVAL
    for base, size in ((0, n), (1, n), (2, row), (3, n)):
        assert e4m3(Q=far[base]) == INVAL and e4m3(scale=far[base]) == INVAL
        for p in shifts(base, M * d, size):
            assert e4m3(Q=p) == INVAL
        for p in shifts(base, 4 * M, size):
            assert e4m3(scale=p) == INVAL
    assert e4m3(scale=_at(0x50000 + M * d - 1)) == INVAL and e4m3(Q=_at(0x60000 + 4 * M - 1)) == INVAL

    M = 4 * 256  # with partial sums
    n, need = M * d * es, pifa.rms_norm_backward_bytes(M, d)
    assert need > 0

    far = [_at(0x1000000 * (i + 1)) for i in range(8)]
    shifts = lambda base, out, size: (_at(0x1000000 * (base + 1) - out + 1), _at(0x1000000 * (base + 1) + size - 1))
    kw = dict(H=far[0], gain=far[1], dY=far[2], dR=far[3], dX=far[4], dgain=far[5], work=far[6])

    def backward(H, gain, dY, dR, dX, dgain, work):
        return lib.rms_norm_backward(H, gain, dY, dR, 1e-5, dX, dgain, M, d, dtype, work, need, None)

    for base, size in ((0, n), (1, row), (2, n), (3, n)):
        for p in shifts(base, n, size):
            assert backward(**{**kw, "dX": p}) == INVAL
        for p in shifts(base, 4 * d, size):
            assert backward(**{**kw, "dgain": p}) == INVAL
        for p in shifts(base, need, size):
            assert backward(**{**kw, "work": p}) == INVAL
    assert backward(**{**kw, "dgain": far[4]}) == INVAL and backward(**{**kw, "work": far[4]}) == INVAL
    assert backward(**{**kw, "work": far[5]}) == INVAL and backward(**{**kw, "dX": far[1]}) == INVAL
    for i in (1, 2, 3):  # not on 4 bytes
        assert backward(**{**kw, "work": _at(0x7000000 + i)}) == UNSUP


def test_streams_of_another_device_are_refused(binding):
    torch, calls = binding

    class Stream:
        cuda_stream = 0x40

        def __init__(self, device_index):
            self.device_index = device_index

    x, y = torch.zeros(2, 64), torch.zeros(2, 64)
    pifa.rms_norm_forward(x, None, 1e-5, Y=y, stream=Stream(-1))  # the binding's device here
    pifa.rms_norm_forward(x, None, 1e-5, Y=y, stream=0x40)
    assert [c[1][-1] for c in calls] == [0x40, 0x40]
    h = pifa._remember(0x5000, d_in=64, d_out=64, dt=pifa.PIFA_BF16, dev=-1)
    try:
        for call in (lambda st: pifa.rms_norm_forward(x, None, 1e-5, Y=y, stream=st),
                     lambda st: pifa.rms_norm_backward(x, None, x, 1e-5, dX=y, need_dgain=False, stream=st),
                     lambda st: pifa.q4_layer_forward(h, x.bfloat16(), y.bfloat16(), stream=st)):
            with pytest.raises(ValueError):
                call(Stream(1))
    finally:
        pifa._forget(h)
    assert len(calls) == 2
