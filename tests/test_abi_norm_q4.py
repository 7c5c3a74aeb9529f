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
