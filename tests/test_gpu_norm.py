"""Norms (rms_norm_forward, _e4m3, _backward) against their fp64 forms.

Tolerances, element by element.  A result is rounded once, by at most half a
step: 2^-8 of it in bf16, 2^-24 in fp32, and in e4m3 2^-4 of it or 2^-10 of the
row's scale.  Behind it stand fp32 sums of at most 128 additions on the way of
one element (a thread's own, then a tree), so the sum of squares is good to 128
* 2^-24 = 2^-17, rho to half of that plus a few roundings: 2^-17 altogether.
"""
import numpy as np
import pytest

from oracle import norm_q4 as o
from paper_2501_19090_amd import inputs

from gpu_util import from_dev, to_dev, torch_mod

pytestmark = pytest.mark.gpu

EPS = 1e-5
FP = 2.0 ** -17
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
WIDTHS = [1, 3, 8, 64, 127, 512, 1000, 2048, 2867, 4096, 8192, 8200, 16391, 33000]


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch_mod().cuda.is_available():
        pytest.skip("no GPU")


def _pifa():
    from paper_2501_19090_amd import pifa
    return pifa


def _rows(M, d, dtype, seed, scale=1.0, outliers=True):
    rng = np.random.default_rng([seed, M, d])
    x = rng.standard_normal((M, d)) * scale
    if outliers and d > 4:
        x[:, rng.integers(0, d, 2)] *= 50.0
    st, x64 = inputs.round_to(x, dtype)
    return to_dev(st), x64


def _gain(d, dtype, seed):
    st, g = inputs.round_to(1.0 + 0.3 * np.random.default_rng(seed).standard_normal((1, d)), dtype)
    return to_dev(st).reshape(d), g[0]


def _tiny(dtype):
    """Below the normal range a rounding is a fixed step."""
    return 2.0 ** -126


def _close(got, want, tol, what):
    off = np.abs(got - want) - tol
    assert np.isfinite(got).all(), what
    assert (off <= 0).all(), (what, float(off.max()), np.unravel_index(off.argmax(), off.shape))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", WIDTHS)
@pytest.mark.parametrize("M", [1, 5, 300])
def test_forward(M, d, dtype):
    pifa, torch = _pifa(), torch_mod()
    x_dev, x = _rows(M, d, dtype, 1)
    r_dev, r = _rows(M, d, dtype, 2)
    g_dev, g = _gain(d, dtype, 3)
    H, Y = torch.full_like(x_dev, float("nan")), torch.full_like(x_dev, float("nan"))
    pifa.rms_norm_forward(x_dev, g_dev, EPS, R=r_dev, H=H, Y=Y)
    torch.cuda.synchronize()
    h, y = o.rms_norm(x, g, EPS, r)
    # h = x + r is one fp32 addition ahead of its rounding
    _close(from_dev(H), h, np.abs(h) * (HALF[dtype] + 2.0 ** -24) + _tiny(dtype), "H")
    _close(from_dev(Y), y, np.abs(y) * (HALF[dtype] + FP) + _tiny(dtype), "Y")
    # neither residual nor gain
    y2 = pifa.rms_norm_forward(x_dev, None, EPS)
    torch.cuda.synchronize()
    _, y = o.rms_norm(x, None, EPS)
    _close(from_dev(y2), y, np.abs(y) * (HALF[dtype] + FP) + _tiny(dtype), "Y alone")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", WIDTHS)
@pytest.mark.parametrize("M", [1, 300])
def test_forward_e4m3(M, d, dtype):
    pifa, torch = _pifa(), torch_mod()
    x_dev, x = _rows(M, d, dtype, 4)
    r_dev, r = _rows(M, d, dtype, 5)
    g_dev, g = _gain(d, dtype, 6)
    H = torch.full_like(x_dev, float("nan"))
    Q, s = pifa.rms_norm_forward_e4m3(x_dev, g_dev, EPS, R=r_dev, H=H)
    torch.cuda.synchronize()
    h, y = o.rms_norm(x, g, EPS, r)
    want = o.e4m3_scale(y)
    s = from_dev(s)
    _close(s, want, want * FP, "scale")
    v = o.e4m3_value(Q.view(torch.uint8).cpu().numpy()) * s[:, None]
    _close(v, y, np.maximum(np.abs(y) * 2.0 ** -4, s[:, None] * 2.0 ** -10) + np.abs(y) * FP, "Q scale")
    _close(from_dev(H), h, np.abs(h) * (HALF[dtype] + 2.0 ** -24) + _tiny(dtype), "H")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", WIDTHS)
@pytest.mark.parametrize("M", [1, 7, 1100])
def test_backward(M, d, dtype):
    pifa, torch = _pifa(), torch_mod()
    if M * d > 4e6:
        M = 270  # more rows than workgroups all the same
    h_dev, h = _rows(M, d, dtype, 7)
    dy_dev, dy = _rows(M, d, dtype, 8, scale=1e-2, outliers=False)
    dr_dev, dr = _rows(M, d, dtype, 9, scale=1e-2, outliers=False)
    g_dev, g = _gain(d, dtype, 10)
    dX, dg = pifa.rms_norm_backward(h_dev, g_dev, dy_dev, EPS, dR=dr_dev)
    dX2, dg2 = pifa.rms_norm_backward(h_dev, g_dev, dy_dev, EPS, dR=dr_dev)
    torch.cuda.synchronize()
    assert torch.equal(dX, dX2) and torch.equal(dg, dg2)  # a fixed order of sums
    want, dgain = o.rms_norm_backward(h, g, dy, EPS, dr)
    p = o.rho(h, EPS)
    # each term is good to 2^-17 of it, the mean to 2^-17 of its terms' magnitudes, rho^3 to three times that
    terms = p * np.abs(g * dy) + p ** 3 * np.abs(h) * np.abs(g * dy * h).mean(1, keepdims=True) + np.abs(dr)
    _close(from_dev(dX), want, np.abs(want) * HALF[dtype] + terms * 4 * FP + _tiny(dtype), "dX")
    # a column's terms are good to 2^-16, their sum takes at most 128 additions on the way of one
    _close(from_dev(dg), dgain, np.abs(dy * h * p).sum(0) * (2 * FP + FP) + 1e-30, "dgain")
    # without gain, residual gradient, or one of the outputs
    only, none = pifa.rms_norm_backward(h_dev, None, dy_dev, EPS, need_dgain=False)
    none2, dg3 = pifa.rms_norm_backward(h_dev, g_dev, dy_dev, EPS, need_dX=False)
    torch.cuda.synchronize()
    assert none is None and none2 is None and torch.equal(dg3, dg)
    want, _ = o.rms_norm_backward(h, None, dy, EPS)
    _close(from_dev(only), want, np.abs(want) * HALF[dtype] + terms * 8 * FP + _tiny(dtype), "dX alone")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_backward_against_differences(dtype):
    """The gradient of sum(Y * dY) by central differences of the forward itself,
    in fp32 sums of its outputs: a random direction, step 2^-6."""
    pifa, torch = _pifa(), torch_mod()
    M, d = 4, 257
    rng = np.random.default_rng(11)
    h = rng.standard_normal((M, d)).astype(np.float32)
    g = (1 + 0.3 * rng.standard_normal(d)).astype(np.float32)
    dy = rng.standard_normal((M, d)).astype(np.float32)
    t = lambda a: torch.from_numpy(a).cuda().to(torch.float32)
    if dtype == "bf16":
        h, g, dy = (torch.from_numpy(a).to(torch.bfloat16).float().numpy() for a in (h, g, dy))
    cast = (lambda a: t(a).to(torch.bfloat16)) if dtype == "bf16" else t
    dX, dg = pifa.rms_norm_backward(cast(h), cast(g), cast(dy), EPS)
    dX, dg = from_dev(dX), from_dev(dg)
    v, w = rng.standard_normal((M, d)).astype(np.float32), rng.standard_normal(d).astype(np.float32)
    step = np.float32(2.0 ** -6)

    def loss(hh, gg):
        return float((pifa.rms_norm_forward(t(hh), t(gg), EPS).double() * t(dy).double()).sum())

    # the second-order remainder of a step of 2^-6 in each element: at most step^2
    # times a few times the size of the terms; fp32 outputs add 2^-24 / step of them
    size = float(np.abs(dy).sum())
    num = (loss(h + step * v, g) - loss(h - step * v, g)) / (2 * step)
    half = 2.0 ** -8 if dtype == "bf16" else 0.0
    assert abs(num - float((dX * v).sum())) <= size * (8 * step ** 2 + 2.0 ** -16) + half * float(np.abs(dX * v).sum())
    num = (loss(h, g + step * w) - loss(h, g - step * w)) / (2 * step)
    assert abs(num - float((dg * w).sum())) <= size * 2.0 ** -14  # linear in the gain


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_unaligned_rows_and_outputs_in_place(dtype):
    """Buffers that start anywhere, H over R, Y over X, dX over dY."""
    pifa, torch = _pifa(), torch_mod()
    M, d = 19, 1003
    x_dev, x = _rows(M, d, dtype, 20)
    r_dev, r = _rows(M, d, dtype, 21)
    g_dev, g = _gain(d, dtype, 22)
    h, y = o.rms_norm(x, g, EPS, r)

    def at(t, off):
        """t's values at an element offset of `off` in a larger buffer of guard values."""
        big = torch.full((t.numel() + 32,), 7.0, dtype=t.dtype, device=t.device)
        big[off:off + t.numel()] = t.reshape(-1)
        return big, big[off:off + t.numel()].view(t.shape)

    for off in (1, 3, 8):
        bx, xv = at(x_dev, off)
        br, rv = at(r_dev, off + 2)
        bg, gv = at(g_dev, off + 1)
        assert pifa.rms_norm_forward(xv, gv, EPS, R=rv, H=rv, Y=xv) is xv
        torch.cuda.synchronize()
        _close(from_dev(rv), h, np.abs(h) * (HALF[dtype] + 2.0 ** -24) + _tiny(dtype), "H over R")
        _close(from_dev(xv), y, np.abs(y) * (HALF[dtype] + FP) + _tiny(dtype), "Y over X")
        for big, o_, n in ((bx, off, M * d), (br, off + 2, M * d)):
            assert (big[:o_] == 7).all() and (big[o_ + n:] == 7).all()
        # 8-bit rows and a gradient at odd places
        qbig = torch.zeros(M * d + 32, dtype=torch.uint8, device="cuda")
        Q = qbig[off:off + M * d].view(M, d).view(torch.float8_e4m3fn)
        q0, s0 = pifa.rms_norm_forward_e4m3(x_dev, g_dev, EPS, R=r_dev)
        q1, s1 = pifa.rms_norm_forward_e4m3(x_dev, gv, EPS, R=r_dev, Q=Q)
        assert torch.equal(q0.view(torch.uint8), q1.view(torch.uint8)) and torch.equal(s0, s1)
        assert (qbig[:off] == 0).all() and (qbig[off + M * d:] == 0).all()
        d0, g0 = pifa.rms_norm_backward(x_dev, g_dev, r_dev, EPS, dR=r_dev)
        by, yv = at(r_dev, off)
        d1, g1 = pifa.rms_norm_backward(x_dev, gv, yv, EPS, dR=yv, dX=yv)
        assert d1 is yv and torch.equal(d0, d1) and torch.equal(g0, g1)
        assert (by[:off] == 7).all() and (by[off + M * d:] == 7).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_special_values_stay_in_their_rows(dtype):
    pifa, torch = _pifa(), torch_mod()
    M, d = 6, 515
    x_dev, x = _rows(M, d, dtype, 30)
    x_dev[1] = 0.0
    x_dev[2, 100] = float("nan")
    x_dev[3, 514] = float("inf")
    x_dev[4] = 1e-30  # squares vanish beside eps
    clean = torch.tensor([0, 5])
    y = pifa.rms_norm_forward(x_dev, None, EPS)
    q, s = pifa.rms_norm_forward_e4m3(x_dev, None, EPS)
    dx, dg = pifa.rms_norm_backward(x_dev, None, x_dev, EPS)
    torch.cuda.synchronize()
    assert (y[1] == 0).all() and (q[1].float() == 0).all() and float(s[1]) == o.TINY
    assert torch.isnan(y[2]).all() and torch.isnan(s[2])
    assert torch.isnan(y[3, 514]) and (y[3, :514] == 0).all() and torch.isnan(s[3])
    assert torch.isfinite(y[clean]).all() and torch.isfinite(dx[clean]).all()
    _close(from_dev(y)[4], o.rms_norm(from_dev(x_dev)[4:5], None, EPS)[1][0], np.full(d, 1e-27 * 0.01), "tiny row")
    assert torch.isnan(dg[100])
    # rows whose largest value needs a scale below the smallest one: it is held at 2^-126
    t = torch.full((1, 64), 1e-38, dtype=x_dev.dtype, device="cuda")
    q, s = pifa.rms_norm_forward_e4m3(t, None, 1.0)
    assert float(s[0]) == o.TINY and abs(float(q[0, 0]) * o.TINY - 1e-38) <= 1e-38 * 2.0 ** -4 + 2.0 ** -8 * 1e-38


def test_no_rows_and_refused_calls():
    pifa, torch = _pifa(), torch_mod()
    x = torch.randn(4, 16, device="cuda", dtype=torch.bfloat16)
    empty = torch.empty(0, 16, device="cuda", dtype=torch.bfloat16)
    assert pifa.rms_norm_forward(empty, None, EPS).shape == (0, 16)
    q, s = pifa.rms_norm_forward_e4m3(empty, None, EPS)
    assert q.shape == (0, 16) and s.numel() == 0
    dX, dg = pifa.rms_norm_backward(empty, None, empty, EPS)
    torch.cuda.synchronize()
    assert dX.numel() == 0 and (dg == 0).all()
    for eps in (0.0, -1.0, float("nan"), float("inf")):
        with pytest.raises(pifa.PifaError):
            pifa.rms_norm_forward(x, None, eps)
    with pytest.raises(pifa.PifaError):
        pifa.rms_norm_forward(x, None, EPS, H=(y := torch.empty_like(x)), Y=y)
    with pytest.raises(TypeError):
        pifa.rms_norm_forward(x, torch.ones(16, device="cuda"), EPS)  # gain of another type
    with pytest.raises(TypeError):
        pifa.rms_norm_forward(x.half(), None, EPS)
    with pytest.raises(ValueError):
        pifa.rms_norm_forward(x.t(), None, EPS)
    with pytest.raises(ValueError):
        pifa.rms_norm_forward(x, None, EPS, R=x[:3])
    with pytest.raises(ValueError):
        pifa.rms_norm_forward(x, None, EPS, R=x.cpu())
    with pytest.raises(ValueError):
        pifa.rms_norm_backward(x, None, x, EPS, dgain=torch.empty(15, device="cuda"))
    big = torch.randn(40, 16, device="cuda", dtype=torch.bfloat16)
    with pytest.raises(pifa.PifaError):
        pifa.rms_norm_backward(big, None, big, EPS, work=torch.empty(8, dtype=torch.uint8, device="cuda"))


def test_captured_and_replayed_beside_eager_work():
    """A graph of norm, 8-bit norm and gradients, replayed on new inputs with
    eager calls between, on a stream of its own."""
    pifa, torch = _pifa(), torch_mod()
    M, d = 70, 1024
    x, r, dy = (torch.randn(M, d, device="cuda").to(torch.bfloat16) for _ in range(3))
    g = torch.randn(d, device="cuda").to(torch.bfloat16)
    H, Y, dX = (torch.empty_like(x) for _ in range(3))
    Q, s = torch.empty(M, d, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(M, device="cuda")
    dg, work = torch.empty(d, device="cuda"), torch.empty(pifa.rms_norm_backward_bytes(M, d), dtype=torch.uint8, device="cuda")

    def calls(H, Y, Q, s, dX, dg, work):
        pifa.rms_norm_forward(x, g, EPS, R=r, H=H, Y=Y)
        pifa.rms_norm_forward_e4m3(x, g, EPS, R=r, Q=Q, scale=s)
        pifa.rms_norm_backward(H, g, dy, EPS, dR=r, dX=dX, dgain=dg, work=work)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        calls(H, Y, Q, s, dX, dg, work)
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            calls(H, Y, Q, s, dX, dg, work)
    for i in range(4):
        for t in (x, r, dy):
            t.copy_(torch.randn(M, d, device="cuda"))
        for t in (H, Y, dX):
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        other = [torch.empty_like(t) for t in (H, Y, Q, s, dX, dg, work)]
        calls(*other)
        torch.cuda.synchronize()
        for a, b in zip((H, Y, Q, s, dX, dg), other):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), i


@pytest.mark.parametrize("d,M", [(1, (1 << 26) + 5), (520, (1 << 21) + 3)])
def test_more_rows_than_one_launch(d, M):
    """The rows behind the first 2^21 of a call: the same values as in a call of their own."""
    pifa, torch = _pifa(), torch_mod()
    x = torch.empty(M, d, dtype=torch.bfloat16, device="cuda")
    x[:, :] = (torch.arange(M, device="cuda") % 251 + 1).to(torch.bfloat16)[:, None]
    x[:, 0] += 1
    g, _ = _gain(d, "bf16", 21)
    Y = pifa.rms_norm_forward(x, g, EPS)
    Q, s = pifa.rms_norm_forward_e4m3(x, g, EPS)
    for m in (0, (1 << 21) - 2, (1 << 21) + 1, M - 2):
        rows = x[m:m + 2].contiguous()
        assert torch.equal(Y[m:m + 2], pifa.rms_norm_forward(rows, g, EPS)), m
        q2, s2 = pifa.rms_norm_forward_e4m3(rows, g, EPS)
        assert torch.equal(Q[m:m + 2].view(torch.uint8), q2.view(torch.uint8)) and torch.equal(s[m:m + 2], s2), m
    # every row of one value of the period is the same row
    assert torch.equal(Y[:M // 251 * 251].view(-1, 251, d)[-1], Y[:251])


@pytest.mark.parametrize("as_handle", [False, True])
def test_workspace_of_a_call_on_another_stream(as_handle):
    """Gradients on a stream of their own, behind work that holds it up: memory
    that is allocated and filled on the current stream meanwhile is not the
    call's workspace."""
    pifa, torch = _pifa(), torch_mod()
    M, d = 1100, 1003
    h_dev, _ = _rows(M, d, "f32", 40)
    dy_dev, _ = _rows(M, d, "f32", 41)
    want_x, want_g = pifa.rms_norm_backward(h_dev, None, dy_dev, EPS)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    n = pifa.rms_norm_backward_bytes(M, d)
    with torch.cuda.stream(side):
        torch.cuda._sleep(50_000_000)
    dX, dg = pifa.rms_norm_backward(h_dev, None, dy_dev, EPS, stream=side.cuda_stream if as_handle else side)
    held_up = not side.query()
    others = [torch.full((n // 4,), 7.0, device="cuda") for _ in range(4)]
    torch.cuda.current_stream().synchronize()
    assert held_up
    side.synchronize()
    assert torch.equal(dg, want_g) and torch.equal(dX, want_x)
    assert all(bool((t == 7).all()) for t in others)


def test_outputs_of_calls_on_another_stream():
    """Outputs a call allocates belong to its stream: a block that the current
    stream still reads is not taken."""
    pifa, torch = _pifa(), torch_mod()
    x_dev, _ = _rows(300, 512, "bf16", 42)
    g_dev, _ = _gain(512, "bf16", 43)
    want = pifa.rms_norm_forward(x_dev, g_dev, EPS)
    wq, ws = pifa.rms_norm_forward_e4m3(x_dev, g_dev, EPS)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream, 0, torch.cuda.default_stream()):
        busy = torch.full_like(x_dev, 3.0)
        torch.cuda._sleep(20_000_000)
        kept = busy.clone()  # reads `busy` behind the sleep
        del busy
        y = pifa.rms_norm_forward(x_dev, g_dev, EPS, stream=stream)
        q, s = pifa.rms_norm_forward_e4m3(x_dev, g_dev, EPS, stream=stream)
        torch.cuda.synchronize()
        assert bool((kept == 3).all())
        assert torch.equal(y, want) and torch.equal(q.view(torch.uint8), wq.view(torch.uint8)) and torch.equal(s, ws)


@pytest.mark.parametrize("d,M", [(512, 17), (512, 16 * 256 + 1), (1024, 9), (2048, 5), (4096, 3), (4096, 517), (8192, 2)])
def test_backward_over_its_rows_keeps_a_bad_value_in_its_column(d, M):
    """dX over H, rows of whole chunks and a last group of rows that is cut: a
    NaN in the last row's dR is that element's of dX, one in its dY that row's of
    dX and that column's of dgain; neither is another column's."""
    pifa, torch = _pifa(), torch_mod()
    h_dev, h = _rows(M, d, "bf16", 50)
    dy_dev, dy = _rows(M, d, "bf16", 51, scale=1e-2, outliers=False)
    dr_dev, dr = _rows(M, d, "bf16", 52, scale=1e-2, outliers=False)
    g_dev, g = _gain(d, "bf16", 53)
    ref_x, ref_g = pifa.rms_norm_backward(h_dev, g_dev, dy_dev, EPS, dR=dr_dev)
    bad_r, bad_y = dr_dev.clone(), dy_dev.clone()
    bad_r[M - 1, 7], bad_y[M - 1, 9] = float("nan"), float("nan")
    torch.cuda.synchronize()
    for _ in range(5):
        over = h_dev.clone()
        dX, dg = pifa.rms_norm_backward(over, g_dev, dy_dev, EPS, dR=bad_r, dX=over)
        assert dX is over and torch.equal(dg, ref_g) and torch.equal(dX[:M - 1], ref_x[:M - 1])
        assert torch.isnan(dX[M - 1, 7]) and int(torch.isnan(dX).sum()) == 1
        over = h_dev.clone()
        dX, dg = pifa.rms_norm_backward(over, g_dev, bad_y, EPS, dR=dr_dev, dX=over)
        assert torch.equal(dX[:M - 1], ref_x[:M - 1]) and torch.isnan(dX[M - 1]).all()
        assert torch.isnan(dg[9]) and int(torch.isnan(dg).sum()) == 1
        dg[9] = ref_g[9]
        assert torch.equal(dg, ref_g)


@pytest.mark.parametrize("d", [300, 1003, 2048, 8192, 16387, 33001])
def test_e4m3_rounds_the_quotient(d):
    """Q is the e4m3 value next to the fp32 quotient Y / scale, ties to even, also
    where the quotient is a midpoint of two of them.  Rows of +-1 and eps = 3 make
    the sums exact, so rms_norm_forward returns the very fp32 values that are
    divided."""
    pifa, torch = _pifa(), torch_mod()
    rng = np.random.default_rng([60, d])
    step = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()
    mid = (step[:-1] + step[1:]) / 2  # 126 midpoints
    x = torch.from_numpy(rng.choice([-1.0, 1.0], (1, d)).astype(np.float32)).cuda()
    ties = 0
    for _ in range(20):
        top = np.float32(rng.uniform(0.5, 400.0))
        g = (mid[rng.integers(0, 126, d)].astype(np.float32) * (top / np.float32(448))).astype(np.float32)
        g[rng.integers(0, d)] = top
        g_dev = torch.from_numpy(g).cuda()
        y = pifa.rms_norm_forward(x, g_dev, 3.0).cpu()
        Q, s = pifa.rms_norm_forward_e4m3(x, g_dev, 3.0)
        s = s.cpu()
        assert torch.equal(s, y.abs().amax(1) / 448)
        q = y / s[:, None]
        ties += int(np.isin(q.abs().numpy(), mid).sum())
        assert torch.equal(Q.view(torch.uint8).cpu(), q.to(torch.float8_e4m3fn).view(torch.uint8))
    assert ties > 5 * d


@pytest.mark.parametrize("d", [300, 2048, 33001])
def test_e4m3_rows_whose_values_overflow(d):
    """A value past fp32 makes the row's scale infinite; what is finite in it is 0, as the quotient is."""
    pifa, torch = _pifa(), torch_mod()
    x = torch.ones(1, d, device="cuda")
    x[0, ::2] = 1.5
    g = torch.ones(d, device="cuda")
    g[2] = 3.4e38
    g[d - 2 + d % 2 - 1] = -2.0
    Q, s = pifa.rms_norm_forward_e4m3(x, g, EPS)
    q = Q.float()[0]
    assert torch.isinf(s[0]) and torch.isnan(q[2])
    q[2] = 0
    assert (q == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [512, 1003, 33001])
def test_backward_of_rows_of_any_size(d, dtype):
    """Rows of zeros beside an eps whose rho^2 is past fp32, rows of 2^-60 and 2^40,
    and rows whose squares overflow (rho is 0 for them) under a dY that u h
    overflows with."""
    pifa, torch = _pifa(), torch_mod()
    M, eps = 40, 2.0 ** -130
    rng = np.random.default_rng([70, d])
    f = np.ones((M, 1))
    f[5], f[6], f[7], f[8], f[9] = 0.0, 2.0 ** -60, 2.0 ** 40, 2.0 ** 80, 2.0 ** 100
    st, h = inputs.round_to(rng.uniform(0.5, 1.0, (M, d)) * f, dtype)
    k = np.ones((M, 1))
    k[5], k[8], k[9] = 2.0 ** -40, 2.0 ** 50, 2.0 ** 60
    yst, dy = inputs.round_to(rng.uniform(0.25, 0.5, (M, d)) * k, dtype)
    gst, g = inputs.round_to(rng.uniform(0.5, 1.5, (1, d)), dtype)
    dX, dg = pifa.rms_norm_backward(to_dev(st), to_dev(gst).reshape(-1), to_dev(yst), eps)
    p = np.where((h * h).sum(1, keepdims=True) > 2.0 ** 128, 0.0, o.rho(h, eps))
    u = g * dy
    back = p * (p * (u * h).mean(1, keepdims=True))
    want, terms = p * (u - h * back), p * (np.abs(u) + np.abs(h * back))
    _close(from_dev(dX), want, np.abs(want) * HALF[dtype] + terms * 4 * FP + _tiny(dtype), "dX")
    _close(from_dev(dg), (dy * h * p).sum(0), np.abs(dy * h * p).sum(0) * 3 * FP, "dgain")
    assert (from_dev(dX)[[8, 9]] == 0).all()


# (type, d): whole rows of every width that has a form of its own, and ragged ones
STEADY = [("bf16", d) for d in (512, 1024, 2048, 4096, 8192, 16384, 500, 1001, 2040, 4093, 8190, 16380)] + \
         [("f32", d) for d in (256, 512, 1024, 2048, 4096, 8192, 255, 1023, 4095, 8191)]


@pytest.mark.parametrize("dtype,d", STEADY)
def test_backward_of_many_rows_a_workgroup(dtype, d):
    """Five or more passes of every workgroup over its rows, the last group of rows
    cut: the loop over two sets of registers, and its end.  fp64 on the GPU."""
    pifa, torch = _pifa(), torch_mod()
    chunks = d // (8 if dtype == "bf16" else 4)
    at_once = 16 if chunks <= 64 else 8 if chunks <= 128 else 4 if chunks <= 256 else 2 if chunks <= 512 else 1
    M = 5 * 256 * at_once + max(1, at_once * 37 - 1 if at_once > 1 else 131)
    rng = torch.Generator(device="cuda").manual_seed(d)
    tdt = torch.bfloat16 if dtype == "bf16" else torch.float32
    h, dy, dr = (torch.randn(M, d, device="cuda", generator=rng).to(tdt) for _ in range(3))
    h[:, 3] *= 50
    g = (1 + 0.3 * torch.randn(d, device="cuda", generator=rng)).to(tdt)
    dX, dg = pifa.rms_norm_backward(h, g, dy, EPS, dR=dr)
    over = h.clone()
    dX2, dg2 = pifa.rms_norm_backward(over, g, dy, EPS, dR=dr, dX=over)
    assert torch.equal(dX, dX2) and torch.equal(dg, dg2)
    h, dy, dr, g = h.double(), dy.double(), dr.double(), g.double()
    p = torch.rsqrt((h * h).mean(1, keepdim=True) + EPS)
    u = g * dy
    want = p * u - p ** 3 * h * (u * h).mean(1, keepdim=True) + dr
    terms = p * u.abs() + p ** 3 * h.abs() * (u * h).abs().mean(1, keepdim=True) + dr.abs()
    off = (dX.double() - want).abs() - want.abs() * HALF[dtype] - terms * 4 * FP
    assert torch.isfinite(dX).all() and float(off.max()) <= 0, float(off.max())
    # at most 7 rows and 16 slots of a workgroup, 16 partial sums of a slice and 16 slices: under 128 additions
    off = (dg.double() - (dy * h * p).sum(0)).abs() - 3 * FP * (dy * h * p).abs().sum(0)
    assert torch.isfinite(dg).all() and float(off.max()) <= 0, float(off.max())


def test_rows_past_2_31_elements():
    """Offsets of the last rows pass 31 bits: the values of a call of their own."""
    pifa, torch = _pifa(), torch_mod()
    M, d = (1 << 21) + 3, 1032
    rng = torch.Generator(device="cuda").manual_seed(80)
    x = torch.empty(M, d, dtype=torch.bfloat16, device="cuda")
    x.normal_(generator=rng)
    g, _ = _gain(d, "bf16", 81)
    last = slice(M - 40, M)
    H = torch.empty_like(x)
    Y = pifa.rms_norm_forward(x, g, EPS, R=x, H=H)
    h2, rows = torch.empty(40, d, dtype=torch.bfloat16, device="cuda"), x[last].clone()
    assert torch.equal(Y[last], pifa.rms_norm_forward(rows, g, EPS, R=rows, H=h2)) and torch.equal(H[last], h2)
    Q, s = pifa.rms_norm_forward_e4m3(x, g, EPS)
    q2, s2 = pifa.rms_norm_forward_e4m3(rows, g, EPS)
    assert torch.equal(Q[last].view(torch.uint8), q2.view(torch.uint8)) and torch.equal(s[last], s2)
    del Q, H
    dX, dg = pifa.rms_norm_backward(x, g, Y, EPS, dR=x)
    dX2, _ = pifa.rms_norm_backward(rows, g, Y[last].clone(), EPS, dR=rows)
    assert torch.equal(dX[last], dX2)
    want, mags = torch.zeros(d, dtype=torch.float64, device="cuda"), torch.zeros(d, dtype=torch.float64, device="cuda")
    for m in range(0, M, 1 << 17):
        h, y = x[m:m + (1 << 17)].double(), Y[m:m + (1 << 17)].double()
        t = y * h * torch.rsqrt((h * h).mean(1, keepdim=True) + EPS)
        want += t.sum(0)
        mags += t.abs().sum(0)
    # a thread adds 2^21 / 256 / 4 rows one by one: 2^11 roundings of 2^-24 of the sum so far, and those of the terms
    assert bool(((dg.double() - want).abs() <= (2.0 ** -13 + 3 * FP) * mags).all())
