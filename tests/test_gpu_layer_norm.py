"""Layer norms (layer_norm_forward, _backward) against their fp64 forms.

Tolerances, element by element.  A result is rounded once, by at most half a
step: 2^-8 of it in bf16, 2^-24 in fp32.  Behind it stand fp32 sums of at most
128 additions on the way of one element (a thread's own, then a tree), good to
128 * 2^-24 = 2^-17 =: FP of their terms' magnitudes.  So the mean is off by at
most dm = FP mean|h|; the centred values by dm beside their own rounding; the mean
of their squares by FP of it and by dm^2 (the first-order part adds up to zero);
rho by half of that relatively; hat = c rho by |hat| (FP + (rho dm)^2) + rho dm.
"""
import numpy as np
import pytest

from oracle import tune as o
from paper_2501_19090_amd import inputs

from gpu_util import from_dev, to_dev, torch_mod

pytestmark = pytest.mark.gpu

EPS = 1e-5
FP = 2.0 ** -17
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
WIDTHS = [1, 3, 8, 64, 127, 512, 1000, 2048, 2867, 4096, 8192, 8200, 16384, 16387, 16391, 33000]
TINY = 2.0 ** -126


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch_mod().cuda.is_available():
        pytest.skip("no GPU")


def _pifa():
    from paper_2501_19090_amd import pifa
    return pifa


def _rows(M, d, dtype, seed, scale=1.0, mean=0.0, outliers=True):
    rng = np.random.default_rng([seed, M, d])
    x = rng.standard_normal((M, d)) * scale + mean
    if outliers and d > 4:
        x[:, rng.integers(0, d, 2)] *= 50.0
    st, x64 = inputs.round_to(x, dtype)
    return to_dev(st), x64


def _vec(d, dtype, seed, mean=1.0):
    st, g = inputs.round_to(mean + 0.3 * np.random.default_rng(seed).standard_normal((1, d)), dtype)
    return to_dev(st).reshape(d), g[0]


def _close(got, want, tol, what):
    off = np.abs(got - want) - tol
    assert np.isfinite(got).all(), what
    assert (off <= 0).all(), (what, float(off.max()), np.unravel_index(off.argmax(), off.shape))


def _hat(h):
    """(rho, hat, bound of hat's error) of rows."""
    c = h - h.mean(1, keepdims=True)
    rho = 1.0 / np.sqrt((c * c).mean(1, keepdims=True) + EPS)
    dm = FP * np.abs(h).mean(1, keepdims=True)
    return rho, c * rho, np.abs(c * rho) * (FP + (rho * dm) ** 2) + rho * dm


def _check_forward(H, Y, x, g, b, r, dtype, what=""):
    h, y = o.layer_norm(x, g, b, EPS, r)
    if H is not None:  # h = x + r is one fp32 addition ahead of its rounding
        _close(from_dev(H), h, np.abs(h) * (HALF[dtype] + 2.0 ** -24) + TINY, what + "H")
    g = 1.0 if g is None else g
    _close(from_dev(Y), y, np.abs(y) * (HALF[dtype] + FP) + np.abs(g) * (_hat(h)[2] + FP * np.abs(_hat(h)[1])) + TINY, what + "Y")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", WIDTHS)
@pytest.mark.parametrize("M", [1, 5, 300])
def test_forward(M, d, dtype):
    pifa, torch = _pifa(), torch_mod()
    x_dev, x = _rows(M, d, dtype, 1, mean=0.5)
    r_dev, r = _rows(M, d, dtype, 2)
    g_dev, g = _vec(d, dtype, 3)
    b_dev, b = _vec(d, dtype, 4, mean=0.0)
    H, Y = torch.full_like(x_dev, float("nan")), torch.full_like(x_dev, float("nan"))
    pifa.layer_norm_forward(x_dev, g_dev, b_dev, EPS, R=r_dev, H=H, Y=Y)
    only, bias = pifa.layer_norm_forward(x_dev, g_dev, None, EPS), pifa.layer_norm_forward(x_dev, None, b_dev, EPS, R=r_dev)
    torch.cuda.synchronize()
    _check_forward(H, Y, x, g, b, r, dtype)
    _check_forward(None, only, x, g, None, None, dtype, "no bias, no residual ")
    _check_forward(None, bias, x, None, b, r, dtype, "no gain ")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [67, 4096, 20000, 50000])
def test_rows_far_from_zero(d, dtype):
    """Rows whose mean is 200 deviations away: the squares of the centred values
    count, not a difference of two large sums."""
    pifa, torch = _pifa(), torch_mod()
    x_dev, x = _rows(6, d, dtype, 5, mean=200.0, outliers=False)
    y = pifa.layer_norm_forward(x_dev, None, None, EPS)
    dy_dev, dy = _rows(6, d, dtype, 6, outliers=False)
    dX, dg, db = pifa.layer_norm_backward(x_dev, None, dy_dev, EPS)
    torch.cuda.synchronize()
    _check_forward(None, y, x, None, None, None, dtype)
    _check_backward(dX, dg, db, x, None, dy, None, dtype)


def _check_backward(dX, dg, db, h, g, dy, dr, dtype):
    want, dgain, dbias = o.layer_norm_backward(h, g, dy, EPS, dr)
    rho, hat, eh = _hat(h)
    u = dy if g is None else dy * g
    mean = lambda a: a.mean(1, keepdims=True)
    au, ahat, dm = np.abs(u), np.abs(hat), FP * np.abs(h).mean(1, keepdims=True)
    # mean(u) is off by FP mean|u|; mean(u hat) by FP of its terms (u - mean(u) has at
    # most |u| + mean|u|) and by what a shift of hat by rho dm makes of mean|u|
    back = 2 * FP * mean((au + mean(au)) * ahat) + mean(au) * rho * dm + np.abs(mean(u * hat)) * (FP + (rho * dm) ** 2)
    terms = au + mean(au) + ahat * np.abs(mean(u * hat))
    tol = rho * (2 * FP * terms + FP * mean(au) + ahat * back + eh * np.abs(mean(u * hat)) + (rho * dm) ** 2 * terms)
    if dX is not None:
        tol = tol + np.abs(want) * HALF[dtype] + (0 if dr is None else FP * np.abs(dr)) + TINY
        _close(from_dev(dX), want, tol, "dX")
    if dg is not None:
        _close(from_dev(dg), dgain, (np.abs(dy) * (eh + FP * ahat)).sum(0) + 1e-30, "dgain")
    if db is not None:
        _close(from_dev(db), dbias, FP * np.abs(dy).sum(0) + 1e-30, "dbias")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", WIDTHS)
@pytest.mark.parametrize("M", [1, 7, 1100])
def test_backward(M, d, dtype):
    pifa, torch = _pifa(), torch_mod()
    if M * d > 4e6:
        M = 270  # more rows than workgroups all the same
    h_dev, h = _rows(M, d, dtype, 7, mean=0.5)
    dy_dev, dy = _rows(M, d, dtype, 8, scale=1e-2, mean=1e-3, outliers=False)
    dr_dev, dr = _rows(M, d, dtype, 9, scale=1e-2, outliers=False)
    g_dev, g = _vec(d, dtype, 10)
    dX, dg, db = pifa.layer_norm_backward(h_dev, g_dev, dy_dev, EPS, dR=dr_dev)
    again = pifa.layer_norm_backward(h_dev, g_dev, dy_dev, EPS, dR=dr_dev)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((dX, dg, db), again))  # a fixed order of sums
    _check_backward(dX, dg, db, h, g, dy, dr, dtype)
    # without gain and residual gradient, and with one output each
    x1, g1, b1 = pifa.layer_norm_backward(h_dev, None, dy_dev, EPS, need_dgain=False, need_dbias=False)
    x2, g2, b2 = pifa.layer_norm_backward(h_dev, g_dev, dy_dev, EPS, need_dX=False, need_dbias=False)
    x3, g3, b3 = pifa.layer_norm_backward(h_dev, g_dev, dy_dev, EPS, need_dX=False, need_dgain=False)
    torch.cuda.synchronize()
    assert g1 is None and b1 is None and x2 is None and b2 is None and x3 is None and g3 is None
    assert torch.equal(g2, dg) and torch.equal(b3, db)
    _check_backward(x1, None, None, h, None, dy, None, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_backward_against_differences(dtype):
    """The gradients of sum(Y * dY) by central differences of the forward itself,
    in fp32: a random direction, step 2^-6."""
    pifa, torch = _pifa(), torch_mod()
    M, d = 4, 257
    rng = np.random.default_rng(11)
    h, dy = (rng.standard_normal((M, d)).astype(np.float32) for _ in range(2))
    g = (1 + 0.3 * rng.standard_normal(d)).astype(np.float32)
    b = rng.standard_normal(d).astype(np.float32)
    t = lambda a: torch.from_numpy(a).cuda()
    if dtype == "bf16":
        h, g, dy = (torch.from_numpy(a).to(torch.bfloat16).float().numpy() for a in (h, g, dy))
    cast = (lambda a: t(a).to(torch.bfloat16)) if dtype == "bf16" else t
    dX, dg, db = (from_dev(a) for a in pifa.layer_norm_backward(cast(h), cast(g), cast(dy), EPS))
    v = rng.standard_normal((M, d)).astype(np.float32)
    w, z = (rng.standard_normal(d).astype(np.float32) for _ in range(2))
    step = np.float32(2.0 ** -6)

    def loss(hh, gg, bb):
        return float((pifa.layer_norm_forward(t(hh), t(gg), t(bb), EPS).double() * t(dy).double()).sum())

    # the second-order remainder of a step of 2^-6 in each element: at most step^2
    # times a few times the size of the terms; fp32 outputs add 2^-24 / step of them
    size = float(np.abs(dy).sum())
    num = (loss(h + step * v, g, b) - loss(h - step * v, g, b)) / (2 * step)
    half = 2.0 ** -8 if dtype == "bf16" else 0.0
    assert abs(num - float((dX * v).sum())) <= size * (8 * step ** 2 + 2.0 ** -16) + half * float(np.abs(dX * v).sum())
    num = (loss(h, g + step * w, b) - loss(h, g - step * w, b)) / (2 * step)
    assert abs(num - float((dg * w).sum())) <= size * 2.0 ** -14  # linear in the gain
    num = (loss(h, g, b + step * z) - loss(h, g, b - step * z)) / (2 * step)
    assert abs(num - float((db * z).sum())) <= size * 2.0 ** -14  # and in the bias


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [1003, 17003, 40003])
def test_unaligned_rows_and_outputs_in_place(d, dtype):
    """Buffers that start anywhere, H over R, Y over X, dX over each of its inputs."""
    pifa, torch = _pifa(), torch_mod()
    M = 19
    x_dev, x = _rows(M, d, dtype, 20)
    r_dev, r = _rows(M, d, dtype, 21)
    g_dev, g = _vec(d, dtype, 22)
    b_dev, b = _vec(d, dtype, 23, mean=0.0)

    def at(t, off):
        """t's values at an element offset of `off` in a larger buffer of guard values."""
        big = torch.full((t.numel() + 32,), 7.0, dtype=t.dtype, device=t.device)
        big[off:off + t.numel()] = t.reshape(-1)
        return big, big[off:off + t.numel()].view(t.shape)

    whole = lambda big, off, n: bool((big[:off] == 7).all() and (big[off + n:] == 7).all())
    for off in (1, 8):
        (bx, xv), (br, rv), (_, gv), (_, bv) = at(x_dev, off), at(r_dev, off + 2), at(g_dev, off + 1), at(b_dev, off + 3)
        assert pifa.layer_norm_forward(xv, gv, bv, EPS, R=rv, H=rv, Y=xv) is xv
        torch.cuda.synchronize()
        _check_forward(rv, xv, x, g, b, r, dtype)
        assert whole(bx, off, M * d) and whole(br, off + 2, M * d)
        want = pifa.layer_norm_backward(x_dev, g_dev, r_dev, EPS, dR=x_dev)
        for i in range(3):
            bufs = [at(t, off + k) for k, t in enumerate((x_dev, r_dev, x_dev))]
            h, dy, dr = (v for _, v in bufs)
            got = pifa.layer_norm_backward(h, gv, dy, EPS, dR=dr, dX=(h, dy, dr)[i])
            torch.cuda.synchronize()
            assert all(torch.equal(a, w) for a, w in zip(got, want)), i
            assert all(whole(big, off + k, M * d) for k, (big, _) in enumerate(bufs))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [515, 40000])
def test_special_values_stay_in_their_rows(d, dtype):
    pifa, torch = _pifa(), torch_mod()
    x_dev, x = _rows(8, d, dtype, 30)
    b_dev, b = _vec(d, dtype, 31)
    x_dev[1] = 0.0
    x_dev[2, 100] = float("nan")
    x_dev[3, 514] = float("inf")
    x_dev[4] = 1e-30   # squares vanish beside eps
    x_dev[6] = 3.0     # a constant row: every centred value is zero
    x_dev[7] = torch.where(torch.arange(d, device="cuda") % 2 == 0, 1e25, -1e25)  # squares past fp32
    clean = [0, 5]
    y = pifa.layer_norm_forward(x_dev, None, b_dev, EPS)
    dx, dg, db = pifa.layer_norm_backward(x_dev, None, x_dev[[0, 1, 1, 1, 0, 5, 0, 0]].contiguous(), EPS)
    torch.cuda.synchronize()
    _check_forward(None, y[clean], from_dev(x_dev)[clean], None, b, None, dtype)
    for m in (1, 6, 7):
        assert torch.equal(y[m], b_dev), m
    assert torch.isnan(y[2]).all() and torch.isnan(y[3]).all()
    assert float((y[4].float() - b_dev.float()).abs().max()) <= 2.0 ** -8 * 3
    assert torch.isfinite(dx[[0, 1, 4, 5, 6]]).all() and (dx[7] == 0).all() and (dx[1] == 0).all()
    assert torch.isnan(dg).all() and torch.isfinite(db).all()  # a NaN row is in every column's sum


def test_no_rows_and_refused_calls():
    pifa, torch = _pifa(), torch_mod()
    x = torch.randn(4, 16, device="cuda", dtype=torch.bfloat16)
    empty = torch.empty(0, 16, device="cuda", dtype=torch.bfloat16)
    assert pifa.layer_norm_forward(empty, None, None, EPS).shape == (0, 16)
    dX, dg, db = pifa.layer_norm_backward(empty, None, empty, EPS)
    torch.cuda.synchronize()
    assert dX.numel() == 0 and (dg == 0).all() and (db == 0).all()
    with pytest.raises(pifa.PifaError):
        pifa.layer_norm_forward(x, None, None, 0.0)
    with pytest.raises(pifa.PifaError):
        pifa.layer_norm_forward(x, None, None, EPS, H=(y := torch.empty_like(x)), Y=y)
    with pytest.raises(TypeError):
        pifa.layer_norm_forward(x, None, torch.ones(16, device="cuda"), EPS)  # a bias of another type
    with pytest.raises(ValueError):
        pifa.layer_norm_forward(x, None, None, EPS, R=x.cpu())
    big = torch.randn(40, 16, device="cuda", dtype=torch.bfloat16)
    with pytest.raises(pifa.PifaError):
        pifa.layer_norm_backward(big, None, big, EPS, work=torch.empty(8, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("d,M", [(1, (1 << 23) + 5), (520, (1 << 21) + 3)])
def test_more_rows_than_one_launch(d, M):
    """The rows behind the first 2^21 of a call: the same values as in a call of their own."""
    pifa, torch = _pifa(), torch_mod()
    x = torch.empty(M, d, dtype=torch.bfloat16, device="cuda")
    x[:, :] = (torch.arange(M, device="cuda") % 251 + 1).to(torch.bfloat16)[:, None]
    x[:, 0] += 1
    g, _ = _vec(d, "bf16", 21)
    Y = pifa.layer_norm_forward(x, g, g, EPS)
    for m in (0, (1 << 21) - 2, (1 << 21) + 1, M - 2):
        assert torch.equal(Y[m:m + 2], pifa.layer_norm_forward(x[m:m + 2].contiguous(), g, g, EPS)), m
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
    want = pifa.layer_norm_backward(h_dev, None, dy_dev, EPS)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a = torch.randn(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(20):
            a = a @ a * 1e-2
    got = pifa.layer_norm_backward(h_dev, None, dy_dev, EPS, stream=side.cuda_stream if as_handle else side)
    junk = [torch.full((pifa.layer_norm_backward_bytes(M, d) // 4,), 3.0, device="cuda") for _ in range(8)]
    torch.cuda.synchronize()
    assert len(junk) == 8 and all(torch.equal(g, w) for g, w in zip(got, want))


def _narrow(h):
    """rho, hat, and the errors of rho (relative) and of hat, of rows whose mean may be
    much larger than their deviations.  The first mean is off by dm = FP mean|h|, and
    so is every c; c's own mean takes that off but for FP of what it sums and the
    roundings of two subtractions.  The mean of the squares loses FP of itself, dm^2
    among it, and what is left of the mean squared."""
    mean = lambda a: a.mean(1, keepdims=True)
    c = h - mean(h)
    var = mean(c * c)
    rho = 1.0 / np.sqrt(var + EPS)
    dm = FP * mean(np.abs(h))
    left = 2 * FP * (mean(np.abs(c)) + dm)
    off = left + 2.0 ** -23 * (np.abs(c) + dm)
    drho = (2 * FP * (var + dm ** 2) + left ** 2) / (var + EPS) + 2.0 ** -22
    hat = c * rho
    return rho, hat, drho, np.abs(hat) * (drho + 2.0 ** -23) + rho * off * (1 + drho), rho * dm


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [2867, 4096, 5000, 16384, 40003])
def test_rows_that_hardly_vary(d, dtype):
    """Constant rows, whose centred values are zero, and rows that vary by a hundred
    thousandth of their size: in fp32, and in bf16 as a sum with a residual that fp32
    holds exactly; the gradients in bf16 from the rounded sum."""
    pifa, torch = _pifa(), torch_mod()
    rng = np.random.default_rng([50, d])
    base = np.array([100.1, 1000.1, -10000.3, 1e5 + 0.7, 1000.1, -100.1, 1000.1, 12345.6])
    x = np.repeat(base[:, None], d, 1)
    x[4:] *= 1 + 1e-5 * rng.standard_normal((4, d))
    g_dev, g = _vec(d, dtype, 51)
    b_dev, b = _vec(d, dtype, 52, mean=0.0)
    dy_dev, dy = _rows(len(base), d, dtype, 53, outliers=False)
    r, r_dev = None, None
    if dtype == "bf16":
        # in steps of 2^-8 of the row's power of two over 2^8: 17 bits in all
        big = inputs.round_to(x, "bf16")[1]
        step = 2.0 ** (np.floor(np.log2(np.abs(base)))[:, None] - 16)
        r_st, r = inputs.round_to(np.clip(np.round((x - big) / step), -256, 256) * step, "bf16")
        x, r_dev = big, to_dev(r_st)
    x_st, x = inputs.round_to(x, dtype)
    h = x if r is None else x + r
    assert np.array_equal(h, h.astype(np.float32))
    H = torch.empty_like(to_dev(x_st))
    Y = pifa.layer_norm_forward(to_dev(x_st), g_dev, b_dev, EPS, R=r_dev, H=H)
    one = [pifa.layer_norm_backward(H[m:m + 1], g_dev, dy_dev[m:m + 1], EPS) for m in range(len(base))]
    torch.cuda.synchronize()
    _, hat, _, eh, _ = _narrow(h)
    y = hat * g + b
    _close(from_dev(Y), y, np.abs(y) * HALF[dtype] + np.abs(g) * eh + 2.0 ** -22 * (np.abs(g * hat) + np.abs(b)), "Y")
    h = from_dev(H)
    mean = lambda a: a.mean(1, keepdims=True)
    rho, hat, drho, eh, off = _narrow(h)
    u = dy * g
    au, back = np.abs(u), np.abs(mean(u * hat))
    # u - mean(u) has at most |u| + mean|u|, c before its mean is taken off |c| + dm; what
    # is left of u's mean, FP of mean|u|, meets the dm
    eb = 2 * FP * mean((au + mean(au)) * (np.abs(hat) + off)) + 2 * off * FP * mean(au) + back * (drho + FP)
    want = [o.layer_norm_backward(h[m:m + 1], g, dy[m:m + 1], EPS) for m in range(len(base))]
    for m, (got, (dx, dg, db)) in enumerate(zip(one, want)):
        i = slice(m, m + 1)
        tol = rho[i] * (2 * FP * (au[i] + mean(au[i])) + eh[i] * back[i] + (np.abs(hat[i]) + eh[i]) * eb[i])
        _close(from_dev(got[0]), dx, tol + np.abs(dx) * (drho[i] + HALF[dtype]) + TINY, "dX %d" % m)
        _close(from_dev(got[1]), dg, (np.abs(dy[i]) * (eh[i] + 2.0 ** -23 * np.abs(hat[i])))[0] + 1e-30, "dgain %d" % m)
        _close(from_dev(got[2]), db, FP * np.abs(dy[m]) + 1e-30, "dbias %d" % m)
