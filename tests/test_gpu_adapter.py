"""Low-rank adapters (adapter_plan, adapter_forward, adapter_backward) against
their fp64 forms.

Tolerances, element by element.  Products of bf16 values are exact in fp32; a
sum takes at most 128 additions on the way of one product (a matrix instruction's
32, a wave's instructions, the waves, the parts of K), so it is good to 128 *
2^-24 = 2^-17 =: FP of its terms' magnitudes.  t and u are good to that, and to 2^-17
of themselves as two bf16 values each; in fp32 results they keep all their bits.  A
bf16 result is rounded by 2^-8 of it at most.
"""
import numpy as np
import pytest

from oracle import tune as o
from paper_2501_19090_amd import inputs

from gpu_util import from_dev, to_dev, torch_mod

pytestmark = pytest.mark.gpu

FP = 2.0 ** -17
HALF = 2.0 ** -8


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch_mod().cuda.is_available():
        pytest.skip("no GPU")


def _pifa():
    from paper_2501_19090_amd import pifa
    return pifa


def _ids(kind, M, n, rng):
    if kind == "runs":
        return np.sort(rng.integers(0, n, M))[::-1].copy().astype(np.int32)
    if kind == "one":
        return np.full(M, n - 1, np.int32)
    if kind == "none":
        return np.full(M, -1, np.int32)
    ids = rng.integers(-1, n, M).astype(np.int32)  # mixed, some without
    ids[rng.integers(0, M, 1 + M // 20)] = rng.choice([n, n + 7, -2 ** 31, 2 ** 31 - 1])
    return ids


class Case:
    def __init__(self, M, d_in, d_out, r, n, kind, seed=1, scaled=True):
        torch = torch_mod()
        rng = np.random.default_rng([seed, M, d_in, d_out, r, n])
        self.ids = _ids(kind, M, n, rng)
        self.n = n

        def dev(shape, scale):
            st, v = inputs.round_to(rng.standard_normal((shape[0], int(np.prod(shape[1:])))) * scale, "bf16")
            return to_dev(st).reshape(shape), v.reshape(shape)

        self.x_dev, self.x = dev((M, d_in), 1.0)
        self.y0_dev, self.y0 = dev((M, d_out), 1.0)
        self.dy_dev, self.dy = dev((M, d_out), 1.0)
        self.dx0_dev, self.dx0 = dev((M, d_in), 1.0)
        self.a_dev, self.a = dev((n, r, d_in), d_in ** -0.5)
        self.b_dev, self.b = dev((n, d_out, r), r ** -0.5)
        self.s = (0.5 + rng.random(n)).astype(np.float32) if scaled else None
        self.s_dev = torch.from_numpy(self.s).cuda() if scaled else None
        self.plan = _pifa().AdapterPlan(torch.from_numpy(self.ids).cuda(), n)

    def forward(self, **kw):
        return _pifa().adapter_forward(self.x_dev, self.a_dev, self.b_dev, self.plan, scale=self.s_dev, **kw)

    def backward(self, **kw):
        return _pifa().adapter_backward(self.x_dev, self.a_dev, self.b_dev, self.plan, self.dy_dev, scale=self.s_dev, **kw)

    def _f(self, x, A, B, y0, s):
        return o.adapter_forward(x, A, B, self.ids, s, y0)

    def check_forward(self, Y, y0):
        torch_mod().cuda.synchronize()
        s = None if self.s is None else self.s.astype(np.float64)
        want = self._f(self.x, self.a, self.b, y0, s)
        # sum_j |b| (|t| + sum |x||a|), twice FP each: t's own error, its two halves, the sum over j
        size = self._f(np.abs(self.x), np.abs(self.a), np.abs(self.b), None if y0 is None else np.abs(y0), s)
        _close(from_dev(Y), want, HALF * np.abs(want) + 4 * FP * size + 1e-30, "Y")

    def check_backward(self, dX, dA, dB, dx0):
        torch_mod().cuda.synchronize()
        s = None if self.s is None else self.s.astype(np.float64)
        want = o.adapter_backward(self.x, self.a, self.b, self.ids, self.dy, s, dx0)
        size = o.adapter_backward(*(np.abs(v) for v in (self.x, self.a, self.b)), self.ids, np.abs(self.dy), s,
                                  None if dx0 is None else np.abs(dx0))
        if dX is not None:
            _close(from_dev(dX), want[0], HALF * np.abs(want[0]) + 4 * FP * size[0] + 1e-30, "dX")
        for got, w, z, name in ((dA, want[1], size[1], "dA"), (dB, want[2], size[2], "dB")):
            if got is not None:
                _close(from_dev(got), w, 2 * FP * z, name)


def _close(got, want, tol, what):
    off = np.abs(got - want) - tol
    assert np.isfinite(got).all(), what
    assert (off <= 0).all(), (what, float(off.max()), np.unravel_index(off.argmax(), off.shape))


SHAPES = [  # M, d_in, d_out, r, n, ids
    (1, 8, 8, 1, 1, "one"), (1, 4096, 4096, 16, 3, "one"), (3, 33, 65, 5, 2, "mixed"), (16, 128, 64, 8, 4, "mixed"),
    (17, 100, 300, 16, 1, "one"), (48, 1024, 1000, 16, 40, "mixed"), (64, 72, 1001, 17, 2, "runs"), (65, 999, 77, 32, 5, "mixed"),
    (200, 31, 31, 33, 3, "mixed"), (300, 2048, 513, 64, 70, "mixed"), (333, 515, 258, 24, 1, "one"), (512, 256, 128, 100, 1, "one"),
    (513, 264, 136, 128, 1, "one"), (700, 1500, 40, 129, 2, "runs"), (1100, 130, 2050, 4, 3, "mixed"), (1025, 64, 64, 48, 1, "one"),
    (1999, 520, 264, 16, 5, "runs"), (2100, 96, 200, 200, 2, "mixed"), (3000, 256, 320, 32, 4000, "mixed"), (40, 64, 64, 16, 3, "none"),
    (70, 3, 5, 2, 2, "mixed"), (70, 7, 130, 40, 2, "mixed"), (600, 6, 4, 9, 1, "one"), (130, 9, 263, 90, 30, "mixed"),
]


@pytest.mark.parametrize("shape", SHAPES)
def test_forward(shape):
    torch = torch_mod()
    c = Case(*shape)
    Y = torch.full_like(c.y0_dev, float("nan"))
    assert c.forward(Y0=c.y0_dev, Y=Y) is Y
    c.check_forward(Y, c.y0)
    assert torch.equal(c.forward(Y0=c.y0_dev), Y)  # a fixed order of sums
    c.check_forward(c.forward(), None)
    without = torch.from_numpy((c.ids < 0) | (c.ids >= c.n)).cuda()
    assert torch.equal(Y[without], c.y0_dev[without])
    assert (c.forward()[without] == 0).all()
    y = c.y0_dev.clone()
    assert c.forward(Y0=y, Y=y) is y and torch.equal(y, Y)


@pytest.mark.parametrize("shape", SHAPES)
def test_backward(shape):
    torch = torch_mod()
    c = Case(*shape, seed=2)
    dX = torch.full_like(c.dx0_dev, float("nan"))
    dA, dB = (torch.full(t.shape, float("nan"), device="cuda") for t in (c.a_dev, c.b_dev))
    c.backward(dX0=c.dx0_dev, dX=dX, dA=dA, dB=dB)
    c.check_backward(dX, dA, dB, c.dx0)
    unused = [a for a in range(c.n) if not (c.ids == a).any()]
    assert (dA[unused] == 0).all() and (dB[unused] == 0).all()
    again = c.backward(dX0=(d := c.dx0_dev.clone()), dX=d)
    assert all(torch.equal(a, b) for a, b in zip(again, (dX, dA, dB)))
    # one output at a time, without a gradient beside
    for k in range(3):
        need = dict(need_dX=k == 0, need_dA=k == 1, need_dB=k == 2)
        got = c.backward(**need)
        assert [g is not None for g in got] == [k == 0, k == 1, k == 2]
        if k:
            assert torch.equal(got[k], (dX, dA, dB)[k])
        else:
            c.check_backward(got[0], None, None, None)


def test_without_a_scale():
    c = Case(90, 200, 100, 12, 3, "mixed", scaled=False)
    c.check_forward(c.forward(Y0=c.y0_dev), c.y0)
    c.check_backward(*c.backward(dX0=c.dx0_dev), c.dx0)


def test_gradients_against_differences():
    """The loss sum(Y dY) is linear in A, in B and in X: its differences over a
    whole step are the gradients, up to the rounding of the outputs to bf16."""
    pifa, torch = _pifa(), torch_mod()
    c = Case(150, 64, 48, 8, 4, "mixed", seed=5)
    dX, dA, dB = (g.double() for g in c.backward())
    loss = lambda x, a, b: pifa.adapter_forward(x, a, b, c.plan, scale=c.s_dev)
    rng = torch.Generator(device="cuda").manual_seed(1)
    for k, (t, grad) in enumerate(((c.x_dev, dX), (c.a_dev, dA), (c.b_dev, dB))):
        v = torch.randn(t.shape, device="cuda", generator=rng).to(torch.bfloat16)
        args = [[c.x_dev, c.a_dev, c.b_dev] for _ in range(2)]
        args[0][k], args[1][k] = v, torch.zeros_like(t)
        y = loss(*args[0]).double()
        assert (loss(*args[1]) == 0).all()
        tol = 2.0 ** -7 * float((y * c.dy_dev.double()).abs().sum()) + 2.0 ** -7 * float((grad * v.double()).abs().sum())
        assert abs(float((y * c.dy_dev.double()).sum()) - float((grad * v.double()).sum())) <= tol, k


@pytest.mark.parametrize("M,n", [(0, 3), (1, 1), (5, 4096), (64, 2), (1000, 30), (1024, 4), (1025, 4), (5000, 700), (70001, 4096),
                                 (1 << 20, 5)])
@pytest.mark.parametrize("kind", ["mixed", "runs", "one", "none"])
def test_plan(M, n, kind):
    """The plan's tiles hold the rows in a stable order by adapter, those without at
    the end; its pieces cover each adapter's tiles in order."""
    pifa, torch = _pifa(), torch_mod()
    rng = np.random.default_rng([M, n])
    ids = _ids(kind, M, n, rng) if M else np.zeros(0, np.int32)
    size = pifa.adapter_plan_bytes(M, n)
    big = torch.full((size + 64,), 123, dtype=torch.uint8, device="cuda")
    pifa.adapter_plan(torch.from_numpy(ids).cuda(), n, big[:size])
    torch.cuda.synchronize()
    assert (big[size:] == 123).all()
    words = big[:size].cpu().numpy().view(np.int32)
    tmax, at = M // 64 + min(n, M) + 1, 16
    head = words[:16]

    def take(k):
        nonlocal at
        at += -(-k // 16) * 16
        return words[at - -(-k // 16) * 16:at]

    tiles, rows = take(2 * tmax), take(64 * tmax)
    pieces, multi = take(4 * (M // 512 + n)), take(3 * (M // 512 + 1))
    bucket = np.where((ids >= 0) & (ids < n), ids, n)
    order = np.argsort(bucket, kind="stable")
    count = np.bincount(bucket, minlength=n + 1)
    start = np.concatenate([[0], np.cumsum(count)])
    first, want_tiles, want_rows, want_pieces, want_multi, slot = [], [], [], [], [], 0
    for a in range(n + 1):
        first.append(len(want_tiles))
        for k in range(0, count[a], 64):
            c = min(64, count[a] - k)
            want_tiles.append((a, c))
            want_rows.append(np.concatenate([order[start[a] + k:start[a] + k + c], np.full(64 - c, -1)]))
        if a < n:
            of = -(-count[a] // 64)
            k = max(1, -(-count[a] // 512))
            want_pieces += [(a, first[a] + 8 * i, min(8, of - 8 * i), slot + i if k > 1 else -1) for i in range(k)]
            if k > 1:
                want_multi.append((a, slot, k))
                slot += k
    assert list(head[:6]) == [M, n, first[n], len(want_tiles), len(want_pieces), len(want_multi)]
    flat = lambda v: np.array(v, np.int32).ravel()
    assert np.array_equal(tiles[:2 * len(want_tiles)], flat(want_tiles))
    assert np.array_equal(rows[:64 * len(want_tiles)], flat(want_rows))
    assert np.array_equal(pieces[:4 * len(want_pieces)], flat(want_pieces))
    assert np.array_equal(multi[:3 * len(want_multi)], flat(want_multi)) and slot <= 2 * (M // 512)


def test_special_values_stay_in_their_rows():
    """A NaN in a row is in its results only; one in an adapter in its rows only."""
    torch = torch_mod()
    c = Case(100, 77, 90, 20, 4, "mixed", seed=7)
    clean, (dX, dA, dB) = c.forward(Y0=c.y0_dev), c.backward(dX0=c.dx0_dev)
    ids = torch.from_numpy(c.ids).cuda()
    row = int((ids == 2).nonzero()[0])
    keep = torch.arange(100, device="cuda") != row
    others = [0, 1, 3]
    for value in (float("nan"), float("inf")):
        x, dy = c.x_dev.clone(), c.dy_dev.clone()
        c.x_dev[row, 3] = value
        y = c.forward(Y0=c.y0_dev)
        assert torch.equal(y[keep], clean[keep]) and not torch.isfinite(y[row]).any()
        c.dy_dev[row, 5] = value
        got = c.backward(dX0=c.dx0_dev)
        assert torch.equal(got[0][keep], dX[keep]) and not torch.isfinite(got[0][row]).any()
        assert torch.equal(got[1][others], dA[others]) and torch.equal(got[2][others], dB[others])
        c.x_dev.copy_(x)
        c.dy_dev.copy_(dy)
    c.a_dev[3, 4, 70] = float("nan")
    c.b_dev[3, 80, 19] = float("nan")
    y, got = c.forward(Y0=c.y0_dev), c.backward(dX0=c.dx0_dev)
    other = ids != 3
    assert torch.equal(y[other], clean[other]) and torch.isnan(y[~other]).all()
    assert torch.equal(got[0][other], dX[other]) and torch.equal(got[1][:3], dA[:3]) and torch.equal(got[2][:3], dB[:3])


@pytest.mark.parametrize("M", [100, 300])
def test_infinite_sums(M):
    """t and u past fp32 are infinite, and so are the results that take them with one
    sign, whichever of them; a row's own, and its adapter's gradients."""
    pifa, torch = _pifa(), torch_mod()
    bf = dict(dtype=torch.bfloat16, device="cuda")
    X, dY = torch.ones(M, 64, **bf), torch.ones(M, 48, **bf)
    X[3], X[4], dY[3], dY[4] = 1e38, -1e38, 1e38, -1e38
    A, B = torch.ones(2, 1, 64, **bf), torch.ones(2, 48, 1, **bf)
    plan = pifa.AdapterPlan(torch.arange(M, dtype=torch.int32, device="cuda") % 2, 2)  # rows 3 and 4: 1 and 0
    Y = pifa.adapter_forward(X, A, B, plan)
    dX, dA, dB = pifa.adapter_backward(X, A, B, plan, dY)
    torch.cuda.synchronize()
    inf = float("inf")
    for out, other in ((Y, 64.0), (dX, 48.0)):
        assert (out[3] == inf).all() and (out[4] == -inf).all()
        assert (out[:3] == other).all() and (out[5:] == other).all()
    # -inf times a negative row is positive: every term of both adapters is, or is finite
    assert (dA == inf).all() and (dB == inf).all()


def test_rows_anywhere_in_a_buffer():
    """Buffers that start at any element, and what lies around them."""
    pifa, torch = _pifa(), torch_mod()
    c = Case(70, 101, 99, 9, 3, "mixed", seed=8)
    want, grads = c.forward(Y0=c.y0_dev), c.backward(dX0=c.dx0_dev)

    def at(t, off):
        big = torch.full((t.numel() + 32,), 7.0, dtype=t.dtype, device="cuda")
        big[off:off + t.numel()] = t.reshape(-1)
        return big, big[off:off + t.numel()].view(t.shape)

    for off in (1, 2, 8):
        put = lambda t, k=0: at(t, off + k)
        (_, x), (_, a), (_, b), (_, s), (_, dy) = put(c.x_dev), put(c.a_dev, 1), put(c.b_dev, 2), put(c.s_dev), put(c.dy_dev, 3)
        by, y = put(c.y0_dev, 1)
        pifa.adapter_forward(x, a, b, c.plan, scale=s, Y0=y, Y=y)
        bx, dx = put(c.dx0_dev)
        (ba, da), (bb, db) = put(grads[1] * 0), put(grads[2] * 0, 1)
        pifa.adapter_backward(x, a, b, c.plan, dy, scale=s, dX0=dx, dX=dx, dA=da, dB=db)
        torch.cuda.synchronize()
        assert torch.equal(y, want) and torch.equal(dx, grads[0]) and torch.equal(da, grads[1]) and torch.equal(db, grads[2])
        for big, k, n in ((by, off + 1, y.numel()), (bx, off, dx.numel()), (ba, off, da.numel()), (bb, off + 1, db.numel())):
            assert (big[:k] == 7).all() and (big[k + n:] == 7).all()


def test_no_rows_and_refused_calls():
    pifa, torch = _pifa(), torch_mod()
    bf = torch.bfloat16
    a, b = torch.ones(2, 4, 16, dtype=bf, device="cuda"), torch.ones(2, 8, 4, dtype=bf, device="cuda")
    x, y = torch.ones(0, 16, dtype=bf, device="cuda"), torch.ones(0, 8, dtype=bf, device="cuda")
    plan = pifa.AdapterPlan(torch.zeros(0, dtype=torch.int32, device="cuda"), 2)
    assert pifa.adapter_forward(x, a, b, plan, Y0=y).shape == (0, 8)
    dX, dA, dB = pifa.adapter_backward(x, a, b, plan, y)
    torch.cuda.synchronize()
    assert dX.shape == (0, 16) and (dA == 0).all() and (dB == 0).all()
    plan = pifa.AdapterPlan(torch.zeros(3, dtype=torch.int32, device="cuda"), 2)
    x, y = torch.ones(3, 16, dtype=bf, device="cuda"), torch.ones(3, 8, dtype=bf, device="cuda")
    with pytest.raises(pifa.PifaError):
        pifa.adapter_forward(x, a, b, plan, work=torch.empty(16, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError):
        pifa.adapter_forward(x, a, b, plan, Y0=y.cpu())
    with pytest.raises(ValueError):
        pifa.adapter_forward(x[:2], a, b, plan)
    with pytest.raises(ValueError):
        pifa.AdapterPlan(torch.zeros(3, dtype=torch.int32), 2)  # ids on the host
    # a plan of another batch in the same memory: nothing is written
    pifa.adapter_plan(torch.zeros(2, dtype=torch.int32, device="cuda"), 2, plan.buffer)
    out = torch.full((3, 8), 5.0, dtype=bf, device="cuda")
    dA = torch.full((2, 4, 16), 5.0, device="cuda")
    pifa.adapter_forward(x, a, b, plan, Y0=y, Y=out)
    pifa.adapter_backward(x, a, b, plan, y, dA=dA, need_dX=False, need_dB=False)
    torch.cuda.synchronize()
    assert (out == 5).all() and (dA == 5).all()


def test_captured_and_replayed_with_other_ids():
    """A graph of plan, forward and gradients, replayed on new rows and ids with
    eager calls between."""
    pifa, torch = _pifa(), torch_mod()
    M, d_in, d_out, r, n = 600, 264, 136, 16, 3
    c = Case(M, d_in, d_out, r, n, "mixed", seed=9)
    ids = torch.zeros(M, dtype=torch.int32, device="cuda")
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    new = lambda: [torch.empty_like(c.y0_dev), torch.empty_like(c.dx0_dev), torch.empty(c.a_dev.shape, device="cuda"),
                   torch.empty(c.b_dev.shape, device="cuda"),
                   torch.empty(pifa.adapter_forward_bytes(M, d_in, d_out, r, n), dtype=torch.uint8, device="cuda"),
                   torch.empty(pifa.adapter_backward_bytes(M, d_in, d_out, r, n), dtype=torch.uint8, device="cuda")]

    def calls(plan, Y, dX, dA, dB, w1, w2):
        plan.update(ids)
        pifa.adapter_forward(c.x_dev, c.a_dev, c.b_dev, plan, scale=c.s_dev, Y0=c.y0_dev, Y=Y, work=w1)
        pifa.adapter_backward(c.x_dev, c.a_dev, c.b_dev, plan, c.dy_dev, scale=c.s_dev, dX0=c.dx0_dev, dX=dX, dA=dA, dB=dB,
                              work=w2)

    out, other = new(), new()
    spare = pifa.AdapterPlan(ids, n)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        calls(c.plan, *out)
    rng = np.random.default_rng(4)
    for kind in ("mixed", "one", "none", "runs"):
        ids.copy_(torch.from_numpy(_ids(kind, M, n, rng)))
        c.x_dev.normal_()
        for t in out[:4]:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        calls(spare, *other)
        torch.cuda.synchronize()
        for a, b in zip(out[:4], other[:4]):
            assert torch.equal(a, b), kind


@pytest.mark.parametrize("as_handle", [False, True])
def test_workspaces_of_calls_on_another_stream(as_handle):
    """Calls on a stream of their own, behind work that holds it up: memory that is
    allocated and filled on the current stream meanwhile is not theirs."""
    pifa, torch = _pifa(), torch_mod()
    c = Case(600, 264, 136, 16, 3, "mixed", seed=10)
    want = [c.forward(Y0=c.y0_dev), *c.backward(dX0=c.dx0_dev)]
    side = torch.cuda.Stream()
    a = torch.randn(4096, 4096, device="cuda")
    ids = torch.from_numpy(c.ids).cuda()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(20):
            a = a @ a * 1e-2
    st = side.cuda_stream if as_handle else side
    plan = pifa.AdapterPlan(ids, 3, stream=st)
    c.plan = plan
    got = [c.forward(Y0=c.y0_dev, stream=st), *c.backward(dX0=c.dx0_dev, stream=st)]
    junk = [torch.full((k,), 3.0, device="cuda") for k in (4096, 1 << 18, 1 << 20, 1 << 21) for _ in range(4)]
    torch.cuda.synchronize()
    assert len(junk) == 16 and all(torch.equal(g, w) for g, w in zip(got, want))


def test_two_streams_share_a_plan():
    """Calls that overlap on two streams, with workspaces and outputs of their own."""
    torch = torch_mod()
    c = Case(700, 520, 260, 24, 6, "mixed", seed=12)
    want_y, want = c.forward(Y0=c.y0_dev), c.backward(dX0=c.dx0_dev)
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for _ in range(5):
        for s in streams:
            got.append((c.forward(Y0=c.y0_dev, stream=s), *c.backward(dX0=c.dx0_dev, stream=s)))
    torch.cuda.synchronize()
    for y, dX, dA, dB in got:
        assert torch.equal(y, want_y) and all(torch.equal(a, b) for a, b in zip((dX, dA, dB), want))


def test_a_plan_of_other_numbers_writes_nothing():
    pifa, torch = _pifa(), torch_mod()
    c = Case(100, 64, 48, 8, 3, "mixed", seed=13)
    for M, n in ((200, 3), (100, 5)):
        other = pifa.AdapterPlan(torch.zeros(M, dtype=torch.int32, device="cuda"), n)
        assert other.buffer.numel() >= pifa.adapter_plan_bytes(100, 3)
        other.M, other.n = 100, 3
        outs = [torch.full(s, 7.0, device="cuda", dtype=t) for s, t in (
            ((100, 48), torch.bfloat16), ((100, 64), torch.bfloat16), ((3, 8, 64), torch.float32), ((3, 48, 8), torch.float32))]
        pifa.adapter_forward(c.x_dev, c.a_dev, c.b_dev, other, Y0=c.y0_dev, Y=outs[0])
        pifa.adapter_backward(c.x_dev, c.a_dev, c.b_dev, other, c.dy_dev, dX0=c.dx0_dev, dX=outs[1], dA=outs[2], dB=outs[3])
        torch.cuda.synchronize()
        assert all(bool((t == 7).all()) for t in outs)


@pytest.mark.parametrize("M,d_in,d_out", [(100, 136, 264), (300, 263, 130), (1100, 5, 131)])
@pytest.mark.parametrize("r", [1, 5, 16, 17, 32, 40, 64, 100, 130])
def test_infinite_operands(M, d_in, d_out, r):
    """One infinity in each operand in turn: results that the formula makes infinite
    have its sign, those that it makes no number are none, the others keep their
    bounds.  (A few t are as close to zero as they are off, far fewer than are met here.)"""
    c = Case(M, d_in, d_out, r, 2, "mixed", seed=14)
    s = c.s.astype(np.float64)
    row = int(np.flatnonzero(c.ids == 1)[3])
    for name, at in (("x", (row, d_in - 2)), ("dy", (row, d_out - 1)), ("a", (1, r - 1, 2)), ("b", (1, d_out - 2, r // 2))):
        for value in (np.inf, -np.inf):
            host, there = getattr(c, name), getattr(c, name + "_dev")
            kept = host[at]
            host[at] = there[at] = value
            with np.errstate(invalid="ignore"):
                want = [c._f(c.x, c.a, c.b, c.y0, s), *o.adapter_backward(c.x, c.a, c.b, c.ids, c.dy, s, c.dx0)]
                size = [c._f(*map(np.abs, (c.x, c.a, c.b, c.y0)), s),
                        *o.adapter_backward(*map(np.abs, (c.x, c.a, c.b)), c.ids, np.abs(c.dy), s, np.abs(c.dx0))]
            got = [from_dev(t) for t in (c.forward(Y0=c.y0_dev), *c.backward(dX0=c.dx0_dev))]
            host[at] = there[at] = kept
            assert not all(np.isfinite(w).all() for w in want)
            for g, w, z, half, what in zip(got, want, size, (HALF, HALF, 0, 0), ("Y", "dX", "dA", "dB")):
                finite, what = np.isfinite(w), (what, name, value)
                assert np.array_equal(g[~finite], w[~finite], equal_nan=True), what
                off = np.abs(g[finite] - w[finite]) - (half * np.abs(w[finite]) + 4 * FP * z[finite] + 1e-30)
                assert np.isfinite(g[finite]).all() and (off <= 0).all(), what


@pytest.mark.parametrize("shape", [
    (130, 100, 9000, 1024, 2, "mixed"), (600, 12001, 64, 300, 1, "one"), (33, 20000, 30001, 201, 2, "mixed"),
    (20, 1 << 19, 40, 5, 2, "mixed"), (70, 33, 1 << 19, 6, 3, "mixed"), (9, 9001, 1001, 1023, 1, "one"), (9, (1 << 19) - 1, 101, 17, 1, "one"),
    (257, 72, 40, 65, 4096, "mixed")])
def test_the_largest_ranks_and_widths(shape):
    """Up to the limits.  A product's way through a sum over K of d columns: 32 additions
    in its instruction, one instruction a wave for each 32 * 4 * 8 columns where K is
    cut into 8 parts (32 * 4 where it is not), 4 waves, 8 parts; over ranks, 32 and two
    for each 32.  Where that passes 128 the bounds grow with it."""
    c = Case(*shape, seed=15)
    M, d_in, d_out, r, n, _ = shape
    tiles = sum(-(-int((c.ids == a).sum()) // 64) for a in range(n))
    target = (3 if r <= 16 else 2) * 256 // (2 * -(-r // 64))  # of a launch of two jobs; the forward cuts as much or more
    split = max(1, min(8, target // tiles))
    steps = max(44 + max(d_in, d_out) // (128 * split), 32 + 2 * -(-r // 32))
    more = max(1.0, steps / 128)

    def close(got, want, size, half, what):
        _close(from_dev(got), want, half * np.abs(want) + 4 * FP * more * size + 1e-30, what)

    s, abs_of = c.s.astype(np.float64), [np.abs(v) for v in (c.x, c.a, c.b)]
    Y = c.forward(Y0=c.y0_dev)
    close(Y, c._f(c.x, c.a, c.b, c.y0, s), c._f(*abs_of, np.abs(c.y0), s), HALF, "Y")
    want = o.adapter_backward(c.x, c.a, c.b, c.ids, c.dy, s, c.dx0)
    size = o.adapter_backward(*abs_of, c.ids, np.abs(c.dy), s, np.abs(c.dx0))
    for got, w, z, half, what in zip(c.backward(dX0=c.dx0_dev), want, size, (HALF, 0, 0), ("dX", "dA", "dB")):
        close(got, w, z, half, what)
