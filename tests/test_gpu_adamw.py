"""AdamW steps (adamw_step) against their definition.

The moments are bit for bit what the formula gives where each fp32 operation is
rounded by itself, their 8-bit codes what the definition's random bits make of
them.  p takes a product, a division and a root of them, each rounded by half a
step of fp32 (2^-24): p (1 - lr decay) is off by 2 * 2^-24 |p|, the update, of
eight rounded operations, by 8 * 2^-24 of itself, p once more by 2^-24.
"""
import numpy as np
import pytest

from oracle import tune as o

from gpu_util import from_dev, torch_mod

pytestmark = pytest.mark.gpu

STEP = 2.0 ** -24
SIZES = [[1], [4095, 4096, 4097], [31, 0, 32, 33, 8192, 5, 100001], [3 * 4096 + 7] * 3]


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch_mod().cuda.is_available():
        pytest.skip("no GPU")


def _pifa():
    from paper_2501_19090_amd import pifa
    return pifa


class Case:
    """Tensors of these sizes, inside larger buffers where `shift`, with their fp32 values on the host."""

    def __init__(self, sizes, bits, grad, copy, seed, shift=0, zero_state=False):
        torch = torch_mod()
        rng = np.random.default_rng(seed)
        self.bits, self.sizes, self.seed = bits, sizes, seed * 1000003
        f = np.float32
        self.p = [f(rng.standard_normal(n) * 0.02) for n in sizes]
        self.g = [torch.from_numpy(f(rng.standard_normal(n) * 10.0 ** rng.uniform(-6, 0, n))).to(grad) for n in sizes]
        if zero_state:
            self.m, self.v = ([np.zeros(n, np.float32) for n in sizes] for _ in range(2))
        else:
            self.m = [f(rng.standard_normal(n) * 10.0 ** rng.uniform(-5, -2, n)) for n in sizes]
            self.v = [f(rng.standard_normal(n) ** 2 * 10.0 ** rng.uniform(-10, -4, n)) for n in sizes]
        self.guards = []

        def dev(t):
            big = torch.full((t.numel() + 2 * shift,), 1, dtype=torch.uint8, device="cuda").to(t.dtype) if t.dtype != torch.uint8 \
                else torch.full((t.numel() + 2 * shift,), 1, dtype=torch.uint8, device="cuda")
            view = big[shift:shift + t.numel()]
            view.copy_(t.cuda())
            self.guards.append((big, shift, t.numel()))
            return view

        d32 = lambda a: dev(torch.from_numpy(a))
        self.p_dev, self.g_dev = [d32(a) for a in self.p], [dev(t) for t in self.g]
        if bits == 32:
            self.states = [(d32(a), d32(b)) for a, b in zip(self.m, self.v)]
        else:
            self.states = []
            for i, n in enumerate(sizes):
                half = np.full(n, 32767)
                code = [o.e4m3_round(a[i], half, 0) if not zero_state else (np.zeros(n, np.uint8), np.zeros(-(-n // 32), np.uint8))
                        for a in (self.m, self.v)]
                self.states.append((dev(torch.from_numpy(code[0][0])).view(torch.float8_e4m3fn),
                                    dev(torch.from_numpy(code[1][0])).view(torch.float8_e4m3fn),
                                    dev(torch.from_numpy(code[0][1])), dev(torch.from_numpy(code[1][1]))))
                self.m[i], self.v[i] = (o.e4m3_values(*c) for c in code)
        self.copies = [torch.zeros(n, dtype=torch.bfloat16, device="cuda") for n in sizes] if copy else None
        self.decay = [0.1 * (i % 3) for i in range(len(sizes))]
        self.opt = _pifa().AdamW(self.p_dev, self.g_dev, weight_decay=self.decay, states=self.states, copies=self.copies,
                                 seed=self.seed)

    def check(self, t, lr, b1, b2, eps, scale, what=""):
        """The state on the device is that after step t from the one on the host, which follows."""
        torch = torch_mod()
        torch.cuda.synchronize()
        for i, n in enumerate(self.sizes):
            g = self.g[i].float().numpy()
            m, v = o.adamw_moments(g, self.m[i], self.v[i], b1, b2, scale)
            s = 1.0 if scale is None else float(np.float32(scale))
            want, _, _ = o.adamw(self.p[i].astype(np.float64), g.astype(np.float64), self.m[i].astype(np.float64),
                                 self.v[i].astype(np.float64), t, lr, b1, b2, eps, self.decay[i], s)
            # from the rounded moments, so that only p's own roundings count
            upd = lr / (1 - b1 ** t) * m.astype(np.float64) / (np.sqrt(v.astype(np.float64) / (1 - b2 ** t)) + eps)
            want = self.p[i].astype(np.float64) * (1 - lr * self.decay[i]) - upd
            got = from_dev(self.p_dev[i])
            tol = STEP * (2 * np.abs(self.p[i]) + 8 * np.abs(upd) + np.abs(want)) + 2.0 ** -149
            assert (np.abs(got - want) <= tol).all(), (what, i, "p", float((np.abs(got - want) - tol).max()))
            if self.bits == 32:
                assert np.array_equal(self.states[i][0].cpu().numpy(), m), (what, i, "m")
                assert np.array_equal(self.states[i][1].cpu().numpy(), v), (what, i, "v")
                self.m[i], self.v[i] = m, v
            else:
                rm, rv = o.random_bits(self.seed & 0xFFFFFFFF, t, i, n)
                for k, (x, bits, least, name) in enumerate(((m, rm, 0, "m"), (v, rv, 1, "v"))):
                    codes, scales = o.e4m3_round(x, bits, least)
                    assert np.array_equal(self.states[i][2 + k].cpu().numpy(), scales), (what, i, name, "scales")
                    have = self.states[i][k].view(torch.uint8).cpu().numpy()
                    # a zero has either sign
                    same = (have == codes) | ((have | codes) == 128)
                    assert same.all(), (what, i, name, np.flatnonzero(~same)[:5])
                    (self.m if k == 0 else self.v)[i] = o.e4m3_values(have, scales)
            if self.copies:
                assert torch.equal(self.copies[i], self.p_dev[i].to(torch.bfloat16)), (what, i, "copy")
            self.p[i] = self.p_dev[i].cpu().numpy().copy()
        for big, shift, n in self.guards:
            one = big.view(torch.uint8) if big.dtype == torch.float8_e4m3fn else big
            assert (one[:shift] == 1).all() and (one[shift + n:] == 1).all(), what


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("grad", ["float32", "bfloat16"])
@pytest.mark.parametrize("sizes", range(len(SIZES)))
def test_steps(sizes, grad, bits):
    """Several steps in a row, numbered and counted on the device, with and without a
    scale of the gradients."""
    torch = torch_mod()
    c = Case(SIZES[sizes], bits, getattr(torch, grad), copy=sizes != 1, seed=sizes + 3)
    scale = torch.tensor([0.37], device="cuda")
    c.opt.step(1e-3, 0.9, 0.95, 1e-8, step=5)
    c.check(5, 1e-3, 0.9, 0.95, 1e-8, None, "numbered")
    assert c.opt.count() == 5
    c.opt.step(2e-3, 0.8, 0.999, 1e-6, grad_scale=scale)
    c.check(6, 2e-3, 0.8, 0.999, 1e-6, 0.37, "counted")
    c.opt.step(0.0, 0.0, 0.0, 1e-8)
    c.check(7, 0.0, 0.0, 0.0, 1e-8, None, "no memory")
    assert c.opt.count() == 7
    c.opt.step(1e-3, 0.9, 0.999, 1e-8, step=1)
    c.check(1, 1e-3, 0.9, 0.999, 1e-8, None, "again")
    c.opt.close()


@pytest.mark.parametrize("bits", [32, 8])
def test_first_steps_of_a_new_state(bits):
    torch = torch_mod()
    c = Case([1000, 77], bits, torch.float32, True, 21, zero_state=True)
    assert c.opt.count() == 0
    for t in (1, 2, 3):
        c.opt.step(1e-3, 0.9, 0.999, 1e-8)
        c.check(t, 1e-3, 0.9, 0.999, 1e-8, None, t)
    c.opt.close()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("shift", [1, 3])
def test_tensors_anywhere_in_a_buffer(shift, bits):
    """Tensors that start at any element, and what lies around them."""
    torch = torch_mod()
    c = Case([4099, 33, 7], bits, torch.bfloat16, False, 31, shift=shift)
    for t in (1, 2):
        c.opt.step(1e-3, step=t)
        c.check(t, 1e-3, 0.9, 0.999, 1e-8, None, t)
    c.opt.close()


def test_states_that_the_class_makes():
    pifa, torch = _pifa(), torch_mod()
    p = torch.randn(50, 40, device="cuda")
    for bits in (32, 8):
        a, g = p.clone(), torch.randn_like(p)
        with pifa.AdamW([a], [g], bits=bits) as opt:
            opt.step(1e-2, eps=1e-12)
            torch.cuda.synchronize()
            # the first step moves every value by lr against its gradient
            assert float((a - (p - 1e-2 * torch.sign(g))).abs().max()) <= 1e-2 * 2.0 ** -20 + 8 * 2.0 ** -24
            assert opt.count() == 1


@pytest.mark.parametrize("bits", [32, 8])
def test_special_values_stay_in_their_values(bits):
    """A NaN or an infinite gradient reaches its own value, and in 8 bits the
    moments of its group of 32; moments of zeros stay zeros."""
    pifa, torch = _pifa(), torch_mod()
    n = 200
    p, g = torch.ones(n, device="cuda"), torch.ones(n, device="cuda")
    g[5], g[70], g[100:132] = float("nan"), float("inf"), 0.0
    with pifa.AdamW([p], [g], bits=bits) as opt:
        opt.step(1e-2)
        torch.cuda.synchronize()
        m, v = (s.float() for s in opt.states[0][:2])
        bad = torch.zeros(n, dtype=torch.bool)
        bad[[5, 70]] = True
        assert torch.isnan(p.cpu()[bad]).all() and torch.isfinite(p.cpu()[~bad]).all()
        assert (p[100:132] == 1).all()
        if bits == 8:
            assert [int(s) for s in opt.states[0][2]].count(255) == 2 and int(opt.states[0][2][0]) == 255
            group = torch.zeros(n, dtype=torch.bool)
            group[0:32] = group[64:96] = True
            assert torch.isnan(m.cpu()[group]).all() and torch.isfinite(m.cpu()[~group]).all()
            assert torch.isnan(v.cpu()[group]).all() and torch.isfinite(v.cpu()[~group]).all()
            opt.step(1e-2)  # a NaN group stays one
            torch.cuda.synchronize()
            assert torch.isnan(p.cpu()[group]).all() and torch.isfinite(p.cpu()[~group]).all()
        else:
            assert torch.isnan(m[5]) and torch.isinf(m[70]) and torch.isinf(v[70]) and torch.isfinite(m.cpu()[~bad]).all()


def test_quotients_at_the_ends_of_the_range():
    """m / (root + eps) past fp32 is infinite, over an infinite root nothing."""
    pifa, torch = _pifa(), torch_mod()
    inf = float("inf")
    p, g = torch.ones(6, device="cuda"), torch.zeros(6, device="cuda")
    m = torch.tensor([1e30, -1e30, 1e30, 0.0, 1e-37, 1e30], device="cuda")
    v = torch.tensor([0.0, 0.0, inf, inf, 0.0, 1.0], device="cuda")
    with pifa.AdamW([p], [g], states=[(m, v)]) as opt:
        opt.step(1.0, 0.5, 0.5, 1e-37, step=60)
        torch.cuda.synchronize()
    got = p.double().cpu()
    assert got[:4].tolist() == [-inf, inf, 1.0, 1.0]
    # m / 2 over eps, and over the root of v / 2: at most eight roundings of fp32, 2^-21
    assert abs(float(got[4]) - 0.5) <= 2.0 ** -21 and abs(float(got[5]) / -(0.5e30 / 0.5 ** 0.5) - 1) <= 2.0 ** -21


@pytest.mark.parametrize("bits", [32, 8])
def test_captured_step_counts_on(bits):
    """A graph of a counted step, replayed with eager calls between: the same bits
    as eager steps; a numbered one replays its number."""
    pifa, torch = _pifa(), torch_mod()
    rng = torch.Generator(device="cuda").manual_seed(3)
    make = lambda: [torch.randn(n, device="cuda", generator=rng) for n in (5000, 37)]
    start, g = make(), [torch.empty(n, device="cuda") for n in (5000, 37)]
    grads = [make() for _ in range(6)]

    def clones():
        p = [t.clone() for t in start]
        return p, pifa.AdamW(p, g, bits=bits, seed=11)

    def set_g(k):
        for a, b in zip(g, grads[k]):
            a.copy_(b)

    want_p, want = clones()
    for k in range(6):
        set_g(k)
        want.step(1e-3)
    got_p, got = clones()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    set_g(0)
    got.step(1e-3)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        got.step(1e-3)
    for k in range(1, 6):
        set_g(k)
        if k == 3:
            got.step(1e-3)
        else:
            graph.replay()
        torch.cuda.synchronize()
    assert got.count() == 6 and want.count() == 6
    for a, b in zip(got_p, want_p):
        assert torch.equal(a, b)
    for s, w in zip(got.states, want.states):
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(s, w))
    got.close()
    want.close()


def test_refused_calls():
    pifa, torch = _pifa(), torch_mod()
    p, g = torch.zeros(8, device="cuda"), torch.zeros(8, device="cuda")
    with pytest.raises(pifa.PifaError):
        pifa.AdamW([p, p], [g, g])  # a tensor twice
    with pytest.raises(pifa.PifaError):
        pifa.AdamW([p], [p])  # a gradient in the parameter's place
    with pytest.raises(ValueError):
        pifa.AdamW([p], [g.cpu()])
    with pifa.AdamW([p], [g]) as opt:
        for kw in (dict(lr=-1.0), dict(lr=float("nan")), dict(lr=1.0, beta1=1.0), dict(lr=1.0, beta2=-0.1),
                   dict(lr=1.0, eps=0.0), dict(lr=1.0, step=-1), dict(lr=1.0, eps=1e-60)):
            with pytest.raises(pifa.PifaError):
                opt.step(**kw)
        with pytest.raises(ValueError):
            opt.step(1e-3, grad_scale=torch.ones(1))
        torch.cuda.synchronize()
        assert (p == 0).all() and opt.count() == 0
    with pifa.AdamW([p[:0]], [g[:0]]) as opt:  # nothing to do, counted all the same
        opt.step(1e-3)
        opt.step(1e-3)
        assert opt.count() == 2


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("lr", [1e-6, 3e-7, 1.5e-7, 2e-5])
def test_small_decays_are_right_on_average(lr, bits):
    """lr * decay of 1.5e-8 to 2e-6, near or below the steps of fp32 at 1: over
    many values the decay is the formula's.  p is rounded once, by half a step (2^-24
    of it) at most, up or down as its update falls, which spans many steps: the
    regression of what p lost beside the update on p has an error of deviation 2^-24
    (sum p^4)^1/2 / sum p^2 at most, and six of these are allowed.  The update itself,
    of either sign whatever p is, is good to 8 * 2^-24 of it, likewise."""
    torch = torch_mod()
    c = Case([1, 1 << 20], bits, torch.float32, False, 41)
    g, before = c.g[1].numpy(), c.p[1].astype(np.float64)
    c.opt.step(lr, 0.9, 0.99, 1e-8, step=9)
    torch.cuda.synchronize()
    m, v = o.adamw_moments(g, c.m[1], c.v[1], 0.9, 0.99)
    upd = lr / (1 - 0.9 ** 9) * m.astype(np.float64) / (np.sqrt(v.astype(np.float64) / (1 - 0.99 ** 9)) + 1e-8)
    assert np.median(np.abs(upd) / np.abs(before)) > 16 * STEP
    lost = before - from_dev(c.p_dev[1]) - upd
    got = (before * lost).sum() / (before ** 2).sum()
    off = 6 * STEP * (np.sqrt((before ** 4).sum()) + 8 * np.sqrt((before ** 2 * upd ** 2).sum())) / (before ** 2).sum()
    assert off < 0.05 * lr * c.decay[1] and abs(got - lr * c.decay[1]) <= off, (got, lr * c.decay[1], off)
    c.opt.close()


def test_infinite_parameters_stay_infinite():
    pifa, torch = _pifa(), torch_mod()
    inf = float("inf")
    for decay in (0.0, 0.1):
        p, g = torch.tensor([inf, -inf, 1.0], device="cuda"), torch.ones(3, device="cuda")
        with pifa.AdamW([p], [g], decay) as opt:
            opt.step(1e-3)
            torch.cuda.synchronize()
        assert p[:2].tolist() == [inf, -inf] and abs(float(p[2]) - (1 - 1e-3 * (1 + decay))) <= 2.0 ** -22


def test_a_second_moment_above_zero_stays_above_zero():
    """Beside one that is 2^220 times larger it is less than fp32 holds of the group's units."""
    pifa, torch = _pifa(), torch_mod()
    n = 64
    p, g = torch.ones(n, device="cuda"), torch.full((n,), 1e-15, device="cuda")
    g[3], g[40:] = 1e18, 0.0
    with pifa.AdamW([p], [g], bits=8, seed=5) as opt:
        opt.step(1e-3, 0.9, 0.999, 1e-8, step=2)
        torch.cuda.synchronize()
        _, v = o.adamw_moments(g.cpu().numpy(), np.zeros(n, np.float32), np.zeros(n, np.float32), 0.9, 0.999)
        codes, scales = o.e4m3_round(v, o.random_bits(5, 2, 0, n)[1], 1)
        have = opt.states[0][1].view(torch.uint8).cpu().numpy()
        assert np.array_equal(have, codes) and np.array_equal(opt.states[0][3].cpu().numpy(), scales)
        assert (have[:40] > 0).all() and (have[40:] == 0).all() and have[4] == 1
