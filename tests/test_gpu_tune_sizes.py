"""Layer norm, adapters and AdamW on tensors of more than 2^31 values: offsets that
do not fit 32 bits.  Rows and values are independent of each other, so what lies
behind the border has the bits of a call of its own."""
from __future__ import annotations

import pytest

from gpu_util import torch_mod

pytestmark = pytest.mark.gpu

EPS = 1e-5


@pytest.fixture(autouse=True)
def _cuda():
    torch = torch_mod()
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


def _pifa():
    from paper_2501_19090_amd import pifa
    return pifa


def test_layer_norm():
    pifa, torch = _pifa(), torch_mod()
    M, d = 2 ** 18 + 3, 8200
    assert M * d > 2 ** 31
    rng = torch.Generator(device="cuda").manual_seed(1)
    make = lambda *s: torch.randn(*s, device="cuda", dtype=torch.bfloat16, generator=rng)
    X, R, g, b = make(M, d), make(M, d), make(d), make(d)
    H = torch.empty_like(X)
    Y = pifa.layer_norm_forward(X, g, b, EPS, R=R, H=H)
    rows = torch.tensor([0, 1, 2 ** 31 // d - 1, 2 ** 31 // d, 2 ** 31 // d + 1, M - 2, M - 1], device="cuda")
    # more than 256 rows, so that both calls take the same number of threads a row
    many = rows.repeat(40)
    h = torch.empty(len(many), d, device="cuda", dtype=torch.bfloat16)
    y = pifa.layer_norm_forward(X[many], g, b, EPS, R=R[many], H=h)
    torch.cuda.synchronize()
    assert torch.equal(Y[many], y) and torch.equal(H[many], h)
    del X, R
    dY, dR = Y.zero_(), make(M, d)
    dY[M - 1] = make(d)
    dX, dgain, dbias = pifa.layer_norm_backward(H, g, dY, EPS, dR=dR)
    dx, dgain1, dbias1 = pifa.layer_norm_backward(H[rows], g, dY[rows], EPS, dR=dR[rows])
    torch.cuda.synchronize()
    assert torch.equal(dX[rows], dx)  # the other rows' gradients add zeros to the sums
    assert torch.equal(dgain, dgain1) and torch.equal(dbias, dbias1)


def test_adapters():
    pifa, torch = _pifa(), torch_mod()
    M, d_in, d_out, r, n = 2 ** 18 + 9, 8200, 24, 4, 2
    assert M * d_in > 2 ** 31
    rng = torch.Generator(device="cuda").manual_seed(2)
    make = lambda *s: torch.randn(*s, device="cuda", dtype=torch.bfloat16, generator=rng)
    X, A, B, Y0, dY, dX0 = make(M, d_in), make(n, r, d_in) * 2 ** -6, make(n, d_out, r), make(M, d_out), make(M, d_out), make(M, d_in)
    ids = torch.randint(-1, n, (M,), device="cuda", dtype=torch.int32, generator=rng)
    plan = pifa.AdapterPlan(ids, n)
    Y = pifa.adapter_forward(X, A, B, plan, Y0=Y0)
    dX, dA, dB = pifa.adapter_backward(X, A, B, plan, dY, dX0=dX0)
    torch.cuda.synchronize()
    fp = 2.0 ** -17
    want, size = ([torch.zeros_like(A, dtype=torch.float64), torch.zeros_like(B, dtype=torch.float64)] for _ in range(2))
    for m in range(0, M, 16384):
        i = slice(m, min(m + 16384, M))
        x, y0, dy, dx0 = (v[i].double() for v in (X, Y0, dY, dX0))
        near = lambda got, w, z, rounded: ((got.double() - w).abs() <= (2.0 ** -8 * w.abs() if rounded else 0) + 4 * fp * z + 1e-30).all()
        y, ys, dx, dxs = y0.clone(), y0.abs(), dx0.clone(), dx0.abs()
        for a in range(n):
            mine = (ids[i] == a).double()[:, None]
            Aa, Ba = A[a].double(), B[a].double()
            t, ts = mine * (x @ Aa.T.contiguous()), mine * (x.abs() @ Aa.abs().T.contiguous())
            u, us = mine * (dy @ Ba), mine * (dy.abs() @ Ba.abs())
            y += t @ Ba.T.contiguous()
            ys += ts @ Ba.abs().T.contiguous()
            dx += u @ Aa
            dxs += us @ Aa.abs()
            want[0][a] += u.T.contiguous() @ x
            size[0][a] += us.T.contiguous() @ x.abs()
            want[1][a] += dy.T.contiguous() @ t
            size[1][a] += dy.abs().T.contiguous() @ ts
        assert near(Y[i], y, ys, True) and near(dX[i], dx, dxs, True), m
    # on a product's way: 32 additions in its instruction, 5 instructions, 8 waves and at
    # most 250 pieces of 512 rows, so 2 FP of the terms' magnitudes; t and u add FP
    for got, w, z in zip((dA, dB), want, size):
        assert ((got.double() - w).abs() <= 3 * fp * z).all()


def test_adamw():
    pifa, torch = _pifa(), torch_mod()
    n, tail = 2 ** 31 + 4101, 10000
    p = torch.linspace(-1, 1, n, device="cuda")
    g = torch.full((n,), 0.25, device="cuda", dtype=torch.bfloat16)
    m, v = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    g[-tail:] = torch.randn(tail, device="cuda").bfloat16()
    v[-tail:] = torch.rand(tail, device="cuda")
    part = [t[-tail:].clone() for t in (p, g, m, v)]
    with pifa.AdamW([p], [g], 0.1, states=[(m, v)]) as whole, pifa.AdamW([part[0]], [part[1]], 0.1, states=[tuple(part[2:])]) as end:
        whole.step(1e-2)
        end.step(1e-2)
        torch.cuda.synchronize()
    for got, want in zip((p, m, v), (part[0], part[2], part[3])):
        assert torch.equal(got[-tail:], want)
    assert bool((m[:-tail] != 0).all()) and bool((v[:-tail] != 0).all())
