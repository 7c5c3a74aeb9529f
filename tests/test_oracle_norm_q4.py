"""Pins of the fp64 norm and 4-bit oracle: closed forms, differences, torch's
8-bit type, and the microscaling format's definition."""
import numpy as np
import pytest

from oracle import norm_q4 as o


def test_norm_closed_forms():
    # a constant row of c has root mean square |c|; eps only matters near zero
    h, y = o.rms_norm(np.full((2, 7), -3.0), np.arange(7.0), 1e-30, np.full((2, 7), 1.0))
    assert np.array_equal(h, np.full((2, 7), -2.0))
    np.testing.assert_allclose(y, np.tile(-np.arange(7.0), (2, 1)), rtol=1e-14)
    _, y = o.rms_norm(np.zeros((1, 5)), None, 1e-6)
    assert np.array_equal(y, np.zeros((1, 5)))
    # scaling a row by a power of two leaves its norm alone (eps aside)
    x = np.random.default_rng(0).standard_normal((3, 33))
    np.testing.assert_allclose(o.rms_norm(x, None, 1e-30)[1], o.rms_norm(8 * x, None, 1e-30)[1], rtol=1e-13)


@pytest.mark.parametrize("with_gain,with_dr", [(True, True), (False, True), (True, False)])
def test_norm_gradient_against_differences(with_gain, with_dr):
    rng = np.random.default_rng(3)
    M, d, eps = 3, 9, 1e-3
    h, dy = rng.standard_normal((M, d)), rng.standard_normal((M, d))
    gain = rng.standard_normal(d) if with_gain else None
    dr = rng.standard_normal((M, d)) if with_dr else None

    def loss(h, g):
        return (o.rms_norm(h, g, eps)[1] * dy).sum() + (0 if dr is None else (h * dr).sum())

    dx, dg = o.rms_norm_backward(h, gain, dy, eps, dr)
    step = 1e-6
    for m in range(M):
        for k in range(d):
            e = np.zeros((M, d))
            e[m, k] = step
            assert abs((loss(h + e, gain) - loss(h - e, gain)) / (2 * step) - dx[m, k]) < 1e-7
    g = np.ones(d) if gain is None else gain
    for k in range(d):
        e = np.zeros(d)
        e[k] = step
        assert abs((loss(h, g + e) - loss(h, g - e)) / (2 * step) - dg[k]) < 1e-7


def test_e4m3_values_are_torchs():
    torch = pytest.importorskip("torch")
    bits = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(bits).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(o.e4m3_value(bits), want)


def test_mx_weights_fields():
    # codes 0..15 in one row's first half, scale 2^(130 - 127); a NaN scale behind it
    codes = np.zeros((1, 32), np.uint8)
    codes[0, :8] = [c | ((c + 1) << 4) for c in range(0, 16, 2)]
    w = o.mx_weights(codes, np.array([[130, 255]], np.uint8))
    assert np.array_equal(w[0, :16], 8 * np.array([0, .5, 1, 1.5, 2, 3, 4, 6, 0, -.5, -1, -1.5, -2, -3, -4, -6]))
    assert np.isnan(w[0, 32:]).all()


def test_mx_candidates_of_representable_and_hard_groups():
    rng = np.random.default_rng(5)
    v = np.concatenate([o.E2M1, -o.E2M1])[rng.integers(0, 16, (4, 64))]
    v[:, ::32] = 6.0  # the group's largest magnitude
    w = v * 2.0 ** -9
    cand, pick = o.mx_candidates(w)
    assert (pick == 0).all() and np.array_equal(cand[0][1], w) and (cand[0][0] == 118).all()
    # one weight just under 8 units: past 6 with the first scale, so the second is closer
    w = np.zeros((1, 32))
    w[0, 3] = 7.9
    cand, pick = o.mx_candidates(w)
    assert pick[0, 0] == 1 and cand[1][1][0, 3] == 8.0 and cand[0][1][0, 3] == 6.0
    # ties to even: 2.5 -> 2, 3.5 -> 4, 5 -> 4, 0.25 -> 0, 0.75 -> 1, 1.75 -> 2
    w = np.zeros((1, 32))
    w[0, :7] = [6, 2.5, 3.5, 5, 0.25, 0.75, 1.75]
    assert np.array_equal(o.mx_candidates(w)[0][0][1][0, :7], [6, 2, 4, 4, 0, 1, 2])
