"""The fp64 forms of layer norms, adapters and AdamW against differences, closed
forms and each other."""
import numpy as np
import pytest

from oracle import tune as o

RNG = np.random.default_rng(5)


def _diff(f, x, v, step=1e-6):
    return (f(x + step * v) - f(x - step * v)) / (2 * step)


def test_layer_norm_rows_have_mean_zero_and_unit_variance():
    x = RNG.standard_normal((7, 50)) * 3 + 11
    _, y = o.layer_norm(x, None, None, 1e-12)
    assert np.abs(y.mean(1)).max() < 1e-12 and np.abs((y * y).mean(1) - 1).max() < 1e-10
    g, b = RNG.standard_normal(50), RNG.standard_normal(50)
    h, z = o.layer_norm(x - 4, g, b, 1e-12, r=np.full_like(x, 4.0))
    assert np.allclose(h, x) and np.allclose(z, y * g + b)
    assert np.allclose(o.layer_norm(x + 100, None, None, 1e-12)[1], y)  # a shift of a row changes nothing


def test_layer_norm_gradients_against_differences():
    x, dy, g, b, dr = (RNG.standard_normal(s) for s in ((4, 9), (4, 9), 9, 9, (4, 9)))
    dx, dg, db = o.layer_norm_backward(x, g, dy, 1e-5)
    for arr, grad, f in ((x, dx, lambda a: (o.layer_norm(a, g, b, 1e-5)[1] * dy).sum()),
                         (g, dg, lambda a: (o.layer_norm(x, a, b, 1e-5)[1] * dy).sum()),
                         (b, db, lambda a: (o.layer_norm(x, g, a, 1e-5)[1] * dy).sum())):
        v = RNG.standard_normal(arr.shape)
        assert abs(_diff(f, arr, v) - (grad * v).sum()) < 1e-7
    assert np.allclose(o.layer_norm_backward(x, g, dy, 1e-5, dr)[0], dx + dr)
    wrong = o.layer_norm_backward(x, g, dy * 1.01, 1e-5)[0]
    assert np.abs(wrong - dx).max() > 1e-4


def test_adapters_are_dense_layers_of_their_rows():
    n, r, d_in, d_out = 4, 3, 11, 7
    A, B, s = RNG.standard_normal((n, r, d_in)), RNG.standard_normal((n, d_out, r)), RNG.random(n) + 0.5
    ids = np.array([2, 0, -1, 2, 9, 0, 2])
    x, y0 = RNG.standard_normal((7, d_in)), RNG.standard_normal((7, d_out))
    y = o.adapter_forward(x, A, B, ids, s, y0)
    for m, a in enumerate(ids):
        want = y0[m] if not 0 <= a < n else y0[m] + s[a] * B[a] @ (A[a] @ x[m])
        assert np.allclose(y[m], want)
    assert np.allclose(o.adapter_forward(x, A, B, ids, s), y - y0)


def test_adapter_gradients_against_differences():
    n, r, d_in, d_out = 3, 2, 5, 6
    A, B, s = RNG.standard_normal((n, r, d_in)), RNG.standard_normal((n, d_out, r)), RNG.random(n) + 0.5
    ids = np.array([2, 0, -1, 2, 0])
    x, dy, dx0 = RNG.standard_normal((5, d_in)), RNG.standard_normal((5, d_out)), RNG.standard_normal((5, d_in))
    dx, dA, dB = o.adapter_backward(x, A, B, ids, dy, s)
    for arr, grad, f in ((x, dx, lambda a: (o.adapter_forward(a, A, B, ids, s) * dy).sum()),
                         (A, dA, lambda a: (o.adapter_forward(x, a, B, ids, s) * dy).sum()),
                         (B, dB, lambda a: (o.adapter_forward(x, A, a, ids, s) * dy).sum())):
        v = RNG.standard_normal(arr.shape)
        assert abs(_diff(f, arr, v) - (grad * v).sum()) < 1e-7
    assert (dA[1] == 0).all() and (dB[1] == 0).all() and (dx[2] == 0).all()
    assert np.allclose(o.adapter_backward(x, A, B, ids, dy, s, dx0)[0], dx + dx0)


def test_adamw_first_step_and_decay():
    p, g = RNG.standard_normal(20), RNG.standard_normal(20)
    z = np.zeros(20)
    p1, m, v = o.adamw(p, g, z, z, 1, 1e-2, 0.9, 0.999, 1e-12, decay=0.5)
    # the first step's moments are the gradient and its square once their bias is off
    assert np.allclose(p1, p * (1 - 1e-2 * 0.5) - 1e-2 * np.sign(g)) and np.allclose(m, 0.1 * g) and np.allclose(v, 1e-3 * g * g)
    same = o.adamw(p, 4 * g, z, z, 1, 1e-2, 0.9, 0.999, 1e-12, decay=0.5, grad_scale=0.25)
    assert all(np.allclose(a, b) for a, b in zip(same, (p1, m, v)))
    m32, v32 = o.adamw_moments(g, z, z, 0.9, 0.999)
    assert m32.dtype == np.float32 and np.allclose(m32, m, rtol=1e-6) and np.allclose(v32, v, rtol=1e-6)


def test_e4m3_codes_and_values():
    assert E4M3_MAX == 448 and np.all(np.diff(o.E4M3_UNITS) > 0)
    # values that have a code keep it, whatever the bits
    for k in (-40, 0, 17):
        x = np.float32(o.E4M3_UNITS[:127] / 512 * 2.0 ** k)
        x = np.concatenate([x, -x, x[-2:]])
        x[::32] = 448 * 2.0 ** k  # the scale of every group
        for b in (0, 65535):
            codes, scales = o.e4m3_round(x, np.full(x.size, b), 0)
            assert (scales == 127 + k).all() and np.array_equal(o.e4m3_values(codes, scales), x)
    # the smallest scale that holds the largest value
    for top, k in ((448.0, 0), (448.1, 1), (224.0, -1), (224.1, 0), (1.0, -8), (1e-45, -126), (0.0, -126), (3e38, 120)):
        assert o.e4m3_round(np.float32([top] * 5), np.zeros(5, np.int64), 0)[1][0] == 127 + k, top
    codes, scales = o.e4m3_round(np.float32([1.0] * 31 + [np.nan] + [2.0] * 40), np.zeros(72, np.int64), 0)
    assert list(scales) == [255, 127 - 7, 127 - 7] and (codes[:32] == 127).all() and np.isnan(o.e4m3_values(codes, scales)[:32]).all()


E4M3_MAX = o.E4M3_UNITS[126] / 512


def test_stochastic_rounding_is_unbiased():
    """The mean of many roundings: within 6 deviations of the value, and above
    zero nothing becomes zero where that is asked."""
    n = 1 << 16
    bits, other = o.random_bits(7, 3, 2, n)
    assert abs(bits.mean() - 32767.5) < 6 * 18919 / np.sqrt(n) and abs(other.mean() - 32767.5) < 6 * 18919 / np.sqrt(n)
    assert abs(np.corrcoef(bits, other)[0, 1]) < 6 / np.sqrt(n) and abs(np.corrcoef(bits[1:], bits[:-1])[0, 1]) < 6 / np.sqrt(n)
    assert len(np.unique(bits)) > 0.6 * 65536  # 1 - 1/e of them
    for value in (300.0, 3.3, 0.1, 2.0 ** -9 * 0.3):
        x = np.full(n, value, np.float32)
        x[::32] = 448.0
        codes, scales = o.e4m3_round(x, bits, 0)
        got = o.e4m3_values(codes, scales)[np.arange(n) % 32 != 0].astype(np.float64)
        assert len(np.unique(got)) == 2
        assert abs(got.mean() - value) < 6 * got.std() / np.sqrt(got.size)
        codes, _ = o.e4m3_round(x, bits, 1)
        assert (codes > 0).all()


@pytest.mark.parametrize("beta2", [0.95, 0.999])
def test_moments_in_8_bits_follow_those_in_64(beta2):
    """2000 steps of noise with a scale that drops on the way: v stays within its
    expected spread; rounded to nearest it would not move."""
    rng = np.random.default_rng(9)
    n = 32 * 64
    codes, scales = np.zeros(n, np.uint8), np.zeros(n // 32, np.uint8)
    v64 = np.zeros(n)
    for t in range(1, 2001):
        g = rng.standard_normal(n) * (1.0 if t < 500 else 0.2)
        v64 = beta2 * v64 + (1 - beta2) * g * g
        v = np.float32(beta2) * o.e4m3_values(codes, scales) + np.float32(1 - beta2) * np.float32(g * g)
        codes, scales = o.e4m3_round(v, o.random_bits(1, t, 0, n)[1], 1)
    ratio = o.e4m3_values(codes, scales) / v64
    # deviation 0.2 of v by element; the mean over 2048 of them, 8 deviations of it
    assert abs(ratio.mean() - 1) < 8 * 0.25 / np.sqrt(n) + 0.02 and ratio.std() < 0.4 and ratio.min() > 0.1


@pytest.mark.parametrize("beta2,steps", [(0.95, 400), (0.999, 3000)])
def test_small_second_moments_in_a_group_with_a_large_one(beta2, steps):
    """v of 1e-2 to 1e-4 of its group's largest is right on average; from about a unit
    of the group (the smallest code) down it stays at one."""
    rng = np.random.default_rng(9)
    groups, share = 128, np.array([1e-2, 1e-3, 1e-4, 1e-6, 1e-8])
    kind = np.tile(np.concatenate([[-1], np.arange(30) % 5, [-1]]), groups)
    size = np.where(kind < 0, 1.0, np.sqrt(share[kind]))
    n = size.size
    codes, scales, v64 = np.zeros(n, np.uint8), np.zeros(groups, np.uint8), np.zeros(n)
    got, want, units = np.zeros(n), np.zeros(n), np.zeros(n)
    for t in range(1, steps + 1):
        g = rng.standard_normal(n) * size
        v64 = beta2 * v64 + (1 - beta2) * g * g
        v = np.float32(beta2) * o.e4m3_values(codes, scales) + np.float32(1 - beta2) * np.float32(g * g)
        codes, scales = o.e4m3_round(v, o.random_bits(1, t, 0, n)[1], 1)
        if 2 * t > steps:
            have = o.e4m3_values(codes, scales).astype(np.float64)
            got, want = got + have, want + v64
            units += have / 2.0 ** (np.repeat(scales.astype(float), 32) - 127 - 9) / (steps - steps // 2)
    for k in range(3):  # 768 values, deviation 0.2 each: six of the mean's
        assert abs(got[kind == k].sum() / want[kind == k].sum() - 1) < 6 * 0.2 / np.sqrt(768), share[k]
    for k in (3, 4):
        assert (units[kind == k] >= 1).all() and units[kind == k].mean() < 2, share[k]
        assert got[kind == k].sum() > 3 * want[kind == k].sum()
