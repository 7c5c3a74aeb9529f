"""4-bit layers against the fp64 product of the weights their codes stand for.

Tolerances, element by element.  An output is rounded once to bf16: 2^-8 of it.
fp32 sums: K / 32 additions of at most 2^-23 of the terms' magnitudes so far on
the way of one term (fewer: the K range is split over waves), 2^-15 of the sum of
magnitudes at K = 8192.  A 16x16x128 step of 8-bit rows cuts the 32 products
of a group off at 2^-14 of the largest: 32 * 2^-14 = 2^-9 of the product of the
group's largest value in the row and in the weights.  The norm's form rounds its rows to bf16 first: 2^-8 of every term,
which adds up to at most 2^-8 of the sum of magnitudes.
"""
import os
import re

import numpy as np
import pytest

from oracle import norm_q4 as o
from paper_2501_19090_amd import inputs

from gpu_util import from_dev, rel_fro, to_dev, torch_mod

pytestmark = pytest.mark.gpu

EPS = 1e-5
SUMS = 2.0 ** -15
SHAPES = [(32, 1), (32, 16), (64, 17), (96, 40), (128, 63), (160, 64), (256, 1000), (512, 130), (1024, 333), (2048, 256),
          (4096, 97), (11008, 48)]
ROWS = [1, 2, 7, 16, 17, 33, 64, 65, 130, 257, 500]


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch_mod().cuda.is_available():
        pytest.skip("no GPU")


def _pifa():
    from paper_2501_19090_amd import pifa
    return pifa


def _codes(d_in, d_out, seed, spread=4):
    """Random codes and scales 2^-spread .. 2^spread around 1 / sqrt(d_in), and the weights they stand for."""
    rng = np.random.default_rng([seed, d_in, d_out])
    codes = rng.integers(0, 256, (d_out, d_in // 2), dtype=np.uint8)
    mid = 127 - int(np.log2(d_in) / 2)
    scales = rng.integers(mid - spread, mid + spread + 1, (d_out, d_in // 32)).astype(np.uint8)
    return codes, scales, o.mx_weights(codes, scales)


def _dev(a):
    return torch_mod().from_numpy(np.ascontiguousarray(a)).cuda()


def _layer(d_in, d_out, seed, spread=4):
    codes, scales, w = _codes(d_in, d_out, seed, spread)
    return _pifa().Q4Layer.from_mx(_dev(codes), _dev(scales)), w


def _x(M, d_in, seed):
    st, x = inputs.round_to(np.random.default_rng([seed, M, d_in]).standard_normal((M, d_in)), "bf16")
    return to_dev(st), x


def _check(got, want, mags, frac, what):
    got = from_dev(got)
    assert np.isfinite(got).all(), what
    off = np.abs(got - want) - (np.abs(want) * 2.0 ** -8 + mags * frac)
    assert (off <= 0).all(), (what, float(off.max()), np.unravel_index(off.argmax(), off.shape))


def _guarded(M, N):
    torch = torch_mod()
    big = torch.full((M * N + 64,), -17.0, dtype=torch.bfloat16, device="cuda")
    return big, big[:M * N].view(M, N)


@pytest.mark.parametrize("shape", SHAPES)
def test_forward(shape):
    torch = torch_mod()
    d_in, d_out = shape
    layer, w = _layer(d_in, d_out, 1)
    with layer:
        for M in ROWS:
            x_dev, x = _x(M, d_in, 2)
            big, Y = _guarded(M, d_out)
            layer(x_dev, Y)
            torch.cuda.synchronize()
            _check(Y, x @ w.T, np.abs(x) @ np.abs(w).T, SUMS, (shape, M))
            assert (big[M * d_out:] == -17).all()


@pytest.mark.parametrize("shape", SHAPES)
def test_forward_e4m3(shape):
    torch = torch_mod()
    d_in, d_out = shape
    layer, w = _layer(d_in, d_out, 3)
    with layer:
        for M in ROWS:
            rng = np.random.default_rng([4, M, d_in])
            q = rng.integers(0, 256, (M, d_in)).astype(np.uint8)
            q[(q & 127) == 127] = 0
            s = (2.0 ** rng.uniform(-12, 4, M)).astype(np.float32)
            x = o.e4m3_value(q)
            big, Y = _guarded(M, d_out)
            layer.forward_e4m3(_dev(q).view(torch.float8_e4m3fn), _dev(s), Y)
            torch.cuda.synchronize()
            f = s.astype(np.float64)[:, None]
            top = lambda a: np.abs(a).reshape(a.shape[0], -1, 32).max(axis=2)
            cut = 2.0 ** -9 * (top(x) @ top(w).T) + SUMS * (np.abs(x) @ np.abs(w).T)
            _check(Y, f * (x @ w.T), f * cut, 1.0, (shape, M))
            assert (big[M * d_out:] == -17).all()


@pytest.mark.parametrize("M,d_in,d_out", [
    (18, 96, 20), (2054, 96, 33), (2080, 1120, 33), (34, 96, 4114), (65, 544, 8310), (65, 2080, 8308), (2090, 2080, 386),
    (33, 96, 8200), (33, 352, 8576), (196, 224, 12524), (129, 96, 10963), (259, 96, 13206), (267, 32, 13064),
    (521, 96, 13453), (778, 96, 14177), (708, 2080, 10990), (2050, 96, 8100), (300, 64, 60000)])
def test_every_tile(M, d_in, d_out):
    """Sizes at which each of the tiles is the one picked, in bf16, e4m3 or both:
    16 x 32, 32 x 32, 32 x 64, 32 x 128, 64 x 64 (both depths), 64 x 128, 128 x
    128 (both forms), 128 x 256 and 256 x 256, all with ragged ends (fp64 on the
    GPU: the products are large)."""
    torch = torch_mod()
    layer, w = _layer(d_in, d_out, 31)
    with layer:
        x_dev, _ = _x(M, d_in, 32)
        q = x_dev.float().to(torch.float8_e4m3fn)
        s = torch.rand(M, device="cuda") + 0.5
        wd = _dev(w)
        top = lambda a: a.abs().view(a.shape[0], -1, 32).amax(2)
        for x, f, run in ((x_dev.double(), 1.0, lambda Y: layer(x_dev, Y)),
                          (q.double(), s.double()[:, None], lambda Y: layer.forward_e4m3(q, s, Y))):
            big, Y = _guarded(M, d_out)
            run(Y)
            want = f * (x @ wd.t().contiguous())
            mags = SUMS * (x.abs() @ wd.abs().t().contiguous())
            if torch.is_tensor(f):
                mags = f * (mags + 2.0 ** -9 * (top(x) @ top(wd).t().contiguous()))
            off = (Y.double() - want).abs() - want.abs() * 2.0 ** -8 - mags
            assert torch.isfinite(Y).all() and float(off.max()) <= 0, (M, d_in, d_out, float(off.max()))
            assert (big[M * d_out:] == -17).all()


@pytest.mark.parametrize("with_r,with_gain,with_h", [(True, True, True), (False, True, False), (True, False, True),
                                                     (False, False, True)])
@pytest.mark.parametrize("shape", [(32, 5), (96, 40), (1024, 333), (4096, 97)])
def test_norm_forward(shape, with_r, with_gain, with_h):
    torch = torch_mod()
    d_in, d_out = shape
    layer, w = _layer(d_in, d_out, 5)
    g_st, g = inputs.round_to(1.0 + 0.3 * np.random.default_rng(6).standard_normal((1, d_in)), "bf16")
    g_dev = to_dev(g_st).reshape(-1) if with_gain else None
    with layer:
        for M in (1, 3, 7, 16, 17, 90):
            x_dev, x = _x(M, d_in, 7)
            r_dev, r = _x(M, d_in, 8) if with_r else (None, None)
            h, y = o.rms_norm(x, g[0] if with_gain else None, EPS, r)
            big, Y = _guarded(M, d_out)
            hbig, H = _guarded(M, d_in) if with_h else (None, None)
            layer.norm_forward(x_dev, g_dev, EPS, R=r_dev, H=H, Y=Y)
            torch.cuda.synchronize()
            mags = np.abs(y) @ np.abs(w).T
            _check(Y, y @ w.T, mags, 2.0 ** -8 + 2 * SUMS, (shape, M))
            assert rel_fro(from_dev(Y), y @ w.T) < 5e-3  # both roundings are 1.7e-3 rms
            assert (big[M * d_out:] == -17).all()
            if with_h:
                off = np.abs(from_dev(H) - h) - np.abs(h) * (2.0 ** -8 + 2.0 ** -24)
                assert (off <= 2.0 ** -126).all() and (hbig[M * d_in:] == -17).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(32, 1), (96, 40), (1024, 77)])
def test_quantized_weights(shape, dtype):
    """q4_layer_create against both candidates of every group: the weights are
    one candidate's, to the bit, and the better one's unless their errors are
    nearly the same (fp32 sums of 32 squares: 2^-18)."""
    pifa, torch = _pifa(), torch_mod()
    d_in, d_out = shape
    rng = np.random.default_rng([9, d_in])
    w = rng.standard_normal((d_out, d_in)) * 2.0 ** rng.integers(-20, 20, (d_out, d_in // 32)).repeat(32, axis=1)
    w[0, :32] = 0.0
    st, w = inputs.round_to(w, dtype)
    with pifa.Q4Layer(to_dev(st)) as layer:
        codes, scales = (t.cpu().numpy() for t in layer.read())
        # read, made again from what was read, and read again: the same bytes
        with pifa.Q4Layer.from_mx(_dev(codes), _dev(scales)) as again:
            c2, s2 = (t.cpu().numpy() for t in again.read())
        x_dev, x = _x(3, d_in, 10)
        Y = layer(x_dev)
        torch.cuda.synchronize()
    assert np.array_equal(codes, c2) and np.array_equal(scales, s2)
    got = o.mx_weights(codes, scales)
    _check(Y, x @ got.T, np.abs(x) @ np.abs(got).T, SUMS, "product")
    cand, pick = o.mx_candidates(w)
    for c in range(2):
        took = scales == cand[c][0]
        rows = np.repeat(took, 32, axis=1)
        assert np.array_equal(got[rows], cand[c][1][rows])
        worse = took & (pick != c) & (cand[0][0] != cand[1][0])
        assert (np.abs(cand[0][2] - cand[1][2])[worse] <= 2.0 ** -18 * cand[0][2][worse]).all()
    assert ((scales == cand[0][0]) | (scales == cand[1][0])).all()
    assert scales[0, 0] == 127 and (codes[0, :16] & 0x77 == 0).all()


def test_quantizing_ends_of_the_range():
    pifa, torch = _pifa(), torch_mod()
    w = np.zeros((6, 32), np.float32)
    w[0, 0], w[1, 1], w[2, 2] = np.inf, np.nan, 3.4e38
    w[3, 3] = 2.0 ** -126
    w[4, 4] = 2.0 ** -149
    w[5] = 2.0 ** -120
    with pifa.Q4Layer(_dev(w)) as layer:
        codes, scales = (t.cpu().numpy() for t in layer.read())
        x = torch.ones(1, 32, dtype=torch.bfloat16, device="cuda")
        y = from_dev(layer(x))[0]
        q = torch.ones(1, 32, device="cuda").to(torch.float8_e4m3fn)
        y8 = from_dev(layer.forward_e4m3(q, torch.ones(1, device="cuda")))[0]
    v = o.mx_weights(codes, scales)
    assert scales[0, 0] == 255 and scales[1, 0] == 255 and np.isnan(v[:2]).all()
    assert abs(v[2, 2] / 3.4e38 - 1) <= 0.25 and np.count_nonzero(v[2]) == 1
    assert abs(v[3, 3] * 2.0 ** 126 - 1) <= 0.25 and (v[4] == 0).all()
    assert np.array_equal(v[5], w[5].astype(np.float64))
    for got in (y, y8):
        assert np.isnan(got[:2]).all() and got[4] == 0
        assert abs(got[5] / 2.0 ** -115 - 1) <= 2.0 ** -8


def test_nan_and_infinite_rows_stay_in_their_rows():
    torch = torch_mod()
    d_in, d_out = 224, 50
    layer, w = _layer(d_in, d_out, 11)
    with layer:
        for M in (5, 16, 40, 80, 300):
            x_dev, x = _x(M, d_in, 12)
            bad = x_dev.clone()
            bad[1, 3], bad[M - 1, 223] = float("nan"), float("inf")
            good, got = from_dev(layer(x_dev)), from_dev(layer(bad))
            keep = [m for m in range(M) if m not in (1, M - 1)]
            assert np.array_equal(good[keep], got[keep])
            assert np.isnan(got[1]).all() and not np.isfinite(got[M - 1][w[:, 223] != 0]).any()
            q = x_dev.float().to(torch.float8_e4m3fn)
            s = torch.ones(M, device="cuda")
            ref = from_dev(layer.forward_e4m3(q, s))
            qb = q.view(torch.uint8).clone()
            qb[1, 100] = 0x7F
            got = from_dev(layer.forward_e4m3(qb.view(torch.float8_e4m3fn), s))
            keep = [m for m in range(M) if m != 1]
            assert np.isnan(got[1]).all() and np.array_equal(ref[keep], got[keep])


def test_last_rows_of_a_batch_are_all_that_is_read():
    """Rows behind the last one are neither read nor written: the buffers end there."""
    torch = torch_mod()
    d_in, d_out = 352, 30
    layer, w = _layer(d_in, d_out, 13)
    with layer:
        for M in (1, 15, 31, 63, 200):
            big = torch.full(((M + 300) * d_in,), float("nan"), dtype=torch.bfloat16, device="cuda")
            x_dev, x = _x(M, d_in, 14)
            big[:M * d_in] = x_dev.reshape(-1)
            Ybig, Y = _guarded(M, d_out)
            layer(big[:M * d_in].view(M, d_in), Y)
            torch.cuda.synchronize()
            _check(Y, x @ w.T, np.abs(x) @ np.abs(w).T, SUMS, M)
            assert (Ybig[M * d_out:] == -17).all()


def test_a_block_end_to_end():
    """Residual, norm and layer as a block runs them: apart, in one call, and
    with 8-bit rows; the three agree within their roundings."""
    pifa, torch = _pifa(), torch_mod()
    d, ff = 1024, 2752
    w = np.random.default_rng(15).standard_normal((ff, d)) / 32
    g_dev = (1 + 0.2 * torch.randn(d, device="cuda")).to(torch.bfloat16)
    with pifa.Q4Layer(to_dev(inputs.round_to(w, "bf16")[0])) as layer:
        wq = o.mx_weights(*(t.cpu().numpy() for t in layer.read()))
        # 4-bit weights of a normal matrix: 11.7% off; its product as much
        assert rel_fro(wq, w) < 0.13
        for M in (1, 12, 40, 300):
            x_dev, x = _x(M, d, 16)
            r_dev, r = _x(M, d, 17)
            H, H2, H3 = (torch.empty_like(x_dev) for _ in range(3))
            apart = layer(pifa.rms_norm_forward(x_dev, g_dev, EPS, R=r_dev, H=H))
            one = layer.norm_forward(x_dev, g_dev, EPS, R=r_dev, H=H2)
            q, s = pifa.rms_norm_forward_e4m3(x_dev, g_dev, EPS, R=r_dev, H=H3)
            eight = layer.forward_e4m3(q, s)
            torch.cuda.synchronize()
            assert torch.equal(H, H2) and torch.equal(H, H3)
            _, y = o.rms_norm(x, from_dev(g_dev), EPS, r)
            want = y @ wq.T
            assert rel_fro(from_dev(apart), want) < 5e-3 and rel_fro(from_dev(one), want) < 5e-3
            assert rel_fro(from_dev(eight), want) < 2.0 ** -4  # half a step of e4m3, at most
            if M > 16:
                assert torch.equal(apart, one)


def test_trained_pifa_block():
    """norm -> PIFA layer and back: the norm's gradient takes the layer's dX."""
    import oracle
    pifa, torch = _pifa(), torch_mod()
    d_in, d_out, r, M = 256, 320, 96, 40
    U, V = inputs.lowrank_factors(d_out, d_in, r, seed=7)
    lay = oracle.build_pifa(U @ V, r)
    wp_st, wp = inputs.round_to(lay["Wp"], "bf16")
    c_st, c = inputs.round_to(lay["C"], "bf16")
    x_dev, x = _x(M, d_in, 18)
    r_dev, res = _x(M, d_in, 19)
    g_st, g = inputs.round_to(1.0 + 0.3 * np.random.default_rng(20).standard_normal((1, d_in)), "bf16")
    g_dev = to_dev(g_st).reshape(-1)
    dy_st, dy = inputs.round_to(0.1 * np.random.default_rng(21).standard_normal((M, d_out)), "bf16")
    with pifa.PifaLayer(to_dev(wp_st), to_dev(c_st), lay["pivot_idx"], lay["nonpivot_idx"], d_out) as layer:
        H = torch.empty_like(x_dev)
        N = pifa.rms_norm_forward(x_dev, g_dev, EPS, R=r_dev, H=H)
        Y = layer(N)
        dN, dH = torch.empty_like(N), torch.empty_like(N)
        pifa.pifa_layer_backward(layer.handle, N, Y, to_dev(dy_st), dX=dN)
        _, dg = pifa.rms_norm_backward(H, g_dev, dN, EPS, dR=r_dev, dX=dH)
        torch.cuda.synchronize()
    W = np.zeros((d_out, d_in))
    W[lay["pivot_idx"]], W[lay["nonpivot_idx"]] = wp, c @ wp
    h, n = o.rms_norm(x, g[0], EPS, res)
    want, dgain = o.rms_norm_backward(h, g[0], dy @ W, EPS, res)
    assert rel_fro(from_dev(Y), n @ W.T) < 1e-2   # the layer's bar, its input rounded as well
    assert rel_fro(from_dev(dH), want) < 1e-2 and rel_fro(from_dev(dg), dgain) < 1e-2


def test_no_rows_and_refused_calls():
    pifa, torch = _pifa(), torch_mod()
    layer, _ = _layer(64, 24, 22)
    bf = torch.bfloat16
    with layer:
        assert layer(torch.empty(0, 64, dtype=bf, device="cuda")).shape == (0, 24)
        x, y = torch.zeros(40, 64, dtype=bf, device="cuda"), torch.zeros(40, 24, dtype=bf, device="cuda")
        assert layer.norm_forward(x[:0], None, EPS).shape == (0, 24)
        with pytest.raises(ValueError):
            layer(x[:, :32].contiguous(), y)  # too short
        with pytest.raises(ValueError):
            layer(x, y[:39])
        with pytest.raises(TypeError):
            layer(x.float(), y)
        with pytest.raises(ValueError):
            layer(x.cpu(), y)
        flat = torch.zeros(40 * 64 + 8, dtype=bf, device="cuda")
        with pytest.raises(pifa.PifaError) as e:
            layer(flat[1:40 * 64 + 1].view(40, 64), y)  # not on 16 bytes
        assert e.value.status == pifa.PIFA_ERR_UNSUPPORTED
        for H in (x, y.view(-1)[:24 * 40]):
            with pytest.raises((pifa.PifaError, ValueError)):
                layer.norm_forward(x, None, EPS, H=H, Y=y)
        with pytest.raises(pifa.PifaError):
            layer.norm_forward(x, None, 0.0)
        assert pifa.q4_layer_weight_bytes(layer.handle) == 24 * (32 + 2)
    codes, scales = torch.zeros(4, 20, dtype=torch.uint8, device="cuda"), torch.zeros(4, 2, dtype=torch.uint8, device="cuda")
    with pytest.raises(pifa.PifaError) as e:
        pifa.Q4Layer.from_mx(codes, scales)  # d_in 40
    assert e.value.status == pifa.PIFA_ERR_UNSUPPORTED
    with pytest.raises(ValueError):
        pifa.Q4Layer.from_mx(torch.zeros(4, 32, dtype=torch.uint8, device="cuda"), scales[:2])


def test_captured_and_replayed_beside_eager_work():
    """Graphs of every form, for few and many rows, replayed on new inputs with
    eager calls and a growing workspace between."""
    pifa, torch = _pifa(), torch_mod()
    d_in, d_out = 512, 200
    layer, w = _layer(d_in, d_out, 23)
    g = (1 + 0.2 * torch.randn(d_in, device="cuda")).to(torch.bfloat16)
    with layer:
        fresh, _ = _layer(d_in, d_out, 23)
        for M in (3, 50, 300):
            x, r = (torch.randn(M, d_in, device="cuda").to(torch.bfloat16) for _ in range(2))
            q, s = torch.empty(M, d_in, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(M, device="cuda")
            outs = [torch.empty(M, d_out, dtype=torch.bfloat16, device="cuda") for _ in range(3)]
            H = torch.empty_like(x)
            layer.reserve(M)

            def calls(lay, outs, H, q, s):
                lay(x, outs[0])
                pifa.rms_norm_forward_e4m3(x, g, EPS, R=r, Q=q, scale=s)
                lay.forward_e4m3(q, s, outs[1])
                lay.norm_forward(x, g, EPS, R=r, H=H, Y=outs[2])

            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.stream(side):
                calls(layer, outs, H, q, s)
                side.synchronize()
                with torch.cuda.graph(graph, stream=side):
                    calls(layer, outs, H, q, s)
            # the workspace grows behind the graph's back: what it captured stays valid
            layer.reserve(4 * M + 100)
            for i in range(3):
                for t in (x, r):
                    t.copy_(torch.randn(M, d_in, device="cuda"))
                for t in outs:
                    t.fill_(float("nan"))
                graph.replay()
                torch.cuda.synchronize()
                o2, H2 = [torch.empty_like(t) for t in outs], torch.empty_like(H)
                calls(fresh, o2, H2, torch.empty_like(q), torch.empty_like(s))
                torch.cuda.synchronize()
                assert torch.equal(H, H2), (M, i)
                for a, b in zip(outs, o2):
                    assert torch.equal(a, b), (M, i)
        fresh.close()


def test_capture_does_not_grow_the_workspace():
    pifa, torch = _pifa(), torch_mod()
    layer, _ = _layer(64, 24, 24)
    with layer:
        x, y = torch.zeros(40, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(40, 24, dtype=torch.bfloat16, device="cuda")
        side = torch.cuda.Stream()
        graph = torch.cuda.CUDAGraph()
        status = None
        with torch.cuda.stream(side):
            with torch.cuda.graph(graph, stream=side):
                y.add_(1)
                try:
                    layer.norm_forward(x, None, EPS, Y=y)
                except pifa.PifaError as e:
                    status = e.status
        assert status == pifa.PIFA_ERR_TOO_LARGE
        layer.reserve(40)
        layer.norm_forward(x, None, EPS, Y=y)
        torch.cuda.synchronize()
        assert (y == 0).all()


def test_two_streams_at_once():
    """Products of one layer need no workspace: calls on two streams may overlap."""
    torch = torch_mod()
    layer, w = _layer(1024, 512, 25)
    with layer:
        xs = [_x(M, 1024, 26 + M) for M in (4, 100)]
        want = [layer(x) for x, _ in xs]
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream() for _ in xs]
        outs = [torch.empty_like(t) for t in want]
        for _ in range(10):
            for st, (x, _), y in zip(streams, xs, outs):
                with torch.cuda.stream(st):
                    layer(x, y)
        torch.cuda.synchronize()
        for a, b in zip(outs, want):
            assert torch.equal(a, b)


@pytest.mark.parametrize("M,d_in,d_out", [(16, 4096, 16400), (13, 8192, 16387), (9, 8160, 20000), (12, 4096, 16400)])
def test_wide_outputs_of_few_rows(M, d_in, d_out):
    """More than 1024 groups of 16 columns: tiles of 16 x 128 above 49152 elements
    of X, the form of few rows at just as many, ragged in every direction."""
    torch = torch_mod()
    layer, w = _layer(d_in, d_out, 41)
    with layer:
        x, _ = _x(M, d_in, 42)
        wd = _dev(w)
        big, Y = _guarded(M, d_out)
        layer(x, Y)
        want = x.double() @ wd.t().contiguous()
        mags = SUMS * (x.double().abs() @ wd.abs().t().contiguous())
        off = (Y.double() - want).abs() - want.abs() * 2.0 ** -8 - mags
        assert torch.isfinite(Y).all() and float(off.max()) <= 0, float(off.max())
        torch.cuda.synchronize()
        assert bool((big[M * d_out:] == -17).all())


@pytest.mark.parametrize("M", [1, 40])
def test_outputs_over_inputs_are_refused(M):
    """Y over an input (each by one element at its end) is refused, next to it is not."""
    torch, pifa = torch_mod(), _pifa()
    d = 256
    layer, _ = _layer(d, d, 51)
    n = M * d
    with layer:
        layer.reserve(M)
        buf = torch.zeros(4 * n + d, dtype=torch.bfloat16, device="cuda")
        lib, h, at = pifa.lib(), layer.handle, lambda i: buf.data_ptr() + 2 * i
        inval = pifa.PIFA_ERR_INVALID_ARG
        norm = lambda X, R, g, Y: lib.q4_layer_norm_forward(h, at(X), R and at(R), g and at(g), EPS, None, at(Y), M, None)
        assert lib.q4_layer_forward(h, at(0), at(n - 1), M, None) == inval
        assert lib.q4_layer_forward(h, at(n), at(1), M, None) == inval
        assert lib.q4_layer_forward(h, at(0), at(n), M, None) == pifa.PIFA_OK
        scale = torch.ones(M, device="cuda")
        assert lib.q4_layer_forward_e4m3(h, at(0), scale.data_ptr(), at(n // 2 - 1), M, None) == inval
        assert lib.q4_layer_forward_e4m3(h, at(2 * n), at(n - 2), at(0), M, None) == inval
        assert lib.q4_layer_forward_e4m3(h, at(0), scale.data_ptr(), at(n // 2), M, None) == pifa.PIFA_OK
        assert norm(0, None, None, 0) == inval and norm(0, None, None, n - 1) == inval
        assert norm(0, n, None, 2 * n - 1) == inval and norm(0, n, 3 * n, 3 * n + d - 1) == inval
        assert norm(0, n, 3 * n, 2 * n) == pifa.PIFA_OK
        torch.cuda.synchronize()


@pytest.mark.parametrize("M,d_in,d_out", [((1 << 19) + 21, 32, 3), (65, 32, (1 << 26) + 5)])
def test_more_than_one_launch(M, d_in, d_out):
    """Rows behind the first slice of a call, and slices of few rows of many outputs."""
    torch, pifa = torch_mod(), _pifa()
    rng = torch.Generator(device="cuda").manual_seed(5)
    codes = torch.randint(0, 256, (d_out, d_in // 2), dtype=torch.uint8, device="cuda", generator=rng)
    scales = torch.full((d_out, d_in // 32), 125, dtype=torch.uint8, device="cuda")
    x = torch.randn(M, d_in, device="cuda", generator=rng).bfloat16()
    q, s = x.float().to(torch.float8_e4m3fn), torch.rand(M, device="cuda", generator=rng) + 0.5
    grid = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64, device="cuda")
    with pifa.Q4Layer.from_mx(codes, scales) as layer:
        for out, X, f in ((layer(x), x, None), (layer.forward_e4m3(q, s), q, s)):
            assert out.shape == (M, d_out)
            n0 = max(0, d_out - 40)
            c = codes[n0:].int()
            w = torch.stack((grid[c & 15], grid[c >> 4]), 2).view(d_out - n0, d_in) / 4
            a = X.double() * (1 if f is None else f.double()[:, None])
            got, want = out[:, n0:].double(), a @ w.t().contiguous()
            mags = a.abs() @ w.abs().t().contiguous()
            cut = 0 if f is None else 2.0 ** -9 * a.abs().amax(1)[:, None] * w.abs().amax(1)[None, :]
            off = (got - want).abs() - want.abs() * 2.0 ** -8 - SUMS * mags - cut
            assert torch.isfinite(got).all() and float(off.max()) <= 0, float(off.max())
            del out


@pytest.mark.parametrize("M,d_in,d_out", [(773, 576, 1242), (895, 2880, 1172), (797, 32, 2706), (898, 4032, 2263),
                                          (843, 32, 6922), (899, 1728, 13164)])
def test_tiles_with_one_wave_along_the_rows(M, d_in, d_out):
    """Sizes at which bf16 rows take 64 x 128 (both depths) and 128 x 128 tiles, and those next to them."""
    test_every_tile(M, d_in, d_out)


def test_batches_of_sequences():
    """X of more than two dimensions: every row is multiplied, Y keeps the leading ones."""
    torch, pifa = torch_mod(), _pifa()
    layer, _ = _layer(128, 48, 61)
    with layer:
        x, _ = _x(15, 128, 62)
        gain = torch.ones(128, dtype=torch.bfloat16, device="cuda")
        q, s = pifa.rms_norm_forward_e4m3(x.view(3, 5, 128), gain, EPS)
        for lead in ((3, 5), (15, 1), (1, 3, 5)):
            b = x.view(*lead, 128)
            assert torch.equal(layer(b), layer(x).view(*lead, 48))
            assert torch.equal(layer.norm_forward(b, gain, EPS), layer.norm_forward(x, gain, EPS).view(*lead, 48))
            assert torch.equal(layer.forward_e4m3(q.view(*lead, 128), s), layer.forward_e4m3(q.view(15, 128), s).view(*lead, 48))
        assert layer(x[4]).shape == (48,) and torch.equal(layer(x[4]), layer(x[4:5])[0])
        for bad in (x.view(30, 64), x.view(5, 384)):
            with pytest.raises(ValueError):
                layer(bad)


@pytest.mark.parametrize("M,d_in,d_out", [(1, 4096, 1000), (1, 12288, 40), (2, 2080, 16400), (3, 4096, 257), (8, 1536, 5000),
                                          (8, 32, 17), (5, 96, 16500), (7, 1728, 33)])
def test_norm_of_few_rows_keeps_its_rows(M, d_in, d_out):
    """Few rows are multiplied as two bf16 values each, 2^-8 2^-8 = 2^-16 from the
    row; rho and the products' inputs add fp32 roundings (2^-17), the sums 2^-15.
    Beside those only the output's rounding is left, also where a few columns
    carry the row."""
    torch = torch_mod()
    layer, w = _layer(d_in, d_out, 71)
    with layer:
        for seed in (72, 73):
            rng = np.random.default_rng([seed, M, d_in])
            spikes = np.ones(d_in)
            spikes[rng.integers(0, d_in, 3)] = 60.0
            st, x = inputs.round_to(rng.standard_normal((M, d_in)) * spikes, "bf16")
            rst, r = inputs.round_to(rng.standard_normal((M, d_in)), "bf16")
            gst, g = inputs.round_to(rng.uniform(0.5, 1.5, d_in), "bf16")
            big, Y = _guarded(M, d_out)
            H = torch.empty(M, d_in, dtype=torch.bfloat16, device="cuda")
            layer.norm_forward(to_dev(st), to_dev(gst), EPS, R=to_dev(rst), H=H, Y=Y)
            rows = (x + r) * o.rho(x + r, EPS) * g
            _check(Y, rows @ w.T, np.abs(rows) @ np.abs(w).T, 2.0 ** -16 + 2.0 ** -17 + SUMS, (M, d_in, d_out, seed))
            assert bool((big[M * d_out:] == -17).all())
            off = np.abs(from_dev(H) - (x + r)) - np.abs(x + r) * 2.0 ** -8
            assert (off <= 0).all()


@pytest.mark.parametrize("M,d_in,d_out", [(2, 8192, 700), (4, 4096, 5000), (8, 2048, 16400), (3, 33024, 40), (1, 12320, 97), (8, 1568, 15)])
def test_norm_in_its_own_launch_keeps_few_rows(M, d_in, d_out):
    test_norm_of_few_rows_keeps_its_rows(M, d_in, d_out)


def test_outputs_of_calls_on_another_stream():
    """Y of a call on a stream of its own is not memory that the current stream still reads."""
    torch, pifa = torch_mod(), _pifa()
    layer, _ = _layer(512, 256, 81)
    with layer:
        x, _ = _x(40, 512, 82)
        q, s = pifa.rms_norm_forward_e4m3(x, None, EPS)
        layer.reserve(40)
        calls = (lambda **kw: layer(x, **kw), lambda **kw: layer.forward_e4m3(q, s, **kw),
                 lambda **kw: layer.norm_forward(x, None, EPS, **kw))
        side = torch.cuda.Stream()
        for call in calls:
            want = call()
            torch.cuda.synchronize()
            busy = torch.full_like(want, 3.0)
            torch.cuda._sleep(20_000_000)
            kept = busy.clone()
            del busy
            got = call(stream=side)
            torch.cuda.synchronize()
            assert bool((kept == 3).all()) and torch.equal(got, want)


@pytest.mark.parametrize("M,d_in", [(2, 4096), (4, 4096), (3, 33024)])
def test_norm_of_few_rows_next_to_the_end_of_the_range(M, d_in):
    """A value past the largest bf16 that fp32 still holds is two finite bf16
    values, not an infinity and its opposite.  One weight a row, so the product is
    that value's (one launch, two launches, rows read twice)."""
    torch, pifa = torch_mod(), _pifa()
    d_out = 40
    codes, scales = np.zeros((d_out, d_in // 2), np.uint8), np.full((d_out, d_in // 32), 27, np.uint8)
    codes[:, 2] = 1 + np.arange(d_out) % 7  # column 4, 2^-100 times 0.5 .. 6
    w = o.mx_weights(codes, scales)
    x = np.ones((M, d_in))
    x[:, : d_in * 3 // 5] = 1 + 2.0 ** -7
    gain = np.zeros(d_in)
    gain[4] = 1.9921875 * 2.0 ** 127  # the largest bf16
    r = np.zeros((M, d_in))
    # one launch holds X + R times the gain, two launches the normed row
    r[:, 4] = 2.0 ** -8 - 2.0 ** -7 if M * d_in <= 12288 else 0.0
    h, y = o.rms_norm(x, gain, EPS, r)
    held = (h * gain if M * d_in <= 12288 else y)[:, 4]
    assert ((held > 1.998 * 2.0 ** 127) & (held < 2.0 ** 128)).all()
    dev = lambda a: to_dev(inputs.round_to(a, "bf16")[0])
    with pifa.Q4Layer.from_mx(_dev(codes), _dev(scales)) as layer:
        got = layer.norm_forward(dev(x), dev(gain[None]).reshape(-1), EPS, R=dev(r))
    _check(got, y @ w.T, np.abs(y) @ np.abs(w).T, 2.0 ** -16 + 2.0 ** -17 + SUMS, (M, d_in))


def _norm_want(x, r, gain, w):
    """Y and its terms' magnitudes where rho is of fp32 sums: 0 past their range."""
    h = x + r
    with np.errstate(all="ignore"):
        p = np.where((h * h).sum(1, keepdims=True) > 2.0 ** 128, 0.0, o.rho(h, EPS))
        y = h * p * gain
        return y @ w.T, np.abs(y) @ np.abs(w).T


@pytest.mark.parametrize("M,d_in,d_out", [(1, 4096, 40), (7, 1728, 300), (8, 64, 17), (8, 2080, 40), (20, 512, 40)])
def test_norm_of_rows_of_any_size(M, d_in, d_out):
    """Rows from 2^-110 to 2^127 (past 2^64 their squares overflow, and the norm is
    0) beside ordinary ones, which keep their values; in one launch and in two."""
    torch = torch_mod()
    layer, w = _layer(d_in, d_out, 91)
    with layer:
        st, x0 = inputs.round_to(np.random.default_rng([92, M]).uniform(0.5, 1, (M, d_in)), "bf16")
        rst, r0 = inputs.round_to(np.random.default_rng([93, M]).uniform(-0.25, 0.25, (M, d_in)), "bf16")
        gst, g = inputs.round_to(np.random.default_rng(94).uniform(0.5, 1.5, d_in), "bf16")
        plain = layer.norm_forward(to_dev(st), to_dev(gst), EPS, R=to_dev(rst))
        for k in (-110, -70, -31, -12, 30, 39, 41, 56, 70, 100, 126):
            f = np.ones((M, 1))
            f[M // 2] = 2.0 ** k
            dev = lambda a: to_dev(inputs.round_to(a * f, "bf16")[0])
            H = torch.empty(M, d_in, dtype=torch.bfloat16, device="cuda")
            Y = layer.norm_forward(dev(x0), to_dev(gst), EPS, R=dev(r0), H=H)
            want, mags = _norm_want(x0 * f, r0 * f, g, w)
            two = 2.0 ** -16 if M <= 8 else 2.0 ** -8  # rows as two bf16 values, or as one
            frac = two + 2.0 ** -17 + SUMS
            _check(Y, want, mags + 2.0 ** -126 / frac, frac, (M, d_in, k))
            keep = [m for m in range(M) if m != M // 2]
            assert torch.equal(Y[keep], plain[keep]), k
            assert (np.abs(from_dev(H) - (x0 + r0) * f) <= np.abs(x0 + r0) * f * 2.0 ** -8).all()


@pytest.mark.parametrize("M,d_in", [(4, 512), (4, 4096), (30, 512)])
def test_norm_and_product_agree_on_what_is_not_finite(M, d_in):
    """An infinity or a NaN in a row makes all of it NaN, as norm and product apart do, and no other."""
    torch, pifa = torch_mod(), _pifa()
    layer, _ = _layer(d_in, 40, 95)
    with layer:
        x, _ = _x(M, d_in, 96)
        r, _ = _x(M, d_in, 97)
        plain = layer.norm_forward(x, None, EPS, R=r)
        for bad in (float("inf"), float("-inf"), float("nan")):
            for a, b in ((x.clone(), r), (x, r.clone())):
                (a if a is not x else b)[2, d_in - 3] = bad
                Y = layer.norm_forward(a, None, EPS, R=b)
                apart = layer(pifa.rms_norm_forward(a, None, EPS, R=b))
                assert torch.isnan(Y[2]).all() and torch.isnan(apart[2]).all()
                keep = [m for m in range(M) if m != 2]
                assert torch.equal(Y[keep], plain[keep])


@pytest.mark.parametrize("M", [1, 3])
@pytest.mark.parametrize("scale", [187, 188, 226])
def test_norm_with_weights_next_to_the_end_of_the_range(M, scale):
    """Weights of 2^60 to 2^99 by rows of 2^38: the normed rows' products are in range."""
    pifa = _pifa()
    d_in, d_out = 256, 24
    rng = np.random.default_rng([98, M])
    codes = rng.integers(0, 256, (d_out, d_in // 2), dtype=np.uint8)
    scales = rng.integers(scale - 3, scale + 1, (d_out, d_in // 32)).astype(np.uint8)
    scales[3, 1] = scale
    w = o.mx_weights(codes, scales)
    st, x = inputs.round_to(rng.standard_normal((M, d_in)) * 2.0 ** 38, "bf16")
    with pifa.Q4Layer.from_mx(_dev(codes), _dev(scales)) as layer:
        Y = layer.norm_forward(to_dev(st), None, EPS)
    want, mags = _norm_want(x, np.zeros_like(x), np.ones(d_in), w)
    _check(Y, want, mags, 2.0 ** -16 + 2.0 ** -17 + SUMS, (M, scale))


def _forms():
    """The library's table of tiles for more than 16 rows, and the one it picks, read
    from its source: (names, [bf16, e4m3] rows of (rows, columns, then the times))."""
    with open(os.path.join(os.path.dirname(_pifa().__file__), "csrc", "pifa.hip")) as f:
        src = f.read()
    names = re.findall(r"kQ4T(\w+)", src[src.index("enum Q4Forms"):src.index("kQ4FormCount")])
    body = src[src.index("kQ4FormTable[2]"):]
    body = body[body.index("=") + 1:body.index(";")]
    rows = [[float(v) for v in r.split(",")] for r in re.findall(r"\{([-\d., ]+)\}", body)]
    rows = [r + [0.0] * (8 - len(r)) for r in rows]
    assert len(rows) == 2 * len(names)
    return names, (rows[:len(names)], rows[len(names):])


def _picked(act, M, N, K):
    names, table = _forms()
    best = None
    for name, (bm, bn, *t) in zip(names, table[act]):
        if t[0] == 0:
            continue
        tiles = -(-M // int(bm)) * -(-N // int(bn))
        at_once = [t[0] + t[1] * K / 1000, t[2] + t[3] * K / 1000, t[4] + t[5] * K / 1000]
        most = 3 if t[5] > 0 else 2 if t[3] > 0 else 1
        rounds, rest = divmod(tiles, 256 * most)
        cost = rounds * at_once[most - 1] + (at_once[(rest - 1) // 256] if rest else 0.0)
        if best is None or cost < best[0]:
            best = cost, name
    return best[1]


def _product_on_the_gpu(act, M, d_in, d_out, seed, sums=SUMS):
    """A product of bf16 (act 0) or 8-bit rows (1) against 64 bits, weights made on the GPU."""
    torch, pifa = torch_mod(), _pifa()
    rng = torch.Generator(device="cuda").manual_seed(seed)
    codes = torch.randint(0, 256, (d_out, d_in // 2), dtype=torch.uint8, device="cuda", generator=rng)
    scales = torch.randint(118, 127, (d_out, d_in // 32), dtype=torch.uint8, device="cuda", generator=rng)
    grid = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64, device="cuda")
    w = torch.stack((grid[codes.int() & 15], grid[codes.int() >> 4]), 2).view(d_out, d_in)
    w *= torch.exp2(scales.double() - 127).repeat_interleave(32, dim=1)
    x = torch.randn(M, d_in, device="cuda", generator=rng).bfloat16()
    big, Y = _guarded(M, d_out)
    with pifa.Q4Layer.from_mx(codes, scales) as layer:
        if act == 0:
            layer(x, Y)
            a = x.double()
        else:
            q = x.float().to(torch.float8_e4m3fn)
            f = torch.rand(M, device="cuda", generator=rng) + 0.5
            layer.forward_e4m3(q, f, Y)
            a = q.double() * f.double()[:, None]
        torch.cuda.synchronize()
    want = a @ w.t().contiguous()
    tol = want.abs() * 2.0 ** -8 + sums * (a.abs() @ w.abs().t().contiguous())
    if act == 1:
        top = lambda v: v.abs().view(v.shape[0], -1, 32).amax(2)
        tol += 2.0 ** -9 * (top(a) @ top(w).t().contiguous())
    off = (Y.double() - want).abs() - tol
    assert torch.isfinite(Y).all() and float(off.max()) <= 0, (act, M, d_in, d_out, float(off.max()))
    assert bool((big[M * d_out:] == -17).all())


# Every tile at sizes that pick it, where its groups of waves take many more K
# tiles than they have stages (the larger K another parity of steps), ragged ends.
DEEP = [(0, "16x32", 17, 100, (11072, 11296)), (0, "32x32", 1054, 100, (11488, 11808)), (0, "32x64", 2065, 102, (4288, 4384)),
        (0, "32x128", 2050, 199, (4288, 4384)), (0, "64x64Deep", 2077, 399, (4192, 4384)), (0, "64x64", 2421, 391, (2112, 2208)),
        (0, "64x128Deep", 65, 11277, (3104, 3232)), (0, "64x128", 2348, 858, (2080, 2144)),
        (0, "128x128Deep", 229, 8202, (4192, 4256)), (0, "128x128Pair", 2250, 2727, (2112, 2144)),
        (0, "128x256", 2331, 6619, (2080, 2144)), (0, "256x256", 1962, 6330, (2080, 2144)),
        (1, "16x32", 19, 100, (11104, 11296)), (1, "32x32", 1028, 100, (11200, 11296)), (1, "32x64", 2059, 103, (6240, 6688)),
        (1, "32x128", 1608, 583, (6176, 6688)), (1, "64x64", 2054, 196, (4192, 4384)), (1, "64x128", 2347, 406, (2080, 2208)),
        (1, "128x128", 2562, 794, (2112, 2208)), (1, "128x128Pair", 2317, 1672, (2080, 2208)),
        (1, "256x256", 2209, 5517, (2112, 2208))]


def test_deep_sizes_cover_every_tile():
    names, table = _forms()
    assert {(a, n) for a, n, *_ in DEEP} == {(a, n) for a in (0, 1) for n, row in zip(names, table[a]) if row[2]}


@pytest.mark.parametrize("act,tile,M,d_out,depths", DEEP)
def test_every_tile_runs_its_ring_many_times(act, tile, M, d_out, depths):
    for d_in in depths:
        assert _picked(act, M, d_out, d_in) == tile
        _product_on_the_gpu(act, M, d_in, d_out, 101)


@pytest.mark.parametrize("act", [0, 1])
@pytest.mark.parametrize("d_out", [250, 5000, 8193, 11008, 16400])
@pytest.mark.parametrize("M", [1, 2, 3, 8, 16])
def test_few_rows_of_wide_layers(M, d_out, act):
    """Up to 16 rows at 1, 2 and 4 groups of columns a workgroup, K of many blocks with a cut one."""
    for d_in in (2080, 4192):
        _product_on_the_gpu(act, M, d_in, d_out, 102)


def test_workspace_is_reserved_during_a_capture():
    """Reserving during a capture leaves it valid, and the captured call takes what was reserved."""
    torch, pifa = torch_mod(), _pifa()
    layer, _ = _layer(64, 24, 111)
    with layer:
        x, _ = _x(40, 64, 112)
        want = layer.norm_forward(x, None, EPS)
        fresh, _ = _layer(64, 24, 111)
        torch.cuda.synchronize()
        y, eager = torch.zeros_like(want), torch.zeros_like(want)
        side, other = torch.cuda.Stream(), torch.cuda.Stream()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.stream(side):
            with torch.cuda.graph(graph, stream=side):
                fresh.reserve(40)
                fresh.norm_forward(x, None, EPS, Y=y)
                layer.reserve(800)
        for _ in range(3):
            y.zero_()
            graph.replay()
            layer.norm_forward(x, None, EPS, Y=eager, stream=other)
            torch.cuda.synchronize()
            assert torch.equal(y, want) and torch.equal(eager, want)
        fresh.close()


@pytest.mark.parametrize("M", [9, 12, 16, 17, 33, 130])
@pytest.mark.parametrize("d_in,d_out", [(512, 200), (4096, 16400)])
def test_norm_of_more_rows_is_norm_and_product(M, d_in, d_out):
    """From 9 rows on the rows are rounded to bf16 as separate calls round them, and nothing else is."""
    torch, pifa = torch_mod(), _pifa()
    layer, _ = _layer(d_in, d_out, 121)
    with layer:
        (x, _), (r, _) = _x(M, d_in, 122), _x(M, d_in, 123)
        g = (1 + 0.2 * torch.randn(d_in, device="cuda")).to(torch.bfloat16)
        H, H2 = torch.empty_like(x), torch.empty_like(x)
        apart = layer(pifa.rms_norm_forward(x, g, EPS, R=r, H=H))
        assert torch.equal(layer.norm_forward(x, g, EPS, R=r, H=H2), apart) and torch.equal(H, H2)


@pytest.mark.parametrize("act", [0, 1])
@pytest.mark.parametrize("d_in,rows", [(32640, (1, 2, 3)), (32768, (1, 2)), (65536, (1, 2, 16, 40)), (1 << 21, (1, 2, 16, 20, 70, 257))])
def test_deep_layers(d_in, rows, act):
    """Up to the largest d_in: rows at the end of what LDS holds, and offsets of 256
    rows below 2^31.  One lane's chain of sums is at most d_in / 32 additions of
    2^-23 of the terms."""
    for M in rows:
        _product_on_the_gpu(act, M, d_in, 40, 103, max(SUMS, d_in / 32 * 2.0 ** -23))
