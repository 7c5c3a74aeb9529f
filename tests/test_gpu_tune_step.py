"""Layer norm, layer, adapters, their gradients and the AdamW step together, as a
fine-tuning step runs them: each against its fp64 form on the values that the GPU
had before it, and the whole step captured into a graph against eager steps."""
import numpy as np
import pytest

from oracle import tune as o
from paper_2501_19090_amd import inputs

from gpu_util import DeviceLayer, from_dev, rel_fro, torch_mod

pytestmark = pytest.mark.gpu

EPS, LR = 1e-5, 1e-2
M, D, R_LAYER, R, N = 200, 256, 96, 8, 3


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch_mod().cuda.is_available():
        pytest.skip("no GPU")


class Step:
    """y = layer(norm(x + r)) + adapters; the loss is half the squared distance to a target."""

    def __init__(self, bits):
        from paper_2501_19090_amd import pifa
        self.pifa, torch = pifa, torch_mod()
        rng = np.random.default_rng(8)
        U, V = inputs.lowrank_factors(R_LAYER, D, R_LAYER, 9)
        piv, npiv = inputs.random_partition(D, R_LAYER, seed=9)
        self.layer = DeviceLayer(piv, npiv, U @ V, rng.standard_normal((D - R_LAYER, R_LAYER)) * 0.2, "bf16")
        t = lambda *s, scale=1.0: torch.from_numpy((rng.standard_normal(s) * scale).astype(np.float32)).cuda()
        bf = lambda x: x.to(torch.bfloat16)
        self.x, self.r, self.target = bf(t(M, D)), bf(t(M, D)), bf(t(M, D))
        self.ids = torch.from_numpy(rng.integers(-1, N, M).astype(np.int32)).cuda()
        self.scale = torch.full((N,), 2.0, device="cuda")
        # masters in fp32, and what the kernels read, kept by the step
        self.master = [t(D, scale=0.1) + 1, t(D, scale=0.1), t(N, R, D, scale=D ** -0.5), t(N, D, R, scale=0.1)]
        self.gain, self.bias, self.A, self.B = self.work = [bf(m) for m in self.master]
        self.grads = [torch.empty_like(m) for m in self.master]
        self.H, self.N_, self.Y, self.dY, self.dN, self.dH = (torch.empty_like(self.x) for _ in range(6))
        self.plan = pifa.AdapterPlan(self.ids, N)
        e = lambda n: torch.empty(n, dtype=torch.uint8, device="cuda")
        self.w1, self.w2 = e(pifa.adapter_forward_bytes(M, D, D, R, N)), e(pifa.adapter_backward_bytes(M, D, D, R, N))
        self.w3 = e(pifa.layer_norm_backward_bytes(M, D))
        self.opt = pifa.AdamW(self.master, self.grads, weight_decay=[0.0, 0.0, 0.1, 0.1], bits=bits, copies=self.work, seed=4)

    def forward(self):
        p = self.pifa
        p.layer_norm_forward(self.x, self.gain, self.bias, EPS, R=self.r, H=self.H, Y=self.N_)
        p.pifa_forward(self.layer.handle, self.N_, self.Y)
        p.adapter_forward(self.N_, self.A, self.B, self.plan, scale=self.scale, Y0=self.Y, Y=self.Y, work=self.w1)

    def run(self):
        p = self.pifa
        self.plan.update(self.ids)
        self.forward()
        self.dY.copy_(self.Y - self.target)
        p.pifa_layer_backward(self.layer.handle, self.N_, self.Y, self.dY, dX=self.dN)
        p.adapter_backward(self.N_, self.A, self.B, self.plan, self.dY, scale=self.scale, dX0=self.dN, dX=self.dN,
                           dA=self.grads[2], dB=self.grads[3], work=self.w2)
        p.layer_norm_backward(self.H, self.gain, self.dN, EPS, dX=self.dH, dgain=self.grads[0], dbias=self.grads[1], work=self.w3)
        self.opt.step(LR)

    def close(self):
        self.opt.close()
        self.layer.close()


@pytest.mark.parametrize("bits", [32, 8])
def test_each_part_on_the_values_before_it(bits):
    torch = torch_mod()
    s = Step(bits)
    try:
        ids = s.ids.cpu().numpy()
        for step in range(1, 4):
            before = [from_dev(w) for w in s.work]
            masters = [m.double().cpu().numpy() for m in s.master]
            states = [[x.clone() for x in st] for st in s.opt.states]
            s.run()
            torch.cuda.synchronize()
            gain, bias, A, B = before
            scale = np.full(N, 2.0)
            n, dy = from_dev(s.N_), from_dev(s.dY)
            h, want = o.layer_norm(from_dev(s.x), gain, bias, EPS, from_dev(s.r))
            assert rel_fro(n, want) <= 2.0 ** -8
            y = o.adapter_forward(n, A, B, ids, scale, s.layer.oracle(n))
            # the layer's output is rounded to bf16, then the sum (each 2^-8 at most) within the layer's own 5e-3
            assert rel_fro(from_dev(s.Y), y) <= 5e-3 + 2.0 ** -8
            dx, dA, dB = o.adapter_backward(n, A, B, ids, dy, scale)
            assert rel_fro(from_dev(s.grads[2]), dA) <= 2.0 ** -16 and rel_fro(from_dev(s.grads[3]), dB) <= 2.0 ** -16
            dense = s.layer.oracle(np.eye(D))  # row k: the output of the k-th unit vector
            dx = dx + dy @ dense.T
            assert rel_fro(from_dev(s.dN), dx) <= 5e-3 + 2.0 ** -8
            dh, dg, db = o.layer_norm_backward(from_dev(s.H), gain, from_dev(s.dN), EPS)
            assert rel_fro(from_dev(s.dH), dh) <= 2.0 ** -8 + 2.0 ** -16
            assert rel_fro(from_dev(s.grads[0]), dg) <= 2.0 ** -16 and rel_fro(from_dev(s.grads[1]), db) <= 2.0 ** -16
            assert s.opt.count() == step
            for k, (p, g, st) in enumerate(zip(masters, s.grads, states)):
                m, v = (x.float().cpu().numpy() for x in st[:2])
                if bits == 8:
                    m, v = (o.e4m3_values(x.view(torch.uint8).cpu().numpy().ravel(), sc.cpu().numpy()).reshape(p.shape)
                            for x, sc in zip(st[:2], st[2:]))
                want, _, _ = o.adamw(p, g.double().cpu().numpy(), m.astype(np.float64), v.astype(np.float64), step, LR, 0.9, 0.999,
                                     1e-8, [0.0, 0.0, 0.1, 0.1][k])
                # v is good to a few roundings, so the update, at most lr / sqrt(1 - 0.999), is to 2^-20 of itself
                off = np.abs(s.master[k].double().cpu().numpy() - want)
                assert off.max() <= 2.0 ** -22 * np.abs(p).max() + 2.0 ** -20 * 32 * LR, (step, k, off.max())
                assert torch.equal(s.work[k], s.master[k].to(torch.bfloat16))
    finally:
        s.close()


@pytest.mark.parametrize("bits", [32, 8])
def test_whole_step_in_a_graph(bits):
    """Replays with an eager step between: the same bits as eager steps."""
    torch = torch_mod()
    want, got = Step(bits), Step(bits)
    try:
        for _ in range(6):
            want.run()
        got.run()  # the layer's workspaces grow here
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got.run()
        for k in range(5):
            if k == 2:
                got.run()
            else:
                graph.replay()
            torch.cuda.synchronize()
        for a, b in zip(got.master + got.work + [got.Y, got.dH], want.master + want.work + [want.Y, want.dH]):
            assert torch.equal(a, b)
        assert got.opt.count() == 6
    finally:
        want.close()
        got.close()
