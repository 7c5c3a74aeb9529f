"""Norms and 4-bit layers as timed cases, with their plain forms.

The operators that stand around a compressed linear layer: the residual's
addition with the root-mean-square norm whose rows the layer reads (in bf16,
fp32, or in 8 bits with a scale per row), that norm's gradients, and layers
with 4-bit weights (e2m1 codes, one power-of-two scale per 32 of a row) on bf16
rows, on 8-bit rows, or on the norm's input directly.  Sizes are those of the
LLaMA layers in ``cases.py``, ragged row counts and odd widths beside them.
"""
from __future__ import annotations

import math

import torch

own = False  # True: the library's entry points; False: elementary torch operations

DEVICE = "cuda"
EPS = 1e-5
GROUP = 32  # weights of a row that share a scale
E4M3_MAX = 448.0
TINY = 2.0 ** -126  # smallest row scale

# Bounds of a drawn case: those of the largest listed ones.
MAX_NORM = 4096 * 8192
MAX_WEIGHTS = 8192 * 28672
MAX_PRODUCT = 4096 * 4096 * 11008


def listed():
    return [
        # one decoded token between two blocks: latency is all there is
        {"name": "norm_m1_d4096", "kind": "norm", "m": 1, "d": 4096, "dtype": "bf16", "residual": True},
        # a prompt's residual stream at the widest model: bandwidth
        {"name": "norm_m4096_d8192", "kind": "norm", "m": 4096, "d": 8192, "dtype": "bf16", "residual": True},
        # a ragged prompt whose next layer reads 8-bit rows
        {"name": "norm_e4m3_m1999_d4096", "kind": "norm_e4m3", "m": 1999, "d": 4096, "dtype": "bf16",
         "residual": True},
        # fine-tuning at the batch of the layers' backward pass
        {"name": "norm_backward_m4096_d4096", "kind": "norm_backward", "m": 4096, "d": 4096, "dtype": "bf16",
         "residual": True},
        # fine-tuning in full precision, a short ragged batch of odd rows
        {"name": "norm_backward_f32_m333_d2867", "kind": "norm_backward", "m": 333, "d": 2867, "dtype": "f32",
         "residual": False},
        # one token through the largest projection: 125 MB of weights
        {"name": "q4_up28672_m1", "kind": "q4", "d_in": 8192, "d_out": 28672, "m": 1},
        # concurrent sequences through an MLP projection, a ragged handful
        {"name": "q4_up11008_m57", "kind": "q4", "d_in": 4096, "d_out": 11008, "m": 57},
        # the prompt of an MLP projection
        {"name": "q4_up11008_m4096", "kind": "q4", "d_in": 4096, "d_out": 11008, "m": 4096},
        # eight concurrent sequences, rows in 8 bits, an attention projection
        {"name": "q4_e4m3_attn_m8", "kind": "q4_e4m3", "d_in": 4096, "d_out": 4096, "m": 8},
        # a ragged prompt in 8 bits through the MLP's way back
        {"name": "q4_e4m3_down11008_m1999", "kind": "q4_e4m3", "d_in": 11008, "d_out": 4096, "m": 1999},
        # one token: residual, norm and the attention block's q, k, v in one call
        {"name": "q4_norm_qkv_m1", "kind": "q4_norm", "d_in": 4096, "d_out": 12288, "m": 1},
        # a short ragged prompt: residual, norm and the MLP's gate and up projections in one call
        {"name": "q4_norm_gate_up_m203", "kind": "q4_norm", "d_in": 4096, "d_out": 22016, "m": 203},
    ]


def _logint(rng, lo, hi, step=1):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)) * step))


def draw(rng):
    kind = rng.choice(["norm", "norm_e4m3", "norm_backward", "q4", "q4", "q4_e4m3", "q4_norm"])
    if kind.startswith("norm"):
        d = _logint(rng, 64, 16384)
        if rng.random() < 0.5:
            d = (d + 7) // 8 * 8
        return {"kind": kind, "m": min(_logint(rng, 1, 8192), MAX_NORM // (2 * d)), "d": d,
                "dtype": rng.choice(["bf16", "bf16", "f32"]), "residual": rng.random() < 0.7}
    d_in = _logint(rng, 256, 16384, GROUP)
    d_out = min(_logint(rng, 256, 28672), MAX_WEIGHTS // d_in)
    m = max(1, min(_logint(rng, 1, 4096), MAX_PRODUCT // (d_in * d_out)))
    return {"kind": kind, "d_in": d_in, "d_out": d_out, "m": m}


# ------------------------------------------------------------------ inputs
def _generator(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(int(seed) * 9973 + 29)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEVICE)


def _stream_rows(g, m, d, dtype):
    """Rows of a residual stream: normal values and a few channels far above the rest."""
    x = _randn(g, m, d)
    x[:, torch.randint(0, d, (3,), generator=g, device=DEVICE)] *= 30.0
    return x.to(dtype)


def _e4m3_rows(x):
    scale = (x.abs().amax(1, keepdim=True) / E4M3_MAX).clamp_min(TINY)
    return (x / scale).to(torch.float8_e4m3fn), scale[:, 0].contiguous()


def _q4_weights(g, d_out, d_in):
    """Codes (two to a byte, the lower index in the low half) and scales of normal weights."""
    w = (_randn(g, d_out, d_in) * d_in ** -0.5).view(d_out, d_in // GROUP, GROUP)
    e = torch.floor(torch.log2(w.abs().amax(2).clamp_min(TINY))) - 2
    mid = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=DEVICE)
    code = torch.bucketize(torch.abs(w * torch.exp2(-e)[:, :, None]), mid).to(torch.uint8)
    code = (code + 8 * (w < 0).to(torch.uint8)).view(d_out, d_in)
    return code[:, 0::2] + 16 * code[:, 1::2], (e + 127).to(torch.uint8)


def _dtype(case):
    return torch.float32 if case.get("dtype") == "f32" else torch.bfloat16


def _inputs(case, seed):
    """Device inputs of a case, from the seed alone."""
    g = _generator(seed)
    kind, m = case["kind"], case["m"]
    if kind.startswith("norm"):
        d, dt = case["d"], _dtype(case)
        s = {"X": _stream_rows(g, m, d, dt), "gain": (1 + 0.2 * _randn(g, d)).to(dt)}
        s["R"] = _stream_rows(g, m, d, dt) if case["residual"] else None
        if kind == "norm_backward":
            s["dY"] = (1e-2 * _randn(g, m, d)).to(dt)
            s["R"] = (1e-2 * _randn(g, m, d)).to(dt) if case["residual"] else None
        return s
    d_in = case["d_in"]
    s = {}
    s["codes"], s["scales"] = _q4_weights(g, case["d_out"], d_in)
    if kind == "q4":
        s["X"] = _randn(g, m, d_in).to(torch.bfloat16)
    elif kind == "q4_e4m3":
        s["Q"], s["row_scale"] = _e4m3_rows(_randn(g, m, d_in))
    else:
        s["X"], s["R"] = _stream_rows(g, m, d_in, torch.bfloat16), _stream_rows(g, m, d_in, torch.bfloat16)
        s["gain"] = (1 + 0.2 * _randn(g, d_in)).to(torch.bfloat16)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["kind"] = case["kind"]
    if "codes" in s:
        # the values of the 16 codes: sign, two bits of exponent, one of mantissa
        s["values"] = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0,
                                    -6.0], device=DEVICE)
    if own:
        from paper_2501_19090_amd import pifa
        if "codes" in s:
            # weights laid out once, as a serving program keeps them
            s["layer"] = pifa.Q4Layer.from_mx(s.pop("codes"), s.pop("scales"))
            s["Y"] = torch.empty((case["m"], case["d_out"]), dtype=torch.bfloat16, device=DEVICE)
            if case["kind"] == "q4_norm":
                s["H"] = torch.empty_like(s["X"])
                s["layer"].reserve(case["m"])
        elif case["kind"] == "norm_backward":
            s["dX"] = torch.empty_like(s["X"])
            s["dgain"] = torch.empty(case["d"], dtype=torch.float32, device=DEVICE)
            s["work"] = torch.empty(pifa.rms_norm_backward_bytes(case["m"], case["d"]), dtype=torch.uint8,
                                    device=DEVICE)
        else:
            s["H"] = torch.empty_like(s["X"]) if case["residual"] else None
            if case["kind"] == "norm":
                s["Y"] = torch.empty_like(s["X"])
            else:
                s["Q"] = torch.empty(s["X"].shape, dtype=torch.float8_e4m3fn, device=DEVICE)
                s["row_scale"] = torch.empty(case["m"], dtype=torch.float32, device=DEVICE)
    return s


# ------------------------------------------------------------------ plain forms
def _normed(s):
    """(H, its norm), both in 32 bits."""
    h = s["X"].float()
    if s["R"] is not None:
        h = h + s["R"].float()
    return h, h * torch.rsqrt((h * h).mean(1, keepdim=True) + EPS) * s["gain"].float()


def _q4_dequantized(s):
    d_out, groups = s["scales"].shape
    codes = s["codes"].to(torch.int32)
    w = torch.stack((s["values"][codes & 15], s["values"][codes >> 4]), dim=2).view(d_out, groups, GROUP)
    return (w * torch.exp2(s["scales"].float() - 127)[:, :, None]).view(d_out, groups * GROUP)


def _plain(s):
    kind = s["kind"]
    if kind == "norm":
        h, y = _normed(s)
        return {"H": h.to(s["X"].dtype) if s["R"] is not None else None, "Y": y.to(s["X"].dtype)}
    if kind == "norm_e4m3":
        h, y = _normed(s)
        q, scale = _e4m3_rows(y)
        return {"H": h.to(s["X"].dtype) if s["R"] is not None else None, "Q": q, "scale": scale}
    if kind == "norm_backward":
        h, dy = s["X"].float(), s["dY"].float()
        rho = torch.rsqrt((h * h).mean(1, keepdim=True) + EPS)
        u = dy * s["gain"].float()
        dx = rho * u - rho ** 3 * h * (u * h).mean(1, keepdim=True)
        if s["R"] is not None:
            dx = dx + s["R"].float()
        return {"dX": dx.to(s["X"].dtype), "dgain": (dy * h * rho).sum(0)}
    w = _q4_dequantized(s)
    if kind == "q4":
        return {"Y": (s["X"].float() @ w.t()).to(torch.bfloat16)}
    if kind == "q4_e4m3":
        return {"Y": (s["row_scale"][:, None] * (s["Q"].float() @ w.t())).to(torch.bfloat16)}
    h, y = _normed(s)
    return {"H": h.to(torch.bfloat16), "Y": (y @ w.t()).to(torch.bfloat16)}


def run(state):
    if not own:
        return _plain(state)
    from paper_2501_19090_amd import pifa
    s, kind = state, state["kind"]
    if kind == "norm":
        pifa.rms_norm_forward(s["X"], s["gain"], EPS, R=s["R"], H=s["H"], Y=s["Y"])
        return {"H": s["H"], "Y": s["Y"]}
    if kind == "norm_e4m3":
        pifa.rms_norm_forward_e4m3(s["X"], s["gain"], EPS, R=s["R"], H=s["H"], Q=s["Q"], scale=s["row_scale"])
        return {"H": s["H"], "Q": s["Q"], "scale": s["row_scale"]}
    if kind == "norm_backward":
        pifa.rms_norm_backward(s["X"], s["gain"], s["dY"], EPS, dR=s["R"], dX=s["dX"], dgain=s["dgain"],
                               work=s["work"])
        return {"dX": s["dX"], "dgain": s["dgain"]}
    if kind == "q4":
        return {"Y": s["layer"](s["X"], s["Y"])}
    if kind == "q4_e4m3":
        return {"Y": s["layer"].forward_e4m3(s["Q"], s["row_scale"], s["Y"])}
    s["layer"].norm_forward(s["X"], s["gain"], EPS, R=s["R"], H=s["H"], Y=s["Y"])
    return {"H": s["H"], "Y": s["Y"]}


def work(case):
    kind, m = case["kind"], case["m"]
    if kind.startswith("norm"):
        d, es = case["d"], 4 if case["dtype"] == "f32" else 2
        rows = m * d
        if kind == "norm_backward":
            return {"bytes": es * (rows * (4 if case["residual"] else 3) + d) + 4 * d, "flops": 10 * rows}
        inout = es * (rows * (3 if case["residual"] else 1) + d)
        return {"bytes": inout + (es * rows if kind == "norm" else rows + 4 * m), "flops": 6 * rows}
    d_in, d_out = case["d_in"], case["d_out"]
    bytes_ = d_out * (d_in // 2 + d_in // GROUP) + 2 * m * d_out
    if kind == "q4":
        bytes_ += 2 * m * d_in
    elif kind == "q4_e4m3":
        bytes_ += m * d_in + 4 * m
    else:
        bytes_ += 2 * (3 * m * d_in + d_in)
    return {"bytes": bytes_, "flops": 2 * m * d_in * d_out}


# ------------------------------------------------------------------ reference
def _q4_exact(s):
    """The 4-bit weights in 64 bits, from the fields of the codes."""
    codes = torch.stack((s["codes"] % 16, torch.div(s["codes"], 16, rounding_mode="floor")), dim=2).flatten(1)
    field = (codes % 8).double()
    e, frac = torch.floor(field / 2), torch.remainder(field, 2)
    mag = torch.where(e > 0, (1 + frac / 2) * torch.pow(2.0, e - 1), frac / 2)
    w = torch.where(codes >= 8, -mag, mag)
    return w * torch.repeat_interleave(torch.pow(2.0, s["scales"].double() - 127), GROUP, dim=1)


def exact(case, seed):
    s, kind = _inputs(case, seed), case["kind"]
    if kind == "norm_backward":
        h, dy, gain = s["X"].double(), s["dY"].double(), s["gain"].double()
        norm = torch.sqrt(h.square().mean(1, keepdim=True) + EPS)
        hat = h / norm
        u = dy * gain
        dx = (u - hat * (u * hat).mean(1, keepdim=True)) / norm
        return {"dX": dx if s["R"] is None else dx + s["R"].double(), "dgain": (dy * hat).sum(0)}
    if kind in ("norm", "norm_e4m3", "q4_norm"):
        h = s["X"].double() if s["R"] is None else s["X"].double() + s["R"].double()
        y = h / torch.sqrt(h.square().mean(1, keepdim=True) + EPS) * s["gain"].double()
        if kind == "q4_norm":
            return {"H": h, "Y": y @ _q4_exact(s).t().contiguous()}
        h = None if s["R"] is None else h
        if kind == "norm":
            return {"H": h, "Y": y}
        scale = torch.clamp(y.abs().amax(1), min=TINY * E4M3_MAX) / E4M3_MAX
        return {"H": h, "Q": y / scale[:, None], "scale": scale}
    w = _q4_exact(s).t().contiguous()
    if kind == "q4":
        return {"Y": s["X"].double() @ w}
    return {"Y": (s["Q"].to(torch.float64) @ w) * s["row_scale"].double()[:, None]}
