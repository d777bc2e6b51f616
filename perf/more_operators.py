"""The training operators of the feed-forward half of a block as they are timed and checked: what a case is, its
inputs, its plain form and its exact values.

Two operators, each with its backward pass; pre-norm they are used as  N = Norm(H);  H' = H + GLU(N):
  glu, glu_bwd     the gated feed-forward sub-layer  (act(X Wg^T) * (X Wu^T)) Wd^T  (+ R), and the gradients of X and of
                   the three weights
  norm, norm_bwd   the residual's sum and its norm  Z = X + R, Y = Norm(Z),  and the gradients of Z, gamma and beta

`run` computes them with elementary torch operations in 32 bits; with `own` set it calls the library.
"""
import math

import numpy as np
import torch

own = False

D = 128
EPS = 1e-5
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
ACTS = ["silu", "gelu", "relu"]


# ---------------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------------
def listed():
    return [
        # a single node whose row has changed
        {"name": "glu-one-row", "op": "glu", "n": 1, "d_ff": 512, "act": "silu", "res": True},
        # one level of a layered circuit
        {"name": "glu-level", "op": "glu", "n": 2000, "d_ff": 512, "act": "silu", "res": True},
        # two thirds of four times the width, as gated layers take it to keep the number of weights; odd row count
        {"name": "glu-odd", "op": "glu", "n": 70001, "d_ff": 344, "act": "gelu", "res": False},
        # a whole circuit of a million gates
        {"name": "glu-million", "op": "glu", "n": 1010000, "d_ff": 512, "act": "silu", "res": True},
        # a wide layer
        {"name": "glu-wide", "op": "glu", "n": 101000, "d_ff": 2048, "act": "relu", "res": True},
        # gradients of a mini-batch of one level
        {"name": "glu-bwd-level", "op": "glu_bwd", "n": 2000, "d_ff": 512, "act": "silu"},
        # gradients at an odd size
        {"name": "glu-bwd-odd", "op": "glu_bwd", "n": 70001, "d_ff": 344, "act": "gelu"},
        # gradients of a training step on a million gates
        {"name": "glu-bwd-million", "op": "glu_bwd", "n": 1010000, "d_ff": 512, "act": "silu"},
        # a short batch in 32 bits
        {"name": "norm-small-odd", "op": "norm", "n": 777, "rms": False, "type": "f32"},
        # a million rows
        {"name": "norm-million", "op": "norm", "n": 1010000, "rms": False, "type": "bf16"},
        # its backward pass on 32-bit rows, odd row count, root mean square
        {"name": "norm-bwd-odd", "op": "norm_bwd", "n": 250007, "rms": True, "type": "f32", "res": True},
        # a million rows backwards
        {"name": "norm-bwd-million", "op": "norm_bwd", "n": 1010000, "rms": False, "type": "bf16", "res": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["glu", "glu_bwd", "norm", "norm_bwd"])
    n = _log(rng, 1, 1000000)
    if op.startswith("glu"):
        d_ff = 8 * _log(rng, 1, max(1, min(256, 63000000 // n)))
        case = {"op": op, "n": n, "d_ff": d_ff, "act": rng.choice(ACTS)}
        return dict(case, res=rng.random() < 0.5) if op == "glu" else case
    case = {"op": op, "n": n, "rms": rng.random() < 0.5, "type": rng.choice(["bf16", "f32"]) if n < 500000 else "bf16"}
    return dict(case, res=rng.random() < 0.5) if op == "norm_bwd" else case


# ---------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 2654435761 % (1 << 31))


def _normal(gen, shape, std=1.0, dtype=torch.float32):
    return (torch.randn(shape, generator=gen, device="cuda") * std).to(dtype)


def _rows(gen, n, dtype, spread=1.0):
    """Activation rows: normal, with a row factor spread over some binades and a few strong features."""
    x = torch.randn((n, D), generator=gen, device="cuda")
    x *= torch.exp2(spread * torch.randn((n, 1), generator=gen, device="cuda"))
    x *= 1.0 + 2.0 * (torch.rand((1, D), generator=gen, device="cuda") < 0.05)
    return x.to(dtype)


def prepare(case, seed):
    gen = _generator(seed)
    op, n = case["op"], case["n"]
    s = dict(case)
    if op in ("glu", "glu_bwd"):
        f, bf = case["d_ff"], torch.bfloat16
        s["x"] = _rows(gen, n, bf, 0.3)
        s["wg"], s["wu"] = _normal(gen, (f, D), 0.09, bf), _normal(gen, (f, D), 0.09, bf)
        s["wd"] = _normal(gen, (D, f), 1.0 / math.sqrt(f), bf)
        if op == "glu":
            s["r"] = _rows(gen, n, bf) if case["res"] else None
            s["y"] = [torch.zeros((n, D), dtype=bf, device="cuda")]
        else:
            s["dy"] = _rows(gen, n, bf)
            s["y"] = [torch.zeros(shape, dtype=bf, device="cuda") for shape in ((n, D), (f, D), (f, D), (D, f))]
    else:
        dtype = TYPES[case["type"]]
        s["gamma"], s["beta"] = 1.0 + _normal(gen, (D,), 0.2), _normal(gen, (D,), 0.2)
        if op == "norm":
            s["x"], s["r"] = _rows(gen, n, dtype), _rows(gen, n, dtype)
            s["y"] = [torch.zeros((n, D), dtype=dtype, device="cuda") for _ in range(2)]
        else:
            s["z"], s["dy"] = _rows(gen, n, dtype), _rows(gen, n, dtype)
            s["dr"] = _rows(gen, n, dtype) if case["res"] else None
            s["y"] = [torch.zeros((n, D), dtype=dtype, device="cuda")] + [torch.zeros(D, device="cuda") for _ in range(2)]
    if own:
        from paper_2502_01681_b200 import dg4
        s["graph"] = dg4.dg4_graph_create(np.zeros(n + 1, np.int32), np.zeros(0, np.int32), np.zeros(n, np.int32), 1)
        s["desc"] = dg4.desc(8, dg4.DG4_F32 if case.get("type") == "f32" else dg4.DG4_BF16, 0.25,
                             residual=bool(case.get("res")), rms_norm=bool(case.get("rms")))
        size = 0
        if op == "glu_bwd":
            size = dg4.dg4_glu_bwd_workspace_bytes(s["graph"], s["desc"], case["d_ff"])
        elif op == "norm_bwd":
            size = dg4.dg4_norm_bwd_workspace_bytes(s["graph"], s["desc"])
        s["ws"] = torch.empty(max(size, 16), dtype=torch.uint8, device="cuda")
        s["act_id"] = {"silu": dg4.DG4_ACT_SILU, "gelu": dg4.DG4_ACT_GELU, "relu": dg4.DG4_ACT_RELU}.get(case.get("act"))
    return s


# ---------------------------------------------------------------------------------------------------
# the operators
# ---------------------------------------------------------------------------------------------------
def _call(s):
    from paper_2502_01681_b200 import dg4
    g, d, y, op = s["graph"], s["desc"], s["y"], s["op"]
    if op == "glu":
        dg4.dg4_glu_fwd(g, d, s["x"], s["wg"], s["wu"], s["wd"], s["act_id"], s["r"], y[0])
    elif op == "glu_bwd":
        dg4.dg4_glu_bwd(g, d, s["x"], s["wg"], s["wu"], s["wd"], s["act_id"], s["dy"], y[0], y[1], y[2], y[3], s["ws"])
    elif op == "norm":
        dg4.dg4_add_norm_fwd(g, d, s["x"], s["r"], s["gamma"], s["beta"], EPS, y[0], y[1])
    else:
        dg4.dg4_norm_bwd(g, d, s["z"], s["gamma"], EPS, s["dy"], s["dr"], y[0], y[1], y[2], s["ws"])


def _act(x, kind):
    """The activation and its derivative."""
    if kind == "relu":
        return x.clamp(min=0.0), (x > 0).float()
    if kind == "silu":
        p, dp = x, 1.0
    else:                                             # gelu, by its tanh form: x * sigmoid(2 c (x + a x^3))
        c, a = 2.0 * math.sqrt(2.0 / math.pi), 0.044715
        p, dp = c * (x + a * x * x * x), c * (1.0 + 3.0 * a * x * x)
    e = torch.exp(-p.abs())
    small, big = e / (1.0 + e), 1.0 / (1.0 + e)       # sigmoid of -|p| and of |p|: neither cancels
    sig, rest = torch.where(p >= 0, big, small), torch.where(p >= 0, small, big)
    return x * sig, sig * (1.0 + x * rest * dp)


def _plain_glu(s):
    x = s["x"].float()
    h = _act(x @ s["wg"].float().t(), s["act"])[0] * (x @ s["wu"].float().t())
    y = h @ s["wd"].float().t()
    s["y"][0].copy_(y if s["r"] is None else y + s["r"].float())


def _plain_glu_bwd(s):
    x, dy, wg, wu, wd = (s[k].float() for k in ("x", "dy", "wg", "wu", "wd"))
    a, da = _act(x @ wg.t(), s["act"])
    u = x @ wu.t()
    s["y"][3].copy_(dy.t() @ (a * u))
    dh = dy @ wd
    dg, du = dh * u * da, dh * a
    s["y"][1].copy_(dg.t() @ x)
    s["y"][2].copy_(du.t() @ x)
    s["y"][0].copy_(dg @ wg + du @ wu)


def _plain_centre(z, rms):
    c = z if rms else z - z.mean(-1, keepdim=True)
    inv = 1.0 / torch.sqrt((c * c).mean(-1, keepdim=True) + EPS)
    return c * inv, inv


def _plain_norm(s):
    z = s["x"].float() + s["r"].float()
    s["y"][0].copy_(z)
    s["y"][1].copy_(_plain_centre(z, s["rms"])[0] * s["gamma"] + s["beta"])


def _plain_norm_bwd(s):
    dy = s["dy"].float()
    c, inv = _plain_centre(s["z"].float(), s["rms"])
    s["y"][1].copy_((dy * c).sum(0, dtype=torch.float64))
    s["y"][2].copy_(dy.sum(0, dtype=torch.float64))
    t = dy * s["gamma"]
    d = t - c * (t * c).mean(-1, keepdim=True)
    if not s["rms"]:
        d = d - t.mean(-1, keepdim=True)
    d = d * inv
    s["y"][0].copy_(d if s["dr"] is None else d + s["dr"].float())


def run(state):
    if own:
        _call(state)
    elif state["op"] == "glu":
        _plain_glu(state)
    elif state["op"] == "glu_bwd":
        _plain_glu_bwd(state)
    elif state["op"] == "norm":
        _plain_norm(state)
    else:
        _plain_norm_bwd(state)
    return state["y"]


def work(case):
    op, n = case["op"], case["n"]
    if op in ("glu", "glu_bwd"):
        f = case["d_ff"]
        rows, weights, products = (2 + case["res"], 3, 3) if op == "glu" else (3, 6, 8)
        return {"bytes": 2 * D * (n * rows + f * weights), "flops": 2 * n * D * f * products}
    es = 2 if case["type"] == "bf16" else 4
    rows = 4 if op == "norm" else 3 + case["res"]
    return {"bytes": n * D * es * rows + 8 * D, "flops": n * D * (8 if op == "norm" else 16)}


# ---------------------------------------------------------------------------------------------------
# exact values, in 64 bits: the definitions forward, differentiated by torch
# ---------------------------------------------------------------------------------------------------
def _exact_sublayer(x, wg, wu, wd, act):
    g = torch.nn.functional.linear(x, wg)
    if act == "gelu":
        a = torch.nn.functional.gelu(g, approximate="tanh")
    else:
        a = torch.relu(g) if act == "relu" else g * torch.sigmoid(g)
    return torch.nn.functional.linear(a * torch.nn.functional.linear(x, wu), wd)


def _exact_glu(s):
    w = [s[k].double() for k in ("wg", "wu", "wd")]
    y = torch.cat([_exact_sublayer(x.double(), *w, s["act"]) for x in s["x"].split(65536)])
    return [y if s["r"] is None else y + s["r"].double()]


def _exact_glu_bwd(s):
    w = [s[k].double().requires_grad_() for k in ("wg", "wu", "wd")]
    dx = []
    for x, dy in zip(s["x"].split(65536), s["dy"].split(65536)):
        x = x.double().requires_grad_()
        _exact_sublayer(x, *w, s["act"]).backward(dy.double())
        dx.append(x.grad)
    return [torch.cat(dx)] + [p.grad for p in w]


def _exact_norm_of(z, gamma, beta, rms):
    if rms:
        return z * torch.rsqrt(z.pow(2).mean(1, keepdim=True) + EPS) * gamma + beta
    return torch.nn.functional.layer_norm(z, (D,), gamma, beta, EPS)


def _exact_norm(s):
    z = s["x"].double() + s["r"].double()
    return [z, _exact_norm_of(z, s["gamma"].double(), s["beta"].double(), s["rms"])]


def _exact_norm_bwd(s):
    z, gamma, beta = (s[k].double().requires_grad_() for k in ("z", "gamma", "beta"))
    _exact_norm_of(z, gamma, beta, s["rms"]).backward(s["dy"].double())
    return [z.grad if s["dr"] is None else z.grad + s["dr"].double(), gamma.grad, beta.grad]


def exact(case, seed):
    s = prepare(case, seed)
    return {"glu": _exact_glu, "glu_bwd": _exact_glu_bwd, "norm": _exact_norm, "norm_bwd": _exact_norm_bwd}[case["op"]](s)
