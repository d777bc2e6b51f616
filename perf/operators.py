"""The serving operators as they are timed and checked: what a case is, its inputs, its plain form and its exact values.

Four operators, used together when one circuit batch carries the rows of many requests:
  qkv, out   the shared projections with a low-rank adapter per request beside them
  kv8        K and V rows quantised to 8 bits as they are written to the table, and read back
  attn       sparse attention over the 8-bit table, for all nodes or for a list of them
  norm       norms after a sub-layer and before the next one, fused with the gate and the scaled residual

`run` computes them with elementary torch operations in 32 bits; with `own` set it calls the library.
"""
import math

import numpy as np
import torch

own = False

D = 128
EPS = 1e-5
MAX_CODE = 448.0          # largest finite e4m3 value
ROW_BYTES = 288           # a table row: 16 pieces of 8 K codes and 8 V codes, then 16 pairs of scale exponents
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---------------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------------
def listed():
    return [
        # one token of each of 64 requests, every one with an adapter of its own: a decoding step
        {"name": "qkv-one-row-each", "op": "qkv", "n": 64, "rows": 64, "segs": 64, "adapters": 64, "rank": 16},
        # a large batch: a million gates of 200 circuits, 40 adapters, the last rows not in use
        {"name": "qkv-million", "op": "qkv", "n": 1010000, "rows": 1009873, "segs": 200, "adapters": 40, "rank": 16},
        # a small circuit, odd lengths, the smallest rank, with the residual
        {"name": "out-small-odd", "op": "out", "n": 2064, "rows": 2051, "segs": 7, "adapters": 5, "rank": 8},
        # the same million gates through the output projection, the largest rank
        {"name": "out-million", "op": "out", "n": 1010000, "rows": 1010000, "segs": 90, "adapters": 12, "rank": 64},
        # one finished level of the level-by-level order: its rows alone are refreshed
        {"name": "kv8-level", "op": "kv8", "n": 101000, "count": 2000, "heads": 8, "type": "bf16"},
        # a whole table in 16-bit storage
        {"name": "kv8-million", "op": "kv8", "n": 1010000, "count": 0, "heads": 8, "type": "bf16"},
        # a whole table from 32-bit rows, odd length
        {"name": "kv8-f32", "op": "kv8", "n": 250007, "count": 0, "heads": 4, "type": "f32"},
        # one level's queries over the table, direct fan-ins
        {"name": "attn-level", "op": "attn", "n": 101000, "count": 2000, "per_level": 2000, "win": 13.0, "hops": 1,
         "heads": 8, "type": "bf16"},
        # all gates of a large circuit, cones of two hops
        {"name": "attn-million", "op": "attn", "n": 1010000, "count": 0, "per_level": 160, "win": 16.0, "hops": 2,
         "heads": 8, "type": "bf16"},
        # wide cones, up to 63 members
        {"name": "attn-wide", "op": "attn", "n": 101000, "count": 0, "per_level": 200, "win": 14.0, "hops": 5,
         "heads": 4, "type": "bf16"},
        # a short batch of requests, one gate vector each
        {"name": "norm-small-odd", "op": "norm", "n": 777, "rows": 770, "segs": 9, "gates": 4, "rms": False, "type": "bf16"},
        # a million rows
        {"name": "norm-million", "op": "norm", "n": 1010000, "rows": 1010000, "segs": 200, "gates": 40, "rms": True,
         "type": "bf16"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["qkv", "out", "kv8", "attn", "norm"])
    if op in ("qkv", "out"):
        rank = rng.choice([8, 16, 24, 32, 40, 48, 56, 64])
        n = _log(rng, 1, 1000000)
        segs = min(_log(rng, 1, 512), max(1, n))
        adapters = min(_log(rng, 1, 64), 640 // rank)
        rows = n if rng.random() < 0.5 else max(1, n - rng.randrange(0, 1 + n // 50 + 3))
        return {"op": op, "n": n, "rows": rows, "segs": segs, "adapters": adapters, "rank": rank}
    if op == "norm":
        n = _log(rng, 1, 1000000)
        return {"op": op, "n": n, "rows": n, "segs": min(_log(rng, 1, 512), n), "gates": _log(rng, 1, 64),
                "rms": rng.random() < 0.5, "type": rng.choice(["bf16", "f32"]) if n < 500000 else "bf16"}
    if op == "kv8":
        n = _log(rng, 1, 1000000)
        return {"op": op, "n": n, "count": rng.choice([0, _log(rng, 1, n)]), "heads": rng.choice([1, 2, 4, 8, 16]),
                "type": rng.choice(["bf16", "f32"]) if n < 500000 else "bf16"}
    hops = rng.choice([1, 2, 2, 3, 4, 5])
    n = _log(rng, 300, 1000000 if hops <= 2 else 90000)
    return {"op": op, "n": n, "count": rng.choice([0, _log(rng, 1, n)]), "per_level": _log(rng, 20, 250),
            "win": round(rng.uniform(6.0, 16.0), 3), "hops": hops, "heads": rng.choice([1, 2, 4, 8, 16]),
            "type": rng.choice(["bf16", "f32"]) if n < 200000 else "bf16"}


# ---------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 2654435761 % (1 << 31))


def _normal(gen, shape, std=1.0, dtype=torch.float32):
    return (torch.randn(shape, generator=gen, device="cuda") * std).to(dtype)


def _rows(gen, n, dtype):
    """Activation rows: normal, with a row factor spread over a few binades and some strong features."""
    x = torch.randn((n, D), generator=gen, device="cuda")
    x *= torch.exp2(torch.randn((n, 1), generator=gen, device="cuda"))
    x *= 1.0 + 4.0 * (torch.rand((1, D), generator=gen, device="cuda") < 0.05)
    return x.to(dtype)


def _segments(gen, rows, segs, ids):
    """Ascending row offsets of the requests (some may be empty) and the adapter or gate of each (-1: none)."""
    if segs >= rows:
        ptr = torch.arange(segs + 1, device="cuda").clamp(max=rows)
    else:
        cuts = (torch.rand(segs - 1, generator=gen, device="cuda", dtype=torch.float64) * rows).long().sort().values
        ptr = torch.cat([cuts.new_zeros(1), cuts, cuts.new_full((1,), rows)])
    seg_id = torch.randint(-1, ids, (segs,), generator=gen, device="cuda")
    return ptr.int(), seg_id.int()


def _fanins(gen, n, per_level, win):
    """Direct fan-ins [n, 2] (-1: none).  Levels are blocks of per_level ids; a gate draws its fan-ins from a
    window of 2^U ids, U in [4, win), that ends where its own level begins; three gates in ten have one fan-in."""
    ids = torch.arange(n, device="cuda")
    start = ids // per_level * per_level
    width = torch.exp2(4.0 + (win - 4.0) * torch.rand(n, generator=gen, device="cuda", dtype=torch.float64))
    width = torch.minimum(width.long(), start).clamp(min=1)
    r = torch.rand((2, n), generator=gen, device="cuda", dtype=torch.float64)
    f = start - 1 - (r * width).long().clamp(max=width - 1)
    f = torch.where(start > 0, f, -1)
    f[1] = torch.where(torch.rand(n, generator=gen, device="cuda") < 0.3, -1, f[1])
    return f.t().contiguous(), (ids // per_level).int()


def _cones(fan, hops):
    """[n, 2^(hops+1) - 1]: the members of the fan-in cone of each node, itself first, -1 where there is none."""
    ids = torch.arange(fan.shape[0], device=fan.device, dtype=torch.int32)[:, None]
    fan = fan.int()
    cone = ids
    for _ in range(hops):
        parts = [torch.where(fan[:, j:j + 1] >= 0, cone[fan[:, j].clamp(min=0).long()], -1) for j in (0, 1)]
        cone = torch.cat([ids] + parts, 1)
    cone = cone.sort(dim=1, descending=True).values          # the node itself is its own largest member
    again = torch.cat([torch.zeros_like(cone[:, :1], dtype=torch.bool), cone[:, 1:] == cone[:, :-1]], 1)
    return torch.where(again, -1, cone)


def _circuit(fan):
    has = fan >= 0
    ptr = torch.cat([torch.zeros(1, dtype=torch.long, device=fan.device), has.sum(1).cumsum(0)])
    return ptr.int().cpu().numpy(), fan[has].int().cpu().numpy()


def _edgeless(n):
    return np.zeros(n + 1, np.int32), np.zeros(0, np.int32), np.zeros(n, np.int32)


def _nodes(gen, n, count):
    return torch.randperm(n, generator=gen, device="cuda")[:count].int() if count else None


def _quantise(x, heads):
    """Codes and scale exponents: per row and head the smallest k >= -127 with max|x| <= 448 * 2^k."""
    x = x.float().view(-1, heads, D // heads)
    top = x.abs().amax(-1)
    m, e = torch.frexp(top.double())                          # top = m * 2^e, m in [0.5, 1)
    k = torch.where(top > 0, e - 9 + (m > 0.875).int(), -127).clamp(min=-127)
    code = (x.double() * torch.exp2(-k.double())[..., None]).float().to(torch.float8_e4m3fn)
    return code, k


def _table(k, v, heads):
    n = k.shape[0]
    t = torch.zeros((n, ROW_BYTES), dtype=torch.uint8, device="cuda")
    for i, x in enumerate((k, v)):
        code, e = _quantise(x, heads)
        t[:, :256].view(n, 16, 2, 8)[:, :, i] = code.view(torch.uint8).view(n, 16, 8)
        t[:, 256:].view(n, 16, 2)[:, :heads, i] = (e + 127).to(torch.uint8)
    return t


def prepare(case, seed):
    gen = _generator(seed)
    op, n = case["op"], case["n"]
    s = dict(case)
    circuit = None
    if op in ("qkv", "out"):
        n_out = 384 if op == "qkv" else D
        s["x"] = _rows(gen, n, torch.bfloat16)
        s["w"] = _normal(gen, (n_out, D), 0.08, torch.bfloat16)
        s["a"] = _normal(gen, (case["adapters"], case["rank"], D), 0.09, torch.bfloat16)
        s["b"] = _normal(gen, (case["adapters"], n_out, case["rank"]), 0.05, torch.bfloat16)
        s["scale"] = 0.5 + torch.rand(case["adapters"], generator=gen, device="cuda")
        s["seg_ptr"], s["seg_id"] = _segments(gen, case["rows"], case["segs"], case["adapters"])
        s["res"] = _rows(gen, n, torch.bfloat16) if op == "out" else None
        s["y"] = [torch.zeros((n, D), dtype=torch.bfloat16, device="cuda") for _ in range(n_out // D)]
        s["heads"], s["type"] = 8, "bf16"
    elif op == "kv8":
        dtype = TYPES[case["type"]]
        s["k"], s["v"] = _rows(gen, n, dtype), _rows(gen, n, dtype)
        s["nodes"] = _nodes(gen, n, case["count"])
        s["t"] = torch.zeros((n, ROW_BYTES), dtype=torch.uint8, device="cuda")
        s["y"] = [torch.zeros((n, D), dtype=dtype, device="cuda") for _ in range(2)]
    elif op == "attn":
        dtype = TYPES[case["type"]]
        fan, level = _fanins(gen, n, case["per_level"], case["win"])
        s["cone"] = _cones(fan, case["hops"])
        circuit = _circuit(fan) + (level.cpu().numpy(),)
        s["q"] = _normal(gen, (n, D), 1.5, dtype)
        s["t"] = _table(_rows(gen, n, torch.float32), _rows(gen, n, torch.float32), case["heads"])
        s["nodes"] = _nodes(gen, n, case["count"])
        s["y"] = [torch.zeros((n, D), dtype=dtype, device="cuda")]
    else:
        dtype = TYPES[case["type"]]
        s["x"], s["res"] = _rows(gen, n, dtype), _rows(gen, n, dtype)
        s["res_scale"] = 0.75
        s["gate"] = _normal(gen, (case["gates"], D), 0.6)
        s["seg_ptr"], s["seg_id"] = _segments(gen, case["rows"], case["segs"], case["gates"])
        s["post"] = (1.0 + _normal(gen, (D,), 0.2), None if case["rms"] else _normal(gen, (D,), 0.2))
        s["pre"] = (1.0 + _normal(gen, (D,), 0.2), None if case["rms"] else _normal(gen, (D,), 0.2))
        s["y"] = [torch.zeros((n, D), dtype=dtype, device="cuda") for _ in range(2)]
        s["heads"] = 8
    if own:
        from paper_2502_01681_b200 import dg4
        row_ptr, col_idx, level = circuit or _edgeless(n)
        s["graph"] = dg4.dg4_graph_create(row_ptr, col_idx, level, case.get("hops", 1))
        s["desc"] = dg4.desc(s["heads"], dg4.DG4_BF16 if s["type"] == "bf16" else dg4.DG4_F32,
                             (s["heads"] / D) ** 0.5, residual=op == "out", rms_norm=bool(case.get("rms")))
        if op in ("qkv", "out"):
            s["ad"] = dg4.adapters(s["a"], s["b"], s["scale"])
        if "seg_ptr" in s:
            s["seg"] = dg4.segments(s["seg_ptr"], s["seg_id"])
    return s


# ---------------------------------------------------------------------------------------------------
# the operators
# ---------------------------------------------------------------------------------------------------
def _call(s):
    from paper_2502_01681_b200 import dg4
    g, d, y = s["graph"], s["desc"], s["y"]
    if s["op"] == "qkv":
        dg4.dg4_qkv_project_adapters(g, d, s["x"], s["w"], s["ad"], s["seg"], y[0], y[1], y[2])
    elif s["op"] == "out":
        dg4.dg4_out_project_adapters(g, d, s["x"], s["w"], s["ad"], s["seg"], s["res"], y[0])
    elif s["op"] == "kv8":
        dg4.dg4_kv8_write(g, d, s["k"], s["v"], s["t"], s["nodes"])
        dg4.dg4_kv8_read(g, d, s["t"], y[0], y[1], s["nodes"])
    elif s["op"] == "attn":
        dg4.dg4_sparse_attn_kv8_fwd(g, d, s["q"], s["t"], y[0], s["nodes"])
    else:
        dg4.dg4_norm_gate_fwd(g, d, s["x"], s["res"], s["res_scale"], s["gate"], s["seg"], s["post"], s["pre"], EPS,
                              y[0], y[1])


def _id_of_row(s):
    lens = (s["seg_ptr"][1:] - s["seg_ptr"][:-1]).long()
    return torch.repeat_interleave(s["seg_id"], lens, output_size=s["rows"])


def _plain_project(s):
    m = s["rows"]
    x = s["x"][:m].float()
    n_ad, rank, _ = s["a"].shape
    y = x @ s["w"].float().t()
    u = (x @ s["a"].float().view(n_ad * rank, D).t()).view(m, n_ad, rank)
    mine = _id_of_row(s)[:, None] == torch.arange(n_ad, device="cuda", dtype=torch.int32)
    u = torch.where(mine[..., None], u * s["scale"][:, None], 0.0)
    y += u.view(m, n_ad * rank) @ s["b"].float().transpose(1, 2).reshape(n_ad * rank, -1)
    if s["res"] is not None:
        y += s["res"][:m].float()
    for i, out in enumerate(s["y"]):
        out[:m] = y[:, i * D:(i + 1) * D]


def _plain_kv8(s):
    for x, out in zip((s["k"], s["v"]), s["y"]):
        at = slice(None) if s["nodes"] is None else s["nodes"].long()
        code, e = _quantise(x[at], s["heads"])
        out[at] = (code.float() * torch.exp2(e.float())[..., None]).view(-1, D).to(out.dtype)


def _read_table(t, heads, i):
    n = t.shape[0]
    code = t[:, :256].view(n, 16, 2, 8)[:, :, i].contiguous().view(torch.float8_e4m3fn).float().view(n, heads, D // heads)
    e = t[:, 256:].view(n, 16, 2)[:, :heads, i].float() - 127.0
    return code * torch.exp2(e)[..., None]


def _plain_attn(s):
    h = s["heads"]
    at = slice(None) if s["nodes"] is None else s["nodes"].long()
    cone = s["cone"][at].long()
    k, v = (_read_table(s["t"], h, i) for i in (0, 1))
    q = s["q"][at].float().view(-1, 1, h, D // h)
    u = cone.clamp(min=0)
    score = (k[u] * q).sum(-1) * (h / D) ** 0.5
    score = torch.where((cone >= 0)[..., None], score, -math.inf)
    p = torch.exp(score - score.amax(1, keepdim=True))
    p = p / p.sum(1, keepdim=True)
    s["y"][0][at] = (v[u] * p[..., None]).sum(1).reshape(-1, D).to(s["y"][0].dtype)


def _plain_norm_of(x, gamma, beta, rms):
    c = x if rms else x - x.mean(-1, keepdim=True)
    y = c / torch.sqrt((c * c).mean(-1, keepdim=True) + EPS) * gamma
    return y if beta is None else y + beta


def _plain_norm(s):
    m = s["rows"]
    at = _id_of_row(s).long()[:, None]
    gate = torch.where(at >= 0, s["gate"][at[:, 0].clamp(min=0)], 1.0)
    r = s["res_scale"] * s["res"][:m].float() + gate * _plain_norm_of(s["x"][:m].float(), *s["post"], s["rms"])
    s["y"][0][:m] = r
    s["y"][1][:m] = _plain_norm_of(r, *s["pre"], s["rms"])


def run(state):
    if own:
        _call(state)
    elif state["op"] in ("qkv", "out"):
        _plain_project(state)
    elif state["op"] == "kv8":
        _plain_kv8(state)
    elif state["op"] == "attn":
        _plain_attn(state)
    else:
        _plain_norm(state)
    return state["y"]


def work(case):
    op, n = case["op"], case["n"]
    if op in ("qkv", "out"):
        m, r, n_out = case["rows"], case["rank"], 384 if op == "qkv" else D
        used = min(case["adapters"], case["segs"])
        return {"bytes": m * 2 * (D + n_out + (D if op == "out" else 0)) + 2 * n_out * D + used * 2 * r * (D + n_out) + 8 * case["segs"],
                "flops": 2 * m * (D * n_out + r * (D + n_out))}
    es = 2 if case["type"] == "bf16" else 4
    if op == "norm":
        m = case["rows"]
        return {"bytes": m * 4 * D * es + case["gates"] * 4 * D + 8 * case["segs"], "flops": m * D * 20}
    m = case["count"] or n
    if op == "kv8":                                   # both directions: K, V and the table row, once each
        return {"bytes": m * (4 * D * es + 2 * ROW_BYTES + (8 if case["count"] else 0)), "flops": m * D * 12}
    members = sum(1.7 ** i for i in range(case["hops"] + 1))
    return {"bytes": m * (2 * D * es + 4 * members) + min(n, m * members) * ROW_BYTES, "flops": m * members * 4 * D}


# ---------------------------------------------------------------------------------------------------
# exact values, in 64 bits
# ---------------------------------------------------------------------------------------------------
def _exact_project(s):
    x, w = s["x"].double(), s["w"].double()
    y = torch.zeros((s["n"], w.shape[0]), dtype=torch.float64, device="cuda")
    ptr, ids = s["seg_ptr"].tolist(), s["seg_id"].tolist()
    for lo, hi, i in zip(ptr[:-1], ptr[1:], ids):
        y[lo:hi] = torch.matmul(x[lo:hi], w.T)
        if i >= 0:
            delta = torch.matmul(s["b"][i].double(), s["a"][i].double()) * s["scale"][i].double()
            y[lo:hi] += torch.matmul(x[lo:hi], delta.T)
        if s["res"] is not None:
            y[lo:hi] += s["res"][lo:hi].double()
    return [y[:, i * D:(i + 1) * D].contiguous() for i in range(w.shape[0] // D)]


def _exact_kv8(s):
    """Each element is moved to the nearest multiple of its step: 2^-3 of its binade, no finer than 2^-9 of the scale."""
    got = []
    at = torch.arange(s["n"], device="cuda") if s["nodes"] is None else s["nodes"].long()
    for x in (s["k"], s["v"]):
        y = torch.zeros((s["n"], D), dtype=torch.float64, device="cuda")
        z = x[at].double().view(at.numel(), s["heads"], -1)
        top = z.abs().amax(-1, keepdim=True)
        k = torch.full_like(top, -127.0)
        k = torch.maximum(k, torch.ceil(torch.log2(top.clamp(min=2.0 ** -140) / MAX_CODE) - 1e-3))
        k = torch.where(top > MAX_CODE * torch.exp2(k), k + 1, k)
        k = torch.where((top <= MAX_CODE * torch.exp2(k - 1)) & (k > -127), k - 1, k)
        z = z / torch.exp2(k)
        step = torch.exp2(torch.frexp(z)[1].double().clamp(min=-5) - 4)
        z = torch.round(z / step) * step * torch.exp2(k)           # torch.round takes ties to the even multiple
        y[at] = z.view(-1, D)
        got.append(y)
    return got


def _exact_attn(s):
    h, n = s["heads"], s["n"]
    byte = s["t"].long()
    def read(i):
        c = byte[:, :256].view(n, 16, 2, 8)[:, :, i].reshape(n, D)
        e, m = (c >> 3) & 15, c & 7
        val = torch.where(e > 0, (8 + m).double() * torch.exp2(e.double() - 10), m.double() * 2.0 ** -9)
        val = torch.where(c >= 128, -val, val).view(n, h, D // h)
        return val * torch.exp2(byte[:, 256:].view(n, 16, 2)[:, :h, i].double() - 127)[..., None]
    k, v = read(0), read(1)
    y = torch.zeros((n, D), dtype=torch.float64, device="cuda")
    at = torch.arange(n, device="cuda") if s["nodes"] is None else s["nodes"].long()
    for part in at.split(65536):
        cone = s["cone"][part]
        row, col = torch.nonzero(cone >= 0, as_tuple=True)
        src = cone[row, col].long()
        e = torch.exp(torch.einsum("ehd,ehd->eh", s["q"].double().view(n, h, -1)[part[row]], k[src]) / math.sqrt(D / h))
        z = torch.zeros((part.numel(), h), dtype=torch.float64, device="cuda").index_add_(0, row, e)
        o = torch.zeros((part.numel(), h, D // h), dtype=torch.float64, device="cuda").index_add_(0, row, e[..., None] * v[src])
        y[part] = (o / z[..., None]).view(-1, D)
    return [y]


def _exact_norm(s):
    def norm(x, gamma, beta):
        if s["rms"]:
            return x * torch.rsqrt(x.pow(2).mean(1, keepdim=True) + EPS) * gamma.double()
        var, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
        return (x - mean) * torch.rsqrt(var + EPS) * gamma.double() + beta.double()
    r = torch.zeros((s["n"], D), dtype=torch.float64, device="cuda")
    y = torch.zeros_like(r)
    for lo, hi, i in zip(s["seg_ptr"].tolist()[:-1], s["seg_ptr"].tolist()[1:], s["seg_id"].tolist()):
        if hi > lo:
            g = s["gate"][i].double() if i >= 0 else 1.0
            r[lo:hi] = s["res"][lo:hi].double() * s["res_scale"] + norm(s["x"][lo:hi].double(), *s["post"]) * g
            y[lo:hi] = norm(r[lo:hi], *s["pre"])
    return [r, y]


def exact(case, seed):
    s = prepare(case, seed)
    return {"qkv": _exact_project, "out": _exact_project, "kv8": _exact_kv8, "attn": _exact_attn, "norm": _exact_norm}[case["op"]](s)
