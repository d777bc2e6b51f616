"""GPU tests of the training calls: the gated feed-forward sub-layer and the norm of a residual sum, forward and backward.
The expected values are plain 64-bit formulas; the tolerances count roundings on sums of absolute values: half a step of the
storage type per stored value (bf16 2^-8, fp32 2^-24 of the value), 2^-19 per product of 128 inputs summed in 32 bits
(8 steps of 2^-23 of the sum of absolute values, doubled), and for the tensor cores' longer sums 2^-23 a step."""
import math

import numpy as np
import pytest
import torch

from paper_2502_01681_b200 import dg4

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
HALF = {BF16: 2.0 ** -8, F32: 2.0 ** -24}
TAG = {BF16: dg4.DG4_BF16, F32: dg4.DG4_F32}
ACT = {"silu": dg4.DG4_ACT_SILU, "gelu": dg4.DG4_ACT_GELU, "relu": dg4.DG4_ACT_RELU}
EPS = 1e-5


def edgeless(n):
    return dg4.dg4_graph_create(np.zeros(n + 1, np.int32), np.zeros(0, np.int32), np.zeros(n, np.int32), 1)


def desc(dtype=BF16, **kw):
    return dg4.desc(8, TAG[dtype], 0.25, **kw)


def normal(seed, shape, std=1.0, dtype=BF16):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def strided(t, ld, offset=0):
    """The same rows in a buffer with another row distance, beginning `offset` elements into it; the rest is NaN."""
    buf = torch.full((t.shape[0] * ld + offset,), math.nan, dtype=t.dtype, device="cuda")
    view = buf[offset:].view(t.shape[0], ld)[:, :128]
    view.copy_(t)
    return view


def within(got, want, tol, what=""):
    got = got.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    same = torch.isnan(want) | (got == want)                             # infinities too
    off = torch.where(same, torch.zeros_like(want), (got - want).abs() / tol.clamp(min=1e-300))
    assert float(off.max()) <= 1.0, (what, float(off.max()), int(off.argmax()))


def workspace(size):
    return torch.full((size,), 0xff, dtype=torch.uint8, device="cuda") if size else None    # stale bytes: NaN in every type


# ---------------------------------------------------------------------------------------------------
# gated sub-layer
# ---------------------------------------------------------------------------------------------------
def act64(g, kind):
    """act, act' and a bound of |act''|, in 64 bits."""
    if kind == "relu":
        return g.clamp(min=0), (g > 0).double(), 0.0
    if kind == "silu":
        p, dp = g, torch.ones_like(g)
    else:
        c = math.sqrt(2 / math.pi)
        p, dp = 2 * c * (g + 0.044715 * g ** 3), 2 * c * (1 + 3 * 0.044715 * g ** 2)
    s = torch.sigmoid(p)
    return g * s, s + g * torch.sigmoid(-p) * s * torch.nan_to_num(dp), 1.2


def glu_case(seed, n, d_ff):
    x = normal(seed, (n, 128))
    return x, normal(seed + 1, (d_ff, 128), 0.09), normal(seed + 2, (d_ff, 128), 0.09), normal(seed + 3, (128, d_ff), 1 / math.sqrt(d_ff))


def hidden64(x, wg, wu, kind):
    x, wg, wu = x.double(), wg.double(), wu.double()
    g, u = x @ wg.T, x @ wu.T
    eg, eu = 2.0 ** -19 * (x.abs() @ wg.abs().T), 2.0 ** -19 * (x.abs() @ wu.abs().T)       # how far G and U may be off
    a, da, curve = act64(g, kind)
    # 2^-20: the exponential and the reciprocal, a few units of the last place
    ea = (da.abs() + curve * eg) * eg + 2.0 ** -20 * a.abs() if kind != "relu" else eg
    eda = curve * eg + 2.0 ** -19 * (1 + a.abs()) if kind != "relu" else (g.abs() <= eg).double()
    return g, u, eg, eu, a, da, ea, eda


def glu_ref(x, wg, wu, wd, kind, res=None):
    _, u, _, eu, a, _, ea, _ = hidden64(x, wg, wu, kind)
    h, wd = a * u, wd.double()
    y = h @ wd.T
    steps = 2.0 ** -23 * (wd.shape[1] / 16 + 1)
    tol = (h.abs() * (2.0 ** -8 + steps) + ea * u.abs() + a.abs() * eu + ea * eu) @ wd.abs().T
    spread = ((h * h) @ (wd * wd).T).sum()                                # variance of the hidden values' rounding, of 2^-16 / 3
    if res is not None:
        y = y + res.double()
    tol = tol * (1 + 2.0 ** -8) + 2.0 ** -8 * y.abs()
    return y, tol, 2.0 ** -16 / 3 * (spread + (y * y).sum())


SHAPES = [  # rows, d_ff: one row, one block, ragged rows and blocks, several tiles and one, two, three blocks to a pair of CTAs
    (1, 8), (1, 512), (2, 64), (127, 64), (128, 72), (129, 200), (255, 128), (256, 344), (257, 520), (2051, 512), (2000, 1032),
    (19000, 64), (38001, 64), (57001, 128), (57001, 192), (60001, 40), (40001, 320), (700, 8192),
    (1, 2048), (1, 768), (300, 776), (513, 1544), (256, 2056), (3000, 896), (900, 4096)]       # few rows: pairs share a tile's blocks


@pytest.mark.parametrize("kind", ["silu", "gelu", "relu"])
@pytest.mark.parametrize("n,d_ff", SHAPES)
def test_glu_forward_matches_the_formula(n, d_ff, kind):
    x, wg, wu, wd = glu_case(n + d_ff, n, d_ff)
    for res in (None, normal(77, (n, 128))):
        y = torch.full_like(x, math.nan)
        g = edgeless(n)
        dg4.dg4_glu_fwd(g, desc(residual=True), x, wg, wu, wd, ACT[kind], res, y)
        want, tol, var = glu_ref(x, wg, wu, wd, kind, res)
        within(y, want, tol, (n, d_ff, kind))
        # the roundings are independent: their sum of squares stays near its expectation (3 times for the few samples of a row)
        assert float((y.double() - want).square().sum()) <= (3.0 if n < 8 else 1.5) * float(var)
        assert dg4.dg4_graph_poll_status(g) == dg4.DG4_OK


def glu_bwd_ref(x, wg, wu, wd, kind, dy):
    g, u, eg, eu, a, da, ea, eda = hidden64(x, wg, wu, kind)
    x, wg, wu, wd, dy = (t.double() for t in (x, wg, wu, wd, dy))
    h, eh = dy @ wd, 2.0 ** -19 * (dy.abs() @ wd.abs())
    dg, du, v = h * u * da, h * a, a * u
    edg = (eh * u.abs() + h.abs() * eu + eh * eu) * (da.abs() + eda) + (h * u).abs() * eda + 2.0 ** -21 * dg.abs()
    edu = eh * (a.abs() + ea) + h.abs() * ea + 2.0 ** -21 * du.abs()
    ev = ea * u.abs() + (a.abs() + ea) * eu
    half = 2.0 ** -8
    rows = 2.0 ** -23 * (x.shape[0] / 16 + 1) + 2.0 ** -22                # sums over the rows, and over their groups

    def sum_of(terms):                                                   # (value, its error, factor) triples: sum of value * factor
        want = sum(p @ q for p, _, q in terms)
        tol = sum((p.abs() * (half + rows) + e * (1 + half)) @ q.abs() for p, e, q in terms)
        var = sum(((p * p) @ (q * q)).sum() for p, _, q in terms)
        return want, tol * (1 + half) + half * want.abs(), 2.0 ** -16 / 3 * (var + (want * want).sum())
    return (sum_of([(dg, edg, wg), (du, edu, wu)]), sum_of([(dg.T, edg.T, x)]), sum_of([(du.T, edu.T, x)]),
            tuple(t.T if torch.is_tensor(t) and t.dim() == 2 else t for t in sum_of([(v.T, ev.T, dy)])))


def glu_grads(x, wg, wu, wd):
    return [torch.full_like(t, math.nan) for t in (x, wg, wu, wd)]


@pytest.mark.parametrize("kind", ["silu", "gelu", "relu"])
@pytest.mark.parametrize("n,d_ff", SHAPES)
def test_glu_backward_matches_the_formula(n, d_ff, kind):
    x, wg, wu, wd = glu_case(n + 3 * d_ff, n, d_ff)
    dy = normal(5, (n, 128))
    out = glu_grads(x, wg, wu, wd)
    g, d = edgeless(n), desc()
    ws = workspace(dg4.dg4_glu_bwd_workspace_bytes(g, d, d_ff))
    dg4.dg4_glu_bwd(g, d, x, wg, wu, wd, ACT[kind], dy, *out, ws)
    for name, got, (want, tol, var) in zip(("dX", "dW_gate", "dW_up", "dW_down"), out, glu_bwd_ref(x, wg, wu, wd, kind, dy)):
        within(got, want, tol, (name, n, d_ff, kind))
        if kind != "relu":                                               # (a gate near zero may count on the other side)
            assert float((got.double() - want).square().sum()) <= (4.0 if n < 8 or d_ff < 64 else 1.5) * float(var), name
    assert dg4.dg4_graph_poll_status(g) == dg4.DG4_OK


def test_glu_gradients_match_differences():
    n, d_ff = 300, 136
    x, wg, wu, wd = glu_case(9, n, d_ff)
    dy = normal(6, (n, 128))
    for kind in ("silu", "gelu"):
        out = glu_grads(x, wg, wu, wd)
        g, d = edgeless(n), desc()
        dg4.dg4_glu_bwd(g, d, x, wg, wu, wd, ACT[kind], dy, *out, workspace(dg4.dg4_glu_bwd_workspace_bytes(g, d, d_ff)))
        at = [t.double() for t in (x, wg, wu, wd)]

        def loss(p):
            return float(((act64(p[0] @ p[1].T, kind)[0] * (p[0] @ p[2].T)) @ p[3].T * dy.double()).sum())
        for i in range(4):
            move = torch.randn_like(at[i])
            step = 1e-5
            ahead, behind = ([t + (s * step * move if j == i else 0) for j, t in enumerate(at)] for s in (1, -1))
            slope = (loss(ahead) - loss(behind)) / (2 * step)
            along = float((out[i].double() * move).sum())
            # the gradient's elements are off by at most 2^-8 of themselves for each of two roundings, independent of the move;
            # six times the standard deviation of their sum
            assert abs(along - slope) <= 6 * 2 * 2.0 ** -8 * float(out[i].double().norm()) + 1e-5 * abs(slope), (kind, i)


def test_glu_strided_rows_and_places_in_the_middle_of_a_buffer():
    n, d_ff = 333, 96
    x, wg, wu, wd = glu_case(21, n, d_ff)
    res, dy = normal(22, (n, 128)), normal(23, (n, 128))
    g, d = edgeless(n), desc(residual=True)
    y, out = torch.empty_like(x), glu_grads(x, wg, wu, wd)
    dg4.dg4_glu_fwd(g, d, x, wg, wu, wd, ACT["silu"], res, y)
    ws = workspace(dg4.dg4_glu_bwd_workspace_bytes(g, d, d_ff))
    dg4.dg4_glu_bwd(g, d, x, wg, wu, wd, ACT["silu"], dy, *out, ws)
    for ld, offset in ((136, 8), (256, 128), (1000, 24)):
        xs, rs, dys = strided(x, ld, offset), strided(res, ld + 8, offset), strided(dy, ld + 16, offset)
        ys, dxs = strided(torch.zeros_like(x), ld + 24, offset), strided(torch.zeros_like(x), ld + 32, offset)
        dg4.dg4_glu_fwd(g, d, xs, wg, wu, wd, ACT["silu"], rs, ys)
        assert torch.equal(ys, y)
        assert bool(torch.isnan(ys.as_strided((n - 1, 24), (ys.stride(0), 1), ys.storage_offset() + 128)).all())   # between the rows
        again = glu_grads(x, wg, wu, wd)
        dg4.dg4_glu_bwd(g, d, xs, wg, wu, wd, ACT["silu"], dys, dxs, *again[1:], ws)
        assert torch.equal(dxs, out[0]) and all(torch.equal(p, q) for p, q in zip(again[1:], out[1:]))


def test_glu_in_place():
    n, d_ff = 60001, 72
    x, wg, wu, wd = glu_case(31, n, d_ff)
    res, dy = normal(32, (n, 128)), normal(33, (n, 128))
    g, d = edgeless(n), desc(residual=True)
    y, out = torch.empty_like(x), glu_grads(x, wg, wu, wd)
    dg4.dg4_glu_fwd(g, d, x, wg, wu, wd, ACT["gelu"], res, y)
    for over in (x.clone(), res.clone()):
        args = (over, res) if torch.equal(over, x) else (x, over)
        dg4.dg4_glu_fwd(g, d, args[0], wg, wu, wd, ACT["gelu"], args[1], over)
        assert torch.equal(over, y)
    post = torch.empty_like(x)                                           # X is the residual too
    dg4.dg4_glu_fwd(g, d, x, wg, wu, wd, ACT["gelu"], x, post)
    over = x.clone()
    dg4.dg4_glu_fwd(g, d, over, wg, wu, wd, ACT["gelu"], over, over)
    assert torch.equal(over, post)
    dg4.dg4_glu_bwd(g, d, x, wg, wu, wd, ACT["gelu"], dy, out[0], None, None, None)      # frozen weights: no workspace
    for over in (x.clone(), dy.clone()):
        args = (over, dy) if torch.equal(over, x) else (x, over)
        dg4.dg4_glu_bwd(g, d, args[0], wg, wu, wd, ACT["gelu"], args[1], over, None, None, None)
        assert torch.equal(over, out[0])


def test_glu_few_rows_in_place_and_with_wide_strides():
    for n, d_ff in ((5, 2048), (700, 1000)):                             # four pairs to a tile, and two
        x, wg, wu, wd = glu_case(35, n, d_ff)
        res, dy = normal(36, (n, 128)), normal(37, (n, 128))
        g, d = edgeless(n), desc(residual=True)
        y, dx = torch.empty_like(x), torch.empty_like(x)
        dg4.dg4_glu_fwd(g, d, x, wg, wu, wd, ACT["silu"], res, y)
        dg4.dg4_glu_bwd(g, d, x, wg, wu, wd, ACT["silu"], dy, dx, None, None, None)
        xs, rs, dys, out = strided(x, 200, 8), strided(res, 136, 16), strided(dy, 144, 8), strided(x, 1000, 24)
        dg4.dg4_glu_fwd(g, d, xs, wg, wu, wd, ACT["silu"], rs, out)
        assert torch.equal(out, y)
        assert n == 1 or bool(torch.isnan(out.as_strided((n - 1, 24), (1000, 1), out.storage_offset() + 128)).all())
        dg4.dg4_glu_fwd(g, d, xs, wg, wu, wd, ACT["silu"], rs, rs)
        assert torch.equal(rs, y)
        dg4.dg4_glu_bwd(g, d, xs, wg, wu, wd, ACT["silu"], dys, out, None, None, None)
        assert torch.equal(out, dx)
        dg4.dg4_glu_bwd(g, d, xs, wg, wu, wd, ACT["silu"], dys, dys, None, None, None)
        assert torch.equal(dys, dx)
        dg4.dg4_glu_fwd(g, d, xs, wg, wu, wd, ACT["silu"], res, xs)
        assert torch.equal(xs, y)


def test_glu_parts_of_the_gradients_are_the_same_bits_every_time():
    for n, d_ff in ((77, 512), (30001, 200)):
        x, wg, wu, wd = glu_case(41, n, d_ff)
        dy = normal(42, (n, 128))
        g, d = edgeless(n), desc()
        ws = workspace(dg4.dg4_glu_bwd_workspace_bytes(g, d, d_ff))
        first = glu_grads(x, wg, wu, wd)
        dg4.dg4_glu_bwd(g, d, x, wg, wu, wd, ACT["silu"], dy, *first, ws)
        for parts in ((1, 1), (1, 0), (0, 1)):
            out = glu_grads(x, wg, wu, wd)
            call = [out[0] if parts[0] else None] + (out[1:] if parts[1] else [None] * 3)
            for _ in range(3):
                dg4.dg4_glu_bwd(g, d, x, wg, wu, wd, ACT["silu"], dy, *call, ws)
            assert all(p is None or torch.equal(p, q) for p, q in zip(call, first))


@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_glu_activation_over_the_whole_range(kind):
    """Y = act(g) of chosen values: unit weights pick the gate's value from X, a one from X, and one hidden unit per output."""
    values = [0.0, -0.0, 1e-30, -1e-30, 1e-3, -1e-3, 0.5, -0.5, 3, -3, 9, -9, 20, -20, 21, -21.5, 22, -22, 25, -30, 31, -43, 44, -60, 80,
              -85, 100, 1e4, -1e4, 1e18, -1e18, 1e30, -1e30, 3e38, -3e38]
    if kind == "gelu":                                                   # its own tail ends at -13 or so
        values = [v for v in values if not -100 < v < -12.5] + [-4, -6, -8, -10, -12]
    rows = torch.tensor(values, dtype=F32).to(BF16)
    n = len(values)
    x = torch.zeros((n, 128), dtype=BF16)
    for k in range(16):                                                  # every value in every place of a group of sixteen
        x[:, k] = rows.roll(k)
    x[:, 127] = 1
    wg, wu, wd = torch.zeros((16, 128)), torch.zeros((16, 128)), torch.zeros((128, 16))
    for k in range(16):
        wg[k, k] = wu[k, 127] = wd[k, k] = 1
    x, wg, wu, wd = x.cuda(), wg.to(BF16).cuda(), wu.to(BF16).cuda(), wd.to(BF16).cuda()
    y = torch.empty_like(x)
    dg4.dg4_glu_fwd(edgeless(n), desc(), x, wg, wu, wd, ACT[kind], None, y)
    want = act64(x[:, :16].double(), kind)[0]
    want = torch.where(x[:, :16].double() < -1000, torch.zeros_like(want), want)
    # the exponent's own rounding is worth its size times 2^-23; below 2^-126 values are zero
    tol = want.abs() * (2.0 ** -8 + 2.0 ** -20 + 2.0 ** -22 * (x[:, :16].double().abs().clamp(max=100) ** (1 if kind == "silu" else 3))) + 2.0 ** -126
    within(y[:, :16], want, tol, kind)
    assert not bool(y[:, 16:].any())
    dy = torch.zeros_like(x)
    dy[:, :16] = 1
    dx = torch.empty_like(x)
    dg4.dg4_glu_bwd(edgeless(n), desc(), x, wg, wu, wd, ACT[kind], dy, dx, None, None, None)
    g = x[:, :16].double()
    slope = act64(g.clamp(-1000, 1000), kind)[1]
    # s + g s (1 - s) p': its two parts may cancel, and 1 - s is known to 2^-24
    sig = torch.sigmoid(g if kind == "silu" else 2 * math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3))
    size = sig + (g * sig).abs() * (1 if kind == "silu" else (1 + 0.11 * g * g).clamp(max=1e5))
    size = torch.where(g < -1000, torch.zeros_like(size), size)
    within(dx[:, :16], slope, 2.0 ** -8 * slope.abs() + 2.0 ** -17 * torch.where(g > 1000, torch.ones_like(size), size) + 2.0 ** -120, kind)


def test_glu_values_stay_in_their_rows_and_units():
    n, d_ff = 200, 152
    x, wg, wu, wd = glu_case(51, n, d_ff)
    dy = normal(52, (n, 128))
    g, d = edgeless(n), desc()
    y, out = torch.empty_like(x), glu_grads(x, wg, wu, wd)
    ws = workspace(dg4.dg4_glu_bwd_workspace_bytes(g, d, d_ff))
    dg4.dg4_glu_fwd(g, d, x, wg, wu, wd, ACT["silu"], None, y)
    dg4.dg4_glu_bwd(g, d, x, wg, wu, wd, ACT["silu"], dy, *out, ws)
    for poison in (math.nan, math.inf, -math.inf):
        xp, dyp = x.clone(), dy.clone()
        xp[17, 3] = dyp[130, 5] = poison
        yp, outp = torch.empty_like(x), glu_grads(x, wg, wu, wd)
        dg4.dg4_glu_fwd(g, d, xp, wg, wu, wd, ACT["silu"], None, yp)
        dg4.dg4_glu_bwd(g, d, xp, wg, wu, wd, ACT["silu"], dyp, *outp, ws)
        keep = torch.ones(n, dtype=torch.bool, device="cuda")
        keep[17] = False
        assert torch.equal(yp[keep], y[keep]) and not bool(torch.isfinite(yp[17]).any())
        keep[130] = False
        assert torch.equal(outp[0][keep], out[0][keep])
    # a hidden unit's weights that are not numbers spoil its own gradients alone (the rows behind the last would add 0 * inf)
    for poison in (math.nan, math.inf):
        wgp = wg.clone()
        wgp[70] = poison
        outp = glu_grads(x, wg, wu, wd)
        dg4.dg4_glu_bwd(g, d, x, wgp, wu, wd, ACT["silu"], dy, *outp, ws)
        keep = torch.ones(d_ff, dtype=torch.bool, device="cuda")
        keep[70] = False
        assert torch.equal(outp[1][keep], out[1][keep]) and torch.equal(outp[2][keep], out[2][keep])
        assert torch.equal(outp[3][:, keep], out[3][:, keep])
    wup = wu.clone()
    wup[:, 7] = math.inf                                                 # every U is infinite: ReLU gates of one row decide
    one = edgeless(1)
    xg = torch.zeros((1, 128), dtype=BF16, device="cuda")
    xg[0, 7] = 1
    outp = glu_grads(xg, wg, wu, wd)
    dg4.dg4_glu_bwd(one, d, xg, wg, wup, wd, ACT["relu"], dy[:1], *outp, None)
    _, u, _, _, a, da, _, _ = hidden64(xg, wg, wup, "relu")
    du = (dy[:1].double() @ wd.double()) * a
    assert bool(torch.isfinite(outp[2]).all()) and float((outp[2][:, 7].double() - du[0]).abs().max()) <= 2.0 ** -6 * float(du.abs().max())


@pytest.mark.parametrize("kind", ["silu", "gelu", "relu"])
def test_glu_gates_that_are_not_numbers_are_not_lost(kind):
    n, d_ff = 40, 96
    x, wg, wu, wd = glu_case(55, n, d_ff)
    dy = normal(56, (n, 128))
    g, d = edgeless(n), desc()
    for unit in (0, 41, 95):
        wgp = wg.clone()
        wgp[unit, 5] = math.nan                                          # one gate of every row
        y, out = torch.empty_like(x), glu_grads(x, wg, wu, wd)
        dg4.dg4_glu_fwd(g, d, x, wgp, wu, wd, ACT[kind], None, y)
        assert bool(torch.isnan(y).all())
        dg4.dg4_glu_bwd(g, d, x, wgp, wu, wd, ACT[kind], dy, *out, workspace(dg4.dg4_glu_bwd_workspace_bytes(g, d, d_ff)))
        assert bool(torch.isnan(out[2][unit]).all()) and bool(torch.isnan(out[3][:, unit]).all()) and bool(torch.isnan(out[0]).all())


def test_glu_offsets_past_32_bits():
    n, ld = 20000, 131072                                                # 5.2 GB from the first row to the last
    x, wg, wu, wd = glu_case(61, n, 64)
    res, dy = normal(62, (n, 128)), normal(63, (n, 128))
    g, d = edgeless(n), desc(residual=True)
    y, out = torch.empty_like(x), glu_grads(x, wg, wu, wd)
    ws = workspace(dg4.dg4_glu_bwd_workspace_bytes(g, d, 64))
    dg4.dg4_glu_fwd(g, d, x, wg, wu, wd, ACT["silu"], res, y)
    dg4.dg4_glu_bwd(g, d, x, wg, wu, wd, ACT["silu"], dy, *out, ws)
    big = torch.empty((n, ld), dtype=BF16, device="cuda")
    xs, rs, ys, dxs = (big[:, i * 128:(i + 1) * 128] for i in range(4))
    xs.copy_(x)
    rs.copy_(res)
    dg4.dg4_glu_fwd(g, d, xs, wg, wu, wd, ACT["silu"], rs, ys)
    assert torch.equal(ys, y)
    again = glu_grads(x, wg, wu, wd)
    dg4.dg4_glu_bwd(g, d, xs, wg, wu, wd, ACT["silu"], dy, dxs, *again[1:], ws)
    assert torch.equal(dxs, out[0]) and all(torch.equal(p, q) for p, q in zip(again[1:], out[1:]))


# ---------------------------------------------------------------------------------------------------
# norm of a residual sum
# ---------------------------------------------------------------------------------------------------
def norm64(z, rms, eps=EPS):
    """(xh, inv, how far xh may be off): mean and variance are sums of 128 in 32 bits."""
    z = z.double()
    mean = torch.zeros_like(z[:, :1]) if rms else z.mean(1, keepdim=True)
    c = z - mean
    inv = (c.square().mean(1, keepdim=True) + eps).rsqrt()
    xh = c * inv
    off = 2.0 ** -20 * (xh.abs() + inv * (0 if rms else 1) * z.abs().mean(1, keepdim=True))
    return xh, inv, off + xh.abs() * off.square().mean(1, keepdim=True).sqrt()


def norm_rows(seed, n, dtype):
    z = torch.randn((n, 128), generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")
    z = z * torch.exp2(torch.arange(n, device="cuda")[:, None] % 13 - 6.0) + (torch.arange(n, device="cuda")[:, None] % 3 - 1.0) * 4
    if n > 3:
        z[1], z[2] = 0.0, 3.0                                            # a row of zeros, a constant row
    return z.to(dtype)


NORM_ROWS = [1, 2, 31, 32, 33, 77, 128, 129, 1000, 9473, 100003]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("n", NORM_ROWS)
def test_add_norm_forward_matches_the_formula(n, rms, dtype):
    x, r = norm_rows(n, n, dtype), normal(n + 1, (n, 128), 0.5, dtype)
    gamma, beta = 1 + normal(1, (128,), 0.3, F32), normal(2, (128,), 0.3, F32)
    g, d = edgeless(n), desc(dtype, rms_norm=rms)
    for res, b, keep in ((r, beta, True), (None, None, True), (r, None, False)):
        z, y = (torch.full_like(x, math.nan) for _ in range(2))
        dg4.dg4_add_norm_fwd(g, d, x, res, gamma, b, EPS, z if keep else None, y)
        sum_ = x.double() + (res.double() if res is not None else 0)
        xh, inv, off = norm64(sum_, rms)
        off = off + 2.0 ** -23 * inv * (x.double().abs() + sum_.abs())   # the sum is held in 32 bits
        want = xh * gamma.double() + (b.double() if b is not None else 0)
        tol = off * gamma.double().abs() + 2.0 ** -22 * (xh * gamma.double()).abs() + HALF[dtype] * want.abs() * (1 + 2.0 ** -8) + 2.0 ** -23 * want.abs()
        within(y, want, tol, (n, rms))
        if keep:
            within(z, sum_, HALF[dtype] * sum_.abs() * (1 + 2.0 ** -8) + 2.0 ** -24 * sum_.abs(), "Z")
        else:
            assert bool(torch.isnan(z).all())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("n", NORM_ROWS)
def test_norm_backward_matches_the_formula(n, rms, dtype):
    z, dy, dr = norm_rows(n + 7, n, dtype), normal(n + 8, (n, 128), 1.0, dtype), normal(n + 9, (n, 128), 1.0, dtype)
    gamma = 1 + normal(3, (128,), 0.3, F32)
    g, d = edgeless(n), desc(dtype, rms_norm=rms)
    ws = workspace(dg4.dg4_norm_bwd_workspace_bytes(g, d))
    xh, inv, off = norm64(z, rms)
    t = dy.double() * gamma.double()
    m2 = (t * xh).mean(1, keepdim=True)
    base = t - xh * m2 - (0 if rms else t.mean(1, keepdim=True))
    et = 2.0 ** -20 * (t.abs() + t.abs().mean(1, keepdim=True)) + off * m2.abs() + xh.abs() * (
        (t.abs() * off).mean(1, keepdim=True) + 2.0 ** -20 * (t * xh).abs().mean(1, keepdim=True)) + 2.0 ** -21 * (xh * m2).abs()
    rel = 2.0 ** -20 + (xh.abs() * off).mean(1, keepdim=True)            # how far inv may be off, of itself
    adds = 2.0 ** -24 * (n / 4000 + 30)                                  # sums over rows: a lane's own, then trees
    want_g, want_b = (dy.double() * xh).sum(0), dy.double().sum(0)
    tol_g = (dy.double().abs() * (off + 2.0 ** -23 * xh.abs())).sum(0) + adds * (dy.double() * xh).abs().sum(0)
    for res, parts in ((dr, (1, 1, 1)), (None, (1, 1, 1)), (dr, (1, 0, 0)), (None, (0, 1, 0)), (None, (0, 0, 1)), (None, (1, 0, 1))):
        dz, dgm, dbt = torch.full_like(z, math.nan), torch.full((128,), math.nan, device="cuda"), torch.full((128,), math.nan, device="cuda")
        out = [p if use else None for p, use in zip((dz, dgm, dbt), parts)]
        dg4.dg4_norm_bwd(g, d, z, gamma, EPS, dy, res, *out, ws if parts[1] or parts[2] else None)
        want = inv * base + (res.double() if res is not None else 0)
        tol = inv * (et + base.abs() * rel) + (HALF[dtype] * (1 + 2.0 ** -8) + 2.0 ** -22) * want.abs() + 2.0 ** -23 * (inv * base).abs()
        for name, got, ref, bound, use in (("dZ", dz, want, tol, parts[0]), ("dgamma", dgm, want_g, tol_g, parts[1]),
                                           ("dbeta", dbt, want_b, adds * dy.double().abs().sum(0), parts[2])):
            if use:
                within(got, ref, bound, (name, n, rms))
            else:
                assert bool(torch.isnan(got).all())


def test_norm_gradients_match_differences():
    n = 200
    z, dy = normal(1, (n, 128), 1.0, F32), normal(2, (n, 128), 1.0, F32)
    gamma, beta = 1 + normal(3, (128,), 0.3, F32), normal(4, (128,), 0.3, F32)
    for rms in (False, True):
        out = [torch.empty_like(t) for t in (z, gamma, beta)]
        g, d = edgeless(n), desc(F32, rms_norm=rms)
        dg4.dg4_norm_bwd(g, d, z, gamma, EPS, dy, None, *out, workspace(dg4.dg4_norm_bwd_workspace_bytes(g, d)))
        at = [t.double() for t in (z, gamma, beta)]

        def loss(p):
            return float(((norm64(p[0], rms)[0] * p[1] + p[2]) * dy.double()).sum())
        for i in range(3):
            move = torch.randn_like(at[i])
            ahead, behind = ([t + (s * 1e-5 * move if j == i else 0) for j, t in enumerate(at)] for s in (1, -1))
            slope = (loss(ahead) - loss(behind)) / 2e-5
            size = float((out[i].double() * move).abs().sum())
            assert abs(float((out[i].double() * move).sum()) - slope) <= 2.0 ** -18 * size + 1e-6 * abs(slope) + 1e-6, (rms, i)


def test_norm_in_place_strided_and_the_same_bits_every_time():
    n = 5001
    for dtype in (BF16, F32):
        x, r, dy, dr = (normal(70 + i, (n, 128), 1.0, dtype) for i in range(4))
        gamma, beta = 1 + normal(3, (128,), 0.3, F32), normal(4, (128,), 0.3, F32)
        g, d = edgeless(n), desc(dtype)
        z, y, dz, dgm, dbt = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x), torch.empty_like(gamma), torch.empty_like(gamma)
        ws = workspace(dg4.dg4_norm_bwd_workspace_bytes(g, d))
        dg4.dg4_add_norm_fwd(g, d, x, r, gamma, beta, EPS, z, y)
        dg4.dg4_norm_bwd(g, d, z, gamma, EPS, dy, dr, dz, dgm, dbt, ws)
        a, b = x.clone(), r.clone()                                      # Z over X, Y over R, and crossed
        dg4.dg4_add_norm_fwd(g, d, a, b, gamma, beta, EPS, a, b)
        assert torch.equal(a, z) and torch.equal(b, y)
        a, b = x.clone(), r.clone()
        dg4.dg4_add_norm_fwd(g, d, a, b, gamma, beta, EPS, b, a)
        assert torch.equal(b, z) and torch.equal(a, y)
        for over in range(3):
            args = [z.clone(), dy.clone(), dr.clone()]
            p, q = torch.empty_like(gamma), torch.empty_like(gamma)
            dg4.dg4_norm_bwd(g, d, args[0], gamma, EPS, args[1], args[2], args[over], p, q, ws)
            assert torch.equal(args[over], dz) and torch.equal(p, dgm) and torch.equal(q, dbt)
        step = 8 if dtype == BF16 else 4
        xs, rs, zs, ys = (strided(t, 128 + (i + 1) * step, step) for i, t in enumerate((x, r, z, y)))
        dg4.dg4_add_norm_fwd(g, d, xs, rs, gamma, beta, EPS, zs, ys)
        assert torch.equal(zs, z) and torch.equal(ys, y)
        dys, drs, dzs = strided(dy, 136, step), strided(dr, 144, 2 * step), strided(dy, 152, step)
        p, q = torch.empty_like(gamma), torch.empty_like(gamma)
        dg4.dg4_norm_bwd(g, d, zs, gamma, EPS, dys, drs, dzs, p, q, ws)
        assert torch.equal(dzs, dz) and torch.equal(p, dgm) and torch.equal(q, dbt)
        assert bool(torch.isnan(dzs.as_strided((n - 1, 24), (152, 1), dzs.storage_offset() + 128)).all())


def test_norm_values_stay_in_their_rows_and_offsets_past_32_bits():
    n, ld = 20000, 131072
    z, dy = normal(80, (n, 128)), normal(81, (n, 128))
    gamma = 1 + normal(3, (128,), 0.3, F32)
    g, d = edgeless(n), desc()
    y, dz, dgm, dbt = torch.empty_like(z), torch.empty_like(z), torch.empty_like(gamma), torch.empty_like(gamma)
    ws = workspace(dg4.dg4_norm_bwd_workspace_bytes(g, d))
    dg4.dg4_add_norm_fwd(g, d, z, None, gamma, None, EPS, None, y)
    dg4.dg4_norm_bwd(g, d, z, gamma, EPS, dy, None, dz, dgm, dbt, ws)
    for poison in (math.nan, math.inf):
        zp, yp, dzp = z.clone(), torch.empty_like(z), torch.empty_like(z)
        zp[4321, 9] = poison
        dg4.dg4_add_norm_fwd(g, d, zp, None, gamma, None, EPS, None, yp)
        dg4.dg4_norm_bwd(g, d, zp, gamma, EPS, dy, None, dzp, None, None, None)
        keep = torch.arange(n, device="cuda") != 4321
        assert torch.equal(yp[keep], y[keep]) and torch.equal(dzp[keep], dz[keep]) and bool(torch.isnan(yp[4321]).any())
    big = torch.empty((n, ld), dtype=BF16, device="cuda")
    zs, ys, dys, dzs = (big[:, i * 128:(i + 1) * 128] for i in range(4))
    zs.copy_(z)
    dys.copy_(dy)
    p, q = torch.empty_like(gamma), torch.empty_like(gamma)
    dg4.dg4_add_norm_fwd(g, d, zs, None, gamma, None, EPS, None, ys)
    dg4.dg4_norm_bwd(g, d, zs, gamma, EPS, dys, None, dzs, p, q, ws)
    assert torch.equal(ys, y) and torch.equal(dzs, dz) and torch.equal(p, dgm) and torch.equal(q, dbt)


# ---------------------------------------------------------------------------------------------------
# together, captured, on streams; error paths
# ---------------------------------------------------------------------------------------------------
class SubLayer:
    """A pre-norm feed-forward sub-layer with its buffers: N = Norm(H), H' = H + GLU(N), and its gradients."""
    def __init__(self, n, d_ff, seed):
        self.g, self.d = edgeless(n), desc(residual=True)
        self.h, self.wg, self.wu, self.wd = glu_case(seed, n, d_ff)
        self.gamma, self.beta = 1 + normal(seed + 5, (128,), 0.2, F32), normal(seed + 6, (128,), 0.2, F32)
        self.up = normal(seed + 7, (n, 128))
        self.norm, self.out, self.dn, self.dh = (torch.empty_like(self.h) for _ in range(4))
        self.grads = [torch.empty_like(t) for t in (self.wg, self.wu, self.wd, self.gamma, self.beta)]
        self.ws = workspace(max(dg4.dg4_glu_bwd_workspace_bytes(self.g, self.d, d_ff), dg4.dg4_norm_bwd_workspace_bytes(self.g, self.d), 16))

    def step(self, kind="silu"):
        dg4.dg4_add_norm_fwd(self.g, self.d, self.h, None, self.gamma, self.beta, EPS, None, self.norm)
        dg4.dg4_glu_fwd(self.g, self.d, self.norm, self.wg, self.wu, self.wd, ACT[kind], self.h, self.out)
        dg4.dg4_glu_bwd(self.g, self.d, self.norm, self.wg, self.wu, self.wd, ACT[kind], self.up, self.dn, *self.grads[:3], self.ws)
        dg4.dg4_norm_bwd(self.g, self.d, self.h, self.gamma, EPS, self.dn, self.up, self.dh, *self.grads[3:], self.ws)

    def results(self):
        return [t.clone() for t in (self.out, self.dh, *self.grads)]


def test_a_sub_layer_trains_forward_and_backward():
    n, d_ff = 1500, 344
    for kind in ("silu", "gelu"):
        s = SubLayer(n, d_ff, 90)
        s.step(kind)
        p = [t.double().requires_grad_() for t in (s.h, s.wg, s.wu, s.wd, s.gamma, s.beta)]
        nrm = torch.nn.functional.layer_norm(p[0], (128,), p[4], p[5], EPS)
        act = torch.nn.functional.silu if kind == "silu" else lambda t: torch.nn.functional.gelu(t, approximate="tanh")
        out = p[0] + (act(nrm @ p[1].T) * (nrm @ p[2].T)) @ p[3].T
        out.backward(s.up.double())
        for got, want in zip(s.results(), (out.detach(), *(t.grad for t in p))):
            # a chain of at most four independent roundings to bf16 (norm, hidden values, dN, the result): each adds at most 2^-8 of
            # the norm, by their squares
            assert float((got.double() - want).norm()) <= 2 * 2.0 ** -8 * float(want.norm())


def test_captured_calls_and_two_streams_give_the_same_bits():
    subs = [SubLayer(3001, 200, 100), SubLayer(40000, 72, 110), SubLayer(5, 512, 120)]
    want = []
    for s in subs:
        s.step()
        want.append(s.results())
    # on streams of their own, all at once, several times
    streams = [torch.cuda.Stream() for _ in subs]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, st in zip(subs, streams):
            with torch.cuda.stream(st):
                s.step()
    torch.cuda.synchronize()
    for s, w in zip(subs, want):
        assert all(torch.equal(p, q) for p, q in zip(s.results(), w))
    # captured, and replayed with other inputs in the same buffers
    for s, w in zip(subs, want):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            s.step()
        keep = s.h.clone(), s.up.clone()
        s.h.copy_(normal(7, s.h.shape))
        s.up.copy_(normal(8, s.h.shape))
        graph.replay()
        torch.cuda.synchronize()
        other = s.results()
        s.step()
        assert all(torch.equal(p, q) for p, q in zip(s.results(), other))
        s.h.copy_(keep[0])
        s.up.copy_(keep[1])
        graph.replay()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(s.results(), w))
        del graph


def test_calls_one_after_the_other_see_one_another():
    """The weights' kernel begins beside dX's, the reductions behind their sums: what follows on the stream sees both done."""
    n, d_ff = 2500, 128
    s = SubLayer(n, d_ff, 130)
    s.step()
    want = s.results()
    for _ in range(30):
        for t in (s.dn, s.dh, *s.grads):
            t.fill_(math.nan)
        s.step()
        got = [t + 0 for t in (s.out, s.dh, *s.grads)]                   # a kernel of torch's right behind
        s.dn.fill_(math.nan)
        assert all(torch.equal(p, q) for p, q in zip(got, want))


@pytest.mark.parametrize("n,d_ff", [(1, 8), (700, 200), (40001, 512), (10, 2048), (600, 800)])
def test_waits_that_run_out_are_reported_and_leave_the_calls_usable(n, d_ff):
    s = SubLayer(n, d_ff, 140)
    s.step()
    want = s.results()
    bad = edgeless(n)
    dg4.dg4_debug_set_poll_limit(1)
    try:
        y, out = torch.empty_like(s.h), glu_grads(s.h, s.wg, s.wu, s.wd)
        dg4.dg4_glu_fwd(bad, s.d, s.norm, s.wg, s.wu, s.wd, ACT["silu"], s.h, y)
        torch.cuda.synchronize()
        dg4.dg4_glu_fwd(bad, s.d, s.norm, s.wg, s.wu, s.wd, ACT["silu"], None, y)
        torch.cuda.synchronize()
        dg4.dg4_glu_bwd(bad, s.d, s.norm, s.wg, s.wu, s.wd, ACT["silu"], s.up, out[0], None, None, None)
        torch.cuda.synchronize()
        dg4.dg4_glu_bwd(bad, s.d, s.norm, s.wg, s.wu, s.wd, ACT["silu"], s.up, *out, s.ws)
        torch.cuda.synchronize()
    finally:
        dg4.dg4_debug_set_poll_limit(0)
    assert dg4.dg4_graph_poll_status(bad) == dg4.DG4_ERR_TIMEOUT
    s.step()
    assert dg4.dg4_graph_poll_status(s.g) == dg4.DG4_OK
    assert all(torch.equal(p, q) for p, q in zip(s.results(), want))


def test_refusals():
    n, d_ff = 300, 64
    x, wg, wu, wd = glu_case(150, n, d_ff)
    g, d, f32 = edgeless(n), desc(), desc(F32)
    y, grads = torch.empty_like(x), glu_grads(x, wg, wu, wd)
    vec = torch.ones(128, device="cuda")
    ws = workspace(dg4.dg4_glu_bwd_workspace_bytes(g, d, d_ff))
    nws = workspace(dg4.dg4_norm_bwd_workspace_bytes(g, d))
    assert ws is not None and nws is not None
    silu = ACT["silu"]
    odd = torch.empty(n * 128 + 8, dtype=BF16, device="cuda")[1:n * 128 + 1].view(n, 128)
    uneven = torch.empty((n, 132), dtype=BF16, device="cuda")[:, :128]
    big = [torch.zeros(s, dtype=BF16, device="cuda") for s in ((8200, 128), (8200, 128), (128, 8200))]
    tiny = [torch.zeros(s, dtype=BF16, device="cuda") for s in ((12, 128), (12, 128), (128, 12))]
    nan = float("nan")
    INV, UNS = dg4.DG4_ERR_INVALID_ARG, dg4.DG4_ERR_UNSUPPORTED
    calls = [
        (UNS, lambda: dg4.dg4_glu_fwd(g, f32, x, wg, wu, wd, silu, None, y)),
        (UNS, lambda: dg4.dg4_glu_fwd(g, d, x, wg, wu, wd, 3, None, y)),
        (UNS, lambda: dg4.dg4_glu_fwd(g, d, x, *big, silu, None, y)),
        (UNS, lambda: dg4.dg4_glu_fwd(g, d, x, *tiny, silu, None, y)),
        (INV, lambda: dg4.dg4_glu_fwd(g, d, odd, wg, wu, wd, silu, None, y)),
        (INV, lambda: dg4.dg4_glu_fwd(g, d, x, wg, wu, wd, silu, None, uneven)),
        (INV, lambda: dg4.dg4_glu_fwd(g, desc(residual=True), x, wg, wu, wd, silu, odd, y)),
        (INV, lambda: dg4.dg4_glu_bwd(g, d, x, wg, wu, wd, silu, odd, *grads, ws)),
        (INV, lambda: dg4.dg4_glu_bwd(g, d, x, wg, wu, wd, silu, y, *grads, None)),
        (INV, lambda: dg4.dg4_glu_bwd(g, d, x, wg, wu, wd, silu, y, *grads, ws[:-1])),
        (INV, lambda: dg4.dg4_glu_bwd(g, d, x, wg, wu, wd, silu, y, *grads, torch.empty(ws.numel() + 8, dtype=torch.uint8, device="cuda")[8:])),
        (INV, lambda: dg4.dg4_glu_bwd(g, d, x, wg, wu, wd, silu, y, None, None, None, None)),
        (INV, lambda: dg4.dg4_glu_bwd(g, d, x, wg, wu, wd, silu, y, x, *grads[1:], ws)),
        (INV, lambda: dg4.dg4_glu_bwd(g, d, x, wg, wu, wd, silu, y, y, *grads[1:], ws)),
        (UNS, lambda: dg4.dg4_glu_bwd(g, f32, x, wg, wu, wd, silu, y, *grads, ws)),
        (INV, lambda: dg4.dg4_glu_bwd(g, d, x, wg, wu, wd, silu, y, grads[0], wg, *grads[2:], ws)),
        (INV, lambda: dg4.dg4_glu_bwd(g, d, x, wg, wu, wd, silu, y, grads[0], grads[1], grads[1], grads[3], ws)),
        (INV, lambda: dg4.dg4_glu_fwd(g, d, x, wg, wu, wd, silu, None, x.as_strided((n // 2, 128), (256, 1)))),
        (INV, lambda: dg4.dg4_add_norm_fwd(g, d, x, None, vec, None, -1.0, None, y)),
        (INV, lambda: dg4.dg4_add_norm_fwd(g, d, x, None, vec, None, nan, None, y)),
        (INV, lambda: dg4.dg4_add_norm_fwd(g, d, x, None, None, None, EPS, None, y)),
        (INV, lambda: dg4.dg4_add_norm_fwd(g, d, x, None, vec, None, EPS, y, y)),
        (INV, lambda: dg4.dg4_add_norm_fwd(g, d, x, odd, vec, None, EPS, None, y)),
        (INV, lambda: dg4.dg4_norm_bwd(g, d, x, vec, EPS, y, None, None, None, None, nws)),
        (INV, lambda: dg4.dg4_norm_bwd(g, d, x, vec, EPS, y, None, None, vec, vec, nws)),
        (INV, lambda: dg4.dg4_norm_bwd(g, d, x, vec, EPS, y, None, None, torch.empty(128, device="cuda"), None, None)),
        (INV, lambda: dg4.dg4_norm_bwd(g, d, x, vec, EPS, y, None, None, torch.empty(128, device="cuda"), None, nws[:-4])),
        (INV, lambda: dg4.dg4_norm_bwd(g, d, x, vec, -1e-9, y, None, y, None, None, None)),
        (INV, lambda: dg4.dg4_norm_bwd(g, d, x, vec, EPS, y, uneven, y, None, None, None)),
    ]
    launches = dg4.dg4_launch_count()
    for i, (status, call) in enumerate(calls):
        with pytest.raises(dg4.Dg4Error) as e:
            call()
        assert e.value.status == status and e.value.detail, i
    dg4.dg4_debug_override_current_device(1)                             # as if another GPU were current on this thread
    try:
        for call in (lambda: dg4.dg4_glu_fwd(g, d, x, wg, wu, wd, silu, None, y), lambda: dg4.dg4_glu_bwd(g, d, x, wg, wu, wd, silu, y, *grads, ws),
                     lambda: dg4.dg4_add_norm_fwd(g, d, x, None, vec, None, EPS, None, y),
                     lambda: dg4.dg4_norm_bwd(g, d, x, vec, EPS, y, None, grads[0], None, None, None)):
            with pytest.raises(dg4.Dg4Error) as e:
                call()
            assert e.value.status == INV
    finally:
        dg4.dg4_debug_override_current_device(-1)
    with pytest.raises(ValueError):
        dg4.dg4_glu_bwd(g, d, x, wg, wu, wd, silu, y, grads[0], grads[1], None, None, ws)
    assert dg4.dg4_launch_count() == launches                            # nothing was started
    for t in ("d = 64", 64), ("heads", 3):
        bad = desc()
        setattr(bad, "d" if t[1] == 64 else "heads", t[1])
        with pytest.raises(dg4.Dg4Error):
            dg4.dg4_glu_fwd(g, bad, x, wg, wu, wd, silu, None, y)
