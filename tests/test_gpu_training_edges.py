"""GPU tests of the training calls at their edges; the expected values and tolerances are built as in test_gpu_training.py."""
import math

import pytest
import torch

from paper_2502_01681_b200 import dg4
from test_gpu_training import ACT, BF16, SubLayer, act64, desc, edgeless, glu_case, glu_grads, normal, within, workspace

pytestmark = pytest.mark.gpu


def test_sums_over_many_rows_do_not_drift():
    """Products of one sign: what the tensor cores' accumulators cut off adds up.  They take 16 rows to an addition, each worth a
    unit of the last place (2^-23 of the sum) at the most in the mean; 131 072 rows are 8 192 additions, and beyond that their
    number does not grow.  The rounding to bf16 is even to both sides: over 8 192 elements its mean stays below
    4 * 2^-8 / sqrt(3 * 8192) = 1e-4."""
    n, d_ff, some = 2000003, 4808, 64                                    # one sum over all rows where their number sets no bound
    x, dy = normal(1, (n, 128)).abs_(), normal(2, (n, 128)).abs_()
    wg, wu = normal(3, (d_ff, 128), 0.02).abs_(), normal(4, (d_ff, 128), 0.02).abs_()
    wd = normal(5, (128, d_ff), 0.02).abs_()
    g, d = edgeless(n), desc()
    out = [torch.full_like(t, math.nan) for t in (wg, wu, wd)]
    ws = workspace(dg4.dg4_glu_bwd_workspace_bytes(g, d, d_ff))
    dg4.dg4_glu_bwd(g, d, x, wg, wu, wd, ACT["silu"], dy, None, *out, ws)
    want = [torch.zeros((some, 128), dtype=torch.float64, device="cuda") for _ in range(3)]
    w = [t.double() for t in (wg[-some:], wu[-some:], wd[:, -some:])]
    for xs, dys in zip(x.split(100000), dy.split(100000)):
        xs, dys = xs.double(), dys.double()
        a, da, _ = act64(xs @ w[0].T, "silu")
        u, h = xs @ w[1].T, dys @ w[2]
        for to, t, other in zip(want, (h * u * da, h * a, a * u), (xs, xs, dys)):
            to += t.T @ other
    for name, got, ref in zip(("dW_gate", "dW_up", "dW_down"), (out[0][-some:], out[1][-some:], out[2][:, -some:].T), want):
        off = (got.double() - ref) / ref
        assert abs(float(off.mean())) <= 8192 * 2.0 ** -23 + 1e-4, name
        assert float(off.abs().max()) <= 2.0 ** -8 + 8192 * 2.0 ** -23 + 1e-4, name


@pytest.mark.parametrize("n,d_ff", [(1500, 1024), (700, 768), (1100, 1544), (2000, 520), (400, 2048), (300, 4096)])
def test_dx_has_the_same_bits_with_and_without_the_weights_gradients(n, d_ff):
    x, wg, wu, wd = glu_case(n, n, d_ff)
    dy = normal(n + 9, (n, 128))
    g, d = edgeless(n), desc()
    out, alone = glu_grads(x, wg, wu, wd), torch.full_like(x, math.nan)
    dg4.dg4_glu_bwd(g, d, x, wg, wu, wd, ACT["silu"], dy, *out, workspace(dg4.dg4_glu_bwd_workspace_bytes(g, d, d_ff)))
    dg4.dg4_glu_bwd(g, d, x, wg, wu, wd, ACT["silu"], dy, alone, None, None, None)
    assert torch.equal(out[0], alone)


def test_relu_gates_that_are_closed_or_not_numbers_backward():
    n, d_ff, unit = 40, 96, 41
    x, wg, wu, wd = glu_case(201, n, d_ff)
    dy = normal(202, (n, 128))
    g, d = edgeless(n), desc()
    ws = workspace(dg4.dg4_glu_bwd_workspace_bytes(g, d, d_ff))
    wgp = wg.clone()
    wgp[unit, 5] = math.nan                                              # one gate of every row: its gradients are not numbers
    out = glu_grads(x, wg, wu, wd)
    dg4.dg4_glu_bwd(g, d, x, wgp, wu, wd, ACT["relu"], dy, *out, ws)
    assert bool(torch.isnan(out[1][unit]).all()) and bool(torch.isnan(out[2][unit]).all()) and bool(torch.isnan(out[3][:, unit]).all())
    keep = torch.arange(d_ff, device="cuda") != unit
    assert bool(torch.isfinite(out[1][keep]).all()) and bool(torch.isfinite(out[2][keep]).all())
    # an infinite U behind a closed gate: the gate's gradient is zero (0 * inf stays in act(G) U and so in W_down's gradient)
    xc = x.clone()
    xc[:, 5], xc[:, 6] = 1.0, 1.0
    wgc, wuc = wg.clone(), wu.clone()
    wgc[unit, 5], wuc[unit, 6] = -1000.0, math.inf
    out, ref = glu_grads(x, wg, wu, wd), glu_grads(x, wg, wu, wd)
    dg4.dg4_glu_bwd(g, d, xc, wgc, wuc, wd, ACT["relu"], dy, *out, ws)
    assert not bool(out[1][unit].any()) and not bool(out[2][unit].any())
    wuc[unit, 6] = 0.0
    dg4.dg4_glu_bwd(g, d, xc, wgc, wuc, wd, ACT["relu"], dy, *ref, ws)
    assert torch.equal(out[1], ref[1]) and torch.equal(out[2][keep], ref[2][keep]) and torch.equal(out[3][:, keep], ref[3][:, keep])
    # dX: that unit's U row is infinite, and its factor dU = dA * 0 meets it in the last product
    assert torch.equal(out[0][:, torch.arange(128, device="cuda") != 6], ref[0][:, torch.arange(128, device="cuda") != 6])


@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_gates_far_out_keep_what_bf16_can_hold(kind):
    """act(g) is a normal number some way past the gates whose sigmoid is below 2^-126."""
    values = [-80.0, -86.0, -87.5, -88.0, -88.5, -89.0, -90.0, -91.0] if kind == "silu" else [-9.5, -9.75, -9.9375, -10.0, -10.0625, -10.125, -10.5]
    n = len(values)
    x = torch.zeros((n, 128), dtype=BF16)
    for k in range(16):                                                  # every value in every place of a group of sixteen
        x[:, k] = torch.tensor(values).roll(k).to(BF16)
    x[:, 127] = 1
    wg, wu, wd = torch.zeros((16, 128)), torch.zeros((16, 128)), torch.zeros((128, 16))
    for k in range(16):
        wg[k, k] = wu[k, 127] = wd[k, k] = 1
    x, wg, wu, wd = x.cuda(), wg.to(BF16).cuda(), wu.to(BF16).cuda(), wd.to(BF16).cuda()
    y = torch.empty_like(x)
    dg4.dg4_glu_fwd(edgeless(n), desc(), x, wg, wu, wd, ACT[kind], None, y)
    g = x[:, :16].double()
    want = act64(g, kind)[0]
    # two roundings to bf16; the exponent p(g) is known to 2^-22 of itself, and a sigmoid of 2^-126 >> k to 2^-(23 - k), k < 8
    c = 2 * math.sqrt(2 / math.pi)
    size = g.abs() if kind == "silu" else c * (g.abs() + 0.044715 * g.abs() ** 3)
    part = 2 * 2.0 ** -8 + 2.0 ** -21 * size + 2.0 ** -15
    within(y[:, :16], want, want.abs() * part + 2.0 ** -126 * 2.0 ** -7, kind)
    dy, dx = torch.zeros_like(x), torch.empty_like(x)
    dy[:, :16] = 1
    dg4.dg4_glu_bwd(edgeless(n), desc(), x, wg, wu, wd, ACT[kind], dy, dx, None, None, None)
    slope = act64(g, kind)[1]
    terms = (want / g).abs() + want.abs() * (1 if kind == "silu" else c * (1 + 3 * 0.044715 * g * g))     # s and g s (1 - s) p'
    within(dx[:, :16], slope, terms * part + 2.0 ** -126 * 2.0 ** -7, kind)


def test_calls_behind_copies_fills_events_and_joined_streams():
    """The kernels may begin before what is in front of them on the stream has ended: not before a copy, a fill or another
    stream's work has."""
    n, d_ff = 30001, 136
    s = SubLayer(n, d_ff, 210)
    h, up = s.h.clone(), s.up.clone()
    s.step()
    want = s.results()
    side, aside = torch.cuda.Stream(), torch.cuda.Stream()

    def spoil():
        for t in (s.h, s.up, s.norm, s.out, s.dn, s.dh, *s.grads):
            t.fill_(math.nan)

    def chain():
        now = torch.cuda.current_stream()
        spoil()
        s.h.copy_(h)                                                     # a copy right in front of a call
        dg4.dg4_add_norm_fwd(s.g, s.d, s.h, None, s.gamma, s.beta, 1e-5, None, s.norm)
        side.wait_stream(now)
        aside.wait_stream(now)
        with torch.cuda.stream(side):                                    # two streams' work is joined in front of the next ones
            dg4.dg4_glu_fwd(s.g, s.d, s.norm, s.wg, s.wu, s.wd, ACT["silu"], s.h, s.out)
        with torch.cuda.stream(aside):
            s.up.fill_(1.0)
            torch.cuda._sleep(200000)                                    # some 0.1 ms: what comes behind the join has to wait
            s.up.copy_(up)
        now.wait_stream(side)
        now.wait_stream(aside)
        dg4.dg4_glu_bwd(s.g, s.d, s.norm, s.wg, s.wu, s.wd, ACT["silu"], s.up, s.dn, *s.grads[:3], s.ws)
        side.wait_stream(now)
        with torch.cuda.stream(side):                                    # a call behind another stream's weights' kernel
            dg4.dg4_norm_bwd(s.g, s.d, s.h, s.gamma, 1e-5, s.dn, s.up, s.dh, *s.grads[3:], s.ws2)
        now.wait_stream(side)

    s.ws2 = workspace(max(dg4.dg4_norm_bwd_workspace_bytes(s.g, s.d), 16))
    for _ in range(10):
        chain()
        got = s.results()
        assert all(torch.equal(p, q) for p, q in zip(got, want))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        chain()
    for _ in range(5):
        spoil()
        graph.replay()
        got = s.results()
        assert all(torch.equal(p, q) for p, q in zip(got, want))
    del graph


def test_workspace_sizes_are_the_handle_s_whichever_device_is_current():
    g, d = edgeless(5000), desc()
    want = dg4.dg4_glu_bwd_workspace_bytes(g, d, 512), dg4.dg4_norm_bwd_workspace_bytes(g, d)
    assert min(want) > 0
    dg4.dg4_debug_override_current_device(1)                             # as if another GPU were current on this thread
    try:
        assert (dg4.dg4_glu_bwd_workspace_bytes(g, d, 512), dg4.dg4_norm_bwd_workspace_bytes(g, d)) == want
    finally:
        dg4.dg4_debug_override_current_device(-1)


def test_several_rounds_of_row_groups_beside_dx():
    """128 blocks and 2 345 tiles: three groups one after the other on the SMs that one group takes."""
    n, d_ff = 300033, 8192
    x, wg, wu, wd = glu_case(220, n, d_ff)
    dy = normal(221, (n, 128))
    g, d = edgeless(n), desc()
    size = dg4.dg4_glu_bwd_workspace_bytes(g, d, d_ff)
    assert size > dg4.dg4_glu_bwd_workspace_bytes(edgeless(131072), d, d_ff) == 0
    ws, out, parts = workspace(size), glu_grads(x, wg, wu, wd), glu_grads(x, wg, wu, wd)
    for _ in range(2):
        dg4.dg4_glu_bwd(g, d, x, wg, wu, wd, ACT["gelu"], dy, *out, ws)
    dg4.dg4_glu_bwd(g, d, x, wg, wu, wd, ACT["gelu"], dy, parts[0], None, None, None, None)
    dg4.dg4_glu_bwd(g, d, x, wg, wu, wd, ACT["gelu"], dy, None, *parts[1:], ws)
    assert all(torch.equal(p, q) for p, q in zip(out, parts)) and all(bool(torch.isfinite(t).all()) for t in out)
    assert dg4.dg4_graph_poll_status(g) == dg4.DG4_OK
