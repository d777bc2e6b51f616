"""More GPU tests of the serving calls: long runs of short requests, strides and alignments, extreme and non-finite
values.  Formulas and tolerances are those of test_gpu_serving.py."""
import numpy as np
import pytest
import torch

from paper_2502_01681_b200 import dg4
from tests.test_gpu_serving import (BF16, HALF, U32, attn_ref, circuit, desc, edgeless, f64, gated_ref, hard_rows, i32,
                                    make_adapters, normal, project_ref, table_ref, vectors, within)

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------------------------------------------
# projections with adapters
# ---------------------------------------------------------------------------------------------------
def project_ref_by_adapter(x, w, ad, ptr, ids, res=None):
    """project_ref with the rows of one adapter taken together: it is one formula per row, and thousands of products of a
    few rows are slow on the CPU."""
    of_row = torch.from_numpy(np.repeat(ids, np.diff(ptr)))
    y, tol = (torch.zeros((x.shape[0], w.shape[0]), dtype=torch.float64) for _ in range(2))
    for i in sorted(set(ids)):
        at = torch.nonzero(of_row == i)[:, 0]
        on = at.cuda()
        y[at], tol[at], _ = project_ref(x[on], w, ad, [0, len(at)], [i], None if res is None else res[on])
    return y, tol


@pytest.mark.parametrize("rank,residual", [(16, True), (16, False), (64, True), (64, False), (8, True)])
def test_out_projection_over_thousands_of_short_requests(rank, residual):
    """Some forty items per CTA, the adapter (or none) another at nearly every one: the next item's product runs ahead of
    this one's second product all along.  Every repetition gives the same bits."""
    rng = np.random.default_rng(11)
    count = 6000
    lens = rng.choice([1, 2, 7, 31, 32, 33, 64], size=count)
    ptr = np.concatenate([[0], np.cumsum(lens)]).tolist()
    n, ids = ptr[-1], rng.integers(-1, 8, size=count).tolist()
    g = edgeless(n)
    o, w, res, ad = normal(1, (n, 128)), normal(2, (128, 128), 0.1), normal(4, (n, 128)), make_adapters(3, 8, rank, 128)
    seg = dg4.segments(i32(ptr), i32(ids))
    first = torch.empty((n, 128), dtype=BF16, device="cuda")
    dg4.dg4_out_project_adapters(g, desc(residual=residual), o, w, ad, seg, res, first)
    y, tol = project_ref_by_adapter(o, w, ad, ptr, ids, res if residual else None)
    within(first, y, tol)
    for _ in range(30):
        again = torch.zeros_like(first)
        dg4.dg4_out_project_adapters(g, desc(residual=residual), o, w, ad, seg, res, again)
        assert torch.equal(first, again)
    assert dg4.dg4_graph_poll_status(g) == 0


@pytest.mark.parametrize("n_out", [128, 384])
@pytest.mark.parametrize("before,between,behind", [(0, 20_000_000, 0), (0, 40, 17), (1000, 3_000_000, 5000), (15, 16, 1)])
def test_long_runs_of_empty_requests(before, between, behind, n_out):
    """Empty requests in front of the first row, inside one CTA's share of the items (some have rows next to them), and at
    the end."""
    n = 148 * 3 * 128
    g = edgeless(n)
    ptr = torch.cat([torch.full((k,), v, dtype=torch.int32) for k, v in
                     ((before + 1, 0), (between + 1, 1), (30, 2), (2, 700), (behind + 1, n))]).cuda()
    ids = torch.full((ptr.numel() - 1,), -1, dtype=torch.int32, device="cuda")
    rows = torch.nonzero(ptr[1:] > ptr[:-1])[:, 0]               # the requests that have rows
    ids[rows] = i32(k % 3 for k in range(len(rows)))
    x, w, ad = normal(1, (n, 128)), normal(2, (n_out, 128), 0.1), make_adapters(3, 3, 16, n_out)
    got, want = ([torch.full((n, 128), 7.0, dtype=BF16, device="cuda") for _ in range(n_out // 128)] for _ in range(2))
    few = dg4.segments(torch.cat([ptr[rows], ptr[-1:]]), ids[rows].contiguous())

    def call(seg, out):
        if n_out == 128:
            dg4.dg4_out_project_adapters(g, desc(), x, w, ad, seg, None, *out)
        else:
            dg4.dg4_qkv_project_adapters(g, desc(), x, w, ad, seg, *out)

    call(dg4.segments(ptr, ids), got)
    call(few, want)
    torch.cuda.synchronize()
    assert dg4.dg4_graph_poll_status(g) == 0
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and not any(bool((a == 7.0).all(1).any()) for a in got)


@pytest.mark.parametrize("count", [40, 700, 5000])
@pytest.mark.parametrize("seed", range(4))
def test_many_unsorted_offsets_stay_inside_the_tensors(seed, count):
    """Which rows are written is then unspecified, but nothing outside is, and no wait runs out."""
    rng = np.random.default_rng(seed)
    n = 900
    spread = [(0, n), (-50, n + 50), (-2 ** 31, 2 ** 31 - 1), (n - 3, n + 3)][seed]
    ptr = rng.integers(*spread, size=count + 1)
    ptr[rng.random(count + 1) < 0.4] = ptr[0]                    # runs of equal ones among them
    seg = dg4.segments(i32(ptr.tolist()), i32(rng.integers(-2, 5, size=count).tolist()))
    g = edgeless(n)
    x, res = normal(1, (n, 128)), normal(4, (n, 128))
    for rank in (16, 64):
        buf = torch.full((n + 512, 512), 3.0, dtype=BF16, device="cuda")
        out = [buf[256:256 + n, 128 * j:128 * (j + 1)] for j in range(4)]
        dg4.dg4_qkv_project_adapters(g, desc(), x, normal(2, (384, 128), 0.1), make_adapters(3, 3, rank, 384), seg, *out[:3])
        dg4.dg4_out_project_adapters(g, desc(residual=True), x, normal(2, (128, 128), 0.1), make_adapters(3, 3, rank, 128), seg, res, out[3])
        torch.cuda.synchronize()
        assert bool((buf[:256] == 3.0).all()) and bool((buf[256 + n:] == 3.0).all())
    buf = torch.full((n + 512, 256), 3.0, dtype=BF16, device="cuda")
    one = (torch.ones(128, device="cuda"), None)
    dg4.dg4_norm_gate_fwd(g, desc(), x, res, 1.0, normal(5, (3, 128), 0.7, torch.float32), seg, one, one, 1e-5,
                          buf[256:256 + n, :128], buf[256:256 + n, 128:])
    torch.cuda.synchronize()
    assert bool((buf[:256] == 3.0).all()) and bool((buf[256 + n:] == 3.0).all())
    assert dg4.dg4_graph_poll_status(g) == 0


# ---------------------------------------------------------------------------------------------------
# attention over the table
# ---------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [BF16, torch.float32])
@pytest.mark.parametrize("hops,heads", [(1, 8), (2, 1), (2, 16), (3, 4), (4, 16)])
@pytest.mark.parametrize("q_exp,k_exp", [(122, -121), (60, -60), (-118, 117)])
def test_scores_of_ordinary_size_from_large_and_small_factors(hops, heads, dtype, q_exp, k_exp):
    """Queries near one end of the range and keys near the other: their products are ordinary numbers."""
    g, lists = circuit(13, 12, 150, hops)
    n = g.n
    q, k = normal(1, (n, 128), 2.0 ** q_exp, dtype), normal(2, (n, 128), 2.0 ** k_exp, dtype)
    v = normal(3, (n, 128), 1.0, dtype)
    t, o, d = torch.empty((n, 288), dtype=torch.uint8, device="cuda"), torch.empty_like(q), desc(heads, dtype)
    dg4.dg4_kv8_write(g, d, k, v, t)
    dg4.dg4_sparse_attn_kv8_fwd(g, d, q, t, o)
    want, tol = attn_ref(q, *table_ref(k, v, heads)[1], lists, heads, d.scale, range(n), dtype)
    within(o, want, tol)


@pytest.mark.parametrize("dtype", [BF16, torch.float32])
@pytest.mark.parametrize("hops,heads", [(1, 8), (2, 8), (2, 1), (3, 4), (4, 16)])
@pytest.mark.parametrize("v_exp,spread", [(115, 0), (-110, 0), (0, 40), (0, 110)])
def test_values_of_any_size(v_exp, spread, hops, heads, dtype):
    """Values near both ends of the range, and members' values that lie many binades apart."""
    g, lists = circuit(17, 12, 150, hops)
    n = g.n
    q, k = normal(1, (n, 128), 1.0, dtype), normal(2, (n, 128), 1.0, dtype)
    power = v_exp + (torch.arange(n, device="cuda") * 7 % (2 * spread + 1) - spread)
    v = (normal(3, (n, 128), 1.0, torch.float32) * torch.exp2(power.float())[:, None]).to(dtype)
    t, o, d = torch.empty((n, 288), dtype=torch.uint8, device="cuda"), torch.empty_like(q), desc(heads, dtype)
    dg4.dg4_kv8_write(g, d, k, v, t)
    dg4.dg4_sparse_attn_kv8_fwd(g, d, q, t, o)
    want, tol = attn_ref(q, *table_ref(k, v, heads)[1], lists, heads, d.scale, range(n), dtype)
    within(o, want, tol + 2.0 ** -132)                           # below 2^-126 a bf16 number's step is 2^-133, an fp32 one's finer


@pytest.mark.parametrize("dtype", [BF16, torch.float32])
@pytest.mark.parametrize("hops,heads", [(2, 8), (2, 16), (3, 4)])
@pytest.mark.parametrize("q_exp,k_exp", [(122, -121), (2, -1)])
def test_a_negative_scale_is_that_of_the_negated_queries(q_exp, k_exp, hops, heads, dtype):
    g, _ = circuit(13, 12, 150, hops)
    n = g.n
    q, k, v = (normal(i, (n, 128), 2.0 ** e, dtype) for i, e in ((1, q_exp), (2, k_exp), (3, 0)))
    t, o, o2, d = torch.empty((n, 288), dtype=torch.uint8, device="cuda"), torch.empty_like(q), torch.empty_like(q), desc(heads, dtype)
    dg4.dg4_kv8_write(g, d, k, v, t)
    dg4.dg4_sparse_attn_kv8_fwd(g, d, -q, t, o)
    dg4.dg4_sparse_attn_kv8_fwd(g, dg4.desc(heads, d.dtype, -d.scale), q, t, o2)
    assert bool(torch.isfinite(o).all()) and torch.equal(o, o2)  # signs are exact


@pytest.mark.parametrize("dtype", [BF16, torch.float32])
@pytest.mark.parametrize("hops,heads", [(2, 8), (2, 1), (3, 8)])
def test_the_largest_scores_choose_their_members(hops, heads, dtype):
    """Scores near the top of the range: the members with the largest share the weight, whatever the distance."""
    g, lists = circuit(14, 12, 150, hops)
    n = g.n
    level = torch.arange(n, device="cuda") % 7
    k = (1.0 + level / 8.0)[:, None].expand(n, 128).to(dtype).contiguous()      # e4m3 numbers
    q = torch.full((n, 128), 2.0 ** 117, dtype=dtype, device="cuda")            # scores of about 2^121
    v = normal(3, (n, 128), 1.0, dtype)
    t, o, d = torch.empty((n, 288), dtype=torch.uint8, device="cuda"), torch.empty_like(q), desc(heads, dtype)
    dg4.dg4_kv8_write(g, d, k, v, t)
    dg4.dg4_sparse_attn_kv8_fwd(g, d, q, t, o)
    vals = table_ref(k, v, heads)[1][1]
    of = level.cpu()
    want = torch.stack([vals[u[of[u] == of[u].max()]].mean(0) for u in (torch.as_tensor(np.asarray(x, np.int64)) for x in lists)])
    # equal weights: the sum's roundings, the weights' to fp16 (none: they are powers of two times one scale) and the output's
    mag = torch.stack([vals[u[of[u] == of[u].max()]].abs().mean(0) for u in (torch.as_tensor(np.asarray(x, np.int64)) for x in lists)])
    half = 2.0 ** -8 if dtype == BF16 else 2.0 ** -24
    rel = 2.0 ** -20 + (2.0 ** -11 if dtype == BF16 else 0.0)
    within(o, want, rel * mag + half * (want.abs() + rel * mag) + 1e-300)


@pytest.mark.parametrize("dtype", [BF16, torch.float32])
@pytest.mark.parametrize("hops,heads", [(2, 8), (3, 8), (4, 16), (5, 1)])
@pytest.mark.parametrize("q_exp", [6, 13, 20, 60])
def test_large_scores_cost_the_values_no_precision(q_exp, hops, heads, dtype):
    """Scores of 10^3, 10^5, 10^7 and more, a member's values scaled by its own power of two: where a member has all the
    weight the output is its value, however large the score is."""
    g, lists = circuit(15, 12, 150, hops)
    n = g.n
    level, power = torch.arange(n, device="cuda") % 7, torch.arange(n, device="cuda") % 9 - 4
    k = (1.0 + level / 8.0)[:, None].expand(n, 128).to(dtype).contiguous()      # e4m3 numbers
    q = torch.full((n, 128), 2.0 ** q_exp, dtype=dtype, device="cuda")          # the dot products are exact
    v = (normal(3, (n, 128), 1.0, torch.float32) * torch.exp2(power.float())[:, None]).to(dtype)
    t, o, d = torch.empty((n, 288), dtype=torch.uint8, device="cuda"), torch.empty_like(q), desc(heads, dtype)
    dg4.dg4_kv8_write(g, d, k, v, t)
    dg4.dg4_sparse_attn_kv8_fwd(g, d, q, t, o)
    vals = table_ref(k, v, heads)[1][1]
    of = level.cpu()
    best = [u[of[u] == of[u].max()] for u in (torch.as_tensor(np.asarray(x, np.int64)) for x in lists)]
    want, mag = torch.stack([vals[u].mean(0) for u in best]), torch.stack([vals[u].abs().mean(0) for u in best])
    # equal weights; the next member's is below 2^-40 of them (a step in k is 46 or more in log2 units, values differ by
    # some 2^12 at most: 2^-30 in the sum).  The sum's roundings, the weights' to fp16 (bf16 rows) and the output's.
    half = 2.0 ** -8 if dtype == BF16 else 2.0 ** -24
    rel = 2.0 ** -20 + (2.0 ** -11 if dtype == BF16 else 0.0)
    top = torch.stack([vals[torch.as_tensor(np.asarray(x, np.int64))].abs().amax(0) for x in lists])
    err = rel * mag + 2.0 ** -30 * top
    within(o, want, err + half * (want.abs() + err) + 1e-300)


@pytest.mark.parametrize("dtype", [BF16, torch.float32])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("hops", [2, 4])
def test_a_poisoned_query_reaches_its_own_head_only(hops, bad, dtype):
    """Every score of that head is not a number or infinite, so the head is not a number; a node that is its own only
    member takes its values whatever its query holds."""
    g, lists = circuit(8, 10, 200, hops)
    n, d = g.n, desc(8, dtype)
    q, k, v = normal(1, (n, 128), 1.0, dtype), normal(2, (n, 128), 1.0, dtype), normal(3, (n, 128), 1.0, dtype)
    t, o, o2 = torch.empty((n, 288), dtype=torch.uint8, device="cuda"), torch.empty_like(q), torch.empty_like(q)
    dg4.dg4_kv8_write(g, d, k, v, t)
    dg4.dg4_sparse_attn_kv8_fwd(g, d, q, t, o)
    hit = {3: 0, 60: 20, 61: 127, n - 1: 64}                     # node 3 is an input
    for node, at in hit.items():
        q[node, at] = bad
    dg4.dg4_sparse_attn_kv8_fwd(g, d, q, t, o2)
    assert len(lists[3]) == 1
    for node in range(n):
        for h in range(8):
            at = slice(16 * h, 16 * h + 16)
            if node in hit and hit[node] // 16 == h and len(lists[node]) > 1:
                assert bool(torch.isnan(o2[node, at]).all()), (node, h)
            else:
                assert torch.equal(o[node, at], o2[node, at]), (node, h)


# ---------------------------------------------------------------------------------------------------
# strides and alignments
# ---------------------------------------------------------------------------------------------------
def placed(x, ld, first, fill=7.0):
    """A copy of x in rows `ld` apart whose first element stands at column `first` of a buffer, and the buffer."""
    buf = torch.full((x.shape[0], ld), fill, dtype=x.dtype, device="cuda")
    view = buf[:, first:first + 128]
    view.copy_(x)
    return view, buf


@pytest.mark.parametrize("dtype,ld,first", [(torch.float32, 132, 0), (torch.float32, 136, 4), (torch.float32, 140, 8),
                                            (torch.float32, 136, 8), (BF16, 136, 0), (BF16, 152, 8), (BF16, 384, 128)])
@pytest.mark.parametrize("heads,n", [(8, 203), (1, 34), (16, 95)])
def test_table_of_rows_at_any_16_byte_place(heads, n, dtype, ld, first):
    """fp32 rows 32 bytes apart move 32 bytes at a time, others 16: the same codes and values either way."""
    g, d = edgeless(n), desc(heads, dtype)
    k, v = hard_rows(1, n, dtype), hard_rows(2, n, dtype).flip(0).contiguous()
    want, vals = table_ref(k, v, heads)
    (k2, _), (v2, _) = placed(k, ld, first), placed(v, 128, 0) if n % 2 else placed(v, ld, first)
    t = torch.full((n, 288), 9, dtype=torch.uint8, device="cuda")
    dg4.dg4_kv8_write(g, d, k2, v2, t)
    assert torch.equal(t.cpu(), want)
    (k3, kb), (v3, vb) = placed(k, ld, first), placed(v, ld, first)
    k3.zero_(), v3.zero_()
    dg4.dg4_kv8_read(g, d, t, k3, v3)
    for got, val, buf in ((k3, vals[0], kb), (v3, vals[1], vb)):
        fine = ~torch.isnan(val)
        assert torch.equal(torch.isnan(got).cpu(), ~fine)
        assert torch.equal(got.cpu()[fine], val.to(torch.float32).to(dtype)[fine])
        assert bool((buf[:, :first] == 7.0).all()) and bool((buf[:, first + 128:] == 7.0).all())


@pytest.mark.parametrize("dtype", [BF16, torch.float32])
@pytest.mark.parametrize("hops,heads", [(1, 8), (2, 8), (2, 16), (3, 4), (4, 16)])
def test_attention_with_strided_queries_outputs_and_table(hops, heads, dtype):
    g, _ = circuit(16, 12, 180, hops)
    n, d = g.n, desc(heads, dtype)
    q, k, v = normal(1, (n, 128), 1.5, dtype), normal(2, (n, 128), 2.0, dtype), normal(3, (n, 128), 1.0, dtype)
    t, o = torch.empty((n, 288), dtype=torch.uint8, device="cuda"), torch.empty_like(q)
    dg4.dg4_kv8_write(g, d, k, v, t)
    dg4.dg4_sparse_attn_kv8_fwd(g, d, q, t, o)
    far = torch.full((n, 352), 5, dtype=torch.uint8, device="cuda")
    far[:, 32:320] = t
    for nodes in (None, i32([n - 1, 3, 3, 0, n // 2])):
        (q2, _), (o2, buf) = placed(q, 160, 8), placed(torch.full_like(q, 7.0), 200, 64)
        dg4.dg4_sparse_attn_kv8_fwd(g, d, q2, far[:, 32:320], o2, nodes)
        on = torch.ones(n, dtype=torch.bool, device="cuda")
        if nodes is not None:
            on.zero_()
            on[nodes.long()] = True
        assert torch.equal(o2[on], o[on]) and bool((o2[~on] == 7.0).all())
        assert bool((buf[:, :64] == 7.0).all()) and bool((buf[:, 192:] == 7.0).all())
    q3, _ = placed(q, 160, 8)                                    # in place
    dg4.dg4_sparse_attn_kv8_fwd(g, d, q3, t, q3)
    assert torch.equal(q3, o)


# ---------------------------------------------------------------------------------------------------
# infinities and NaN through the gated norms
# ---------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [BF16, torch.float32])
@pytest.mark.parametrize("rms", [False, True])
def test_non_finite_values_follow_the_formula_and_stay_in_their_rows(rms, dtype):
    n, rs = 300, 0.75
    g, d = edgeless(n), desc(dtype=dtype, rms_norm=rms)
    ptr, ids = [0, 40, 41, 44, 200, n - 20], [0, 2, 1, -1, 2]
    s, r = normal(1, (n, 128), 3.0, dtype), normal(2, (n, 128), 2.0, dtype)
    gate, post, pre = normal(3, (3, 128), 0.7, torch.float32), vectors(4), vectors(6)
    seg = dg4.segments(i32(ptr), i32(ids))

    def call(s, r, gate):
        out = [torch.full((n, 128), 7.0, dtype=dtype, device="cuda") for _ in range(2)]
        dg4.dg4_norm_gate_fwd(g, d, s, r, rs, gate, seg, post, pre, 1e-5, *out)
        return out

    clean = call(s, r, gate)
    nan, inf = float("nan"), float("inf")
    s2, r2, gate2 = s.clone(), r.clone(), gate.clone()
    s2[10, 5], s2[50, 127], s2[60, 0], s2[n - 3, 4] = nan, inf, -inf, nan
    r2[70, 64], r2[80, 1], r2[81], r2[n - 2, 3] = -inf, nan, inf, inf
    gate2[1, 9], gate2[1, 10] = inf, nan                         # the request of rows 41 to 43
    got = call(s2, r2, gate2)
    hit = torch.zeros(n, dtype=torch.bool)
    hit[[10, 50, 60, 70, 80, 81, 41, 42, 43]] = True
    rest = ~hit.cuda()
    for a, b in zip(got, clean):
        assert torch.equal(a[rest], b[rest])                     # rows of no request (7.0) among them
    gates = torch.ones((n, 128), dtype=torch.float64)
    for lo, hi, i in zip(ptr[:-1], ptr[1:], ids):
        gates[lo:hi] = f64(gate2)[i] if i >= 0 else 1.0

    def norm(x, gamma, beta):
        c = x if rms else x - x.mean(1, keepdim=True)
        return c * torch.rsqrt((c * c).mean(1, keepdim=True) + 1e-5) * f64(gamma) + f64(beta)

    p = norm(f64(s2), *post)
    want_r = rs * f64(r2) + gates * p
    want_y = norm(want_r, *pre)
    # finite elements of these rows: some twenty roundings of terms of at most this size (the rows' values are of order
    # one, sums over a row taken in 12 roundings), and the output's own
    size = (rs * f64(r2)).abs() + gates.abs() * (p.abs() + f64(post[1]).abs())
    for what, a, want, mag in (("R_out", got[0], want_r, size), ("Y", got[1], want_y, want_y.abs() + f64(pre[1]).abs())):
        a, want, mag = f64(a)[hit], want[hit], mag[hit]
        assert torch.equal(torch.isnan(a), torch.isnan(want)), what
        assert torch.equal(torch.isinf(a), torch.isinf(want)) and bool((a[torch.isinf(a)] == want[torch.isinf(a)]).all()), what
        fine = torch.isfinite(want)
        tol = 40 * U32 * mag + HALF[dtype] * (want.abs() + 40 * U32 * mag)
        assert bool(((a - want).abs()[fine] <= tol[fine]).all()), what
    # the rows that were not hit are those of the formula
    seen, (wr, tr), (wy, ty) = gated_ref(s, r, rs, gate, ptr, ids, post, pre, 1e-5, rms, dtype)
    on = seen & ~hit
    within(got[0][on.cuda()], wr[on], tr[on], "R_out")
    within(got[1][on.cuda()], wy[on], ty[on], "Y")


# ---------------------------------------------------------------------------------------------------
# what the binding refuses
# ---------------------------------------------------------------------------------------------------
def test_a_gate_without_rows_is_no_gate_of_ones():
    n = 40
    g = edgeless(n)
    x, r2, y = normal(1, (n, 128)), torch.full((n, 128), 7.0, dtype=BF16, device="cuda"), torch.empty((n, 128), dtype=BF16, device="cuda")
    one, seg = (torch.ones(128, device="cuda"), None), dg4.segments(i32([0, n]), i32([0]))
    for gate in (torch.empty((0, 128), device="cuda"), torch.empty(0, device="cuda"), torch.ones((1, 120), device="cuda")):
        with pytest.raises(ValueError):
            dg4.dg4_norm_gate_fwd(g, desc(), x, x, 1.0, gate, seg, one, one, 1e-5, r2, y)
    torch.cuda.synchronize()
    assert bool((r2 == 7.0).all())


def test_a_table_of_wider_elements_is_refused():
    n = 40
    g = edgeless(n)
    x, y = normal(1, (n, 128)), torch.empty((n, 128), dtype=BF16, device="cuda")
    for dtype in (torch.float32, torch.int16):
        t = torch.zeros((n, 288), dtype=dtype, device="cuda")
        with pytest.raises(ValueError):
            dg4.dg4_kv8_write(g, desc(), x, x, t)
        with pytest.raises(ValueError):
            dg4.dg4_kv8_read(g, desc(), t, y, y)
        with pytest.raises(ValueError):
            dg4.dg4_sparse_attn_kv8_fwd(g, desc(), x, t, y)
    for dtype in (torch.uint8, torch.int8, torch.float8_e4m3fn):
        t = torch.empty((n, 288), dtype=dtype, device="cuda")
        dg4.dg4_kv8_write(g, desc(), x, x, t)
        assert torch.equal(t.view(torch.uint8).cpu(), table_ref(x, x, 8)[0])
