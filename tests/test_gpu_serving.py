"""GPU tests of the calls that serve many requests in one batch: projections with an adapter per request, the 8-bit
K | V table and the attention over it, the gated norms.  The expected values are plain 64-bit formulas on the CPU; the
tolerances count roundings: half a step of the storage type per stored value, 2^-24 per 32-bit operation, on sums of
absolute values."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import oracle as orc
from paper_2502_01681_b200 import dg4
from tests.helpers import csr_from_fanins, levels_of, random_dag

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
TAG = {torch.bfloat16: dg4.DG4_BF16, torch.float32: dg4.DG4_F32}
BF16 = torch.bfloat16


def edgeless(n):
    rp, ci = csr_from_fanins([[] for _ in range(n)])
    return dg4.dg4_graph_create(rp, ci, np.zeros(n, np.int32), 1, 0)


def desc(heads=8, dtype=BF16, **kw):
    return dg4.desc(heads, TAG[dtype], (heads / 128.0) ** 0.5, **kw)


def normal(seed, shape, std=1.0, dtype=BF16):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std).to(dtype).cuda()


def i32(x):
    return torch.tensor(list(x), dtype=torch.int32, device="cuda")


def f64(t):
    return t.detach().cpu().double()


def within(got, want, tol, what=""):
    got = f64(got)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    ok = torch.isnan(want) | ((got - want).abs() <= tol)
    assert bool(ok.all()), (what, float(((got - want).abs() / tol.clamp(min=1e-300))[~torch.isnan(want)].max()))


# ---------------------------------------------------------------------------------------------------
# projections with adapters
# ---------------------------------------------------------------------------------------------------
def make_adapters(seed, count, rank, n_out):
    a = normal(seed, (count, rank, 128), 0.1)
    b = normal(seed + 1, (count, n_out, rank), 0.1)
    s = (0.5 + torch.rand(count, generator=torch.Generator().manual_seed(seed + 2))).cuda()
    return dg4.adapters(a, b, s)


def project_ref(x, w, ad, ptr, ids, res=None):
    """(y, tolerance) for the covered rows and the mask of these rows."""
    n, count, rank = x.shape[0], *ad.A.shape[:2]
    x, w, a, b, s = f64(x), f64(w), f64(ad.A), f64(ad.B), f64(ad.scale)
    y = torch.zeros((n, w.shape[0]), dtype=torch.float64)
    tol, seen = torch.zeros_like(y), torch.zeros(n, dtype=torch.bool)
    for lo, hi, i in zip(ptr[:-1], ptr[1:], ids):
        if hi <= lo:
            continue
        r, seen[lo:hi] = x[lo:hi], True
        out = r @ w.T
        t = 128 * U32 * (r.abs() @ w.abs().T)                     # 128 products, added in some order
        if 0 <= i < count:
            u = s[i] * (r @ a[i].T)
            out = out + u @ b[i].T
            mag = u.abs() @ b[i].abs().T
            # U: 128 products and the scale in 32 bits, then half a step of bf16; then `rank` more products
            t = t + 2.0 ** -8 * mag + 132 * U32 * s[i] * ((r.abs() @ a[i].abs().T) @ b[i].abs().T) * (1 + 2.0 ** -8)
            t = t + rank * U32 * (mag * (1 + 2.0 ** -8) + r.abs() @ w.abs().T)
        if res is not None:
            out = out + f64(res)[lo:hi]
        y[lo:hi] = out
        tol[lo:hi] = t * 1.01 + 2.0 ** -8 * (out.abs() + t)
    return y, tol, seen


LAYOUTS = {
    "one": lambda n: ([0, n], [1]),
    "each": lambda n: (list(range(n + 1)), [i % 4 - 1 for i in range(n)]),
    "ragged": lambda n: ([0, n // 7, n // 7, n // 3, n // 3 + n // 5, n], [0, 2, -1, 1, 2]),
    "gaps": lambda n: ([n // 9, n // 4, n // 2, n - n // 8], [2, 99, 0]),
    "alternating": lambda n: ([0] + [n * k // 8 for k in range(1, 9)], [0, -1, 0, 0, 1, -7, 1, 2]),
}


@pytest.mark.parametrize("layout", sorted(LAYOUTS))
@pytest.mark.parametrize("n,rank", [(1, 8), (31, 16), (128, 64), (129, 24), (257, 32), (1000, 40), (3001, 48), (9000, 56)])
def test_qkv_with_adapters_matches_the_formula(n, rank, layout):
    if layout == "each" and n > 4000:
        pytest.skip("covered by the smaller sizes")
    g = edgeless(n)
    ptr, ids = LAYOUTS[layout](n)
    x, w = normal(1, (n, 128)), normal(2, (384, 128), 0.1)
    ad = make_adapters(3, 3, rank, 384)
    q, k, v = (torch.full((n, 128), 7.0, dtype=BF16, device="cuda") for _ in range(3))
    dg4.dg4_qkv_project_adapters(g, desc(), x, w, ad, dg4.segments(i32(ptr), i32(ids)), q, k, v)
    torch.cuda.synchronize()
    assert dg4.dg4_graph_poll_status(g) == 0
    y, tol, seen = project_ref(x, w, ad, ptr, ids)
    for j, out in enumerate((q, k, v)):
        within(out[seen.cuda()], y[seen, j * 128:(j + 1) * 128], tol[seen, j * 128:(j + 1) * 128], j)
        assert bool((out[~seen.cuda()] == 7.0).all())           # rows of no request stay as they were


@pytest.mark.parametrize("n,rank,layout", [(1, 64, "one"), (130, 8, "ragged"), (500, 16, "each"), (2051, 32, "gaps"),
                                           (40000, 64, "alternating"), (40001, 8, "ragged")])
@pytest.mark.parametrize("residual", [True, False])
def test_out_projection_with_adapters_matches_the_formula(n, rank, layout, residual):
    g = edgeless(n)
    ptr, ids = LAYOUTS[layout](n)
    o, w, res = normal(1, (n, 128)), normal(2, (128, 128), 0.1), normal(4, (n, 128))
    ad = make_adapters(3, 3, rank, 128)
    seg = dg4.segments(i32(ptr), i32(ids))
    out = torch.full((n, 128), 7.0, dtype=BF16, device="cuda")
    dg4.dg4_out_project_adapters(g, desc(residual=residual), o, w, ad, seg, res, out)
    y, tol, seen = project_ref(o, w, ad, ptr, ids, res if residual else None)
    within(out[seen.cuda()], y[seen], tol[seen])
    assert bool((out[~seen.cuda()] == 7.0).all())
    if residual:                                                # in place on the residual: the same bits
        h = res.clone()
        dg4.dg4_out_project_adapters(g, desc(residual=True), o, w, ad, seg, h, h)
        assert torch.equal(h[seen.cuda()], out[seen.cuda()])
        assert torch.equal(h[~seen.cuda()], res[~seen.cuda()])


def test_many_requests_of_every_length():
    rng = np.random.default_rng(5)
    lens = rng.choice([0, 0, 1, 2, 31, 32, 33, 127, 128, 129, 300], size=1500)
    ptr = np.concatenate([[0], np.cumsum(lens)]).tolist()
    n, ids = ptr[-1], rng.integers(-1, 9, size=1500).tolist()
    g = edgeless(n)
    x, w, ad = normal(1, (n, 128)), normal(2, (384, 128), 0.1), make_adapters(3, 8, 16, 384)
    q, k, v = (torch.empty((n, 128), dtype=BF16, device="cuda") for _ in range(3))
    seg = dg4.segments(i32(ptr), i32(ids))
    dg4.dg4_qkv_project_adapters(g, desc(), x, w, ad, seg, q, k, v)
    y, tol, seen = project_ref(x, w, ad, ptr, ids)
    assert bool(seen.all())
    for j, out in enumerate((q, k, v)):
        within(out, y[:, j * 128:(j + 1) * 128], tol[:, j * 128:(j + 1) * 128], j)
    again = [torch.empty_like(q) for _ in range(3)]
    dg4.dg4_qkv_project_adapters(g, desc(), x, w, ad, seg, *again)
    assert all(torch.equal(p, r) for p, r in zip((q, k, v), again))


def test_without_adapters_the_projection_is_the_plain_one():
    n = 5000
    g = edgeless(n)
    x, w = normal(1, (n, 128)), normal(2, (384, 128), 0.1)
    want = [torch.empty((n, 128), dtype=BF16, device="cuda") for _ in range(3)]
    got = [torch.empty_like(t) for t in want]
    dg4.dg4_qkv_project(g, desc(), x, w, *want)
    seg = dg4.segments(i32([0, 100, n]), i32([-1, 3]))
    dg4.dg4_qkv_project_adapters(g, desc(), x, w, make_adapters(3, 3, 16, 384), seg, *got)
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_no_segments_means_adapter_zero_everywhere():
    n = 700
    g = edgeless(n)
    x, w, ad = normal(1, (n, 128)), normal(2, (128, 128), 0.1), make_adapters(3, 3, 16, 128)
    a, b = (torch.empty((n, 128), dtype=BF16, device="cuda") for _ in range(2))
    dg4.dg4_out_project_adapters(g, desc(), x, w, ad, None, None, a)
    dg4.dg4_out_project_adapters(g, desc(), x, w, ad, dg4.segments(i32([0, n]), i32([0])), None, b)
    assert torch.equal(a, b)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_request_poisons_its_own_rows_only(bad):
    n = 1000
    g = edgeless(n)
    ptr, ids = [0, 5, 100, 101, 130, 400, n], [0, 1, 2, 0, 1, 2]
    seg = dg4.segments(i32(ptr), i32(ids))
    x, w, ad = normal(1, (n, 128)), normal(2, (384, 128), 0.1), make_adapters(3, 3, 24, 384)
    want = [torch.empty((n, 128), dtype=BF16, device="cuda") for _ in range(3)]
    got = [torch.empty_like(t) for t in want]
    dg4.dg4_qkv_project_adapters(g, desc(), x, w, ad, seg, *want)
    x2, b2, a2 = x.clone(), ad.B.clone(), ad.A.clone()
    x2[100] = bad                                               # the one row of the third request
    b2[1], a2[1, 3] = bad, bad                                  # adapter 1: the second and the fifth
    dg4.dg4_qkv_project_adapters(g, desc(), x2, w, dg4.adapters(a2, b2, ad.scale), seg, *got)
    clean = torch.ones(n, dtype=torch.bool, device="cuda")
    clean[5:101], clean[130:400] = False, False
    for a, b in zip(want, got):
        assert torch.equal(a[clean], b[clean])
        assert not bool(torch.isfinite(b[~clean]).all(1).any())


def test_strided_rows_and_interleaved_outputs():
    n = 333
    g = edgeless(n)
    x, w, ad = normal(1, (n, 200))[:, :128], normal(2, (384, 128), 0.1), make_adapters(3, 2, 16, 384)
    seg = dg4.segments(i32([0, 200, n]), i32([1, 0]))
    want = [torch.empty((n, 128), dtype=BF16, device="cuda") for _ in range(3)]
    dg4.dg4_qkv_project_adapters(g, desc(), x.contiguous(), w, ad, seg, *want)
    buf = torch.full((n, 400), 3.0, dtype=BF16, device="cuda")
    dg4.dg4_qkv_project_adapters(g, desc(), x, w, ad, seg, buf[:, 256:384], buf[:, :128], buf[:, 128:256])
    assert torch.equal(buf[:, 256:384], want[0]) and torch.equal(buf[:, :128], want[1]) and torch.equal(buf[:, 128:256], want[2])
    assert bool((buf[:, 384:] == 3.0).all())


def test_row_offsets_pass_32_bits():
    n, ld = 20000, 131072                                        # 5 GB from the first row to the last
    g = edgeless(n)
    x, w, ad, res = normal(1, (n, 128)), normal(2, (128, 128), 0.1), make_adapters(3, 3, 16, 128), normal(5, (n, 128))
    seg = dg4.segments(i32([0, 7000, n - 3]), i32([2, 0]))
    gate, post, pre = normal(6, (3, 128), 0.7, torch.float32), vectors(7), vectors(9)
    want, r2, y = (torch.zeros((n, 128), dtype=BF16, device="cuda") for _ in range(3))
    dg4.dg4_out_project_adapters(g, desc(residual=True), x, w, ad, seg, res, want)
    dg4.dg4_norm_gate_fwd(g, desc(), want, res, 0.5, gate, seg, post, pre, 1e-5, r2, y)
    far = torch.zeros((n, ld), dtype=BF16, device="cuda")
    a, b, c, d, e = (far[:, 256 * i: 256 * i + 128] for i in range(5))
    a.copy_(x), b.copy_(res)
    dg4.dg4_out_project_adapters(g, desc(residual=True), a, w, ad, seg, b, c)
    dg4.dg4_norm_gate_fwd(g, desc(), c, b, 0.5, gate, seg, post, pre, 1e-5, d, e)
    torch.cuda.synchronize()
    assert torch.equal(c, want) and torch.equal(d, r2) and torch.equal(e, y)
    assert not bool(far[:, 128:256].any()) and not bool(far[:, 1152:2048].any())


def test_wild_offsets_stay_inside_the_tensors():
    n = 640
    g = edgeless(n)
    big = 2 ** 31 - 1
    x, w, ad = normal(1, (n, 128)), normal(2, (128, 128), 0.1), make_adapters(3, 2, 8, 128)
    for ptr in ([-5, 100, big], [300, 100, 500], [big, big, -big], [-big, -1, 0], [n, n + 1, n + 2]):
        buf = torch.full((n + 512, 128), 3.0, dtype=BF16, device="cuda")
        dg4.dg4_out_project_adapters(g, desc(), x, w, ad, dg4.segments(i32(ptr), i32([0, big])), None, buf[256:256 + n])
        torch.cuda.synchronize()
        assert bool((buf[:256] == 3.0).all()) and bool((buf[256 + n:] == 3.0).all())
        dg4.dg4_norm_gate_fwd(g, desc(), x, x, 1.0, torch.ones(1, 128, device="cuda"), dg4.segments(i32(ptr), i32([0, big])),
                              (torch.ones(128, device="cuda"), None), None, 1e-5, buf[256:256 + n], None)
        torch.cuda.synchronize()
        assert bool((buf[:256] == 3.0).all()) and bool((buf[256 + n:] == 3.0).all())
    assert dg4.dg4_graph_poll_status(g) == 0


@pytest.mark.parametrize("n,rank,out_only", [(200000, 16, False), (200000, 64, False), (300, 16, False), (200000, 16, True), (200000, 64, True)])
def test_adapter_waits_that_run_out_are_reported_and_leave_the_device_usable(n, rank, out_only):
    g, n_out = edgeless(n), 128 if out_only else 384
    ptr, ids = [0, n // 50, n // 2, n], [0, 1, 2]
    x, w, ad, res = normal(1, (n, 128)), normal(2, (n_out, 128), 0.1), make_adapters(3, 3, rank, n_out), normal(9, (n, 128))
    seg = dg4.segments(i32(ptr), i32(ids))
    out = [torch.empty((n, 128), dtype=BF16, device="cuda") for _ in range(n_out // 128)]

    def call(graph):
        if out_only:
            dg4.dg4_out_project_adapters(graph, desc(residual=True), x, w, ad, seg, res, *out)
        else:
            dg4.dg4_qkv_project_adapters(graph, desc(), x, w, ad, seg, *out)

    dg4.dg4_debug_set_poll_limit(1)
    try:
        call(g)
        torch.cuda.synchronize()
    finally:
        dg4.dg4_debug_set_poll_limit(0)
    # one poll of a suspended wait lasts up to 640 ns, so the waits of a call with one item per CTA may all be over in it
    assert dg4.dg4_graph_poll_status(g) in ((dg4.DG4_ERR_TIMEOUT,) if n > 1000 else (0, dg4.DG4_ERR_TIMEOUT))
    g2 = edgeless(n)
    call(g2)
    assert dg4.dg4_graph_poll_status(g2) == 0
    y, tol, _ = project_ref(x, w, ad, ptr, ids, res if out_only else None)
    for j, t in enumerate(out):
        within(t, y[:, j * 128:(j + 1) * 128], tol[:, j * 128:(j + 1) * 128], j)


# ---------------------------------------------------------------------------------------------------
# the 8-bit table
# ---------------------------------------------------------------------------------------------------
E4M3 = np.array([(-1.0 if c & 128 else 1.0) * ((8 + (c & 7)) * 2.0 ** ((c >> 3 & 15) - 10) if c & 120 else (c & 7) * 2.0 ** -9)
                 for c in range(256)])                           # 0x7f and 0xff (NaN) are set apart below


def quantise_ref(x, heads):
    """(codes, exponent bytes, values) by the definition, one slice at a time, in 64 bits."""
    x = f64(x).numpy()
    n, dh = x.shape[0], 128 // heads
    codes, exps, vals = np.zeros((n, 128), np.uint8), np.zeros((n, heads), np.uint8), np.zeros((n, 128))
    pos = E4M3[:127]                                             # the finite non-negative codes, ascending
    for r in range(n):
        for h in range(heads):
            s = x[r, h * dh:(h + 1) * dh]
            at = slice(h * dh, (h + 1) * dh)
            if not np.isfinite(s).all():
                codes[r, at], exps[r, h], vals[r, at] = 0x7F, 255, np.nan
                continue
            top = np.abs(s).max()
            b = max(0, int(np.log2(top / 448.0)) + 120) if top > 0 else 0     # no more than the answer
            while top > 448.0 * 2.0 ** (b - 127):
                b += 1
            assert b == 0 or top > 448.0 * 2.0 ** (b - 128)
            z = np.abs(s) * 2.0 ** (127 - b)
            hi = np.searchsorted(pos, z, side="left").clip(max=126)
            lo = (hi - 1).clip(min=0)
            up = (pos[hi] - z < z - pos[lo]) | ((pos[hi] - z == z - pos[lo]) & (hi % 2 == 0))
            c = np.where(up, hi, lo)
            codes[r, at] = c + np.where(np.signbit(s), 128, 0)
            exps[r, h], vals[r, at] = b, np.sign(s) * pos[c] * 2.0 ** (b - 127)
    return codes, exps, vals


def table_ref(k, v, heads):
    n = k.shape[0]
    t, vals = np.zeros((n, 288), np.uint8), []
    for i, x in enumerate((k, v)):
        codes, exps, val = quantise_ref(x, heads)
        t[:, :256].reshape(n, 16, 2, 8)[:, :, i] = codes.reshape(n, 16, 8)
        t[:, 256:].reshape(n, 16, 2)[:, :heads, i] = exps
        vals.append(torch.from_numpy(val))
    return torch.from_numpy(t), vals


def hard_rows(seed, n, dtype):
    """Rows with every binade, borders of the scale and of the codes, zeros, subnormals and non-finite elements."""
    x = normal(seed, (n, 128), 1.0, torch.float32)
    x *= torch.exp2(torch.arange(n, device="cuda").float() * 5 % 240 - 120)[:, None]
    special = [0.0, 1.75 * 2.0 ** 30, 2.0 ** -126, 2.0 ** -133, 3.0e38, 448.0, 449.0, 452.0, 2.0 ** -9, 1.75 * 2.0 ** -100]
    for i, s in enumerate(special[: max(0, n - 3)]):
        x[i] = s * torch.linspace(-1, 1, 128, device="cuda")
        x[i, 17] = s
    if n > 12:
        x[10, 3], x[11, 40], x[12, 127] = float("inf"), float("nan"), float("-inf")
        x[9] = torch.tensor([1.0 + k / 16 for k in range(128)], device="cuda")      # ties between codes
    if n > 14:
        x[13] = torch.nextafter(torch.tensor(1.75 * 2.0 ** 20), torch.tensor(1e30)).cuda()
        x[14] = torch.nextafter(torch.tensor(1.75 * 2.0 ** 20), torch.tensor(0.0)).cuda()
    return x.to(dtype)


@pytest.mark.parametrize("dtype", [BF16, torch.float32])
@pytest.mark.parametrize("heads,n", [(8, 200), (1, 33), (2, 17), (4, 64), (16, 95), (8, 1)])
def test_kv8_codes_are_the_definition_bit_for_bit(heads, n, dtype):
    g = edgeless(n)
    k, v = hard_rows(1, n, dtype), hard_rows(2, n, dtype).flip(0).contiguous()
    t = torch.full((n, 320), 9, dtype=torch.uint8, device="cuda")
    dg4.dg4_kv8_write(g, desc(heads, dtype), k, v, t)
    want, vals = table_ref(k, v, heads)
    assert torch.equal(t[:, :288].cpu(), want)
    assert bool((t[:, 288:] == 9).all())                         # bytes behind a row are not the table's
    k2, v2 = torch.empty_like(k), torch.empty_like(v)
    dg4.dg4_kv8_read(g, desc(heads, dtype), t, k2, v2)
    for got, val in ((k2, vals[0]), (v2, vals[1])):
        exact = val.to(torch.float32).to(dtype)                  # the values are fp32 numbers
        assert torch.equal(torch.isnan(got).cpu(), torch.isnan(val))
        fine = ~torch.isnan(val)
        assert torch.equal(got.cpu()[fine], exact[fine])


def test_kv8_lists_touch_the_listed_rows_only():
    n, dtype = 300, BF16
    g = edgeless(n)
    k, v = normal(1, (n, 160))[:, :128], normal(2, (n, 128))
    nodes = [5, 299, 5, -1, 0, 300, 17, 2 ** 31 - 1, -2 ** 31, 17]
    t = torch.full((n, 288), 9, dtype=torch.uint8, device="cuda")
    dg4.dg4_kv8_write(g, desc(), k, v, t, i32(nodes))
    want, vals = table_ref(k, v, 8)
    seen = torch.zeros(n, dtype=torch.bool)
    seen[[5, 299, 0, 17]] = True
    assert torch.equal(t.cpu()[seen], want[seen]) and bool((t.cpu()[~seen] == 9).all())
    k2, v2 = (torch.full((n, 128), 7.0, dtype=dtype, device="cuda") for _ in range(2))
    dg4.dg4_kv8_read(g, desc(), t, k2, v2, i32(nodes))
    assert torch.equal(f64(k2)[seen], vals[0][seen]) and torch.equal(f64(v2)[seen], vals[1][seen])
    assert bool((k2.cpu()[~seen] == 7).all()) and bool((v2.cpu()[~seen] == 7).all())
    before = t.clone()
    dg4.dg4_kv8_write(g, desc(), k, v, t, torch.empty(0, dtype=torch.int32, device="cuda"))
    assert torch.equal(t, before)


# ---------------------------------------------------------------------------------------------------
# attention over the table
# ---------------------------------------------------------------------------------------------------
def circuit(seed, n_pi, n_gates, hops, window=40):
    fan = random_dag(np.random.default_rng(seed), n_pi, n_gates, window=window)
    rp, ci = csr_from_fanins(fan)
    g = dg4.dg4_graph_create(rp, ci, levels_of(fan), hops, 0)
    ptr, idx = orc.neighbourhood(rp, ci, hops)
    return g, [idx[a:b] for a, b in zip(ptr[:-1], ptr[1:])]


def attn_ref(q, k, v, lists, heads, scale, nodes, dtype):
    """(o, tolerance) rows of `nodes` from the 64-bit values of the table."""
    q = f64(q)
    o, tol = torch.zeros((len(nodes), 128), dtype=torch.float64), torch.zeros((len(nodes), 128), dtype=torch.float64)
    for r, node in enumerate(nodes):
        u = torch.as_tensor(np.asarray(lists[node], np.int64))
        for h in range(heads):
            at = slice(h * 128 // heads, (h + 1) * 128 // heads)
            kk, vv, qq = k[u][:, at], v[u][:, at], q[node, at]
            if len(u) == 1:
                o[r, at], tol[r, at] = vv[0], HALF[dtype] * vv[0].abs() + 1e-300
                continue
            s = scale * (kk @ qq)
            p = torch.softmax(s, 0)
            # a score in log2 units: d_head products and sums, three factors, the subtraction of the maximum; the
            # exponential and the reciprocal are good to 2^-21; sums over the members
            ds = (128 / heads + 8) * U32 * (scale * (kk.abs() @ qq.abs())).max() + 4 * U32 * s.abs().max()
            rel = 2 * (2 * ds + 2.0 ** -21) + (2 * len(u) + 8) * U32
            if dtype == BF16:
                # the query in fp16 is exact down to 2^-25 of its largest element and off by 2^-40 of that below it
                rel += 4 * scale * 2.0 ** -40 * float((kk.abs().sum(1) * qq.abs().max()).max())
                # each weight is rounded to fp16: half a step of 2^-11 relative to it; the exponents' own rounding in
                # the wide form: half a step of a number below 128 + |score| in log2 units, three times
                rel += 2.0 ** -11 + 3 * 2.0 ** -24 * (128 + 2 * s.abs().max())
            o[r, at] = p @ vv
            mag = p @ vv.abs()
            tol[r, at] = rel * mag * 1.01 + HALF[dtype] * (o[r, at].abs() + rel * mag) + 1e-300
    return o, tol


@pytest.mark.parametrize("dtype", [BF16, torch.float32])
@pytest.mark.parametrize("hops,heads,n_pi,n_gates", [(1, 8, 20, 500), (2, 8, 20, 700), (2, 1, 5, 120), (1, 16, 3, 130), (2, 4, 9, 99),
                                                     (3, 8, 20, 300), (5, 2, 10, 150), (8, 16, 10, 130), (2, 2, 1, 0)])
def test_attention_over_the_table_matches_the_formula(hops, heads, n_pi, n_gates, dtype):
    g, lists = circuit(7, n_pi, n_gates, hops)
    n = g.n
    q, k, v = normal(1, (n, 128), 1.5, dtype), normal(2, (n, 128), 2.0, dtype), normal(3, (n, 128), 1.0, dtype)
    t = torch.empty((n, 288), dtype=torch.uint8, device="cuda")
    dg4.dg4_kv8_write(g, desc(heads, dtype), k, v, t)
    _, vals = table_ref(k, v, heads)
    o = torch.empty_like(q)
    d = desc(heads, dtype)
    dg4.dg4_sparse_attn_kv8_fwd(g, d, q, t, o)
    want, tol = attn_ref(q, *vals, lists, heads, d.scale, range(n), dtype)
    within(o, want, tol)
    # a list gives the same rows bit for bit, wherever they stand in it, and leaves the others alone
    nodes = [n - 1, 0, n - 1, -3, n, n // 2, n // 3]
    part = torch.full_like(q, 7.0)
    dg4.dg4_sparse_attn_kv8_fwd(g, d, q, t, part, i32(nodes))
    seen = torch.zeros(n, dtype=torch.bool, device="cuda")
    seen[[n - 1, 0, n // 2, n // 3]] = True
    assert torch.equal(part[seen], o[seen]) and bool((part[~seen] == 7.0).all())
    inplace = q.clone()
    dg4.dg4_sparse_attn_kv8_fwd(g, d, inplace, t, inplace)
    assert torch.equal(inplace, o)


@pytest.mark.parametrize("hops", [2, 4])
def test_a_poisoned_key_or_value_reaches_its_readers_only(hops):
    g, lists = circuit(8, 10, 200, hops)
    n = g.n
    q, k, v = normal(1, (n, 128)), normal(2, (n, 128)), normal(3, (n, 128))
    t, o, o2 = torch.empty((n, 288), dtype=torch.uint8, device="cuda"), torch.empty_like(q), torch.empty_like(q)
    dg4.dg4_kv8_write(g, desc(), k, v, t)
    dg4.dg4_sparse_attn_kv8_fwd(g, desc(), q, t, o)
    k[60, 20], v[90, 100] = float("inf"), float("nan")            # head 1 of K[60], head 6 of V[90]
    dg4.dg4_kv8_write(g, desc(), k, v, t, i32([60, 90]))
    dg4.dg4_sparse_attn_kv8_fwd(g, desc(), q, t, o2)
    for node in range(n):
        u = set(int(x) for x in lists[node])
        for h in range(8):
            at = slice(16 * h, 16 * h + 16)
            if (h == 1 and 60 in u and len(u) > 1) or (h == 6 and 90 in u):
                assert bool(torch.isnan(o2[node, at]).all()), (node, h)
            else:
                assert torch.equal(o[node, at], o2[node, at]), (node, h)


@pytest.mark.parametrize("hops", [2, 3])
def test_scores_far_apart_and_far_from_zero(hops):
    g, lists = circuit(9, 10, 120, hops)
    n = g.n
    q, k, v = normal(1, (n, 128), 60.0), normal(2, (n, 128), 60.0), normal(3, (n, 128))
    t, o = torch.empty((n, 288), dtype=torch.uint8, device="cuda"), torch.empty_like(q)
    dg4.dg4_kv8_write(g, desc(), k, v, t)
    dg4.dg4_sparse_attn_kv8_fwd(g, desc(), q, t, o)
    _, vals = table_ref(k, v, 8)
    want, tol = attn_ref(q, *vals, lists, 8, desc().scale, range(n), BF16)
    within(o, want, tol)
    # one member's scores overflow to -inf: it weighs nothing, and the others' weights are finite
    q2, k2 = torch.full_like(q, 1.0e30), torch.full_like(k, 1.0e-30)
    k2[50] = -1.0e30
    dg4.dg4_kv8_write(g, desc(), k2, v, t)
    dg4.dg4_sparse_attn_kv8_fwd(g, desc(), q2, t, o)
    readers = [w for w in range(n) if 50 in lists[w] and w != 50 and len(lists[w]) > 1]
    assert readers
    for node in readers:
        u = torch.as_tensor([int(x) for x in lists[node] if x != 50])
        mean = vals[1][u].mean(0)
        assert bool(((f64(o[node]) - mean).abs() <= 2.0 ** -7 * vals[1][u].abs().mean(0)).all())


def test_table_offsets_pass_32_bits():
    g, lists = circuit(10, 4, 70000, 2, window=30000)
    n, ldt = g.n, 65536
    rows = [0, 1, n // 2, n - 2, n - 1]
    q, k, v = normal(1, (n, 128)), normal(2, (n, 128)), normal(3, (n, 128))
    t = torch.zeros((n, ldt), dtype=torch.uint8, device="cuda")
    small = torch.empty((n, 288), dtype=torch.uint8, device="cuda")
    o, o2 = torch.empty_like(q), torch.empty_like(q)
    assert n * ldt > 2 ** 32
    for table, out in ((t, o), (small, o2)):
        dg4.dg4_kv8_write(g, desc(), k, v, table)
        dg4.dg4_sparse_attn_kv8_fwd(g, desc(), q, table, out)
    assert torch.equal(o, o2) and torch.equal(t[rows, :288], small[rows])
    k2, v2 = torch.empty_like(k), torch.empty_like(v)
    dg4.dg4_kv8_read(g, desc(), t, k2, v2)
    _, vals = table_ref(k[rows], v[rows], 8)
    assert torch.equal(f64(k2[rows]), vals[0]) and torch.equal(f64(v2[rows]), vals[1])


# ---------------------------------------------------------------------------------------------------
# norms, gate and residual
# ---------------------------------------------------------------------------------------------------
def norm_ref(x, dx, gamma, beta, eps, rms):
    """Norm of 64-bit rows and the error that an error dx of x and 32-bit arithmetic leave in it."""
    c = x if rms else x - x.mean(1, keepdim=True)
    # the mean: a sum of 128 in 12 roundings; the subtraction
    dc = dx + (0 if rms else dx.mean(1, keepdim=True) + 14 * U32 * x.abs().mean(1, keepdim=True)) + U32 * c.abs()
    var = (c * c).mean(1, keepdim=True) + eps
    sd = var.sqrt()
    # the variance: 20 roundings of positive terms and twice the error of c; the reciprocal root takes half of it
    drel = 12 * U32 + (c.abs() * dc).mean(1, keepdim=True) / var + 4 * U32
    b = 0 if beta is None else f64(beta)
    y = c / sd * f64(gamma) + b
    err = (dc / sd + (c / sd).abs() * drel) * f64(gamma).abs() + 3 * U32 * ((c / sd * f64(gamma)).abs() + (0 if beta is None else b.abs()))
    return y, err


def gated_ref(s, r, rs, gate, ptr, ids, post, pre, eps, rms, dtype):
    n = s.shape[0]
    seen, gates = torch.zeros(n, dtype=torch.bool), torch.ones((n, 128), dtype=torch.float64)
    for lo, hi, i in zip(ptr[:-1], ptr[1:], ids):
        seen[lo:hi] = True
        if gate is not None and 0 <= i < gate.shape[0]:
            gates[lo:hi] = f64(gate)[i]
    x, dx = norm_ref(f64(s), torch.zeros((n, 128), dtype=torch.float64), *post, eps, rms)
    out = rs * f64(r) + gates * x
    dout = gates.abs() * dx + 3 * U32 * ((rs * f64(r)).abs() + (gates * x).abs())
    y, dy = norm_ref(out, dout, *pre, eps, rms)
    return seen, (out, dout * 1.05 + HALF[dtype] * (out.abs() + dout)), (y, dy * 1.05 + HALF[dtype] * (y.abs() + dy))


def vectors(seed, beta=True):
    return (1.0 + normal(seed, (128,), 0.3, torch.float32), normal(seed + 1, (128,), 0.3, torch.float32) if beta else None)


@pytest.mark.parametrize("dtype", [BF16, torch.float32])
@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("n,layout", [(1, "one"), (2, "each"), (33, "gaps"), (257, "ragged"), (777, "alternating"), (5000, "each"),
                                      (70001, "gaps")])
def test_gated_norms_match_the_formula(n, layout, rms, dtype):
    g = edgeless(n)
    ptr, ids = LAYOUTS[layout](n)
    s, r = normal(1, (n, 128), 3.0, dtype), normal(2, (n, 128), 2.0, dtype)
    s[n // 2] += 300.0                                           # a large common offset in one row
    gate, post, pre = normal(3, (3, 128), 0.7, torch.float32), vectors(4, not rms), vectors(6)
    d = desc(dtype=dtype, rms_norm=rms)
    seg = dg4.segments(i32(ptr), i32(ids))
    r2, y = (torch.full((n, 128), 7.0, dtype=dtype, device="cuda") for _ in range(2))
    dg4.dg4_norm_gate_fwd(g, d, s, r, 0.75, gate, seg, post, pre, 1e-5, r2, y)
    seen, (want_r, tol_r), (want_y, tol_y) = gated_ref(s, r, 0.75, gate, ptr, ids, post, pre, 1e-5, rms, dtype)
    on = seen.cuda()
    within(r2[on], want_r[seen], tol_r[seen], "R_out")
    within(y[on], want_y[seen], tol_y[seen], "Y")
    assert bool((r2[~on] == 7.0).all()) and bool((y[~on] == 7.0).all())
    # R_out alone, in place on R; both in place, crossed
    a, b = r.clone(), s.clone()
    dg4.dg4_norm_gate_fwd(g, d, s, a, 0.75, gate, seg, post, None, 1e-5, a, None)
    assert torch.equal(a[on], r2[on]) and torch.equal(a[~on], r[~on])
    a = r.clone()
    dg4.dg4_norm_gate_fwd(g, d, b, a, 0.75, gate, seg, post, pre, 1e-5, b, a)
    assert torch.equal(b[on], r2[on]) and torch.equal(a[on], y[on])


def test_gated_norms_without_gate_or_segments():
    n = 300
    g = edgeless(n)
    s, r, post, pre = normal(1, (n, 160))[:, :128], normal(2, (n, 128)), vectors(3), vectors(5, False)
    r2, y, r3, y3 = (torch.empty((n, 128), dtype=BF16, device="cuda") for _ in range(4))
    dg4.dg4_norm_gate_fwd(g, desc(), s, r, -1.5, None, None, post, pre, 1e-6, r2, y)
    _, (want_r, tol_r), (want_y, tol_y) = gated_ref(s, r, -1.5, None, [0, n], [0], post, pre, 1e-6, False, BF16)
    within(r2, want_r, tol_r)
    within(y, want_y, tol_y)
    one = torch.ones((1, 128), device="cuda")
    dg4.dg4_norm_gate_fwd(g, desc(), s, r, -1.5, one, None, post, pre, 1e-6, r3, y3)
    assert torch.equal(r2, r3) and torch.equal(y, y3)


# ---------------------------------------------------------------------------------------------------
# together, captured, on other streams
# ---------------------------------------------------------------------------------------------------
def test_a_layer_of_them_together_step_by_step_and_captured():
    fan = random_dag(np.random.default_rng(3), 30, 1500, window=60)
    rp, ci = csr_from_fanins(fan)
    g = dg4.dg4_graph_create(rp, ci, levels_of(fan), 2, 0)
    nptr, nidx = orc.neighbourhood(rp, ci, 2)
    lists = [nidx[a:b] for a, b in zip(nptr[:-1], nptr[1:])]
    n, d = g.n, desc(residual=True)
    ptr, ids = [0, 300, 301, 900, n], [1, 0, -1, 2]
    seg = dg4.segments(i32(ptr), i32(ids))
    x, res = normal(1, (n, 128)), normal(2, (n, 128))
    wq, wo = normal(3, (384, 128), 0.1), normal(4, (128, 128), 0.1)
    adq, ado = make_adapters(5, 3, 16, 384), make_adapters(8, 3, 16, 128)
    gate, post, pre = normal(11, (3, 128), 0.7, torch.float32), vectors(12), vectors(14)
    q, k, v, o, s, r2, y = (torch.zeros((n, 128), dtype=BF16, device="cuda") for _ in range(7))
    t = torch.zeros((n, 288), dtype=torch.uint8, device="cuda")

    def layer():
        dg4.dg4_qkv_project_adapters(g, d, x, wq, adq, seg, q, k, v)
        dg4.dg4_kv8_write(g, d, k, v, t)
        dg4.dg4_sparse_attn_kv8_fwd(g, d, q, t, o)
        dg4.dg4_out_project_adapters(g, desc(), o, wo, ado, seg, None, s)
        dg4.dg4_norm_gate_fwd(g, d, s, res, 0.5, gate, seg, post, pre, 1e-5, r2, y)

    layer()
    torch.cuda.synchronize()
    first = [a.clone() for a in (q, k, v, t, o, s, r2, y)]
    want, tol, _ = project_ref(x, wq, adq, ptr, ids)
    for j, a in enumerate((q, k, v)):
        within(a, want[:, j * 128:(j + 1) * 128], tol[:, j * 128:(j + 1) * 128], "qkv"[j])
    table, vals = table_ref(k, v, 8)
    assert torch.equal(t.cpu(), table)
    within(o, *attn_ref(q, *vals, lists, 8, d.scale, range(n), BF16), "attention")
    want, tol, _ = project_ref(o, wo, ado, ptr, ids)
    within(s, want, tol, "output projection")
    _, (wr, tr), (wy, ty) = gated_ref(s, res, 0.5, gate, ptr, ids, post, pre, 1e-5, False, BF16)
    within(r2, wr, tr, "residual")
    within(y, wy, ty, "norm")

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        layer()
    x2 = normal(77, (n, 128))
    for inputs in (x.clone(), x2, x.clone()):
        x.copy_(inputs)
        for a in (q, k, v, o, s, r2, y, t):
            a.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = [a.clone() for a in (q, k, v, t, o, s, r2, y)]
        layer()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (q, k, v, t, o, s, r2, y)))
    assert all(torch.equal(a, b) for a, b in zip(got, first))
    assert dg4.dg4_graph_poll_status(g) == 0


def test_two_streams_at_once_give_the_same_bits():
    n = 60000
    g = edgeless(n)
    w, ad = normal(2, (384, 128), 0.1), make_adapters(3, 3, 32, 384)
    seg = dg4.segments(i32([0, 777, 30000, n]), i32([2, 0, 1]))
    xs = [normal(10 + i, (n, 128)) for i in range(2)]
    want = [[torch.empty((n, 128), dtype=BF16, device="cuda") for _ in range(3)] for _ in xs]
    got = [[torch.empty((n, 128), dtype=BF16, device="cuda") for _ in range(3)] for _ in xs]
    for x, out in zip(xs, want):
        dg4.dg4_qkv_project_adapters(g, desc(), x, w, ad, seg, *out)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]
    for _ in range(5):
        for x, out, st in zip(xs, got, streams):
            dg4.dg4_qkv_project_adapters(g, desc(), x, w, ad, seg, *out, stream=st)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for p, q in zip(want, got) for a, b in zip(p, q))


def test_small_calls_on_three_streams_at_once():
    n = 96                                                       # column blocks on different CTAs, two to an SM
    g = edgeless(n)
    w, wo = normal(2, (384, 128), 0.1), normal(3, (128, 128), 0.1)
    ad, ado = make_adapters(4, 96, 16, 384), make_adapters(7, 96, 16, 128)
    seg = dg4.segments(i32(range(n + 1)), i32((i * 37) % 97 - 1 for i in range(n)))
    xs = [normal(20 + i, (n, 128)) for i in range(3)]
    new = lambda: [torch.zeros((n, 128), dtype=BF16, device="cuda") for _ in range(4)]  # noqa: E731
    want, got, streams = [new() for _ in xs], [new() for _ in xs], [torch.cuda.Stream() for _ in xs]

    def call(x, y, stream):
        dg4.dg4_qkv_project_adapters(g, desc(), x, w, ad, seg, *y[:3], stream=stream)
        dg4.dg4_out_project_adapters(g, desc(residual=True), x, wo, ado, seg, x, y[3], stream=stream)

    for x, y in zip(xs, want):
        call(x, y, None)
    torch.cuda.synchronize()
    for _ in range(50):
        for x, y, st in zip(xs, got, streams):
            call(x, y, st)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for p, q in zip(want, got) for a, b in zip(p, q))
    assert dg4.dg4_graph_poll_status(g) == 0


def test_a_captured_call_reads_the_requests_and_lists_of_its_replay():
    n = 2000
    g, lists = circuit(12, 20, n - 20, 2)
    x, w, ad = normal(1, (n, 128)), normal(2, (384, 128), 0.1), make_adapters(3, 3, 16, 384)
    ptr, ids, nodes = i32([0, 500, n]), i32([0, 1]), i32([3, 4, 5, 6])
    seg = dg4.segments(ptr, ids)
    gate, post = normal(5, (3, 128), 0.7, torch.float32), vectors(6)
    q, k, v, o, r2 = (torch.zeros((n, 128), dtype=BF16, device="cuda") for _ in range(5))
    t = torch.zeros((n, 288), dtype=torch.uint8, device="cuda")

    def step():
        dg4.dg4_qkv_project_adapters(g, desc(), x, w, ad, seg, q, k, v)
        dg4.dg4_kv8_write(g, desc(), k, v, t, nodes)
        dg4.dg4_sparse_attn_kv8_fwd(g, desc(), q, t, o, nodes)
        dg4.dg4_norm_gate_fwd(g, desc(), o, x, 1.0, gate, seg, post, None, 1e-5, r2, None)

    step()
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step()
    for p, i, u in (([0, 1, 2], [2, 2], [0, 1, 2, 1999]), ([7, 1400, 1999], [-1, 0], [1999, 1998, 0, -1]), ([n, n, n], [0, 1], [-1, -1, -1, -1])):
        ptr.copy_(i32(p)), ids.copy_(i32(i)), nodes.copy_(i32(u))
        for a in (q, k, v, o, r2, t):
            a.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = [a.clone() for a in (q, k, v, o, r2, t)]
        for a in (q, k, v, o, r2, t):
            a.zero_()
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (q, k, v, o, r2, t)))
        y, tol, seen = project_ref(x, w, ad, p, i)
        within(q[seen.cuda()], y[seen, :128], tol[seen, :128])
        assert bool((q[~seen.cuda()] == 0).all()) and bool((r2[~seen.cuda()] == 0).all())


# ---------------------------------------------------------------------------------------------------
# refusals
# ---------------------------------------------------------------------------------------------------
def refused(status, call, *args, **kw):
    with pytest.raises(dg4.Dg4Error) as e:
        call(*args, **kw)
    assert e.value.status == status and e.value.detail
    return e.value.detail


def test_refusals():
    n = 64
    g = edgeless(n)
    x, w, wo = normal(1, (n, 128)), normal(2, (384, 128)), normal(3, (128, 128))
    q, k, v = (torch.zeros_like(x) for _ in range(3))
    t = torch.zeros((n, 288), dtype=torch.uint8, device="cuda")
    ad, ado, seg = make_adapters(3, 2, 16, 384), make_adapters(3, 2, 16, 128), dg4.segments(i32([0, n]), i32([0]))
    inv, uns = dg4.DG4_ERR_INVALID_ARG, dg4.DG4_ERR_UNSUPPORTED
    qkv, out, norm = dg4.dg4_qkv_project_adapters, dg4.dg4_out_project_adapters, dg4.dg4_norm_gate_fwd
    refused(uns, qkv, g, desc(), x, w, make_adapters(3, 2, 12, 384), seg, q, k, v)
    refused(uns, qkv, g, desc(), x, w, make_adapters(3, 2, 72, 384), seg, q, k, v)
    refused(uns, qkv, g, desc(dtype=torch.float32), x, w, ad, seg, q, k, v)
    refused(inv, qkv, g, desc(), x, w, ad, dg4.segments(i32([0]), i32([])), q, k, v)
    refused(inv, qkv, g, desc(), x[:, 1:], w, ad, seg, q, k, v)
    refused(inv, out, g, desc(residual=True), x, wo, ado, seg, torch.zeros((n, 132), dtype=BF16, device="cuda")[:, :128], q)
    f = torch.float32
    refused(uns, dg4.dg4_kv8_write, g, desc(32, f), x.float(), x.float(), t)
    refused(inv, dg4.dg4_kv8_write, g, desc(), x, x, torch.zeros((n, 272), dtype=torch.uint8, device="cuda"))
    refused(inv, dg4.dg4_kv8_read, g, desc(), torch.zeros((n, 304), dtype=torch.uint8, device="cuda"), q, k)
    refused(inv, dg4.dg4_sparse_attn_kv8_fwd, g, desc(), x, t, x, i32([0]))
    refused(inv, dg4.dg4_sparse_attn_kv8_fwd, g, desc(), x, torch.zeros(n * 288 + 8, dtype=torch.uint8, device="cuda")[8:].view(n, 288), q)
    one = (torch.ones(128, device="cuda"), None)
    refused(inv, norm, g, desc(), x, x, 1.0, None, None, one, one, -1.0, q, k)
    refused(inv, norm, g, desc(), x, x, float("nan"), None, None, one, one, 1e-5, q, k)
    refused(inv, norm, g, desc(), x, x, 1.0, None, None, one, one, 1e-5, q, q)
    refused(inv, norm, g, desc(), x, x, 1.0, None, None, one, None, 1e-5, q, k)
    refused(inv, norm, g, desc(), x, x, 1.0, torch.ones((2, 128), device="cuda"), None, one, one, 1e-5, q, k)
    lib = dg4.load()
    d = desc()
    assert lib.dg4_kv8_write(g.handle, ctypes.byref(d), x.data_ptr(), 128, x.data_ptr(), 128, t.data_ptr(), 288, None, 5, None) == inv
    assert lib.dg4_kv8_write(g.handle, ctypes.byref(d), x.data_ptr(), 128, x.data_ptr(), 128, t.data_ptr(), 288, None, -1, None) == inv
    dg4.dg4_debug_override_current_device(1)
    try:
        refused(inv, qkv, g, desc(), x, w, ad, seg, q, k, v)
        refused(inv, out, g, desc(), x, wo, ado, seg, None, q)
        refused(inv, dg4.dg4_kv8_write, g, desc(), x, x, t)
        refused(inv, dg4.dg4_kv8_read, g, desc(), t, q, k)
        refused(inv, dg4.dg4_sparse_attn_kv8_fwd, g, desc(), x, t, q)
        refused(inv, norm, g, desc(), x, x, 1.0, None, None, one, one, 1e-5, q, k)
    finally:
        dg4.dg4_debug_override_current_device(-1)
    torch.cuda.synchronize()
