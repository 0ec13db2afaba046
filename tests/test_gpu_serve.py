"""GPU tests of the shared-prefix serving operators against the fp64 oracle (oracle/serving.py).

Tolerances.  An appended row is bit-equal unless rotated; a rotated entry is u c - v s with c
and s right to two fp32 steps and three roundings, then rounded once: half a step of the type
relative to the value plus 4 * 2^-23 (|u| + |v|).  An attention output is sum_x p_x v_x with
weights off by a relative w: a score is a sum of d products in fp32 (at most (d + 4) 2^-24 S,
S = scale * sum |q_f k_f|), which moves p by twice that (numerator and sum), the exponent's
argument in units of log2 is rounded at |s| log2(e) 2^-23, the sum over N tokens adds (N + 8)
2^-24, and the bf16 path rounds each weight to bf16, half a step.  So every entry lies within
half a step |o| + w A, A = sum_x p_x |v_x|.
"""
import numpy as np
import pytest
import torch

import kvsynth
import paper_2607_12550_amd as J
from gpu_util import ctx, note
from oracle import serving as osv

pytestmark = pytest.mark.gpu
DT = {"bf16": (J.JOLT_BF16, torch.bfloat16, 2.0 ** -8), "f32": (J.JOLT_F32, torch.float32, 2.0 ** -24)}


def dev_i(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def f64(x):
    return x.double().cpu().numpy()


def pages_desc(dtype, H, page, d, n_pages, layout="hpd"):
    if layout == "hpd":                 # [page][head][token][d]
        st = (H * page * d, page * d, d)
    elif layout == "phd":               # [page][token][head][d]
        st = (H * page * d, d, H * d)
    else:                               # "kv": keys and values of a page side by side, padded rows
        st = (2 * H * page * (d + 8), page * (d + 8), d + 8)
    return J.page_desc(dtype=DT[dtype][0], n_heads=H, page_size=page, d=d, n_pages=n_pages, stride_page=st[0],
                       stride_head=st[1], stride_token=st[2])


def pools(desc, dtype, layout, fill):
    """(storage, keys view, values view) with views [page][head][token][d] of the pools."""
    n = (2 if layout != "kv" else 1) * desc.n_pages * desc.stride_page
    buf = torch.full((n,), fill, dtype=DT[dtype][1], device="cuda")
    off = desc.n_pages * desc.stride_page if layout != "kv" else desc.n_heads * desc.stride_head
    shape, st = (desc.n_pages, desc.n_heads, desc.page_size, desc.d), (desc.stride_page, desc.stride_head, desc.stride_token, 1)
    return buf, buf.as_strided(shape, st), buf[off:].as_strided(shape, st)


# ------------------------------------------------------------------------------- plan
def _plan_inputs(rng, have, add, page, extra_cols=1, n_pages=None, spare=3):
    need = [-(-h // page) for h in have]
    new = sum(-(-(h + n) // page) for h, n in zip(have, add)) - sum(need)
    n_pages = n_pages or sum(need) + new + spare
    ids = rng.permutation(n_pages)
    table = rng.integers(-5, n_pages + 5, (len(have), max(1, max(-(-(h + n) // page) for h, n in zip(have, add)) + extra_cols)))
    at = 0
    for r, k in enumerate(need):
        table[r, :k] = ids[at:at + k]
        at += k
    return table, ids[at:], n_pages


def _run_plan(have, add, page, free, n_free, table, n_tok, n_pages):
    n = len(have)
    o = dict(table=dev_i(table), kv_len=dev_i([7] * n), q_start=dev_i([7] * (n + 1)), slots=dev_i([7] * n_tok), positions=dev_i([7] * n_tok),
             n_free=dev_i([7]), info=dev_i([7] * 4))
    J.jolt_page_plan(ctx(), pages_desc("bf16", 1, page, 32, n_pages), dev_i(have), dev_i(add), dev_i(free), dev_i([n_free]), o["table"],
                     o["kv_len"], o["q_start"], o["slots"], o["positions"], o["n_free"], o["info"])
    torch.cuda.synchronize()
    return {k: v.cpu().numpy() for k, v in o.items()}


def _same_plan(got, want):
    for k, v in got.items():
        np.testing.assert_array_equal(v, want[k], err_msg=k)


@pytest.mark.parametrize("n_req,hi_have,hi_add,page,spare_tok", [
    (1, 0, 1, 1, 0), (1, 0, 1, 16, 5), (3, 40, 0, 16, 4), (64, 500, 1, 16, 0), (65, 70, 5, 1, 3), (255, 100, 30, 8, 1),
    (256, 1000, 3, 1024, 0), (257, 33, 100, 32, 1000), (1000, 200, 90, 64, 77), (4096, 50, 9, 16, 2)])
def test_page_plan(n_req, hi_have, hi_add, page, spare_tok):
    rng = np.random.default_rng(n_req)
    have, add = rng.integers(0, hi_have + 1, n_req).tolist(), rng.integers(0, hi_add + 1, n_req).tolist()
    if n_req == 1:
        add = [1]
    table, free, n_pages = _plan_inputs(rng, have, add, page)
    n_tok = sum(add) + spare_tok or 1
    note("jolt_page_plan", n_req, hi_have, hi_add, page, n_tok)
    _same_plan(_run_plan(have, add, page, free, len(free), table, n_tok, n_pages),
               osv.plan(have, add, page, free, len(free), table, n_tok, n_pages))


@pytest.mark.parametrize("fault", ["pages", "claimed_pages", "table", "tokens", "negative_have", "negative_add", "huge", "all"])
def test_page_plan_that_cannot_be_served_changes_nothing(fault):
    rng = np.random.default_rng(5)
    have, add, page = [5, 0, 30], [20, 17, 3], 8
    table, free, n_pages = _plan_inputs(rng, have, add, page, extra_cols=0)
    n_free, n_tok = len(free), 40
    if fault in ("pages", "all"):
        n_free = 4
    if fault == "claimed_pages":        # n_free says more than the array holds
        n_free, free = 10 ** 6, free[:4]
    if fault in ("table", "all"):
        table = table[:, :4]
    if fault in ("tokens", "all"):
        n_tok = 39
    if fault in ("negative_have", "all"):
        have[1] = -1
    if fault == "negative_add":
        add[2] = -3
    if fault == "huge":                 # sums past 32 bits
        have[0] = add[0] = have[2] = add[2] = 2 ** 31 - 1
    got, want = (f(have, add, page, free, n_free, table, n_tok, n_pages) for f in (_run_plan, osv.plan))
    assert want["info"][2] != 0 and (got["slots"] == -1).all() and (got["q_start"] == 0).all()
    _same_plan(got, want)


def test_page_plan_keeps_bad_pages_out_of_the_slots():
    rng = np.random.default_rng(6)
    have, add, page = [5, 0, 30], [20, 17, 3], 8
    table, free, n_pages = _plan_inputs(rng, have, add, page)
    table[0, 0], free[-1], free[-2] = n_pages, -7, 2 ** 31 - 1
    got, want = (f(have, add, page, free, len(free), table, 40, n_pages) for f in (_run_plan, osv.plan))
    assert (want["slots"] == -1).any()
    _same_plan(got, want)


# ------------------------------------------------------------------------------- append
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,H,d,page,layout,rope,fused", [
    (1, 1, 32, 1, "hpd", True, False), (7, 3, 64, 16, "phd", True, True), (33, 8, 128, 32, "kv", True, True),
    (64, 8, 128, 16, "hpd", False, False), (130, 40, 64, 64, "hpd", True, False), (5, 2, 32, 1024, "kv", False, True)])
def test_page_append(dtype, n, H, d, page, layout, rope, fused):
    rng = np.random.default_rng(n)
    td, half = DT[dtype][1], DT[dtype][2]
    n_pages = -(-n // page) + 2
    desc = pages_desc(dtype, H, page, d, n_pages, layout)
    buf, Kp, Vp = pools(desc, dtype, layout, 3.5)
    slots = rng.permutation(n_pages * page)[:n]
    slots[rng.random(n) < 0.2] = -1
    slots[rng.random(n) < 0.1] = n_pages * page + 3
    pos = rng.integers(0, 100000, n)
    if fused:                           # rows of a joint projection: strides of their own
        x = torch.randn((n, 3 * H, d), device="cuda", generator=torch.Generator("cuda").manual_seed(n)).to(td)
        K, V = x[:, H:2 * H], x[:, 2 * H:]
    else:
        g = torch.Generator("cuda").manual_seed(n)
        K, V = (torch.randn((n, H, d), device="cuda", generator=g).to(td) for _ in range(2))
    r = (5e5, 777) if rope else None
    note("jolt_page_append", dtype, n, H, d, page, layout, rope)
    before = buf.clone()
    J.jolt_page_append(ctx(), desc, K, V, dev_i(slots), Kp, Vp, positions=dev_i(pos) if rope else None, rope=r)
    torch.cuda.synchronize()
    k64, v64 = f64(K), f64(V)
    want = osv.rotate(k64, pos + r[1], r[0]) if rope else k64
    h = np.roll(np.abs(k64), d // 2, -1)
    tol = half * np.abs(want) + 4 * 2.0 ** -23 * (np.abs(k64) + h) if rope else 0 * want
    gk, gv = f64(Kp), f64(Vp)
    for t, s in enumerate(slots):
        if 0 <= s < n_pages * page:
            assert (np.abs(gk[s // page, :, s % page] - want[t]) <= tol[t]).all(), t
            assert (gv[s // page, :, s % page] == v64[t]).all()
            Kp[s // page, :, s % page] = 3.5
            Vp[s // page, :, s % page] = 3.5
    assert torch.equal(buf, before)     # nothing else was written


# ------------------------------------------------------------------------------- attention
class Batch:
    """Inputs of a prefix-attention call and what the oracle says of them."""

    def __init__(self, dtype, T, have, new, H, G, d, page, seed=0, layout="hpd", pad_rows=0, hole=3.0, big=1.0):
        rng = np.random.default_rng(seed)
        g = torch.Generator("cuda").manual_seed(seed)
        self.dtype, self.T, self.H, self.G, self.d, self.page = dtype, T, H, G, d, page
        td = DT[dtype][1]
        lens = [h + n for h, n in zip(have, new)]
        self.q_start, self.kv_len = np.concatenate([[0], np.cumsum(new)]), np.array(lens)
        self.n_tok = int(self.q_start[-1]) + pad_rows
        need = [-(-x // page) for x in lens]
        n_pages = sum(need) + 2
        ids = rng.permutation(n_pages)
        self.table = np.full((len(have), max(need) + 1), -9)
        self.desc = pages_desc(dtype, H, page, d, n_pages, layout)
        self.buf, self.Kp, self.Vp = pools(self.desc, dtype, layout, hole)
        at, self.tk, self.tv = 0, [], []
        for r, x in enumerate(lens):
            self.table[r, :need[r]] = ids[at:at + need[r]]
            at += need[r]
            k, v = (big * torch.randn((H, x, d), device="cuda", generator=g).to(td) for _ in range(2))
            for s in range(x):
                p = self.table[r, s // page]
                self.Kp[p, :, s % page], self.Vp[p, :, s % page] = k[:, s], v[:, s]
            self.tk.append(k)
            self.tv.append(v)
        self.K, self.V = (big * torch.randn((2, H, max(T, 1), d), device="cuda", generator=g).to(td) for _ in range(2))
        self.Q = torch.randn((max(self.n_tok, 1), H * G, d), device="cuda", generator=g).to(td)
        self.scale = 1 / np.sqrt(d)
        self.prefix = J.cell_desc(dtype=DT[dtype][0], n_layers=2, n_heads=H, T=T, d=d, stride_layer=H * T * d,
                                  stride_head=T * d, stride_token=d) if T else None

    def run(self, max_new=0, pages=True, prefix=True, stream=None, fill=5.25):
        self.O = torch.full_like(self.Q, fill)
        self.lse = torch.full(self.Q.shape[:2], fill, dtype=torch.float32, device="cuda")
        pre = self.prefix if prefix else None
        pg = self.desc if pages else None
        nb = J.jolt_prefix_attend_workspace_size(len(self.kv_len), self.Q.shape[0], self.Q.shape[1], prefix=pre, pages=pg,
                                                 max_pages=self.table.shape[1] if pages else 0, max_new=max_new)
        # NaN in every type, and a guard behind the bytes asked for
        guarded = torch.full((nb + 4096,), 255, dtype=torch.uint8, device="cuda")
        ws = guarded[:nb]
        note("jolt_prefix_attend", self.dtype, "T", self.T, "rows", self.Q.shape[0], "requests", len(self.kv_len), "H", self.H, "G", self.G,
             "d", self.d, "page", self.page, "max_new", max_new)
        J.jolt_prefix_attend(ctx(), self.Q, self.O, dev_i(self.q_start), dev_i(self.kv_len), self.scale, ws, prefix=pre, K_prefix=self.K,
                             V_prefix=self.V, layer=1 if prefix and self.T else 0, pages=pg, K_pages=self.Kp, V_pages=self.Vp,
                             table=dev_i(self.table), max_new=max_new, lse=self.lse, stream=stream)
        torch.cuda.synchronize()
        assert (guarded[nb:] == 255).all()
        return f64(self.O), f64(self.lse)

    def want(self, pages=True, prefix=True):
        H, d = self.H, self.d
        K, V = (f64(x[1]) if prefix and self.T else np.zeros((H, 0, d)) for x in (self.K, self.V))
        none = [np.zeros((H, 0, d))] * len(self.kv_len)
        return osv.prefix_attend(f64(self.Q), K, V, [f64(x) for x in self.tk] if pages else none,
                                 [f64(x) for x in self.tv] if pages else none, self.q_start, self.kv_len if pages else 0 * self.kv_len,
                                 self.scale)

    def check(self, got, want, fill=5.25):
        (O, lse), (wO, wl, A, S) = got, want
        half = DT[self.dtype][2]
        N = self.T + self.kv_len.max()
        rows = np.isfinite(wl) | (wl == -np.inf)
        assert (O[~rows] == fill).all() and (lse[~rows] == fill).all()        # rows of no request
        S, wl = np.where(rows, S, 0), np.where(rows, wl, 0)
        ds = (self.d + 4) * 2.0 ** -24 * S + 2.0 ** -22 * (np.abs(np.where(np.isfinite(wl), wl, 0)) + S)
        w = 2 * ds + (N + 8) * 2.0 ** -24 + (half if self.dtype == "bf16" else 0)
        tol = half * np.abs(wO) + w[..., None] * A
        err = np.abs(O - wO)
        assert (err[rows] <= tol[rows]).all(), (np.nanmax(err[rows] / tol[rows]))
        empty = np.isneginf(wl)
        assert (np.isneginf(lse) == empty)[rows].all()
        ok = rows & ~empty
        assert (np.abs(lse[ok] - wl[ok]) <= (ds + (N + 8) * 2.0 ** -24)[ok]).all()


CASES = [  # T, have, new, H, G, d, page
    (0, [0], [1], 1, 1, 32, 1), (1, [0], [1], 1, 1, 64, 16), (17, [3, 0], [1, 1], 2, 1, 128, 8),
    (300, [40, 7], [1, 1], 4, 2, 64, 16), (65, [0, 31, 32, 33, 63, 64, 65, 127], [1] * 8, 2, 4, 128, 32),
    (1000, [5] * 20, [1] * 20, 2, 5, 128, 16), (129, [100, 0, 3], [3, 5, 2], 8, 4, 128, 64),
    (513, [0, 200], [40, 70], 2, 3, 64, 16), (260, [9, 0, 0, 50], [1, 130, 0, 7], 2, 8, 32, 128),
    (64, [1, 2, 3], [16, 17, 15], 4, 1, 128, 1024), (0, [700, 0, 5], [1, 33, 2], 1, 16, 64, 32),
    (2050, [300], [1], 1, 64, 128, 16), (33, [4] * 70, [1] * 70, 1, 2, 64, 4),
    (700, [20, 0, 33], [8, 5, 7], 40, 4, 128, 16), (400, [31, 0, 32, 1, 63], [1, 2, 8, 1, 3], 2, 4, 32, 32), (0, [0, 1, 31, 32, 33], [1] * 5, 3, 2, 128, 8), (129, [2, 500], [1, 25], 16, 1, 32, 16),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: f"T{c[0]}_r{len(c[1])}_n{sum(c[2])}_H{c[3]}G{c[4]}d{c[5]}p{c[6]}")
def test_prefix_attend(dtype, case):
    T, have, new, H, G, d, page = case
    b = Batch(dtype, T, have, new, H, G, d, page, seed=T + d)
    want = b.want()
    b.check(b.run(max_new=max(new)), want)
    b.check(b.run(), want)                  # the bound on new rows not given


def test_prefix_attend_bound_on_new_rows():
    """A request with more rows than max_new says counts as having none: its rows stay as they were."""
    b = Batch("bf16", 100, [3, 0, 50], [1, 60, 9], 2, 2, 64, 16)
    for m in (1, 2, 8, 9, 59, 60, 61, 10 ** 6):
        want = b.want()
        for r, n in enumerate((1, 60, 9)):
            if n > m:
                for w in want:
                    w[b.q_start[r]:b.q_start[r + 1]] = np.nan
        b.check(b.run(max_new=m), want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prefix_attend_prefix_alone_and_pages_alone(dtype):
    for new in ([1, 1, 0, 1], [30, 1, 2, 40]):
        b = Batch(dtype, 333, [0, 65, 9, 2], new, 4, 2, 64, 16)
        b.check(b.run(pages=False), b.want(pages=False))
        b.check(b.run(prefix=False), b.want(prefix=False))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [[1, 1, 1, 1], [2, 40, 3, 1]])
def test_prefix_attend_rows_that_attend_to_nothing(dtype, new):
    """Tails shorter than their new rows (the first rows attend to nothing there), and empty ones."""
    b = Batch(dtype, 0, [0, 5, 0, 9], new, 2, 4, 64, 8)
    b.kv_len = np.minimum(b.kv_len, [0, 3, 1, 10])
    want = b.want()
    assert np.isneginf(want[1]).any()
    b.check(b.run(max_new=max(new)), want)
    for T in (70, 700):
        b = Batch(dtype, T, [0, 5, 0, 9], new, 2, 4, 64, 8)
        for lens in ([0, 0, 0, 0], [1, 3, 0, 2]):
            b.kv_len = np.minimum(lens, b.kv_len)
            b.check(b.run(max_new=max(new)), b.want())
    b = Batch(dtype, 0, [600, 5, 0, 9], new, 2, 4, 64, 8)     # a table with room for many pages
    b.kv_len = np.minimum(b.kv_len, [600, 3, 1, 0])
    b.check(b.run(max_new=max(new)), b.want())


@pytest.mark.parametrize("layout", ["phd", "kv"])
def test_prefix_attend_layouts_of_pages(layout):
    for new in ([1, 1, 1], [1, 50, 3]):
        b = Batch("bf16", 100, [60, 5, 17], new, 3, 4, 128, 16, layout=layout)
        b.check(b.run(), b.want())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf"), "lowest"])
@pytest.mark.parametrize("T", [50, 600])
@pytest.mark.parametrize("new,d", [([1, 1, 1], 64), ([3, 2, 3], 32), ([7, 5, 8], 128), ([40, 2, 37], 64), ([33, 1, 90], 128)])
def test_prefix_attend_ignores_what_a_row_does_not_attend_to(dtype, bad, new, d, T):
    """Whatever stands in unused page slots, behind the lengths and, for the rows before it, in the last token."""
    bad = float(torch.finfo(DT[dtype][1]).min) if bad == "lowest" else bad
    b = Batch(dtype, T, [60, 5, 17], new, 2, 4, d, 16, hole=bad)
    want, m = b.want(), max(new)
    b.check(b.run(max_new=m), want)
    # the last token of request 0: keys first, then values; every row but the last is as before
    r, last = 0, int(b.kv_len[0]) - 1
    keep = np.ones(b.n_tok, bool)
    keep[b.q_start[1] - 1] = False
    for pool in (b.Kp, b.Vp):
        pool[b.table[r, last // 16], :, last % 16] = bad
        O, lse = b.run(max_new=m)
        for x, y in ((O, want[0]), (lse, want[1])):
            assert np.isfinite(x[keep]).all()
        b2 = [w.copy() for w in want]
        O[~keep], lse[~keep] = b2[0][~keep], b2[1][~keep]
        b.check((O, lse), want)


def test_prefix_attend_value_that_is_not_finite_reaches_the_rows_that_see_it():
    for new, T in (([1, 1], 50), ([4, 40], 50), ([1, 1], 600), ([4, 2], 50), ([4, 2], 600)):
        b = Batch("bf16", T, [60, 5], new, 2, 4, 64, 16)
        b.V[1, 1, 7, 3] = float("inf")
        b.Vp[b.table[0, 0], 0, 2, 5] = float("nan")
        O, _ = b.run(max_new=max(new))
        n0 = int(b.q_start[1])
        assert np.isposinf(O[:, 4:, 3]).all() and np.isfinite(np.delete(O[:, 4:], 3, 2)).all()
        assert np.isnan(O[:n0, :4, 5]).all() and np.isfinite(O[n0:, :4]).all() and np.isfinite(np.delete(O[:, :4], 5, 2)).all()


def test_prefix_attend_scores_far_apart():
    """Scores of several hundred: the maximum moves late and everything else underflows."""
    for dtype in ("bf16", "f32"):
        for new in ([1, 1, 1], [20, 1, 18]):
            b = Batch(dtype, 200, [90, 5, 17], new, 2, 4, 64, 16, big=60.0)
            b.K[1, :, 150] *= 3
            b.check(b.run(), b.want())


def test_prefix_attend_leaves_rows_behind_the_last_request():
    for new, T in (([1, 0, 1], 100), ([30, 2, 0], 100), ([1, 0, 1], 1000)):
        b = Batch("bf16", T, [60, 5, 17], new, 2, 4, 128, 16, pad_rows=37)
        b.Q[b.q_start[-1]:] = float("nan")
        b.check(b.run(max_new=max(new)), b.want())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prefix_attend_rows_do_not_depend_on_their_neighbours(dtype):
    """What stands in rows of no request, and in the other rows, does not move a bit of a row."""
    for new in ([1, 0, 1], [30, 2, 0], [60, 5, 33]):
        b = Batch(dtype, 300, [60, 5, 17], new, 2, 4, 64, 16, pad_rows=37)
        n, n0 = int(b.q_start[-1]), int(b.q_start[1])
        first = b.run()
        for fill in (float("nan"), 1e4, -float("inf")):
            b.Q[n:] = fill
            b.Q[n0:n] = 30 * torch.randn_like(b.Q[n0:n])
            O, lse = b.run()
            assert (O[:n0] == first[0][:n0]).all() and (lse[:n0] == first[1][:n0]).all()


def test_prefix_attend_bounds_lengths_and_pages_that_are_wrong():
    """Lengths past the table, pages outside the pool, starts past the rows: nothing outside is
    read or written (checked on the rows that are still well defined)."""
    for new, T in (([1, 1, 1], 40), ([20, 2, 3], 40), ([1, 1, 1], 640)):
        b = Batch("bf16", T, [60, 5, 17], new, 2, 4, 64, 16)
        want = b.want()
        b.table[1] = [-1] * b.table.shape[1]
        b.table[2, 0] = b.desc.n_pages
        b.kv_len = b.kv_len.copy()
        b.kv_len[1] = 2 ** 31 - 1
        O, lse = b.run(max_new=max(new))
        n0, n1 = int(b.q_start[1]), int(b.q_start[2])
        half = 2.0 ** -7
        assert (np.abs(O[:n0] - want[0][:n0]) <= half * (np.abs(want[0]) + want[2])[:n0]).all()
        only = b.want(pages=False)          # request 1's pages are all outside: the prefix alone
        assert (np.abs(O[n0:n1] - only[0][n0:n1]) <= half * (np.abs(only[0]) + only[2])[n0:n1]).all()
        keep = b.q_start
        b.q_start = np.array([0, n0, b.n_tok + 1000, 2 ** 31 - 1])
        O, _ = b.run(max_new=max(new))
        assert (np.abs(O[:n0] - want[0][:n0]) <= half * (np.abs(want[0]) + want[2])[:n0]).all()
        b.q_start = keep[::-1].copy()
        b.run(max_new=max(new))
        b.q_start = np.array([-2 ** 31, -5, 2 ** 31 - 1, 0])
        b.run(max_new=max(new))


def test_prefix_attend_equal_calls_give_equal_bits_and_streams_do_not_matter():
    b = Batch("bf16", 3000, [60, 5, 17] * 9, [1, 20, 3] * 9, 2, 4, 64, 16)
    O, lse = b.run()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for stream in (None, s, s):
        O2, lse2 = b.run(stream=stream)
        assert (O2 == O).all() and (lse2 == lse).all()


def test_prefix_attend_most_requests():
    rng = np.random.default_rng(0)
    b = Batch("bf16", 5, rng.integers(0, 40, 4096).tolist(), rng.integers(0, 3, 4096).tolist(), 1, 2, 32, 8)
    b.check(b.run(max_new=2), b.want())


def test_prefix_attend_rows_with_strides():
    """Q inside the rows of a joint projection, O inside wider rows; nothing beside O's rows is written."""
    for new in ([1, 1, 0, 2], [30, 1, 2, 40]):
        b = Batch("bf16", 100, [60, 5, 17, 0], new, 2, 4, 64, 16)
        want, n = b.want(), b.n_tok
        wide_q = torch.zeros((n, 8 + 2 * 2, 64), dtype=torch.bfloat16, device="cuda")
        wide_q[:, 2:10] = b.Q
        wide_o = torch.full((n, 9, 64), 7.0, dtype=torch.bfloat16, device="cuda")
        ws = torch.empty(J.jolt_prefix_attend_workspace_size(4, n, 8, prefix=b.prefix, pages=b.desc, max_pages=b.table.shape[1]),
                         dtype=torch.uint8, device="cuda")
        J.jolt_prefix_attend(ctx(), wide_q[:, 2:10], wide_o[:, :8], dev_i(b.q_start), dev_i(b.kv_len), b.scale, ws, prefix=b.prefix,
                             K_prefix=b.K, V_prefix=b.V, layer=1, pages=b.desc, K_pages=b.Kp, V_pages=b.Vp, table=dev_i(b.table))
        torch.cuda.synchronize()
        O, lse = b.run()
        assert (f64(wide_o[:, :8]) == O).all() and (wide_o[:, 8] == 7.0).all()
        b.check((O, lse), want)


def test_prefix_attend_calls_at_once():
    """Calls on several streams, each with a workspace of its own, give what they give alone."""
    bs = [Batch("bf16", 3000 + 500 * i, [60, 500, 17] * 5, new * 5, 2, 4, 64, 16, seed=i) for i, new in enumerate(([1, 1, 1], [1, 20, 3], [2, 1, 2]))]
    alone = [b.run() for b in bs]
    streams = [torch.cuda.Stream() for _ in bs]
    state = [(torch.empty(J.jolt_prefix_attend_workspace_size(15, b.n_tok, 8, prefix=b.prefix, pages=b.desc, max_pages=b.table.shape[1]),
                          dtype=torch.uint8, device="cuda"), dev_i(b.q_start), dev_i(b.kv_len), dev_i(b.table), torch.zeros_like(b.Q)) for b in bs]
    torch.cuda.synchronize()
    for _ in range(5):
        for b, s, (ws, qs, kv, tab, O) in zip(bs, streams, state):
            J.jolt_prefix_attend(ctx(), b.Q, O, qs, kv, b.scale, ws, prefix=b.prefix, K_prefix=b.K, V_prefix=b.V, layer=1, pages=b.desc,
                                 K_pages=b.Kp, V_pages=b.Vp, table=tab, stream=s)
    torch.cuda.synchronize()
    for (O, _), st in zip(alone, state):
        assert (f64(st[4]) == O).all()


def test_long_tails_past_32_bit_offsets():
    """A pool of more than 2^31 elements, with the request's pages at its far end."""
    H, page, d = 8, 1024, 128
    n_pages = (1 << 31) // (H * page * d) + 3
    desc = pages_desc("bf16", H, page, d, n_pages)
    pool = torch.zeros((n_pages, H, page, d), dtype=torch.bfloat16, device="cuda")
    g = torch.Generator("cuda").manual_seed(1)
    x = torch.randn((2, H, page, d), device="cuda", generator=g).bfloat16()
    table = np.array([[n_pages - 1, n_pages - 2]])
    slots = np.concatenate([np.arange(page) + (n_pages - 1) * page, [(n_pages - 2) * page]])
    V = torch.zeros_like(pool)
    k = torch.cat([x[0], x[1][:, :1]], 1).transpose(0, 1).contiguous()
    J.jolt_page_append(ctx(), desc, k, 2 * k, dev_i(slots), pool, V)
    Q = torch.randn((1, H, d), device="cuda", generator=g).bfloat16()
    O, lse = torch.zeros_like(Q), torch.zeros((1, H), device="cuda")
    ws = torch.empty(J.jolt_prefix_attend_workspace_size(1, 1, H, pages=desc, max_pages=2, max_new=1), dtype=torch.uint8, device="cuda")
    J.jolt_prefix_attend(ctx(), Q, O, dev_i([0, 1]), dev_i([page + 1]), 0.1, ws, pages=desc, K_pages=pool, V_pages=V, table=dev_i(table),
                         max_new=1, lse=lse)
    torch.cuda.synchronize()
    kk = f64(k).transpose(1, 0, 2)
    wO, wl, A, _ = osv.prefix_attend(f64(Q), kk[:, :0], kk[:, :0], [kk], [2 * kk], [0, 1], [page + 1], 0.1)
    assert (np.abs(f64(O) - wO) <= 2.0 ** -7 * (np.abs(wO) + A)).all() and (np.abs(f64(lse) - wl) <= 1e-4).all()
    assert int((pool != 0).any(-1).sum()) == H * (page + 1)


def test_tensor_arguments_are_checked_before_the_library():
    """Types, sizes and layouts that do not fit are refused by the binding (the null context would
    end every call before device work)."""
    A = 1 << 20
    pages = J.page_desc(dtype=J.JOLT_BF16, n_heads=8, page_size=16, d=128, n_pages=100, stride_page=8 * 16 * 128,
                        stride_head=16 * 128, stride_token=128)
    z = torch.zeros(4, dtype=torch.int32, device="cuda")
    t = torch.zeros((4, 3), dtype=torch.int32, device="cuda")
    one = torch.zeros(1, dtype=torch.int32, device="cuda")
    args = dict(have=z, add=z, free_pages=z, n_free=one, table=t, kv_len=z.clone(), q_start=torch.zeros(5, dtype=torch.int32, device="cuda"),
                slots=z.clone(), positions=z.clone(), n_free_out=one.clone(), info=z.clone())
    bad = dict(have=z.long(), add=z[:3], n_free=z, table=t[:2], kv_len=t[:, 0], q_start=z, positions=z[:2], n_free_out=z, info=one)
    for k, v in bad.items():
        with pytest.raises(ValueError):
            J.jolt_page_plan(None, pages, **{**args, k: v})
    K = torch.zeros((4, 8, 128), dtype=torch.bfloat16, device="cuda")
    for k, v in ((K.float(), K), (K, K[:, :4]), (K[:3], K), (K.transpose(1, 2), K), (K, K[..., ::2])):
        with pytest.raises(ValueError):
            J.jolt_page_append(None, pages, k, v, z, A, 2 * A)
    Q = torch.zeros((4, 32, 128), dtype=torch.bfloat16, device="cuda")
    qs = torch.zeros(5, dtype=torch.int32, device="cuda")
    for kw in (dict(Q=Q.float()), dict(O=Q[:3]), dict(lse=torch.zeros(4, 32, dtype=torch.float64, device="cuda")), dict(kv_len=z[:2]),
               dict(table=t[:2]), dict(q_start=qs[:3]), dict(Q=Q.transpose(0, 1)), dict(pages=None), dict(Q=Q.cpu())):
        a = dict(Q=Q, O=Q.clone(), q_start=qs, kv_len=z, scale=0.1, ws=A, pages=pages, K_pages=A, V_pages=A, table=t, ws_bytes=1)
        with pytest.raises(ValueError):
            J.jolt_prefix_attend(None, **{**a, **kw})
    ok = dict(Q=Q, O=Q.clone(), q_start=qs, kv_len=z, scale=0.1, ws=A, pages=pages, K_pages=A, V_pages=2 * A, table=t, ws_bytes=1 << 40)
    for call in (lambda: J.jolt_page_plan(None, pages, **args), lambda: J.jolt_page_append(None, pages, K, K, z, A, 2 * A),
                 lambda: J.jolt_prefix_attend(None, **ok)):
        with pytest.raises(J.JoltError, match="ctx is null"):
            call()


# ------------------------------------------------------------------------------- a step
class Server:
    """The three operators as a serving loop uses them, with the oracle's state beside them."""

    def __init__(self, T, n_req, H, G, d, page, n_tok, max_pages, n_pages, seed=0):
        rng = np.random.default_rng(seed)
        self.H, self.G, self.d, self.page, self.T, self.n_pages = H, G, d, page, T, n_pages
        self.desc = pages_desc("bf16", H, page, d, n_pages)
        _, self.Kp, self.Vp = pools(self.desc, "bf16", "hpd", float("nan"))
        self.free = rng.permutation(n_pages)
        self.d_free = dev_i(self.free)
        self.table = dev_i(np.full((n_req, max_pages), -1))
        self.lens = [dev_i([0] * n_req), dev_i([0] * n_req)]
        self.nfree = [dev_i([n_pages]), dev_i([0])]
        self.add, self.q_start, self.info = dev_i([0] * n_req), dev_i([0] * (n_req + 1)), dev_i([0] * 4)
        self.slots, self.pos = dev_i([0] * n_tok), dev_i([0] * n_tok)
        self.q = torch.zeros((n_tok, H * G, d), dtype=torch.bfloat16, device="cuda")
        self.k, self.v = (torch.zeros((n_tok, H, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        self.O, self.lse = torch.zeros_like(self.q), torch.zeros((n_tok, H * G), device="cuda")
        self.tk, self.tv = [[] for _ in range(n_req)], [[] for _ in range(n_req)]

    def prefix(self, K, V):
        self.K, self.V = K, V
        self.pre = J.cell_desc(dtype=J.JOLT_BF16, n_layers=1, n_heads=self.H, T=self.T, d=self.d, stride_layer=self.H * self.T * self.d,
                               stride_head=self.T * self.d, stride_token=self.d)
        nb = J.jolt_prefix_attend_workspace_size(self.add.numel(), self.q.shape[0], self.q.shape[1], prefix=self.pre, pages=self.desc,
                                                 max_pages=self.table.shape[1])
        self.ws = torch.empty(nb, dtype=torch.uint8, device="cuda")

    def step(self, flip, stream=None):
        a, b = (0, 1) if flip == 0 else (1, 0)
        J.jolt_page_plan(ctx(), self.desc, self.lens[a], self.add, self.d_free, self.nfree[a], self.table, self.lens[b], self.q_start,
                         self.slots, self.pos, self.nfree[b], self.info, stream=stream)
        J.jolt_page_append(ctx(), self.desc, self.k, self.v, self.slots, self.Kp, self.Vp, positions=self.pos, rope=(1e4, self.T), stream=stream)
        J.jolt_prefix_attend(ctx(), self.q, self.O, self.q_start, self.lens[b], self.d ** -0.5, self.ws, prefix=self.pre, K_prefix=self.K,
                             V_prefix=self.V, pages=self.desc, K_pages=self.Kp, V_pages=self.Vp, table=self.table, lse=self.lse, stream=stream)

    def inputs(self, add, seed):
        g = torch.Generator("cuda").manual_seed(seed)
        self.add.copy_(dev_i(add))
        for x in (self.q, self.k, self.v):
            x.copy_(torch.randn(x.shape, device="cuda", generator=g))
        t = 0
        for r, n in enumerate(add):
            for _ in range(n):
                pos = [len(self.tk[r]) + self.T]
                self.tk[r].append(osv.rotate(f64(self.k[t:t + 1]), pos, 1e4)[0])
                self.tv[r].append(f64(self.v[t]))
                t += 1
        self.n_rows, self.new = t, add

    def check(self):
        st = lambda x: np.stack(x, 1) if x else np.zeros((self.H, 0, self.d))  # noqa: E731
        qs = np.concatenate([[0], np.cumsum(self.new)])
        O, lse, A, S = osv.prefix_attend(f64(self.q), f64(self.K), f64(self.V), [st(x) for x in self.tk], [st(x) for x in self.tv], qs,
                                         [len(x) for x in self.tk], self.d ** -0.5)
        n = self.n_rows
        # the oracle's keys are not rounded to bf16: each score moves by half a step of its products
        ds = (2.0 ** -8 + (self.d + 4) * 2.0 ** -24) * S[:n]
        w = 2 * ds * np.exp(2 * ds) + 2.0 ** -8 + 2.0 ** -12
        assert (np.abs(f64(self.O[:n]) - O[:n]) <= 2.0 ** -8 * np.abs(O[:n]) + w[..., None] * A[:n]).all()
        assert (np.abs(f64(self.lse[:n]) - lse[:n]) <= ds + 2.0 ** -12).all()
        assert self.info.tolist()[2] == 0


def _decoded_prefix(H, T, d):
    """Keys (with RoPE) and values of one layer, compressed and decompressed by the library."""
    from gpu_util import compress, device_cells, workspace
    kv = kvsynth.make_cache(n_layers=1, n_heads=H, T=T, d=d, dtype="f32")
    cells = [kv[t][:, 0].reshape(H, T, d).astype(np.float64) for t in (0, 1)]
    xs, _, desc = device_cells(cells, "bf16")
    blobs, _ = compress(xs, desc, [J.Params(48, 48, 8, 32, J.JOLT_FACTOR_F16, 0, i) for i in (1, 2)])
    out = [torch.empty((H, T, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    ws = workspace(desc, 2)
    J.jolt_decompress(ctx(), blobs[:1], desc, out[:1], ws, rope=(1e4, 0))
    J.jolt_decompress(ctx(), blobs[1:], desc, out[1:], ws)
    torch.cuda.synchronize()
    return out


STEPS = [[7, 0, 20, 1, 3], [1, 1, 1, 1, 1], [1, 30, 1, 0, 1], [2, 2, 2, 2, 2], [0, 0, 0, 0, 0], [1, 1, 1, 1, 1]]


def test_serving_from_a_compressed_prefix():
    H, T, d = 4, 200, 64
    s = Server(T, 5, H, 2, d, 8, 40, 8, 30)
    s.prefix(*_decoded_prefix(H, T, d))
    for i, add in enumerate(STEPS):
        s.inputs(add, i)
        s.step(i % 2)
        torch.cuda.synchronize()
        s.check()


def test_serving_steps_captured_and_replayed():
    """Two steps (the lengths go back and forth between two buffers) as one graph, replayed with
    other lengths, with eager work and synchronisations between, against the same steps run eagerly."""
    H, T, d = 4, 200, 64
    runs = []
    for captured in (False, True):
        s = Server(T, 5, H, 2, d, 8, 40, 8, 30)
        s.prefix(*_decoded_prefix(H, T, d))
        outs = []
        if captured:
            st = torch.cuda.Stream()
            st.wait_stream(torch.cuda.current_stream())
            graphs = []
            for flip in (0, 1):
                g = torch.cuda.CUDAGraph()
                with torch.cuda.graph(g, stream=st):
                    s.step(flip, stream=torch.cuda.current_stream())
                graphs.append(g)
        for i, add in enumerate(STEPS):
            s.inputs(add, i)
            if captured:
                graphs[i % 2].replay()
            else:
                s.step(i % 2)
            torch.cuda.synchronize()
            s.check()
            outs.append((s.O[:s.n_rows].clone(), s.lse[:s.n_rows].clone(), s.slots.clone(), s.table.clone(), s.info.clone()))
        runs.append(outs)
    for a, b in zip(*runs):
        for x, y in zip(a, b):
            assert torch.equal(x, y)


def test_current_device_and_profile_of_the_operators():
    J.jolt_profile_enable(ctx(), True)
    J.jolt_profile_reset(ctx())
    s = Server(0 + 16, 2, 1, 1, 32, 8, 4, 4, 8)
    s.prefix(*(torch.randn((1, 16, 32), device="cuda").bfloat16() for _ in range(2)))
    s.inputs([1, 2], 0)
    s.step(0)
    torch.cuda.synchronize()
    s.check()
    p = J.jolt_profile_read(ctx())
    J.jolt_profile_enable(ctx(), False)
    assert all(p[k][1] == 1 and p[k][0] > 0 for k in ("page_plan", "page_append", "prefix_attend"))
