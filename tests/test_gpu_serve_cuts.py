"""GPU tests of jolt_prefix_attend over calls that run each of its kernels' forms (serve_cuts.py):
random inputs against the definition in float64, with the tolerances of test_gpu_serve.py, equal
weights over values of which every one counts, and values that show the weights themselves.
"""
import numpy as np
import pytest
import torch

from serve_cuts import CUTS, cut, name
from test_gpu_serve import CASES, DT, Batch

pytestmark = pytest.mark.gpu


def want64(b):
    """What b.want() gives, request by request in float64 on the GPU."""
    H, G, d = b.H, b.G, b.d
    n_all = b.Q.shape[0]
    O, A = (torch.full((n_all, H * G, d), float("nan"), dtype=torch.float64, device="cuda") for _ in range(2))
    lse, S = (torch.full((n_all, H * G), float("nan"), dtype=torch.float64, device="cuda") for _ in range(2))
    for r, length in enumerate(b.kv_len):
        q0, q1 = int(b.q_start[r]), int(b.q_start[r + 1])
        n = q1 - q0
        if n == 0:
            continue
        k, v = (torch.cat(([x[1][:, :b.T]] if b.T else []) + [t[r][:, :length]], 1).double() for x, t in ((b.K, b.tk), (b.V, b.tv)))
        q = b.Q[q0:q1].double().reshape(n, H, G, d).permute(1, 0, 2, 3).reshape(H, n * G, d)
        kt = k.transpose(1, 2).contiguous()
        hidden = torch.arange(k.shape[1], device="cuda") > (b.T + int(length) - n + torch.arange(n, device="cuda"))[:, None]
        hidden = hidden.repeat_interleave(G, 0)
        s = (b.scale * (q @ kt)).masked_fill(hidden, -np.inf)
        top = s.amax(-1, keepdim=True)
        p = (s - top).exp()
        total = p.sum(-1, keepdim=True)

        def put(dst, x):
            dst[q0:q1] = x.reshape(H, n, G, *x.shape[2:]).transpose(0, 1).reshape(n, H * G, *x.shape[2:])
        put(O, p @ v / total)
        put(A, p @ v.abs() / total)
        put(lse, (top + total.log())[..., 0])
        put(S, (b.scale * (q.abs() @ kt.abs())).masked_fill(hidden, 0).amax(-1))
    return tuple(x.cpu().numpy() for x in (O, lse, A, S))


def test_the_definition_on_the_gpu_is_the_oracle():
    b = Batch("bf16", 33, [5, 0, 40], [1, 9, 3], 2, 3, 32, 8, pad_rows=2)
    for x, y in zip(want64(b), b.want()):
        np.testing.assert_allclose(x, y, rtol=1e-10, atol=1e-12)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("call,rows,how,many,join", CUTS, ids=[name(c[0]) for c in CUTS])
def test_every_form_of_the_kernels(dtype, call, rows, how, many, join):
    b = Batch(dtype, *call, seed=call[0])
    assert cut(dtype, call)["prefix_rows"] == rows[dtype != "bf16"]
    b.check(b.run(max_new=max(call[2])), want64(b))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("call", [c[0] for c in CUTS] + CASES, ids=name)
def test_every_token_counts(dtype, call):
    """Queries of zero weigh all tokens alike, 2^-8 or its product with a power of two, and token x
    has the value 1 at feature (x + 5 h) % d and 0 elsewhere: sums are whole multiples of the weight
    and exact, so that an output is off by the rounding of 1 / l, of its product and of itself (half a
    step), and a token that is lost or taken twice moves one by far more.  lse is ln of the
    number of tokens: log2 right to two steps of a value below 16, two roundings of sums
    below 32 and one product, in all below 2^-18."""
    T, have, new, H, G, d, page = call
    b = Batch(dtype, *call)
    b.Q.zero_()
    eye = torch.eye(d, device="cuda", dtype=b.V.dtype)
    heads = 5 * torch.arange(H, device="cuda")[:, None]
    b.V[1] = eye[(torch.arange(b.V.shape[2], device="cuda") + heads) % d]
    at = torch.arange(int(b.kv_len.max()), device="cuda")
    tail = eye[(at + 3 + heads) % d]                                        # [H][tokens][d]
    columns = torch.as_tensor(b.table, device="cuda").clamp(min=0).long()
    for r, length in enumerate(b.kv_len):
        x = at[:int(length)]
        b.Vp[columns[r, x // page], :, x % page] = tail[:, :int(length)].transpose(0, 1)
    O, lse = b.run(max_new=max(new))
    pre = b.V[1][:, :T].double().sum(1)
    running = torch.cat([torch.zeros((H, 1, d), dtype=torch.float64, device="cuda"), tail.double().cumsum(1)], 1)
    tol = DT[dtype][2] + 2.0 ** -22
    for r, length in enumerate(b.kv_len):
        q0, n = int(b.q_start[r]), int(b.q_start[r + 1] - b.q_start[r])
        seen = (int(length) - n + 1 + torch.arange(n, device="cuda")).clamp(min=0)
        count = (T + seen).double()[:, None, None]
        want = ((pre + running[:, seen].transpose(0, 1)) / count).repeat_interleave(G, 1).cpu().numpy()
        assert (np.abs(O[q0:q0 + n] - want) <= tol * want).all(), r
        assert (np.abs(lse[q0:q0 + n] - count.log()[..., 0].cpu().numpy()) <= 2.0 ** -18).all(), r


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_more_heads_than_workgroups_fill_the_chip(dtype):
    for call in ((70, [5, 3], [1, 2], 1024, 1, 32, 8), (300, [500, 0, 2], [1, 2, 1], 600, 2, 64, 16), (200, [3, 40], [40, 2], 513, 1, 64, 16)):
        b = Batch(dtype, *call)
        b.check(b.run(max_new=max(call[2])), want64(b))


@pytest.mark.parametrize("new,T", [([1, 1, 2], 40), ([1, 3, 2], 900), ([40, 1, 9], 300)])
def test_rows_before_the_first_request_are_left(new, T):
    b = Batch("bf16", T, [9, 0, 50], new, 2, 4, 64, 8, pad_rows=11)
    b.q_start = b.q_start + 7
    b.check(b.run(max_new=max(new)), want64(b))


@pytest.mark.parametrize("new,T", [([1, 1, 2], 40), ([1, 3, 2], 900), ([40, 1, 9], 300)])
def test_requests_that_share_pages(new, T):
    """One tail's pages in the tables of two requests, and a page twice in one table."""
    b = Batch("bf16", T, [30, 30 + new[0] - new[1], 70], new, 2, 4, 64, 8)
    b.table[1], b.tk[1], b.tv[1] = b.table[0], b.tk[0], b.tv[0]
    b.table[2, 3] = b.table[2, 1]
    for x in (b.tk, b.tv):
        x[2][:, 24:32] = x[2][:, 8:16]
    b.check(b.run(max_new=max(new)), want64(b))


def _weights_seen(b, where):
    """Values that make an output a row's weights themselves: the unit rows for the d tokens of the prefix
    (where = "prefix") or for the first d tokens of every tail, zero for all others."""
    eye = torch.eye(b.d, device="cuda", dtype=b.V.dtype)
    b.V.zero_()
    if where == "prefix":
        b.V[1, :, :b.d] = eye
    columns = torch.as_tensor(b.table, device="cuda").clamp(min=0).long()
    for r, v in enumerate(b.tv):
        v.zero_()
        if where == "tails":
            v[:, :b.d] = eye[:v.shape[1]]
        x = torch.arange(v.shape[1], device="cuda")
        b.Vp[columns[r, x // b.page], :, x % b.page] = v.transpose(0, 1)


@pytest.mark.parametrize("where", ["prefix", "tails"])
@pytest.mark.parametrize("new,columns", [([1, 1], 0), ([1, 1], 64), ([3, 2], 64), ([40, 2], 0)])
def test_bf16_weights_keep_sixteen_bits(where, new, columns):
    """With values that show the weights every entry is off by the rounding of the output (half a step)
    and by its weight alone: two bf16 terms, the second below 2^-7 of the weight and rounded at
    2^-8 of itself; scores and sums as in test_gpu_serve.py."""
    d = 64
    b = Batch("bf16", d, [d, 9], new, 2, 4, d, 16, seed=3)
    b.table = np.pad(b.table, ((0, 0), (0, max(0, columns - b.table.shape[1]))), constant_values=-1)
    _weights_seen(b, where)
    O, lse = b.run(max_new=max(new))
    want, wl, A, S = want64(b)
    ds = (d + 4) * 2.0 ** -24 * S + 2.0 ** -22 * (np.abs(wl) + S)
    w = 2 * ds + (b.T + b.kv_len.max() + 8) * 2.0 ** -24 + 2.0 ** -15 + 2.0 ** -23
    assert (want > 0).any() and (np.abs(O - want) <= (2.0 ** -8 + w[..., None]) * want).all()


@pytest.mark.parametrize("new,T", [([1, 1], 50), ([1, 1], 600), ([40, 2], 600)])
def test_infinite_value_under_weights_of_one_bit(new, T):
    """Equal weights, which one bf16 term holds exactly: an infinite value stays infinite, of its sign."""
    b = Batch("bf16", T, [60, 5], new, 2, 4, 64, 16)
    b.Q.zero_()
    b.V[1, 1, 7, 3], b.V[1, 0, 9, 5] = float("inf"), -float("inf")
    b.Vp[b.table[0, 0], 0, 2, 6] = float("inf")
    O, _ = b.run(max_new=max(new))
    n0 = int(b.q_start[1])
    assert np.isposinf(O[:, 4:, 3]).all() and np.isneginf(O[:, :4, 5]).all() and np.isposinf(O[:n0, :4, 6]).all()
    for x, f in ((O[:n0, 4:], [3]), (O[:n0, :4], [5, 6]), (O[n0:, :4], [5])):
        assert np.isfinite(np.delete(x, f, 2)).all()
