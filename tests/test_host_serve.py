"""Host-side checks of the shared-prefix serving operators (no GPU needed): the argument
validation of jolt_page_plan, jolt_page_append and jolt_prefix_attend, and the oracle's plan
and attention against each other's plain restatements.

Every call passes a null context, which is looked at last: an argument at fault gives its own
code and message, and a call with none at fault ends at the context without device work.
"""
import ctypes as C

import numpy as np
import pytest

import paper_2607_12550_amd as J
from oracle import attention as oat, serving as osv

A = 1 << 20                                    # an aligned address that nothing reads


def _pages(**kw):
    a = dict(dtype=J.JOLT_BF16, n_heads=8, page_size=16, d=128, n_pages=100, stride_page=8 * 16 * 128,
             stride_head=16 * 128, stride_token=128)
    a.update(kw)
    return J.page_desc(**a)


def _prefix(**kw):
    a = dict(dtype=J.JOLT_BF16, n_layers=4, n_heads=8, T=300, d=128, stride_layer=8 * 300 * 128,
             stride_head=300 * 128, stride_token=128)
    a.update(kw)
    return J.cell_desc(**a)


def _refused(rc, code, word):
    assert rc == code, (rc, J.jolt_last_error())
    assert word in J.jolt_last_error()


def _plan(pages=_pages(), n_req=4, have=A, add=2 * A, free=3 * A, cap=50, n_free=4 * A, table=5 * A, max_pages=10,
          n_tok=64, kv=6 * A, qs=7 * A, slots=8 * A, pos=9 * A, out=10 * A, info=11 * A):
    return J.lib.jolt_page_plan(None, None if pages is None else C.byref(pages), n_req, have, add, free, cap, n_free,
                                table, max_pages, n_tok, kv, qs, slots, pos, out, info, None)


def test_page_plan_refuses_bad_arguments():
    _refused(_plan(), J.JOLT_E_INVAL, "ctx is null")
    _refused(_plan(pages=None), J.JOLT_E_INVAL, "descriptor")
    for p in (0, 3, 24, 2048, -16):
        _refused(_plan(pages=_pages(page_size=p)), J.JOLT_E_INVAL, "page_size")
    for n in (0, -1, 1 << 27):
        _refused(_plan(pages=_pages(n_pages=n)), J.JOLT_E_INVAL, "n_pages")
    for kw in (dict(n_req=0), dict(n_tok=0), dict(max_pages=0), dict(cap=-1)):
        _refused(_plan(**kw), J.JOLT_E_INVAL, "must be")
    _refused(_plan(max_pages=1 << 26), J.JOLT_E_INVAL, "2^30")
    _refused(_plan(n_req=4097), J.JOLT_E_UNSUPPORTED, "4096")
    for kw in ("have", "add", "free", "n_free", "table", "kv", "qs", "slots", "pos", "out", "info"):
        _refused(_plan(**{kw: None}), J.JOLT_E_INVAL, "null argument")
    _refused(_plan(free=None, cap=0), J.JOLT_E_INVAL, "ctx is null")      # an empty stack needs no memory
    for kw in (dict(kv=A), dict(kv=2 * A), dict(out=4 * A)):
        _refused(_plan(**kw), J.JOLT_E_INVAL, "their own")


def _append(pages=_pages(), n_tok=4, slots=A, pos=2 * A, rope=None, K=3 * A, ks=(1024, 128), V=4 * A, vs=(1024, 128),
            Kp=5 * A, Vp=6 * A):
    s = [None if x is None else C.byref(J.RowStrides(*x)) for x in (ks, vs)]
    r = None if rope is None else C.byref(J.Rope(*rope, 0))
    return J.lib.jolt_page_append(None, C.byref(pages), n_tok, slots, pos, r, K, s[0], V, s[1], Kp, Vp, None)


def test_page_append_refuses_bad_arguments():
    _refused(_append(), J.JOLT_E_INVAL, "ctx is null")
    _refused(_append(rope=(1e4, 300)), J.JOLT_E_INVAL, "ctx is null")
    _refused(_append(pos=None), J.JOLT_E_INVAL, "ctx is null")
    _refused(_append(pos=None, rope=(1e4, 0)), J.JOLT_E_INVAL, "null argument")
    for kw in ("slots", "Kp", "Vp"):
        _refused(_append(**{kw: None}), J.JOLT_E_INVAL, "null argument")
    for kw in ("K", "V", "ks", "vs"):
        _refused(_append(**{kw: None}), J.JOLT_E_INVAL, "null")
    for kw in ("K", "V", "Kp", "Vp"):
        _refused(_append(**{kw: 3 * A + 8}), J.JOLT_E_INVAL, "16-byte")
    for st in ((1020, 128), (1024, -8), (-1024, 128), (1024, 4)):
        _refused(_append(ks=st), J.JOLT_E_INVAL, "strides")
    _refused(_append(Vp=5 * A), J.JOLT_E_INVAL, "pool each")
    _refused(_append(n_tok=0), J.JOLT_E_INVAL, "n_tok")
    for rope in ((1.0, 0), (float("nan"), 0), (float("inf"), 0), (1e4, -1)):
        _refused(_append(rope=rope), J.JOLT_E_INVAL, "rope")
    _refused(_append(pages=_pages(d=48)), J.JOLT_E_UNSUPPORTED, "d must")
    _refused(_append(pages=_pages(dtype=7)), J.JOLT_E_INVAL, "dtype")
    for kw in (dict(stride_token=64), dict(stride_head=15 * 128), dict(stride_page=7 * 16 * 128), dict(stride_page=0),
               dict(stride_token=132), dict(stride_head=-2048), dict(stride_page=1 << 58)):
        _refused(_append(pages=_pages(**kw)), J.JOLT_E_INVAL, "strides")
    # tokens outside heads, heads outside pages, and an unused stride of a single page
    for kw in (dict(stride_token=8 * 128, stride_head=128), dict(stride_head=100 * 16 * 128, stride_page=16 * 128),
               dict(n_pages=1, stride_page=0), dict(n_heads=1, stride_head=0)):
        _refused(_append(pages=_pages(**kw)), J.JOLT_E_INVAL, "ctx is null")


def _attend(prefix=_prefix(), K=A, V=2 * A, layer=0, pages=_pages(), Kp=3 * A, Vp=4 * A, table=5 * A, n_req=4, n_tok=8,
            n_q=32, max_pages=10, max_new=0, qst=4096, ost=4096, qs=6 * A, kv=7 * A, Q=8 * A, scale=0.1, O=9 * A,
            lse=None, ws=10 * A, nb=1 << 40, batch=True):
    b = C.byref(J.AttendBatch(n_req, n_tok, n_q, max_pages, max_new, 0, qst, ost)) if batch else None
    return J.lib.jolt_prefix_attend(None, None if prefix is None else C.byref(prefix), K, V, layer,
                                    None if pages is None else C.byref(pages), Kp, Vp, table, b, qs, kv, Q, scale, O,
                                    lse, ws, nb, None)


def test_prefix_attend_refuses_bad_arguments():
    for ok in (dict(), dict(prefix=None, K=None, V=None), dict(pages=None, Kp=None, Vp=None, table=None, kv=None),
               dict(layer=3), dict(max_new=5), dict(lse=11 * A), dict(n_q=8, qst=1024, ost=1024)):
        _refused(_attend(**ok), J.JOLT_E_INVAL, "ctx is null")
    _refused(_attend(batch=False), J.JOLT_E_INVAL, "batch")
    _refused(_attend(prefix=None, pages=None), J.JOLT_E_INVAL, "neither")
    for kw in ("Q", "O", "ws", "qs"):
        _refused(_attend(**{kw: None}), J.JOLT_E_INVAL, "null argument")
    for kw in ("K", "V"):
        _refused(_attend(**{kw: None}), J.JOLT_E_INVAL, "without keys")
    for kw in ("Kp", "Vp", "table", "kv"):
        _refused(_attend(**{kw: None}), J.JOLT_E_INVAL, "without pools")
    for kw in ("K", "V", "Kp", "Vp", "Q", "O"):
        _refused(_attend(**{kw: 8 * A + 8}), J.JOLT_E_INVAL, "16-byte")
    _refused(_attend(ws=10 * A + 128), J.JOLT_E_INVAL, "256-byte")
    for layer in (-1, 4):
        _refused(_attend(layer=layer), J.JOLT_E_INVAL, "layer")
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        _refused(_attend(scale=scale), J.JOLT_E_INVAL, "scale")
    for p in (_prefix(d=64, stride_token=64), _prefix(n_heads=4), _prefix(dtype=J.JOLT_F32)):
        _refused(_attend(prefix=p), J.JOLT_E_INVAL, "differ")
    _refused(_attend(prefix=_prefix(T=1 << 20, stride_head=1 << 27, stride_layer=1 << 30)), J.JOLT_E_UNSUPPORTED, "2^20")
    _refused(_attend(prefix=_prefix(T=0)), J.JOLT_E_INVAL, "T must")
    for kw in (dict(n_req=0), dict(n_tok=0), dict(n_q=0)):
        _refused(_attend(**kw), J.JOLT_E_INVAL, "empty")
    _refused(_attend(n_req=4097), J.JOLT_E_UNSUPPORTED, "requests")
    _refused(_attend(n_q=12), J.JOLT_E_INVAL, "multiple")
    _refused(_attend(n_q=520, qst=1 << 17, ost=1 << 17), J.JOLT_E_UNSUPPORTED, "per key-value head")
    _refused(_attend(n_tok=1 << 23), J.JOLT_E_UNSUPPORTED, "2^28")
    _refused(_attend(max_new=-1), J.JOLT_E_INVAL, "max_new")
    for kw in (dict(qst=4088), dict(ost=4088), dict(qst=4100), dict(ost=4100)):
        _refused(_attend(**kw), J.JOLT_E_INVAL, "strides of Q and O")
    for n in (0, 1 << 26):
        _refused(_attend(max_pages=n), J.JOLT_E_INVAL, "max_pages")
    need = J.jolt_prefix_attend_workspace_size(4, 8, 32, prefix=_prefix(), pages=_pages(), max_pages=10)
    _refused(_attend(nb=need - 1), J.JOLT_E_WORKSPACE, "workspace")
    _refused(_attend(nb=need), J.JOLT_E_INVAL, "ctx is null")


def test_tensors_off_the_gpu_are_refused():
    """The binding takes GPU tensors only; a host tensor never reaches a kernel."""
    import torch
    z = [torch.zeros(n, dtype=torch.int32) for n in (4, 4, 4, 1, 4, 5, 4, 4, 1, 4)]
    t = torch.zeros((4, 3), dtype=torch.int32)
    with pytest.raises(ValueError, match="on the GPU"):
        J.jolt_page_plan(None, _pages(), *z[:4], t, *z[4:])
    K = torch.zeros((4, 8, 128), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="on the GPU"):
        J.jolt_page_append(None, _pages(), K, K, z[0], A, 2 * A)
    Q = torch.zeros((4, 32, 128), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="on the GPU"):
        J.jolt_prefix_attend(None, Q, Q, z[5], z[0], 0.1, A, pages=_pages(), K_pages=A, V_pages=A, table=t, ws_bytes=1)
    with pytest.raises(ValueError, match="must be a tensor"):
        J.jolt_page_append(None, _pages(), [1], K, z[0], A, 2 * A)


# ------------------------------------------------------------------------------ the oracle
def test_oracle_plan_fills_every_slot_once(rng):
    page, n_pages = 8, 64
    have, add = [0, 5, 16, 3], [9, 0, 1, 30]
    ids = rng.permutation(n_pages)
    table = np.full((4, 6), -1)
    at = 0
    for r, h in enumerate(have):
        k = -(-h // page)
        table[r, :k] = ids[at:at + k]
        at += k
    free = ids[at:]
    out = osv.plan(have, add, page, free, len(free), table, 48, n_pages)
    assert out["info"].tolist() == [40, 2 + 0 + 1 + 4, 0, 7] and out["n_free"] == len(free) - 7
    used = out["slots"][:40]
    assert len(set(used.tolist())) == 40 and (out["slots"][40:] == -1).all()
    held = {table[r, x // page] * page + x % page for r, h in enumerate(have) for x in range(h)}
    assert not held & set(used.tolist())
    for r in range(4):                             # a request's rows lie where its table says
        for i in range(add[r]):
            x = have[r] + i
            assert out["slots"][out["q_start"][r] + i] == out["table"][r, x // page] * page + x % page


def test_oracle_prefix_attention_is_plain_attention(rng):
    H, T, d, n_q = 2, 5, 8, 6
    K, V = rng.standard_normal((2, H, T, d))
    tk, tv = rng.standard_normal((2, H, 3, d))
    Q = rng.standard_normal((2, n_q, d))
    O, lse, _, _ = osv.prefix_attend(Q, K, V, [tk], [tv], [0, 2], [3], 0.3)
    for i, seen in enumerate((2, 3)):
        k, v = np.concatenate([K, tk[:, :seen]], 1), np.concatenate([V, tv[:, :seen]], 1)
        np.testing.assert_allclose(O[i], oat.attend(k, v, 0, H, Q[i], 0.3), rtol=1e-12)
        s = 0.3 * np.einsum("htd,hgd->hgt", k, Q[i].reshape(H, 3, d))
        np.testing.assert_allclose(lse[i], np.log(np.exp(s).sum(-1)).reshape(-1), rtol=1e-12)
