"""Host-side checks of the shared-prefix serving operators at the edges of what they accept (no GPU
needed): tensors that do not hold what a descriptor reaches, workspaces of smaller batches, and the
choice of kernels that the GPU tests rely on; and a package without the binding's native checks.
"""
import os
import random
import subprocess
import sys
import types

import pytest
import torch

import paper_2607_12550_amd as J
from serve_cuts import CUTS, cut
from test_host_serve import A, _attend, _pages, _prefix, _refused


def _small(**kw):
    """Pages of 2 heads, 4 tokens and 32 features, 3 of them: 768 elements."""
    return _pages(**{**dict(n_heads=2, page_size=4, d=32, n_pages=3, stride_page=256, stride_head=128, stride_token=32), **kw})


def _cell(**kw):
    """Two layers of 2 heads, 5 tokens and 32 features: 640 elements, 320 of them for layer 0 alone."""
    return _prefix(**{**dict(n_layers=2, n_heads=2, T=5, d=32, stride_layer=320, stride_head=160, stride_token=32), **kw})


def _t(n, dtype=torch.bfloat16):
    return torch.zeros(n, dtype=dtype)


def test_memory_that_a_descriptor_reaches_is_checked():
    """Type, size and device of pools, prefix and workspace; a host tensor is the last to be seen, so
    one that fits in all else shows that."""
    big = torch.zeros(1000, dtype=torch.bfloat16)
    for bad, word in ((_t(768, torch.float32), "bfloat16"), (_t(767), "768 elements"), (big[300:], "768 elements"),
                      (_t(1).expand(768), "768 elements"), (_t(1535, torch.uint8), "768 elements"), (_t(1536, torch.uint8), "on the GPU"), (_t(768), "on the GPU"), (big[232:], "on the GPU"), ([1], "must be a tensor")):
        for K, V, name in ((bad, A, "K_pages"), (A, bad, "V_pages")):
            with pytest.raises(ValueError, match=name) as e:
                J._marshal.pools(_small(), K, V)
            assert word in str(e.value)
    # padded rows, tokens outside heads, and strides of axes of one element, which reach nowhere
    for desc, n in ((_small(stride_token=40, stride_head=160, stride_page=320), 2 * 320 + 160 + 3 * 40 + 32),
                    (_small(stride_token=64, stride_head=32), 768), (_small(n_pages=1, stride_page=1 << 40), 256)):
        with pytest.raises(ValueError, match=f"{n} elements"):
            J._marshal.pools(desc, _t(n - 1), A)
        with pytest.raises(ValueError, match="on the GPU"):
            J._marshal.pools(desc, _t(n), A)
    with pytest.raises(ValueError, match="float32"):
        J._marshal.pools(_small(dtype=J.JOLT_F32), _t(768), A)
    for layer, n in ((0, 320), (1, 640), (5, 320)):
        with pytest.raises(ValueError, match="K_prefix.*%d elements" % n):
            J._marshal.cell(_cell(), layer, _t(n - 1), A)
        with pytest.raises(ValueError, match="V_prefix.*on the GPU"):
            J._marshal.cell(_cell(), layer, A, _t(n))
    assert J._marshal.pools(_small(), A, None) == (A, 0) and J._marshal.cell(_cell(), 0, None, A) == (0, A)


def test_workspaces_are_checked():
    ws = torch.zeros(256, dtype=torch.uint8)
    for a, size, word in ((ws, 257, "257 bytes"), (ws[1:], 256, "256 bytes"), (ws[:1].expand(1 << 20), None, "bytes"), (ws, None, "on the GPU"),
                          (ws.float(), 1024, "on the GPU"), (A, None, "size"), (None, None, "must be a tensor"), (A, -1, "negative")):
        with pytest.raises(ValueError, match=word):
            J._marshal.bytes(a, size, "ws")
    assert J._marshal.bytes(A, 77, "ws") == (A, 77) and J._marshal.bytes(None, 77, "ws") == (0, 77)


def test_host_pools_prefix_and_workspace_never_reach_a_kernel():
    """The public calls look at the memory that they are given before anything else."""
    z = torch.zeros(4, dtype=torch.int32)
    rows = torch.zeros((4, 2, 32), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="V_pages must be a tensor on the GPU"):
        J.jolt_page_append(None, _small(), rows, rows, z, A, _t(768))
    ok = dict(prefix=_cell(), K_prefix=A, V_prefix=2 * A, pages=_small(), K_pages=3 * A, V_pages=4 * A, table=torch.zeros((3, 2), dtype=torch.int32),
              ws_bytes=256)
    for kw, ws, word in ((dict(K_prefix=_t(640)), A, "K_prefix must"), (dict(), _t(256, torch.uint8), "ws must")):
        with pytest.raises(ValueError, match=word):
            J.jolt_prefix_attend(None, rows, rows, z, z[:3], 0.1, ws, **{**ok, **kw})
    with pytest.raises(ValueError, match="table must be a tensor"):
        J._marshal.columns(None, 3, "table")
    for t in (z, ok["table"][:2]):
        with pytest.raises(ValueError, match="n_req, max_pages"):
            J._marshal.columns(t, 3, "table")
    assert J._marshal.columns(ok["table"], 3, "table") == 2


def _size(n_req, n_tok, max_new, T, max_pages, H, G, d, page, dtype):
    pre = None if T == 0 else J.cell_desc(dtype=dtype, n_layers=1, n_heads=H, T=T, d=d, stride_layer=H * T * d, stride_head=T * d, stride_token=d)
    pages = None if max_pages == 0 else J.page_desc(dtype=dtype, n_heads=H, page_size=page, d=d, n_pages=4, stride_page=H * page * d,
                                                    stride_head=page * d, stride_token=d)
    return J.jolt_prefix_attend_workspace_size(n_req, n_tok, H * G, prefix=pre, pages=pages, max_pages=max_pages, max_new=max_new)


def test_a_smaller_batch_needs_no_larger_workspace():
    """Along each size of a batch downwards, and from random batches to random smaller ones."""
    model = dict(H=8, G=4, d=128, page=16, dtype=J.JOLT_BF16)
    for base, axis, hi in ((dict(n_tok=256, max_new=1, T=4096, max_pages=40), "n_req", 256), (dict(n_req=64, max_new=0, T=4096, max_pages=40), "n_tok", 2100),
                           (dict(n_req=64, n_tok=700, T=300, max_pages=40), "max_new", 700), (dict(n_req=3, n_tok=70, max_new=0, max_pages=0), "T", 9000),
                           (dict(n_req=3, n_tok=9, max_new=1, max_pages=4), "T", 70000), (dict(n_req=9, n_tok=9, max_new=1, T=0), "max_pages", 50)):
        last = 0
        for x in range(1, hi + 1, 1 + hi // 2500):
            kw = {**base, **model, axis: x}
            if axis == "n_req":
                kw["n_tok"] = x
            n = _size(**kw)
            assert n >= last, (axis, x)
            last = n
    rng = random.Random(0)

    def log_int(hi):
        return min(hi, int(2 ** rng.uniform(0, hi.bit_length())))
    for _ in range(6000):
        model = dict(H=rng.choice([1, 2, 3, 8, 40, 600]), G=rng.choice([1, 3, 4, 8]), d=rng.choice([32, 64, 128]), page=rng.choice([4, 64]),
                     dtype=rng.choice([J.JOLT_BF16, J.JOLT_F32]))
        top = dict(n_req=log_int(4096), n_tok=log_int(5000), max_new=log_int(600), T=rng.choice([0, log_int(40000)]), max_pages=log_int(300))
        new = min(top["max_new"], top["n_tok"])
        low = {k: max(1, log_int(v)) if v else 0 for k, v in top.items()}
        low["max_new"] = log_int(new)
        if rng.random() < 0.2:              # not given: as many as there are rows
            top["max_new"] = low["max_new"] = 0
        if rng.random() < 0.1:
            low["max_pages"], low["T"] = rng.choice([(0, max(1, low["T"])), (low["max_pages"], 0)])
            if low["T"] and not top["T"]:
                continue
        assert _size(**low, **model) <= _size(**top, **model), (low, top, model)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_calls_run_the_kernels_that_they_are_meant_to_test(dtype):
    """Each call's form, and that the calls together reach every one of both types."""
    seen = set()
    for call, rows, how, many, join in CUTS:
        c, d = cut(dtype, call), call[5]
        assert not c["whole"] and c["prefix_rows"] == rows[dtype != "bf16"] and c["many_rows"] == many and c["join_lanes"] == join
        assert (c["share"] > c["token_tiles"]) == (how == "several") and c["prefix_runs"] > 1
        assert call[0] % (64 if dtype == "bf16" else 32)                     # the last tile of tokens is not full
        seen |= {("prefix", d, c["prefix_rows"]), ("join", d, join), ("long tails", many), ("ends in a row tile", c["token_tiles"] % c["share"] != 0), how}
    assert {("prefix", 64, 64), ("prefix", 64, 128), ("prefix", 128, 64), ("prefix", 128, 128), ("join", 32, 8), ("join", 64, 16), ("join", 128, 32),
            ("join", 128, 64), ("join", 64, 256), ("long tails", 64), ("long tails", 128), ("ends in a row tile", True), "several"} <= seen
    small = cut(dtype, (60, [3, 7], [1, 1], 4, 2, 64, 16))
    few = cut(dtype, (4001, [9] * 17, [1] * 17, 40, 1, 128, 16))
    assert small["whole"] and few["prefix_rows"] == 32 and not few["whole"]


def test_the_cut_refuses_what_the_call_refuses():
    with pytest.raises(J.JoltError, match="multiple"):
        J.jolt_debug_prefix_cut(4, 8, 12, pages=_pages(), max_pages=3)
    assert J.lib.jolt_debug_prefix_cut(None, None, None, None) == J.JOLT_E_INVAL


def test_without_the_native_checks_only_the_serving_calls_are_gone():
    code = """
import sys
sys.modules["paper_2607_12550_amd._marshal"] = None           # an import of it fails
import paper_2607_12550_amd as J
assert J.jolt_q_cap(4096, 4.0) > 0
import torch
z = torch.zeros(4, dtype=torch.int32)
pages = J.page_desc(dtype=J.JOLT_BF16, n_heads=1, page_size=8, d=32, n_pages=1, stride_page=256, stride_head=256, stride_token=32)
for call in (lambda: J.jolt_page_plan(None, pages, *[z] * 11), lambda: J.jolt_page_append(None, pages, z, z, z, z, z),
             lambda: J.jolt_prefix_attend(None, z, z, z, z, 0.1, z, pages=pages)):
    try:
        call()
    except ImportError as e:
        assert "_marshal.so" in str(e) and "build" in str(e), e
    else:
        raise SystemExit("no error")
"""
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=120,
                       cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert r.returncode == 0, r.stdout + r.stderr


def test_the_library_is_built_where_the_native_checks_are_not(monkeypatch, tmp_path):
    from paper_2607_12550_amd import build as B

    def no_compiler():
        raise RuntimeError("no g++")

    def link(cmd, **kw):
        open(cmd[cmd.index("-o") + 1], "w").close()
        return types.SimpleNamespace(returncode=0, stdout="", stderr="")
    monkeypatch.setattr(B, "_compile", lambda src, extra: src)
    monkeypatch.setattr(B, "_marshal", no_compiler)
    monkeypatch.setattr(B, "BUILD", str(tmp_path / "objects"))
    monkeypatch.setattr(B, "OUT", str(tmp_path / "lib.so"))
    monkeypatch.setattr(B, "subprocess", types.SimpleNamespace(run=link))
    with pytest.raises(RuntimeError, match="no g"):
        B.build()
    assert (tmp_path / "lib.so").exists()


def test_scales_whose_scores_in_units_of_log2_overflow_are_refused():
    for scale in (2.0 ** 127, 3e38):
        _refused(_attend(scale=scale), J.JOLT_E_INVAL, "scale")
    for scale in (1e38, 1e-45):
        _refused(_attend(scale=scale), J.JOLT_E_INVAL, "ctx is null")
