"""GPU tests of the shared-prefix serving operators at the edges of what they accept: values near
the largest of their type, and as many rows as an int counts.  Oracle and tolerances are those of
test_gpu_serve.py.
"""
import pytest
import torch

import paper_2607_12550_amd as J
from gpu_util import ctx, note
from test_gpu_serve import Batch, dev_i, pages_desc

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new,T", [([1, 1, 1], 50), ([1, 1, 1], 700), ([40, 2, 37], 700)])
def test_large_values_under_rising_scores(dtype, new, T):
    """Values up to 3e38 whose scores rise along the prefix: every output is a mean of them and
    finite, also where weights against an early maximum would sum past fp32."""
    for mag in (1e35, 1e37, 2e38):
        b = Batch(dtype, T, [60, 5, 17], new, 2, 4, 64, 16)

        def limit(x):
            return (x.double().clamp(-1.5, 1.5) * mag).to(x.dtype)
        for x in (b.V, b.Vp):
            x.copy_(limit(x))
        b.tv = [limit(v) for v in b.tv]
        u = torch.randn(64, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
        b.K[1] = u * torch.linspace(0.05, 2.5, T, device="cuda")[None, :, None] + 0.02 * b.K[1].float()
        b.Q.copy_(u + 0.1 * b.Q.float())
        b.check(b.run(max_new=max(new)), b.want())


def test_append_of_more_rows_than_a_launch_axis_takes():
    """2^24 and more rows of one head; rows at both ends and around the axis's length have slots."""
    n = (1 << 24) + 5
    at = torch.tensor([0, 1, (1 << 22) - 1, 1 << 22, (1 << 23) + 7, (1 << 24) - 1, 1 << 24, n - 1], device="cuda")
    desc = pages_desc("bf16", 1, 8, 32, 2)
    K = torch.zeros((n, 1, 32), dtype=torch.bfloat16, device="cuda")
    K[at] = torch.randn((8, 1, 32), device="cuda", generator=torch.Generator("cuda").manual_seed(0)).bfloat16()
    slots = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    slots[at] = dev_i(range(3, 11))
    Kp, Vp = (torch.full((2, 1, 8, 32), 3.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    note("jolt_page_append", n)
    J.jolt_page_append(ctx(), desc, K, K[:1].expand(n, 1, 32), slots, Kp, Vp)
    torch.cuda.synchronize()
    kp, vp = Kp.view(16, 32), Vp.view(16, 32)
    assert torch.equal(kp[3:11], K[at, 0]) and torch.equal(vp[3:11], K[:1, 0].expand(8, 32))
    for x in (kp, vp):
        assert (x[:3] == 3).all() and (x[11:] == 3).all()


def test_attention_of_more_rows_than_a_launch_axis_takes():
    """2^27 and more output rows of 128 features: with queries of zero over one token of prefix every
    row is that token's value, exactly.  The workspace is about 70 GB, the rows twice 34."""
    n_tok, n_q, d = (1 << 21) + 1, 64, 128
    prefix = J.cell_desc(dtype=J.JOLT_BF16, n_layers=1, n_heads=1, T=1, d=d, stride_layer=d, stride_head=d, stride_token=d)
    nb = J.jolt_prefix_attend_workspace_size(1, n_tok, n_q, prefix=prefix)
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < nb + 4 * n_tok * n_q * d + (8 << 30):
        pytest.skip("needs about 150 GB of free device memory")
    K, V = torch.randn((2, d), device="cuda", generator=torch.Generator("cuda").manual_seed(0)).bfloat16()
    Q = torch.zeros((n_tok, n_q, d), dtype=torch.bfloat16, device="cuda")
    O, ws = torch.full_like(Q, 9.0), torch.empty(nb, dtype=torch.uint8, device="cuda")
    note("jolt_prefix_attend", n_tok, n_q, d, nb)
    J.jolt_prefix_attend(ctx(), Q, O, dev_i([0, n_tok]), None, 0.1, ws, prefix=prefix, K_prefix=K, V_prefix=V)
    torch.cuda.synchronize()
    right = all(bool((O[t:t + (1 << 16)] == V).all()) for t in range(0, n_tok, 1 << 16))
    del Q, O, ws
    torch.cuda.empty_cache()
    assert right


def test_plan_of_as_many_rows_as_an_int_counts():
    """2^31 - 1 packed rows, three quarters of them of requests."""
    page, n_tok, cols = 1024, 2 ** 31 - 1, 1 << 19
    have, add = [0, 1023, 5], [1 << 29, (1 << 29) - 1023, (1 << 29) - 100]
    n_pages = 3 * cols
    free = torch.randperm(n_pages, device="cuda", generator=torch.Generator("cuda").manual_seed(0)).to(torch.int32)
    table = torch.full((3, cols), -1, dtype=torch.int32, device="cuda")
    table[1, 0], table[2, 0] = free[-1], free[-2]
    desc = pages_desc("bf16", 1, page, 32, n_pages)
    torch.cuda.empty_cache()
    slots, pos = (torch.full((n_tok,), 7, dtype=torch.int32, device="cuda") for _ in range(2))
    kv, qs, left, info = (torch.zeros(n, dtype=torch.int32, device="cuda") for n in (3, 4, 1, 4))
    note("jolt_page_plan", n_tok)
    J.jolt_page_plan(ctx(), desc, dev_i(have), dev_i(add), free, dev_i([n_pages - 2]), table, kv, qs, slots, pos, left, info)
    torch.cuda.synchronize()
    starts = [0, add[0], add[0] + add[1], sum(add)]
    assert qs.tolist() == starts and kv.tolist() == [h + n for h, n in zip(have, add)]
    # each takes the pages that it does not hold, in order, from the top down
    want = torch.cat([free[:-2].flip(0)[:cols], free[-1:], free[:-2].flip(0)[cols:2 * cols - 1], free[-2:-1], free[:-2].flip(0)[2 * cols - 1:]])
    assert torch.equal(table.view(-1), want) and info.tolist() == [sum(add), n_pages - 2, 0, n_pages - 2] and left.tolist() == [0]
    step = 1 << 27
    for r in range(3):
        for t in range(starts[r], starts[r + 1], step):
            p = torch.arange(t, min(t + step, starts[r + 1]), device="cuda") - starts[r] + have[r]
            assert torch.equal(pos[t:t + p.numel()], p.int())
            assert torch.equal(slots[t:t + p.numel()], (table[r, p // page] * page + p % page).int())
    for x in (slots, pos):
        assert all(bool((x[t:t + step] == -1).all()) for t in range(sum(add), n_tok, step))
    del slots, pos
    torch.cuda.empty_cache()
