"""Cases of the operators that serve a batch of requests from one shared prefix.

Three operators, each through the package's public entry points:

* ``plan``: block tables and slot maps of a step, built on the GPU from the requests' lengths
  (``jolt_page_plan``);
* ``append``: the step's new key and value rows written into their pages, keys with their rotary
  embedding (``jolt_page_append``);
* ``attend``: attention of the step's queries over the prefix that all requests share and over
  each request's own pages (``jolt_prefix_attend``).

The plain forms compute the same in elementary torch operations in 32 bits (angles in 64).
"""
import itertools
import math
import random

import torch

own = False


# ------------------------------------------------------------------------------- the cases
def _plan(name, n_req, have, new, page, spare=0):
    return dict(name=name, kind="plan", n_req=n_req, have=have, new=new, page=page, spare=spare)


def _append(name, n_tok, H, d, page, bf16, rope):
    return dict(name=name, kind="append", n_tok=n_tok, H=H, d=d, page=page, bf16=bf16, rope=rope)


def _attend(name, n_req, T, have, new, H, G, d, page, bf16=True):
    return dict(name=name, kind="attend", n_req=n_req, T=T, have=have, new=new, H=H, G=G, d=d, page=page, bf16=bf16)


def listed():
    return [
        # one decode step of 64 requests: the smallest call, launches and latency
        _plan("plan_decode_64", 64, 2048, 1, 16),
        # the first step of 500 requests that bring prompts of 1 to 2000 tokens, padded token room
        _plan("plan_prompts_500", 500, 300, 2000, 64, 777),
        # one layer's new rows of a decode step, grouped-query heads, keys with RoPE
        _append("append_decode_gqa", 64, 8, 128, 16, True, True),
        # one layer's new rows of a long prompt step, grouped-query heads, keys with RoPE
        _append("append_prompts_gqa", 32768, 8, 128, 64, True, True),
        # an fp32 cache of 40 heads of 64, a ragged number of rows, rotated before
        _append("append_fp32_mha", 4001, 40, 64, 32, False, False),
        # two requests early in their answers after a short prefix: the smallest attention call
        _attend("attend_small_T300", 2, 300, 40, 1, 4, 2, 64, 16),
        # a decode step of a grouped-query model, 64 requests on a 4096-token prefix
        _attend("attend_gqa_T4096", 64, 4096, 512, 1, 8, 4, 128, 16),
        # the same with many requests on a long prefix: the largest call
        _attend("attend_gqa_T32768", 256, 32768, 1024, 1, 8, 4, 128, 64),
        # a decode step with multi-head attention, a prefix that fills no tile
        _attend("attend_mha_T4001", 17, 4001, 300, 1, 40, 1, 128, 32),
        # prompts of 1 to 384 tokens after the shared prefix, some of them on longer tails
        _attend("attend_prompts_T4096", 16, 4096, 100, 384, 8, 4, 128, 64),
        # no shared prefix: each request's own pages alone, long tails
        _attend("attend_pages_only", 12, 0, 16384, 1, 8, 4, 128, 64),
        # an fp32 cache of a small model, up to five tokens a request (speculative decoding)
        _attend("attend_fp32_T1001", 32, 1001, 200, 5, 4, 2, 64, 16, False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["plan", "append", "attend", "attend", "attend", "attend"])
    page = rng.choice([8, 16, 16, 32, 64, 64, 128])
    if kind == "plan":
        n_req = _log_int(rng, 1, 1024)
        new = rng.choice([1, 1, rng.randint(2, 8), _log_int(rng, 16, 2000)])
        new = min(new, max(1, 131072 // n_req))
        c = _plan("", n_req, _log_int(rng, 1, 8192), new, page, rng.choice([0, 0, rng.randint(1, 999)]))
    elif kind == "append":
        H, d = rng.choice([1, 4, 8, 8, 16, 40]), rng.choice([32, 64, 128, 128])
        bf16 = rng.random() < 0.75
        c = _append("", _log_int(rng, 1, (1 << 25) // (H * d * (1 if bf16 else 2))), H, d, page, bf16, rng.random() < 0.7)
    else:
        bf16 = rng.random() < 0.75
        d = rng.choice([32, 64, 64, 128, 128, 128])
        H = rng.choice([1, 2, 4, 8, 8, 16, 40])
        G = rng.choice([g for g in (1, 2, 3, 4, 4, 5, 8, 8) if g * H <= 64])
        n_req = _log_int(rng, 1, 256)
        T = rng.choice([0] + [_log_int(rng, 60, 32768)] * 5)
        have = _log_int(rng, 1, 2048)
        new = rng.choice([1, 1, 1, rng.randint(2, 8), _log_int(rng, 16, 512)])
        new = min(new, max(1, 4096 // n_req))
        # no more pairs of queries and tokens than the largest listed case (fp32: a sixteenth of them)
        most = (1 << 35) // (1 if bf16 else 16)
        while n_req * new * H * G * (T + have + new) * d > most or n_req * (have + new) * H * d > (1 << 28):
            n_req, T, have = max(1, n_req // 2), T // 2, max(1, have // 2)
        c = _attend("", n_req, T, have, new, H, G, d, page, bf16)
    del c["name"]
    return c


# ------------------------------------------------------------------------------- inputs
def _spread(n, lo, hi):
    """n whole numbers spread over lo .. hi evenly in their logarithm: the same for every seed."""
    if lo == hi:
        return [lo] * n
    return [min(hi, max(lo, round(math.exp(math.log(lo) + (math.log(hi) - math.log(lo)) * (i + 0.5) / n)))) for i in range(n)]


def _lengths(c):
    """(tokens already in the cache, tokens added) of every request, in an order of the case's own."""
    have = [x - 1 for x in _spread(c["n_req"], 1, c["have"] + 1)]
    new = _spread(c["n_req"], 1, c["new"])
    random.Random(c["n_req"]).shuffle(have)
    return list(zip(have, new))


def _up(a, b):
    return -(-a // b)


def _gen(seed, key):
    return torch.Generator(device="cuda").manual_seed((int(seed) & 0x7FFFFFFF) * 1000003 + key)


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _keys(g, *shape):
    """Rows of keys: unit noise around a mean of their own per feature, four features far larger."""
    d = shape[-1]
    size = torch.ones(d, device="cuda")
    size[torch.randperm(d, generator=g, device="cuda")[:4]] = 3.0
    mean = 0.5 * torch.randn(d, generator=g, device="cuda")
    return (torch.randn(shape, generator=g, device="cuda") + mean) * size


def _paged(lens, page, gen, extra):
    """A table of the pages that hold `lens` tokens each, drawn from a pool in no order: (table, pages in the pool, the other pages)."""
    n = torch.tensor([_up(x, page) for x in lens], device="cuda")
    used = int(n.sum())
    ids = torch.randperm(used + extra, generator=gen, device="cuda").to(torch.int32)
    j = torch.arange(max(1, int(n.max())), device="cuda")
    at = (n.cumsum(0) - n)[:, None] + j
    table = torch.where(j < n[:, None], ids[at.clamp(max=ids.numel() - 1)], -1)
    return table, used + extra, ids[used:].contiguous()


def _prepare_plan(c, seed):
    g = _gen(seed, 1)
    lengths = _lengths(c)
    random.Random(seed).shuffle(lengths)
    page, n_tok = c["page"], sum(n for _, n in lengths) + c["spare"]
    taken = sum(_up(h + n, page) - _up(h, page) for h, n in lengths)
    table, pool, free = _paged([h for h, _ in lengths], page, g, taken + 64)
    width = max(_up(h + n, page) for h, n in lengths)
    wide = torch.full((c["n_req"], width), -1, dtype=torch.int32, device="cuda")
    wide[:, :min(width, table.shape[1])] = table[:, :width]
    return dict(have=_ints([h for h, _ in lengths]), add=_ints([n for _, n in lengths]), free=free, n_free=_ints([free.numel()]), table=wide,
                pool=pool, kv_len=_ints([0] * c["n_req"]), q_start=_ints([0] * (c["n_req"] + 1)), n_free_out=_ints([0]),
                info=_ints([0] * 4), slots=_ints([0] * n_tok), positions=_ints([0] * n_tok))


def _prepare_append(c, seed):
    g = _gen(seed, 2)
    n, H, d, page = c["n_tok"], c["H"], c["d"], c["page"]
    dt = torch.bfloat16 if c["bf16"] else torch.float32
    pool = _up(n, page) + 4
    # requests of about 100 rows each, placed in pages in no order
    order = torch.randperm(pool, generator=g, device="cuda")
    t = torch.arange(n, device="cuda")
    slots = (order[t // page] * page + t % page).to(torch.int32)
    return dict(K=_keys(g, n, H, d).to(dt), V=torch.randn((n, H, d), generator=g, device="cuda").to(dt), slots=slots,
                positions=(t % 100 + 7 * (t // 100)).to(torch.int32), pool=pool, offset=4096, base=1e4,
                K_pages=torch.zeros((pool, H, page, d), dtype=dt, device="cuda"),
                V_pages=torch.zeros((pool, H, page, d), dtype=dt, device="cuda"))


def _prepare_attend(c, seed):
    g = _gen(seed, 3)
    T, H, G, d, page = c["T"], c["H"], c["G"], c["d"], c["page"]
    dt = torch.bfloat16 if c["bf16"] else torch.float32
    lengths = _lengths(c)
    random.Random(seed).shuffle(lengths)
    lens = [h + n for h, n in lengths]
    table, pool, _ = _paged(lens, page, g, 3)
    q_start = [0] + list(itertools.accumulate(n for _, n in lengths))
    n_tok = q_start[-1]
    return dict(Q=torch.randn((n_tok, H * G, d), generator=g, device="cuda").to(dt),
                K=_keys(g, H, T, d).to(dt), V=torch.randn((H, T, d), generator=g, device="cuda").to(dt),
                K_pages=_keys(g, pool, H, page, d).to(dt), V_pages=torch.randn((pool, H, page, d), generator=g, device="cuda").to(dt),
                table=table, q_start=_ints(q_start), kv_len=_ints(lens), pool=pool, scale=1.0 / math.sqrt(d),
                O=torch.zeros((n_tok, H * G, d), dtype=dt, device="cuda"),
                lse=torch.zeros((n_tok, H * G), dtype=torch.float32, device="cuda"))


def _page_desc(J, c, pool, H, d):
    P = c["page"]
    return J.page_desc(dtype=J.JOLT_BF16 if c.get("bf16", True) else J.JOLT_F32, n_heads=H, page_size=P, d=d, n_pages=pool,
                       stride_page=H * P * d, stride_head=P * d, stride_token=d)


def prepare(case, seed):
    s = {"plan": _prepare_plan, "append": _prepare_append, "attend": _prepare_attend}[case["kind"]](case, seed)
    s["case"] = case
    if own:
        # what a serving program sets up once: the context, the descriptors, the workspace
        import paper_2607_12550_amd as J
        s["J"], s["ctx"] = J, J.jolt_create(0)
        H, d = case.get("H", 1), case.get("d", 128)
        s["pages"] = _page_desc(J, case, s["pool"], H, d)
        if case["kind"] == "attend":
            T = case["T"]
            s["prefix"] = None if T == 0 else J.cell_desc(dtype=s["pages"].dtype, n_layers=1, n_heads=H, T=T, d=d, stride_layer=H * T * d,
                                                          stride_head=T * d, stride_token=d)
            nb = J.jolt_prefix_attend_workspace_size(case["n_req"], s["Q"].shape[0], s["Q"].shape[1], prefix=s["prefix"], pages=s["pages"],
                                                     max_pages=s["table"].shape[1], max_new=case["new"])
            s["ws"] = torch.empty(nb, dtype=torch.uint8, device="cuda")
    return s


# ------------------------------------------------------------------------------- plain forms
def _plain_plan(s, page):
    have, add, table, free = s["have"].long(), s["add"].long(), s["table"], s["free"]
    total = have + add
    old = (have + page - 1) // page
    taken = (total + page - 1) // page - old
    q_start = torch.cat([torch.zeros_like(add[:1]), add.cumsum(0)])
    before = taken.cumsum(0) - taken
    t = torch.arange(s["slots"].numel(), device=have.device)
    in_use = t < q_start[-1]
    r = torch.bucketize(t, q_start[1:], right=True).clamp(max=have.numel() - 1)
    pos = have[r] + t - q_start[r]
    j = torch.where(in_use, pos // page, 0)
    fresh = j >= old[r]
    top = s["n_free"].long() - 1
    at = (top - before[r] - (j - old[r])).clamp(0, free.numel() - 1)
    ids = torch.where(fresh, free[at], table[r, j]).long()
    slots = torch.where(in_use, ids * page + pos % page, -1)
    # every page that a token lies in is entered; the padded tokens repeat the last one's entry
    last = (q_start[-1] - 1).clamp(min=0)
    k = torch.minimum(t, last)
    table[r[k], j[k]] = ids[k].to(torch.int32)
    new_pages = taken.sum().reshape(1)
    info = torch.cat([q_start[-1:], new_pages, torch.zeros_like(new_pages), new_pages])
    i32 = torch.int32
    return dict(table=table, kv_len=total.to(i32), q_start=q_start.to(i32), slots=slots.to(i32),
                positions=torch.where(in_use, pos, -1).to(i32), n_free=(s["n_free"] - new_pages).to(i32), info=info.to(i32))


def _plain_append(s, page, d, rope):
    K = s["K"].float()
    if rope:
        half = d // 2
        j = torch.arange(half, device=K.device, dtype=torch.float64)
        angle = (s["positions"].double() + s["offset"])[:, None] * s["base"] ** (-2.0 * j / d)
        cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
        a, b = K[..., :half], K[..., half:]
        K = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    at = s["slots"].long()
    s["K_pages"][at // page, :, at % page] = K.to(s["K_pages"].dtype)
    s["V_pages"][at // page, :, at % page] = s["V"]
    return dict(K_pages=s["K_pages"], V_pages=s["V_pages"])


def _plain_attend(s, c):
    H, G, d, T, page = c["H"], c["G"], c["d"], c["T"], c["page"]
    Q, table, lens = s["Q"], s["table"], s["kv_len"].long()
    n_tok, n_req, new = Q.shape[0], c["n_req"], c["new"]
    Qh = Q.float().view(n_tok, H, G, d).permute(1, 0, 2, 3)                        # [H][tok][G][d]
    # tails: every request's pages and its queries, padded to the longest
    t = torch.arange(n_tok, device=Q.device)
    start = s["q_start"].long()
    r = torch.bucketize(t, start[1:], right=True)
    i = t - start[r]
    N = table.shape[1] * page
    ids = table.clamp(min=0).long()

    def tails(pages):
        return pages[ids].float().permute(2, 0, 1, 3, 4).reshape(H, n_req, N, d)
    Qt = torch.zeros((H, n_req, new, G, d), device=Q.device)
    Qt[:, r, i] = Qh
    st = Qt.view(H, n_req, new * G, d) @ tails(s["K_pages"]).transpose(-1, -2).contiguous() * s["scale"]
    x = torch.arange(N, device=Q.device)
    count = start[1:] - start[:-1]
    seen = x < (lens - count)[:, None, None] + torch.arange(new, device=Q.device)[:, None] + 1      # [req][new][N]
    st = st.view(H, n_req, new, G, N).masked_fill(~seen[:, :, None], -math.inf)
    m = st.amax(-1)[:, r, i]                                                        # [H][tok][G]
    if T:
        sp = (Qh.reshape(H, n_tok * G, d) @ s["K"].float().transpose(-1, -2).contiguous() * s["scale"]).view(H, n_tok, G, T)
        m = torch.maximum(m, sp.amax(-1))
    top = torch.zeros((H, n_req, new, G), device=Q.device)
    top[:, r, i] = m
    pt = (st - top[..., None]).exp()
    acc = (pt.view(H, n_req, new * G, N) @ tails(s["V_pages"])).view(H, n_req, new, G, d)[:, r, i]
    total = pt.sum(-1)[:, r, i]
    if T:
        pp = (sp - m[..., None]).exp()
        acc = acc + (pp.view(H, n_tok * G, T) @ s["V"].float()).view(H, n_tok, G, d)
        total = total + pp.sum(-1)
    O = (acc / total[..., None]).permute(1, 0, 2, 3).reshape(n_tok, H * G, d)
    lse = (m + total.log()).permute(1, 0, 2).reshape(n_tok, H * G)
    return dict(O=O.to(Q.dtype), lse=lse)


def run(state):
    s, c = state, state["case"]
    if own:
        J = s["J"]
        if c["kind"] == "plan":
            J.jolt_page_plan(s["ctx"], s["pages"], s["have"], s["add"], s["free"], s["n_free"], s["table"], s["kv_len"], s["q_start"],
                             s["slots"], s["positions"], s["n_free_out"], s["info"])
            return dict(table=s["table"], kv_len=s["kv_len"], q_start=s["q_start"], slots=s["slots"], positions=s["positions"],
                        n_free=s["n_free_out"], info=s["info"])
        if c["kind"] == "append":
            J.jolt_page_append(s["ctx"], s["pages"], s["K"], s["V"], s["slots"], s["K_pages"], s["V_pages"],
                               positions=s["positions"], rope=(s["base"], s["offset"]) if c["rope"] else None)
            return dict(K_pages=s["K_pages"], V_pages=s["V_pages"])
        J.jolt_prefix_attend(s["ctx"], s["Q"], s["O"], s["q_start"], s["kv_len"], s["scale"], s["ws"], prefix=s["prefix"], K_prefix=s["K"],
                             V_prefix=s["V"], pages=s["pages"], K_pages=s["K_pages"], V_pages=s["V_pages"], table=s["table"],
                             max_new=c["new"], lse=s["lse"])
        return dict(O=s["O"], lse=s["lse"])
    if c["kind"] == "plan":
        return _plain_plan(s, c["page"])
    if c["kind"] == "append":
        return _plain_append(s, c["page"], c["d"], c["rope"])
    return _plain_attend(s, c)


def work(case):
    c = case
    if c["kind"] == "plan":
        lengths, page = _lengths(c), c["page"]
        n_tok, new_pages = sum(n for _, n in lengths), sum(_up(h + n, page) - _up(h, page) for h, n in lengths)
        # lengths in and out, the free pages taken and entered, a table entry read per open page, slots and positions
        return dict(bytes=4 * (5 * c["n_req"] + 2 * new_pages + 2 * (n_tok + c["spare"])), flops=0)
    esz = 2 if c["bf16"] else 4
    if c["kind"] == "append":
        rows = c["n_tok"] * c["H"] * c["d"]
        return dict(bytes=4 * rows * esz + 8 * c["n_tok"], flops=3 * rows if c["rope"] else 0)
    lengths = _lengths(c)
    n_tok = sum(n for _, n in lengths)
    kept = c["T"] + sum(h + n for h, n in lengths)
    pairs = sum(n * (c["T"] + h) + n * (n + 1) // 2 for h, n in lengths)
    n_q = c["H"] * c["G"]
    return dict(bytes=2 * kept * c["H"] * c["d"] * esz + n_tok * n_q * (2 * c["d"] * esz + 4), flops=4 * pairs * n_q * c["d"])


# ------------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    """The attention and the appended rows from their definitions in float64, the plan token by token: one request after the other."""
    c = case
    if c["kind"] == "plan":
        s, P = _prepare_plan(c, seed), c["page"]
        have, add, free, table = s["have"].tolist(), s["add"].tolist(), s["free"].tolist(), s["table"].tolist()
        slots, positions, q_start, given = [], [], [0], len(free)
        for r, (h, n) in enumerate(zip(have, add)):
            for pos in range(h, h + n):
                if pos % P == 0:
                    table[r][pos // P] = free.pop()
                slots.append(table[r][pos // P] * P + pos % P)
                positions.append(pos)
            q_start.append(len(slots))
        rest, n = [-1] * c["spare"], given - len(free)
        return dict(table=_ints(table), kv_len=_ints([h + x for h, x in zip(have, add)]), q_start=_ints(q_start), slots=_ints(slots + rest),
                    positions=_ints(positions + rest), n_free=_ints([len(free)]), info=_ints([len(slots), n, 0, n]))
    if c["kind"] == "append":
        s = _prepare_append(c, seed)
        d, P = c["d"], c["page"]
        Kd, Vd = s["K"].double(), s["V"].double()
        if c["rope"]:
            # the pair (j, j + d/2) as a complex number, turned by exp(i angle)
            z = torch.complex(Kd[..., :d // 2], Kd[..., d // 2:])
            freq = torch.exp(-math.log(s["base"]) * torch.arange(0, d, 2, device="cuda", dtype=torch.float64) / d)
            turn = (s["positions"].double() + s["offset"])[:, None, None] * freq
            z = z * torch.polar(torch.ones_like(turn), turn)
            Kd = torch.cat([z.real, z.imag], -1)
        out = {}
        for name, rows in (("K_pages", Kd), ("V_pages", Vd)):
            flat = torch.zeros((s["pool"] * P, c["H"], d), dtype=torch.float64, device="cuda")
            flat[s["slots"].long()] = rows
            out[name] = flat.view(s["pool"], P, c["H"], d).transpose(1, 2).contiguous()
        return out
    s = _prepare_attend(c, seed)
    H, G, d, P = c["H"], c["G"], c["d"], c["page"]
    starts, lens = s["q_start"].tolist(), s["kv_len"].tolist()
    Kp, Vp = s["K"].double(), s["V"].double()
    Os, Ls = [], []
    for r, L in enumerate(lens):
        q0, q1 = starts[r], starts[r + 1]
        ids = s["table"][r, :_up(L, P)].long()
        own_k, own_v = (x[ids].double().transpose(1, 2).reshape(-1, H, d)[:L].transpose(0, 1) for x in (s["K_pages"], s["V_pages"]))
        K, V = torch.cat([Kp, own_k], 1), torch.cat([Vp, own_v], 1)
        # rows ordered (head, group, token): the query heads of one key-value head together
        q = s["Q"][q0:q1].double().view(q1 - q0, H, G, d).permute(1, 2, 0, 3)
        a = (q.reshape(H, -1, d) @ K.transpose(1, 2).contiguous()).view(H, G, q1 - q0, -1) * s["scale"]
        last = c["T"] + L - (q1 - q0) + torch.arange(q1 - q0, device="cuda")
        a[:, :, torch.arange(K.shape[1], device="cuda")[None] > last[:, None]] = -math.inf
        lse = torch.logsumexp(a, -1)
        w = torch.exp(a - lse[..., None])
        o = (w.view(H, -1, K.shape[1]) @ V.contiguous()).view(H, G, q1 - q0, d)
        Os.append(o.permute(2, 0, 1, 3).reshape(q1 - q0, H * G, d))
        Ls.append(lse.permute(2, 0, 1).reshape(q1 - q0, H * G))
    return dict(O=torch.cat(Os), lse=torch.cat(Ls))
