"""The work of several requests behind one shared prefix, as cases to be timed and compared.

A program that serves many requests at once keeps one KV cache for the prefix they share (a system
prompt, a document) and a pool of 64-slot pages for what each request holds behind it.  A step of
it is: the plan (pages, slots, positions, ancestor masks of the step's rows, from the requests'
lengths), then per layer the rotary embedding with the write of the new keys and values, and the
attention of every row to the prefix, its request's pages and its own branch; after the last layer
the scores of the rows' logits (log probabilities of given tokens, entropy, top alternatives); and
after verification the accepted rows' move to the front.

Heads, widths and tree sizes are those of the repository's models and workloads (16, 32 and 40 heads
of 128, the tiny model's heads of 64; trees of 31, 41 and 128 nodes; prefixes of 512 to 2048), and
generic ones beside them: K/V heads shared by 4 or 8 query heads, one token per request, prefixes
up to 8192, vocabularies of 32000 and 128000.

`run` computes an operator in plain torch operations, or where `own` is true through the library.
"""

import math
import random

import torch

own = False

PAGE = 64
NODES = 128  # rows of a request in one step, at most
THETA = 10000.0
NINF = float("-inf")


def _case(op, name=None, **kw):
    c = {"op": op, **kw}
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # one request's tree of the benchmark's size: the smallest plan, where the launch is all there is
        _case("plan", "plan_b1_n31", requests=1, rows=31, ragged=False, held=200, prefix=512, head_dim=128, tree=True, pad=0),
        # a full server's step: 256 requests with trees of up to 41 nodes and long answers, and padding rows
        _case("plan", "plan_b256_n41", requests=256, rows=41, ragged=True, held=2048, prefix=2048, head_dim=128, tree=True, pad=100),
        # eight requests decoding one token each, a 7B model's layer
        _case("store", "store_b8_n1", requests=8, rows=1, ragged=False, held=300, prefix=512, heads=32, kv_heads=32, head_dim=128, pad=0),
        # 64 requests' trees of the benchmark's size
        _case("store", "store_b64_n31", requests=64, rows=31, ragged=True, held=500, prefix=1024, heads=32, kv_heads=32, head_dim=128, pad=7),
        # one request, one token, a short prefix: latency
        _case("attention", "attention_b1_n1_p512", requests=1, rows=1, ragged=False, held=64, prefix=512, heads=32, kv_heads=32, head_dim=128, tree=False, pad=0),
        # 16 requests' trees behind the long prefix of the repository's workloads
        _case("attention", "attention_b16_n31_p2048", requests=16, rows=31, ragged=False, held=200, prefix=2048, heads=32, kv_heads=32, head_dim=128, tree=True, pad=0),
        # 128 requests decoding one token each behind a document, shared K/V heads, ragged answers
        _case("attention", "attention_b128_n1_p8192", requests=128, rows=1, ragged=True, held=1024, prefix=8192, heads=32, kv_heads=8, head_dim=128, tree=False, pad=5),
        # 32 requests' 41-node trees, a 13B model's heads, an odd prefix: the most arithmetic
        _case("attention", "attention_b32_n41_p4099", requests=32, rows=41, ragged=False, held=500, prefix=4099, heads=40, kv_heads=40, head_dim=128, tree=True, pad=0),
        # four requests' accepted branches in the ~1B draft model's pages
        _case("commit", "commit_1b_b4", requests=4, rows=31, ragged=False, held=150, layers=22, kv_heads=16, head_dim=128),
        # 32 requests' accepted branches in a 7B model's pages
        _case("commit", "commit_7b_b32", requests=32, rows=41, ragged=True, held=60, layers=32, kv_heads=32, head_dim=128),
        # the target's scores of the benchmark's tree: every draft token under its parent's distribution
        _case("scores", "scores_n31_v32000", rows=31, vocab=32000, dtype="fp32", k=8, tree=True),
        # a batch of prompts scored at once, a large vocabulary, logits of a bf16 head
        _case("scores", "scores_n1024_v128000", rows=1024, vocab=128000, dtype="bf16", k=20, tree=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _drawn(rng):
    op = rng.choice(["plan", "store", "attention", "attention", "commit", "scores", "scores"])
    heads, kv_heads, head_dim = rng.choice([(4, 4, 64), (4, 2, 64), (16, 16, 128), (32, 32, 128), (32, 8, 128), (40, 40, 128), (64, 8, 128), (24, 8, 64)])
    rows = rng.choice([1, 1, _log(rng, 2, 16), _log(rng, 16, NODES)])
    base = dict(requests=_log(rng, 1, 200), rows=rows, ragged=rng.random() < 0.7, held=rng.choice([0, _log(rng, 1, 4000)]))
    tree, pad = rng.random() < 0.6, rng.choice([0, rng.randrange(1, 70)])
    prefix = rng.choice([0, _log(rng, 1, 300), _log(rng, 300, 8192)])
    if op == "plan":
        return _case(op, **base, prefix=prefix, head_dim=head_dim, tree=tree, pad=pad)
    if op == "store":
        return _case(op, **base, prefix=prefix, heads=heads, kv_heads=kv_heads, head_dim=head_dim, pad=pad)
    if op == "attention":
        return _case(op, **base, prefix=prefix, heads=heads, kv_heads=kv_heads, head_dim=head_dim, tree=tree, pad=pad)
    if op == "commit":
        return _case(op, **base, layers=rng.choice([2, 22, 32, 40]), kv_heads=kv_heads, head_dim=head_dim)
    return _case(op, rows=_log(rng, 1, 2000), vocab=rng.choice([rng.randrange(30, 2000), 32000, rng.randrange(30000, 260000)]),
                 dtype=rng.choice(["fp32", "bf16"]), k=rng.choice([0, 1, rng.randrange(2, 65)]), tree=rng.random() < 0.5)


def draw(rng):
    # at most what the largest listed cases cost, and no more than a state's room
    while True:
        c = _drawn(rng)
        w = work(c)
        room = 0
        if "requests" in c:
            n, held = _lengths(c)
            pages = sum(-(-(h + m) // PAGE) + 1 for h, m in zip(held, n))
            room = pages * PAGE * c.get("kv_heads", 1) * c["head_dim"] * 4 * c.get("layers", 1)
        if w["bytes"] < 5e8 and w["flops"] < 1.1e11 and room < 6e9:
            return c


def _lengths(c):
    """(rows, held tokens) of every request: functions of the case alone."""
    r = random.Random("%d %d %d" % (c["requests"], c["rows"], c["held"]))
    if not c["ragged"]:
        return [c["rows"]] * c["requests"], [c["held"]] * c["requests"]
    n = [r.randint(1, c["rows"]) for _ in range(c["requests"])]
    held = [r.randint(0, c["held"]) for _ in range(c["requests"])]
    if len(n) > 4:
        n[2] = 0  # a request that sits this step out
    return n, held


def work(c):
    if c["op"] == "scores":
        size = 4 if c["dtype"] == "fp32" else 2
        return {"bytes": c["rows"] * (c["vocab"] * size + 8 * c["k"] + 20), "flops": 0}
    n, held = _lengths(c)
    N, Dh = sum(n), c["head_dim"]
    if c["op"] == "plan":
        pages = sum(-(-(h + m) // PAGE) for h, m in zip(held, n))
        return {"bytes": 16 * c["requests"] + 8 * pages + (N + c["pad"]) * (4 + 4 + 4 + 16 + 4 * Dh), "flops": 0}
    if c["op"] == "store":
        return {"bytes": N * ((c["heads"] + 2 * c["kv_heads"]) * Dh * 4 + 4 * Dh + 4), "flops": 6 * N * (c["heads"] + c["kv_heads"]) * Dh // 2}
    if c["op"] == "commit":
        moved = sum(min(3, m - 1) for m in n if m > 0)  # (about three accepted rows a request)
        return {"bytes": moved * c["layers"] * c["kv_heads"] * Dh * 8 + 8 * N, "flops": 0}
    keys = c["prefix"] + sum(h + m for h, m in zip(held, n) if m > 0)
    pairs = sum(m * (c["prefix"] + h + (m + 1) // 2) for h, m in zip(held, n))
    return {"bytes": keys * c["kv_heads"] * Dh * 4 + N * (c["heads"] * Dh * 4 + 16), "flops": 4 * Dh * c["heads"] * pairs}


# ------------------------------------------------------------------ inputs


def _tree(r, n):
    """Parents of a request's n rows: a random tree with branches of up to eight tokens."""
    parent, depth = [-1], [0]
    for i in range(1, n):
        p = r.randrange(i)
        while depth[p] > 7:
            p = r.randrange(i)
        parent.append(p)
        depth.append(depth[p] + 1)
    return parent[:n]


def _requests(c, seed):
    """What the step's host has: row_start, held, parents, the pages each request holds already, the free ones."""
    r = random.Random(seed)
    n, held = _lengths(c)
    B = c["requests"]
    start = [0]
    for m in n:
        start.append(start[-1] + m)
    parent = [p for m in n for p in (_tree(r, m) if c.get("tree") else list(range(-1, m - 1)))]
    pad = c.get("pad", 0)
    have = [-(-h // PAGE) for h in held]
    want = [-(-(h + m) // PAGE) for h, m in zip(held, n)]
    n_pages = sum(want) + 8
    width = max(want) + 1
    order = list(range(n_pages))
    r.shuffle(order)
    table = [[-1] * width for _ in range(B)]
    at = 0
    for b in range(B):
        table[b][:have[b]] = order[at:at + have[b]]
        at += have[b]
    dev = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    return {"n": n, "total": start[-1], "N": start[-1] + pad, "requests": B, "n_pages": n_pages, "width": width,
            "row_start": dev(start), "held": dev(held), "parent": dev(parent + [0] * pad) if parent or pad else dev([0]),
            "block_table": dev(table), "free_pages": dev(order[at:]), "prefix": c.get("prefix", 0), "head_dim": c["head_dim"],
            "longest": max(h + m for h, m in zip(held, n)), "most": max(max(n), 1)}


def _config(c):
    from paper_2309_04255_amd import binding

    H, Dh = c.get("heads", c.get("kv_heads", 4)), c["head_dim"]
    return binding.LlmcadConfig(c.get("layers", 1), H * Dh, H, Dh, 4 * H * Dh, 32000, 1e-6, THETA, 16)


def prepare(c, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(*shape, scale=1.0, dtype=torch.bfloat16):
        return torch.randn(shape, generator=g, device="cuda", dtype=dtype) * scale

    if c["op"] == "scores":
        n, V = c["rows"], c["vocab"]
        x = normal(n, V, scale=2.5, dtype=torch.float32)
        peak = torch.randint(0, V, (n, 1), generator=g, device="cuda")
        x.scatter_add_(1, peak, torch.full((n, 1), 9.0, device="cuda"))  # (a clear favourite)
        tokens = torch.randint(0, V, (n,), generator=g, device="cuda")
        tokens = torch.where(torch.rand(n, generator=g, device="cuda") < 0.5, peak[:, 0], tokens).to(torch.int32)
        s = {"op": "scores", "k": min(c["k"], V), "logits": x if c["dtype"] == "fp32" else x.to(torch.bfloat16), "tokens": tokens, "row_of": None}
        if c["tree"]:  # the draft tokens of a tree, each under its parent's row
            s["row_of"] = torch.tensor([max(p, 0) for p in _tree(random.Random(seed), n)], dtype=torch.int32, device="cuda")
        if own:
            from paper_2309_04255_amd import binding

            s["workspace"] = torch.zeros(binding.token_scores_workspace_bytes(n, V, s["k"]), dtype=torch.uint8, device="cuda")
        return s
    s = {"op": c["op"], **_requests(c, seed)}
    N, Dh = s["N"], c["head_dim"]
    if own:
        from paper_2309_04255_amd import binding

        s["cfg"] = _config(c)
        s["plan"] = torch.empty(binding.batch_plan_bytes(s["cfg"], s["requests"], N), dtype=torch.uint8, device="cuda")
    if c["op"] == "plan":
        return s
    maps = _plain_plan(s)  # (the program's plan of this step)
    s.update(slot=maps["slot"], mask=maps["mask"], rope=maps["rope"])
    Hkv, L = c["kv_heads"], c.get("layers", 1)
    s["kv_heads"] = Hkv
    s["k_pages"] = normal(L, s["n_pages"], Hkv, PAGE, Dh)
    s["v_pages"] = normal(L, s["n_pages"], Hkv, Dh, PAGE)
    if own:
        binding.batch_plan(s["cfg"], s["row_start"], s["held"], s["parent"], s["prefix"], s["block_table"], s["free_pages"], s["n_pages"], s["plan"], N)
    if c["op"] == "commit":
        r = random.Random(seed + 1)
        host, at, path, acc = s["parent"].tolist(), 0, [], []
        for m in s["n"]:
            branch = []
            i = r.randrange(m) if m else -1
            while i >= 0:  # (a node's branch, root first)
                branch.append(i)
                i = host[at + i]
            path += branch[::-1] + [-1] * (m - len(branch))
            acc.append(max(len(branch) - 1, 0))
            at += m
        s["path"] = torch.tensor(path or [0], dtype=torch.int32, device="cuda")
        s["accept_len"] = torch.tensor(acc, dtype=torch.int32, device="cuda")
        return s
    H = c["heads"]
    s["heads"] = H
    if c["op"] == "store":
        # (the fused projection's output: a row's queries, keys and values side by side)
        s["qkv"] = normal(N, (H + 2 * Hkv) * Dh)
        s["q_out"] = torch.zeros(N, H, Dh, dtype=torch.bfloat16, device="cuda")
        return s
    cap = max(-(-c["prefix"] // PAGE), 1) * PAGE
    s["k_cache"] = normal(1, Hkv, cap, Dh)
    s["v_cache"] = normal(1, Hkv, Dh, cap)
    s["q"] = normal(N, H, Dh, scale=1.5)
    s["out"] = torch.zeros(N, H, Dh, dtype=torch.bfloat16, device="cuda")
    if own:
        s["workspace"] = torch.zeros(binding.batch_workspace_bytes(s["cfg"], Hkv, s["requests"], N), dtype=torch.uint8, device="cuda")
    return s


# ------------------------------------------------------------------ plain forms


def _rows(s):
    """(request, its row) of every row; padding rows get the last request and a row past its own."""
    at = torch.arange(s["N"], device="cuda")
    req = torch.searchsorted(s["row_start"][1:].long().contiguous(), at, right=True).clamp(max=s["requests"] - 1)
    return req, at - s["row_start"].long()[req], at < s["total"]


def _plain_plan(s):
    B, N, width = s["requests"], s["N"], s["width"]
    start, held = s["row_start"].long(), s["held"].long()
    n = start[1:] - start[:-1]
    first, last = (held + PAGE - 1) // PAGE, (held + n + PAGE - 1) // PAGE
    need = last - first
    off = torch.cumsum(need, 0) - need
    col = torch.arange(width, device="cuda")
    new = (col >= first[:, None]) & (col < last[:, None])
    take = (off[:, None] + col - first[:, None]).clamp(0, s["free_pages"].numel() - 1)
    s["block_table"].copy_(torch.where(new, s["free_pages"][take], s["block_table"]))
    req, local, real = _rows(s)
    at = (held[req] + local).clamp(max=width * PAGE - 1)
    slot = torch.where(real, s["block_table"].long()[req, at // PAGE] * PAGE + at % PAGE, -1)
    # who descends from whom: (identity + parent links) to the 127th power
    link = torch.zeros(B, NODES, NODES + 1, device="cuda")
    par = s["parent"][:N].long()
    lane = local.clamp(max=NODES - 1)
    link[req, lane, torch.where(real & (par >= 0), par, NODES)] = 1.0
    reach = torch.linalg.matrix_power(link[:, :, :NODES] + torch.eye(NODES, device="cuda"), NODES - 1) > 0
    sees = reach[req, lane] & real[:, None]
    words = (sees.view(N, 4, 32).long() << torch.arange(32, device="cuda")).sum(-1)
    mask = torch.where(words >= 2**31, words - 2**32, words).to(torch.int32)
    pos = torch.where(real, s["prefix"] + held[req] + sees.sum(-1) - 1, 0)
    half = s["head_dim"] // 2
    freq = THETA ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
    ang = pos.double()[:, None] * freq
    rope = torch.stack([torch.cos(ang), torch.sin(ang)], -1).float()
    return {"block_table": s["block_table"], "slot": slot.to(torch.int32), "position": pos.to(torch.int32), "mask": mask, "rope": rope,
            "status": torch.zeros(B, dtype=torch.int32, device="cuda"), "taken": need.sum().to(torch.int32).reshape(1)}


def _plain_store(s):
    T, H, Hkv, Dh = s["total"], s["heads"], s["kv_heads"], s["head_dim"]
    x = s["qkv"][:T].view(T, H + 2 * Hkv, Dh).float()
    cos, sin = s["rope"][:T, None, :, 0], s["rope"][:T, None, :, 1]
    a, b = x[:, :H + Hkv, :Dh // 2], x[:, :H + Hkv, Dh // 2:]
    y = torch.cat([a * cos - b * sin, b * cos + a * sin], -1).to(torch.bfloat16)
    s["q_out"][:T] = y[:, :H]
    slot = s["slot"][:T].long()
    s["k_pages"][0][slot // PAGE, :, slot % PAGE] = y[:, H:]
    s["v_pages"][0][slot // PAGE, :, :, slot % PAGE] = s["qkv"][:T].view(T, H + 2 * Hkv, Dh)[:, H + Hkv:]
    return {"q": s["q_out"], "k_pages": s["k_pages"], "v_pages": s["v_pages"]}


def _plain_attention(s):
    N, B, H, Hkv, Dh, P, most = s["N"], s["requests"], s["heads"], s["kv_heads"], s["head_dim"], s["prefix"], s["most"]
    g = H // Hkv
    q = s["q"].float() / math.sqrt(Dh)
    # the prefix, for all rows at once: running maximum, sum and weighted values
    flat = q.view(N, Hkv, g, Dh).transpose(0, 1).reshape(Hkv, N * g, Dh)
    if P:
        score = flat @ s["k_cache"][0, :, :P].float().transpose(1, 2).contiguous()
        m1 = score.amax(-1, keepdim=True)
        e = torch.exp(score - m1)
        l1, o1 = e.sum(-1, keepdim=True), e @ s["v_cache"][0, :, :, :P].float().transpose(1, 2).contiguous()
    else:
        m1 = torch.full((Hkv, N * g, 1), NINF, device="cuda")
        l1, o1 = torch.zeros_like(m1), torch.zeros_like(flat)
    # each request's own keys, in rows of the longest request's length
    pages = -(-s["longest"] // PAGE)
    table = s["block_table"][:, :pages].long().clamp(min=0)
    k = s["k_pages"][0][table].permute(0, 2, 1, 3, 4).reshape(B, Hkv, pages * PAGE, Dh).float()
    v = s["v_pages"][0][table].permute(0, 2, 1, 4, 3).reshape(B, Hkv, pages * PAGE, Dh).float()
    at = (s["row_start"].long()[:-1, None] + torch.arange(most, device="cuda")).clamp(max=N - 1)
    mine = q[at].view(B, most, Hkv, g, Dh).permute(0, 2, 1, 3, 4).reshape(B, Hkv, most * g, Dh)
    score = (mine @ k.transpose(2, 3).contiguous()).view(B, Hkv, most, g, pages * PAGE)
    t = torch.arange(pages * PAGE, device="cuda")
    node = t - s["held"].long()[:, None]  # the key's row among the request's own, negative for held tokens
    word = s["mask"][at].long().gather(2, (node // 32).clamp(0, 3)[:, None].expand(B, most, -1))
    sees = (node < 0)[:, None] | ((node >= 0) & (node < NODES))[:, None] & ((word >> (node % 32)[:, None]) & 1 > 0)
    score = torch.where(sees[:, None, :, None], score, NINF)
    m2 = score.amax(-1, keepdim=True)
    e = torch.exp(score - torch.where(m2 == NINF, 0.0, m2))
    l2, o2 = e.sum(-1, keepdim=True), (e.view(B, Hkv, most * g, -1) @ v).view(B, Hkv, most, g, Dh)
    # joined, row by row
    req, local, _ = _rows(s)
    local = local.clamp(max=most - 1)
    back = lambda x: x[req, :, local]  # noqa: E731
    m1, l1, o1 = (x.view(Hkv, N, g, -1).transpose(0, 1) for x in (m1, l1, o1))
    m2, l2, o2 = back(m2), back(l2), back(o2)
    m = torch.maximum(m1, m2)
    a1, a2 = torch.exp(m1 - m), torch.exp(m2 - m)
    out = (o1 * a1 + o2 * a2) / (l1 * a1 + l2 * a2)
    s["out"][:s["total"]] = out.reshape(N, H, Dh)[:s["total"]].to(torch.bfloat16)
    return s["out"]


def _plain_commit(s):
    req, local, _ = _rows(s)
    to = s["slot"][:s["N"]].long()
    src = s["path"][:s["N"]].long() if s["N"] else to
    moves = (local >= 1) & (local <= s["accept_len"].long()[req])
    back = to[(s["row_start"].long()[req] + torch.where(moves, src, local))]
    for pool in (s["k_pages"], s["v_pages"].transpose(3, 4)):
        pool[:, to // PAGE, :, to % PAGE] = pool[:, back // PAGE, :, back % PAGE]
    return {"k_pages": s["k_pages"], "v_pages": s["v_pages"]}


def _plain_scores(s):
    x = s["logits"].float()
    row = s["row_of"].long() if s["row_of"] is not None else torch.arange(x.shape[0], device="cuda")
    m = x.amax(-1, keepdim=True)
    d = x - m
    e = torch.exp(d)
    total = e.sum(-1, keepdim=True)
    log = torch.log(total)
    entropy = (log - (e * d).sum(-1, keepdim=True) / total)[:, 0]
    given = d[row, s["tokens"].long()] - log[row, 0]
    top, token = torch.sort(x, dim=-1, descending=True, stable=True)
    k = s["k"]
    return {"logprob": given, "entropy": entropy, "lse": (m + log)[:, 0], "top_token": token[:, :k].to(torch.int32), "top_logprob": top[:, :k] - m - log}


_PLAIN = {"plan": _plain_plan, "store": _plain_store, "attention": _plain_attention, "commit": _plain_commit, "scores": _plain_scores}


def _own(s):
    from paper_2309_04255_amd import binding

    op = s["op"]
    if op == "plan":
        binding.batch_plan(s["cfg"], s["row_start"], s["held"], s["parent"], s["prefix"], s["block_table"], s["free_pages"], s["n_pages"], s["plan"], s["N"])
        v = binding.batch_plan_views(s["cfg"], s["requests"], s["N"], s["plan"])
        return {"block_table": s["block_table"], **{k: v[k] for k in ("slot", "position", "mask", "rope", "status", "taken")}}
    if op == "store":
        N, H, Hkv, Dh = s["N"], s["heads"], s["kv_heads"], s["head_dim"]
        x = s["qkv"].view(N, H + 2 * Hkv, Dh)
        binding.batch_store(s["cfg"], Hkv, 0, x[:, :H], x[:, H:H + Hkv], x[:, H + Hkv:], s["q_out"], s["k_pages"], s["v_pages"], s["plan"], s["requests"])
        return {"q": s["q_out"], "k_pages": s["k_pages"], "v_pages": s["v_pages"]}
    if op == "attention":
        binding.batch_attention(s["cfg"], s["kv_heads"], 0, s["q"], s["k_cache"], s["v_cache"], s["prefix"], s["k_pages"], s["v_pages"],
                                s["block_table"], s["plan"], s["out"], s["workspace"])
        return s["out"]
    if op == "commit":
        binding.batch_commit(s["cfg"], s["kv_heads"], s["k_pages"], s["v_pages"], s["plan"], s["requests"], s["path"], s["accept_len"])
        return {"k_pages": s["k_pages"], "v_pages": s["v_pages"]}
    return binding.token_scores(s["logits"], s["tokens"], s["k"], row_of=s["row_of"], workspace=s["workspace"])


def run(s):
    return _own(s) if own else _PLAIN[s["op"]](s)


# ------------------------------------------------------------------ 64 bits


def _exact_scores(s):
    x = s["logits"].double()
    if x.numel() > 2e8:
        return None
    p = torch.log_softmax(x, -1)
    row = s["row_of"].long() if s["row_of"] is not None else torch.arange(x.shape[0], device="cuda")
    h = -(p.exp() * p).sum(-1)
    return {"logprob": p[row, s["tokens"].long()], "entropy": h, "lse": torch.logsumexp(x, -1),
            "top_token": None, "top_logprob": torch.topk(p, s["k"], -1).values}


def _exact_attention(s):
    """One request after the other: its whole key list, a softmax, the weighted values."""
    H, Hkv, Dh, P = s["heads"], s["kv_heads"], s["head_dim"], s["prefix"]
    out = s["out"].double()
    pk = s["k_cache"][0, :, :P].double()
    pv = s["v_cache"][0, :, :, :P].transpose(1, 2).double()
    start, held, table = s["row_start"].tolist(), s["held"].tolist(), s["block_table"].tolist()
    for b in range(s["requests"]):
        r0, n, h = start[b], start[b + 1] - start[b], held[b]
        if not n:
            continue
        pages = table[b][:-(-(h + n) // PAGE)]
        k = torch.cat([pk, torch.cat([s["k_pages"][0, p].double() for p in pages], 1)[:, :h + n]], 1)
        v = torch.cat([pv, torch.cat([s["v_pages"][0, p].transpose(1, 2).double() for p in pages], 1)[:, :h + n]], 1)
        sees = torch.ones(n, P + h + n, dtype=torch.bool, device="cuda")
        bits = s["mask"][r0:r0 + n].tolist()
        sees[:, P + h:] = torch.tensor([[(w[j // 32] >> (j % 32)) & 1 > 0 for j in range(n)] for w in bits], device="cuda")
        q = s["q"][r0:r0 + n].double().view(n, Hkv, H // Hkv, Dh).permute(1, 2, 0, 3).reshape(Hkv, -1, Dh)
        score = (torch.bmm(q, k.transpose(1, 2).contiguous()) / math.sqrt(Dh)).view(Hkv, H // Hkv, n, -1)
        w = torch.softmax(score.masked_fill(~sees, NINF), -1)
        o = torch.bmm(w.view(Hkv, -1, w.shape[-1]), v.contiguous()).view(Hkv, H // Hkv, n, Dh)
        out[r0:r0 + n] = o.permute(2, 0, 1, 3).reshape(n, H, Dh)
    return out


def _exact_store(s):
    T, H, Hkv, Dh, half = s["total"], s["heads"], s["kv_heads"], s["head_dim"], s["head_dim"] // 2
    x = torch.view_as_complex(torch.stack(s["qkv"][:T].double().view(T, -1, 2, half).unbind(2), -1).contiguous())
    turned = x[:, :H + Hkv] * torch.view_as_complex(s["rope"][:T].double().contiguous())[:, None]
    turned = torch.cat([turned.real, turned.imag], -1)
    q, k, v = s["q_out"].double(), s["k_pages"].double(), s["v_pages"].double()
    q[:T] = turned[:, :H]
    for i, slot in enumerate(s["slot"][:T].tolist()):
        k[0, slot // PAGE, :, slot % PAGE] = turned[i, H:]
        v[0, slot // PAGE, :, :, slot % PAGE] = s["qkv"][i].double().view(-1, Dh)[H + Hkv:]
    return {"q": q, "k_pages": k, "v_pages": v}


def _exact_plan(s):
    out = {"block_table": None, "slot": None, "position": None, "mask": None, "rope": None, "status": None, "taken": None}
    held, par, rows = s["held"].tolist(), s["parent"].tolist(), []
    for b, m in enumerate(s["n"]):
        depth = []
        for p in par[len(rows):len(rows) + m]:
            depth.append(depth[p] + 1 if p >= 0 else 0)
        rows += [s["prefix"] + held[b] + d for d in depth]
    pos = torch.tensor(rows + [0] * (s["N"] - len(rows)), dtype=torch.float64)
    ang = pos[:, None] * torch.exp(-math.log(THETA) * 2.0 * torch.arange(s["head_dim"] // 2, dtype=torch.float64) / s["head_dim"])
    out["rope"] = torch.stack([ang.cos(), ang.sin()], -1)
    return out


def exact(c, seed):
    global own
    was, own = own, False
    try:
        s = prepare(c, seed)
    finally:
        own = was
    # (the moves of `commit` are copies: nothing is computed)
    return {"plan": _exact_plan, "store": _exact_store, "attention": _exact_attention, "commit": lambda s: None, "scores": _exact_scores}[c["op"]](s)
