"""What a step of several requests needs beside its attention, as cases to be timed and compared.

A program that serves requests behind one shared prefix plans a step, stores the new keys and values, runs
the attention, and gets a row of logits per token of its trees.  Around that it has to
  - norm the queries and keys of each head before their rotation, where the model does so (`norm_store`),
  - adjust the logits: penalties for the tokens that a row's own sequence holds already (its request's
    history and its branch of the tree), biases of given tokens, masks of what a grammar allows; and take the
    greedy token of every row (`adjust`),
  - walk the trees along those greedy tokens (`accept`),
  - continue requests from others: several answers to one prompt, beams that change places, requests that
    end (`fork`), and now and then move the pages in use to the front of the pool (`compact`).

Heads, widths and tree sizes are those of the repository's models and workloads (16, 32 and 40 heads of
128, the tiny model's heads of 64; trees of 31 and 41 nodes; a vocabulary of 32000), and generic ones beside
them: K/V heads shared by 4 or 8 query heads, one token per request, vocabularies of 128000 and odd ones.

`run` computes an operator in plain torch operations, or where `own` is true through the library.
"""

import math
import random

import torch

own = False

PAGE = 64
NODES = 128  # rows of a request in one step, at most
THETA = 10000.0
EPS = 1e-6
NINF = float("-inf")


def _case(op, name=None, **kw):
    c = {"op": op, **kw}
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # eight requests decoding one token each, shared K/V heads, a layer of a model with normed queries and keys: latency
        _case("norm_store", "norm_store_b8_n1", requests=8, rows=1, ragged=False, held=300, prefix=512, heads=32, kv_heads=8, head_dim=128, per_head=False, pad=0),
        # 64 requests' trees of the benchmark's size, a gain for each head
        _case("norm_store", "norm_store_b64_n31", requests=64, rows=31, ragged=True, held=500, prefix=1024, heads=32, kv_heads=32, head_dim=128, per_head=True, pad=7),
        # 64 prompts taken in, up to 128 rows each, shared K/V heads: the most bytes
        _case("norm_store", "norm_store_b64_n128", requests=64, rows=128, ragged=False, held=0, prefix=2048, heads=32, kv_heads=8, head_dim=128, per_head=False, pad=0),
        # the benchmark's tree of one request, fp32 logits as the passes return them, a short history: latency
        _case("adjust", "adjust_b1_n31_v32000", requests=1, rows=31, ragged=False, held=200, vocab=32000, dtype="fp32", tree=True, bias=20, masks=0, out=True, pad=0),
        # 32 requests' trees, all of it: penalties, biases and masks of a grammar; the greedy tokens alone are wanted
        _case("adjust", "adjust_b32_n41_v32000", requests=32, rows=41, ragged=True, held=1000, vocab=32000, dtype="fp32", tree=True, bias=100, masks=40, out=False, pad=9),
        # a full server, one token for each of 256 requests with long histories, a large vocabulary, logits of a bf16 head
        _case("adjust", "adjust_b256_n1_v128000", requests=256, rows=1, ragged=True, held=4000, vocab=128000, dtype="bf16", tree=False, bias=30, masks=16, out=True, pad=0),
        # one request's tree of the benchmark's size: the launch is all there is
        _case("accept", "accept_b1_n31", requests=1, rows=31, ragged=False, held=200, pad=0),
        # a full server's trees
        _case("accept", "accept_b1024_n41", requests=1024, rows=41, ragged=True, held=2000, pad=100),
        # four answers to one prompt, the ~1B draft model's pages
        _case("fork", "fork_1b_b4", requests=4, group=4, beams=False, ended=False, held=150, ragged=False, layers=22, kv_heads=16, head_dim=128),
        # 16 prompts of four beams each that change places after a step, some requests end; 40 layers of shared K/V heads
        _case("fork", "fork_beams_b64", requests=64, group=4, beams=True, ended=True, held=400, ragged=True, layers=40, kv_heads=8, head_dim=128),
        # the tiny model's pool after a few requests ended
        _case("compact", "compact_tiny_n300", requests=24, held=500, ragged=True, pages=300, layers=2, kv_heads=4, head_dim=64),
        # a 7B model's pool of 144 pages
        _case("compact", "compact_7b_n144", requests=16, held=400, ragged=True, pages=144, layers=32, kv_heads=32, head_dim=128),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _drawn(rng):
    op = rng.choice(["norm_store", "norm_store", "adjust", "adjust", "adjust", "accept", "fork", "fork", "compact", "compact"])
    heads, kv_heads, head_dim = rng.choice([(4, 4, 64), (4, 2, 64), (16, 16, 128), (32, 32, 128), (32, 8, 128), (40, 40, 128), (64, 8, 128), (24, 8, 64), (10, 2, 128)])
    rows = rng.choice([1, 1, _log(rng, 2, 16), _log(rng, 16, NODES)])
    base = dict(requests=_log(rng, 1, 250), rows=rows, ragged=rng.random() < 0.7, held=rng.choice([0, _log(rng, 1, 4000)]))
    pad = rng.choice([0, rng.randrange(1, 70)])
    pool = dict(layers=rng.choice([1, 2, 22, 32, 40]), kv_heads=kv_heads, head_dim=head_dim)
    if op == "norm_store":
        return _case(op, **base, prefix=rng.choice([0, _log(rng, 1, 8192)]), heads=heads, kv_heads=kv_heads, head_dim=head_dim, per_head=rng.random() < 0.4, pad=pad)
    if op == "adjust":
        return _case(op, **base, vocab=rng.choice([rng.randrange(30, 2000), 32000, rng.randrange(30000, 260000)]), dtype=rng.choice(["fp32", "bf16"]), tree=rng.random() < 0.6,
                     bias=rng.choice([0, _log(rng, 1, 300)]), masks=rng.choice([0, _log(rng, 1, 60)]), out=rng.random() < 0.6, pad=pad)
    if op == "accept":
        return _case(op, **{**base, "requests": _log(rng, 1, 1000)}, pad=pad)
    if op == "fork":
        return _case(op, requests=_log(rng, 2, 200), group=rng.choice([2, 3, 4, 8]), beams=rng.random() < 0.5, ended=rng.random() < 0.5, held=_log(rng, 1, 1500), ragged=rng.random() < 0.7, **pool)
    requests, held = _log(rng, 1, 100), _log(rng, 1, 1500)
    return _case(op, requests=requests, held=held, ragged=rng.random() < 0.7, pages=requests * -(-held // PAGE) + _log(rng, 1, 600), **pool)


def draw(rng):
    # at most what the largest listed cases cost, and no more than a state's room
    while True:
        c = _drawn(rng)
        n, held = _lengths(c)
        pages = c.get("pages") or sum(-(-(h + m) // PAGE) + 1 for h, m in zip(held, n)) + 8
        room = pages * PAGE * c.get("kv_heads", 0) * c.get("head_dim", 0) * 4 * c.get("layers", 1)
        rows = sum(n) + c.get("pad", 0)
        if work(c)["bytes"] < (1.5e8 if c["op"] in ("norm_store", "adjust") else 2e9) and room < 5e9 and rows < 25000 and rows * c.get("vocab", 0) < 4.5e7:
            return c


def _lengths(c):
    """(rows, held tokens) of every request: functions of the case alone."""
    r = random.Random("%d %d %d" % (c["requests"], c.get("rows", 0), c["held"]))
    rows = c.get("rows", 0)
    if not c["ragged"]:
        return [rows] * c["requests"], [c["held"]] * c["requests"]
    n = [r.randint(min(1, rows), rows) for _ in range(c["requests"])]
    held = [r.randint(0, c["held"]) for _ in range(c["requests"])]
    if len(n) > 4:
        n[2] = 0  # a request that sits this step out
    return n, held


def _sources(c):
    """What each request of a `fork` continues from (-1: it ends), and its tokens before: functions of the case alone."""
    r = random.Random("%d %d %d" % (c["requests"], c["group"], c["held"]))
    _, held = _lengths(c)
    B, g = c["requests"], c["group"]
    src = []
    for b in range(B):
        first = b - b % g
        if c["beams"]:  # every beam goes on from one of its group's
            src.append(r.randrange(first, min(first + g, B)))
            held[b] = held[first] if b > first and held[first] else max(held[b], 1)  # (beams are as long as each other)
        else:  # a prompt's answers, in the places of requests that ended before
            src.append(first)
            held[b] = max(held[b], 1) if b == first else 0
        if c["ended"] and r.random() < 0.1:
            src[b] = -1
    return src, held


def _copies(c):
    """Tokens in the last pages that `fork` has to copy."""
    src, held = _sources(c)
    stays = {s for b, s in enumerate(src) if s == b}
    total = 0
    for b, s in enumerate(src):
        if s < 0 or s == b:
            continue
        if s not in stays:
            stays.add(s)  # (the first to come takes the page over)
            continue
        total += held[s] % PAGE
    return total


def work(c):
    n, held = _lengths(c)
    N = sum(n)
    if c["op"] == "norm_store":
        Dh, H, Hkv = c["head_dim"], c["heads"], c["kv_heads"]
        return {"bytes": N * ((H + 2 * Hkv) * Dh * 4 + 4 * Dh + 4) + 2 * (H + Hkv) * Dh, "flops": 6 * N * (H + Hkv) * Dh}
    if c["op"] == "adjust":
        size = 4 if c["dtype"] == "fp32" else 2
        words = -(-c["vocab"] // 32)
        return {"bytes": N * (c["vocab"] * size * (2 if c["out"] else 1) + 28) + 4 * sum(held) + 4 * words * (1 + min(c["masks"], N)) + 4 * c["requests"] * c["bias"], "flops": 0}
    if c["op"] == "accept":
        return {"bytes": N * (16 + 4 + 4 + 4) + 12 * c["requests"], "flops": 0}
    token = c["layers"] * c["kv_heads"] * c["head_dim"] * 4
    if c["op"] == "fork":
        _, held = _sources(c)
        entries = sum(-(-h // PAGE) for h in held)
        return {"bytes": 2 * token * _copies(c) + 8 * entries + 16 * c["requests"] + 4 * (entries + c["requests"] + 8), "flops": 0}
    used = sum(-(-h // PAGE) for h in held)
    moved = used * (c["pages"] - used) / c["pages"]  # (as many as lie past the first `used` pages on average)
    return {"bytes": 2 * token * PAGE * moved + 8 * used, "flops": 0}


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


def _dev(v, dtype=torch.int32):
    return torch.tensor(v, dtype=dtype, device="cuda")


def _requests(c, seed):
    """A step as its program has planned it: the requests' rows, trees and pages, and each row's slot, ancestors, position and angles."""
    r = random.Random(seed)
    n, held = _lengths(c)
    B = c["requests"]
    start = [0]
    for m in n:
        start.append(start[-1] + m)
    total, pad = start[-1], c.get("pad", 0)
    N = max(total + pad, 1)
    parent = [p for m in n for p in (_tree(r, m) if c.get("tree", c["op"] == "accept") else list(range(-1, m - 1)))]
    have = [-(-h // PAGE) for h in held]
    want = [-(-(h + m) // PAGE) for h, m in zip(held, n)]
    n_pages, width = sum(want) + 8, max(want) + 1
    order = list(range(n_pages))
    r.shuffle(order)
    table = [[-1] * width for _ in range(B)]
    at = 0
    for b in range(B):
        table[b][:want[b]] = order[at:at + want[b]]
        at += want[b]
    slot, words, position = [], [], []
    for b, m in enumerate(n):
        sees = []
        for i in range(m):
            p = parent[start[b] + i]
            sees.append((sees[p] if p >= 0 else 0) | 1 << i)
            slot.append(table[b][(held[b] + i) // PAGE] * PAGE + (held[b] + i) % PAGE)
            words.append([((sees[i] >> 32 * k & 0xffffffff) ^ 0x80000000) - 0x80000000 for k in range(4)])
            position.append(c.get("prefix", 0) + held[b] + bin(sees[i]).count("1") - 1)
    half = c.get("head_dim", 64) // 2
    ang = _dev(position + [0] * (N - total), torch.float64)[:, None] * THETA ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
    # (the library's program takes the same pages from its free list, in the same order)
    lent = [table[b][k] for b in range(B) for k in range(have[b], want[b])]
    mine = [[table[b][k] if k < have[b] else -1 for k in range(width)] for b in range(B)]
    return {"op": c["op"], "total": total, "N": N, "requests": B, "n_pages": n_pages, "prefix": c.get("prefix", 0),
            "row_start": _dev(start), "held": _dev(held), "parent": _dev(parent + [0] * (N - total)), "slot": _dev(slot + [-1] * (N - total)),
            "mask": _dev(words + [[0] * 4] * (N - total)), "rope": torch.stack([torch.cos(ang), torch.sin(ang)], -1).float(),
            "block_table": _dev(mine), "free_pages": _dev(lent + order[at:])}


def _config(c):
    from paper_2309_04255_amd import binding

    H, Dh = c.get("heads", c.get("kv_heads", 4)), c.get("head_dim", 64)
    return binding.LlmcadConfig(c.get("layers", 1), H * Dh, H, Dh, 4 * H * Dh, c.get("vocab", 32000), EPS, THETA, 16)


def _planned(c, s):
    """The library's configuration and plan of the step."""
    from paper_2309_04255_amd import binding

    s["cfg"] = _config(c)
    s["plan"] = torch.zeros(binding.batch_plan_bytes(s["cfg"], s["requests"], s["N"]), dtype=torch.uint8, device="cuda")
    binding.batch_plan(s["cfg"], s["row_start"], s["held"], s["parent"], s["prefix"], s["block_table"], s["free_pages"], s["n_pages"], s["plan"], s["N"])


def _words(flags):
    """Truth values [..., V] as 32-bit words [..., ceil(V / 32)], bit t % 32 of word t / 32."""
    V = flags.shape[-1]
    flags = torch.nn.functional.pad(flags, (0, -V % 32)).unflatten(-1, (-1, 32))
    w = (flags.long() << torch.arange(32, device=flags.device)).sum(-1)
    return torch.where(w >= 2**31, w - 2**32, w).to(torch.int32)


def prepare(c, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(*shape, scale=1.0, dtype=torch.bfloat16):
        return torch.randn(shape, generator=g, device="cuda", dtype=dtype) * scale

    def uniform(*shape):
        return torch.rand(shape, generator=g, device="cuda")

    if c["op"] in ("fork", "compact"):
        return _prepare_pool(c, seed, normal)
    s = _requests(c, seed)
    N, B = s["N"], s["requests"]
    if own:
        _planned(c, s)
    if c["op"] == "norm_store":
        H, Hkv, Dh = c["heads"], c["kv_heads"], c["head_dim"]
        s.update(heads=H, kv_heads=Hkv, head_dim=Dh)
        s["k_pages"] = normal(1, s["n_pages"], Hkv, PAGE, Dh)
        s["v_pages"] = normal(1, s["n_pages"], Hkv, Dh, PAGE)
        s["qkv"] = normal(N, (H + 2 * Hkv) * Dh, scale=2.0)  # (the fused projection's output: a row's queries, keys and values side by side)
        s["q_gain"] = 1.0 + normal(*((H, Dh) if c["per_head"] else (Dh,)), scale=0.2)
        s["k_gain"] = 1.0 + normal(*((Hkv, Dh) if c["per_head"] else (Dh,)), scale=0.2)
        s["q_out"] = torch.zeros(N, H, Dh, dtype=torch.bfloat16, device="cuda")
        return s
    if c["op"] == "accept":
        V = 32000
        greedy = torch.randint(0, V, (N,), generator=g, device="cuda", dtype=torch.int32)
        req, local, _ = _rows(s)
        before = greedy[(s["row_start"].long()[req] + s["parent"].long().clamp(min=0)).clamp(max=N - 1)]
        other = torch.randint(0, V, (N,), generator=g, device="cuda", dtype=torch.int32)
        s["tokens"] = torch.where(uniform(N) < 0.6, before, other)  # (a draft that is right more often than not; siblings may agree)
        s["greedy"] = greedy
        s["history"] = torch.zeros(B, c["held"] + c["rows"], dtype=torch.int32, device="cuda")
        s["path"] = torch.full((N,), -7, dtype=torch.int32, device="cuda")
        s["accept_len"] = torch.full((B,), -7, dtype=torch.int32, device="cuda")
        s["next_token"] = torch.full((B,), -7, dtype=torch.int32, device="cuda")
        return s
    V, stride = c["vocab"], max(c["held"], 1)
    words = lambda *shape: (V * uniform(*shape) ** 3).long().clamp(max=V - 1).to(torch.int32)  # noqa: E731  (few tokens are most of a text)
    x = normal(N, V, scale=2.5, dtype=torch.float32)
    x.scatter_add_(1, words(N, 4).long(), torch.full((N, 4), 8.0, device="cuda"))  # (a few favourites)
    s["vocab"], s["bf16"] = V, c["dtype"] == "bf16"
    s["logits"] = x.to(torch.bfloat16) if s["bf16"] else x
    s["tokens"], s["history"] = words(N), words(B, stride)
    s["prompt_len"] = s["held"] // 2
    prefix = torch.zeros(V, dtype=torch.bool, device="cuda")
    prefix[words(min(V, 2000)).long()] = True  # (the tokens of the shared prefix)
    s["seen"] = _words(prefix)
    plain = uniform(B, 1) < 0.2  # (requests without penalties)
    s["penalties"] = torch.where(plain, _dev([1.0, 0.0, 0.0], torch.float32), torch.stack([1.0 + 0.3 * uniform(B), uniform(B), 0.5 * uniform(B)], -1))
    s["bias"] = None
    if c["bias"]:
        r = random.Random(seed + 1)
        count = [r.choice([0, r.randint(0, min(c["bias"], V)), min(c["bias"], V)]) for _ in range(B)]
        start = [0]
        for m in count:
            start.append(start[-1] + m)
        tok = [t for m in count for t in r.sample(range(V), m)]
        s["bias"] = (_dev(start), _dev(tok or [0]), normal(max(len(tok), 1), scale=4.0, dtype=torch.float32))
        s["bias_of"] = _dev([b for b, m in enumerate(count) for _ in range(m)], torch.int64)
    s["allow"] = s["mask_of"] = None
    if c["masks"]:
        share = uniform(c["masks"], 1) ** 2  # (states of a grammar that allow much or little)
        s["allow"] = _words(uniform(c["masks"], V) < share)
        s["mask_of"] = torch.randint(-1, c["masks"], (N,), generator=g, device="cuda", dtype=torch.int32)
    s["out"] = torch.zeros_like(s["logits"]) if c["out"] else None
    s["greedy"] = torch.full((N,), -7, dtype=torch.int32, device="cuda")
    if own:
        from paper_2309_04255_amd import binding

        s["workspace"] = torch.empty(binding.batch_adjust_workspace_bytes(s["cfg"], N), dtype=torch.uint8, device="cuda")
    return s


def _prepare_pool(c, seed, normal):
    r = random.Random(seed)
    B, L, Hkv, Dh = c["requests"], c["layers"], c["kv_heads"], c["head_dim"]
    src, held = _sources(c) if c["op"] == "fork" else (None, _lengths(c)[1])
    have = [-(-h // PAGE) for h in held]
    n_pages, width = c.get("pages") or sum(have) + B + 8, max(max(have), 1) + 1
    order = list(range(n_pages))
    r.shuffle(order)
    table, at = [[-1] * width for _ in range(B)], 0
    for b in range(B):
        table[b][:have[b]] = order[at:at + have[b]]
        at += have[b]
    s = {"op": c["op"], "requests": B, "n_pages": n_pages, "kv_heads": Hkv, "held": _dev(held), "block_table": _dev(table), "table_out": torch.full((B, width), -7, dtype=torch.int32, device="cuda"),
         "k_pages": normal(L, n_pages, Hkv, PAGE, Dh), "v_pages": normal(L, n_pages, Hkv, Dh, PAGE)}
    if c["op"] == "fork":
        s["source"] = _dev(src)
        s["held_out"] = torch.zeros(B, dtype=torch.int32, device="cuda")
        s["free_pages"] = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    if own:
        from paper_2309_04255_amd import binding

        s["cfg"] = _config(c)
        s["workspace"] = torch.empty(binding.batch_pages_workspace_bytes(B, n_pages), dtype=torch.uint8, device="cuda")
    return s


# ------------------------------------------------------------------ plain forms


def _rows(s):
    """(request, its row) of every row, and whether it is one: padding rows get the last request and a row past its own."""
    at = torch.arange(s["N"], device="cuda")
    req = torch.searchsorted(s["row_start"][1:].long().contiguous(), at, right=True).clamp(max=s["requests"] - 1)
    return req, at - s["row_start"].long()[req], at < s["total"]


def _bits(s):
    """Truth values [N, 128]: which rows of its request a row descends from, itself among them."""
    return ((s["mask"].long()[:, :, None] >> torch.arange(32, device="cuda")) & 1).view(s["N"], NODES) > 0


def _plain_norm_store(s):
    T, H, Hkv, Dh = s["total"], s["heads"], s["kv_heads"], s["head_dim"]
    x = s["qkv"][:T].view(T, H + 2 * Hkv, Dh).float()
    y = x[:, :H + Hkv]
    y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS)
    y = y * torch.cat([s["q_gain"].expand(H, Dh), s["k_gain"].expand(Hkv, Dh)]).float()
    cos, sin = s["rope"][:T, None, :, 0], s["rope"][:T, None, :, 1]
    a, b = y[..., :Dh // 2], y[..., Dh // 2:]
    y = torch.cat([a * cos - b * sin, b * cos + a * sin], -1).to(torch.bfloat16)
    s["q_out"][:T] = y[:, :H]
    slot = s["slot"][:T].long()
    s["k_pages"][0][slot // PAGE, :, slot % PAGE] = y[:, H:]
    s["v_pages"][0][slot // PAGE, :, :, slot % PAGE] = s["qkv"][:T].view(T, H + 2 * Hkv, Dh)[:, H + Hkv:]
    return {"q": s["q_out"], "k_pages": s["k_pages"], "v_pages": s["v_pages"]}


def _plain_adjust(s):
    N, B, V = s["N"], s["requests"], s["vocab"]
    req, _, real = _rows(s)
    held, prompt = s["held"].long(), s["prompt_len"].long()
    # how often each token occurs in a request's history (its answer's part), and whether it does at all
    t = torch.arange(s["history"].shape[1], device="cuda")
    at = torch.where(t < held[:, None], s["history"].long(), V)
    seen = torch.zeros(B, V + 1, dtype=torch.bool, device="cuda").scatter_(1, at, True)
    count = torch.zeros(B, V + 1, dtype=torch.int32, device="cuda").scatter_add_(1, at, (t >= prompt[:, None]).to(torch.int32))
    # a row's own branch beside it
    bits = _bits(s)
    lane = torch.arange(NODES, device="cuda")
    token = s["tokens"].long()[(s["row_start"].long()[req][:, None] + lane).clamp(max=N - 1)]
    at = torch.where(bits, token, V)
    answer = held[req][:, None] + torch.cumsum(bits, 1) - 1 >= prompt[req][:, None]
    seen = seen[req].scatter_(1, at, True)[:, :V]
    count = count[req].scatter_add_(1, at, answer.to(torch.int32))[:, :V]
    lanes = torch.arange(32, device="cuda")
    seen |= (((s["seen"][:, None] >> lanes) & 1) > 0).view(-1)[:V]
    x = s["logits"].float()
    rho, presence, frequency = (s["penalties"][req][:, i:i + 1] for i in range(3))
    x = torch.where(seen, torch.where(x > 0, x / rho, x * rho), x)
    x = x - frequency * count
    x = x - torch.where(count > 0, presence, 0.0)
    if s["bias"] is not None:
        m = s["bias_of"].shape[0]
        bias = torch.zeros(B, V, device="cuda")
        bias[s["bias_of"], s["bias"][1][:m].long()] = s["bias"][2][:m]
        x = x + bias[req]
    if s["allow"] is not None:
        allowed = (((s["allow"][:, :, None] >> lanes) & 1) > 0).view(s["allow"].shape[0], -1)[:, :V]
        x = torch.where(allowed[s["mask_of"].long().clamp(min=0)] | (s["mask_of"] < 0)[:, None], x, NINF)
    x = x.to(s["logits"].dtype)
    best = x.amax(-1, keepdim=True)
    first = torch.where(x == best, torch.arange(V, device="cuda"), V).amin(-1)
    first = torch.where(best[:, 0] == NINF, -1, first).to(torch.int32)
    s["greedy"].copy_(torch.where(real, first, s["greedy"]))
    if s["out"] is None:
        return {"greedy": s["greedy"]}
    s["out"][:s["total"]] = x[:s["total"]]
    return {"out": s["out"], "greedy": s["greedy"]}


def _plain_accept(s):
    N, B = s["N"], s["requests"]
    req, local, real = _rows(s)
    start, bits = s["row_start"].long(), _bits(s)
    before = s["greedy"][(start[req] + s["parent"].long().clamp(min=0)).clamp(max=N - 1)]
    wrong = real & (local > 0) & (s["tokens"] != before)
    lane = torch.arange(NODES, device="cuda")
    branch = (start[req][:, None] + lane).clamp(max=N - 1)
    reached = real & ~(bits & wrong[branch]).any(-1)
    depth = bits.sum(-1) - 1
    rank = torch.where(reached, depth * NODES + (NODES - 1 - local), -1)
    best = torch.full((B,), -1, dtype=torch.int64, device="cuda").scatter_reduce_(0, req, rank, "amax")
    last = start[:-1] + NODES - 1 - best % NODES  # the row that the walk ends at
    some = best >= 0
    length = torch.where(some, best // NODES, -1)
    s["accept_len"].copy_(length)
    s["next_token"].copy_(torch.where(some, s["greedy"][last.clamp(0, N - 1)], s["next_token"]))
    # the k-th entry of a path is the k-th ancestor of that row
    mine = bits[last.clamp(0, N - 1)]
    kth = torch.sort((~mine).to(torch.int32), dim=-1, stable=True).indices
    path = torch.where(local <= length[req], kth[req, local.clamp(max=NODES - 1)], -1)
    s["path"].copy_(torch.where(real, path, s["path"]))
    # the accepted tokens join the history
    put = real & (local <= length[req])
    to = s["held"].long()[req] + local
    token = s["tokens"][(start[req] + path.clamp(min=0)).clamp(max=N - 1)]
    put = put & (to < s["history"].shape[1])
    s["history"][req[put], to[put]] = token[put]
    return {k: s[k] for k in ("path", "accept_len", "next_token", "history")}


def _used(s, table, held):
    """Which pages requests hold, and which table entries say so."""
    mine = torch.arange(table.shape[1], device="cuda") * PAGE < held[:, None]
    used = torch.zeros(s["n_pages"] + 1, dtype=torch.bool, device="cuda")
    used[torch.where(mine, table, s["n_pages"]).view(-1)] = True
    return used[:s["n_pages"]], mine


def _free_list(used):
    order = torch.sort(used.to(torch.int32), stable=True).indices
    return torch.where(torch.arange(used.shape[0], device="cuda") < (~used).sum(), order, -1)


def _plain_fork(s):
    B, table, src = s["requests"], s["block_table"].long(), s["source"].long()
    me = torch.arange(B, device="cuda")
    ended, stays = src < 0, src == me
    e = src.clamp(min=0)
    held = torch.where(ended, 0, s["held"].long()[e])
    # a last page that is not full goes on with its own request, or with the first that continues from it; others get a copy
    first = torch.full((B,), B, device="cuda").scatter_reduce_(0, e, torch.where(ended, B, me), "amin")
    copies = ~ended & ~stays & (stays[e] | (first[e] != me)) & (held % PAGE > 0)
    free = _free_list(_used(s, table, s["held"].long())[0])
    page = free[(torch.cumsum(copies, 0) - 1).clamp(min=0)]
    col = torch.arange(table.shape[1], device="cuda")
    new = torch.where(col * PAGE < held[:, None], table[e], -1)
    last = new.gather(1, (held // PAGE).clamp(max=table.shape[1] - 1)[:, None])[:, 0]
    new = torch.where(copies[:, None] & (col == (held // PAGE)[:, None]), page[:, None], new)
    which = copies.nonzero()[:, 0]
    old, to = last[which], page[which]
    filled = torch.arange(PAGE, device="cuda") < (held[which] % PAGE)[:, None]
    k, v = s["k_pages"], s["v_pages"]
    k[:, to] = torch.where(filled[None, :, None, :, None], k[:, old], k[:, to])
    v[:, to] = torch.where(filled[None, :, None, None, :], v[:, old], v[:, to])
    s["table_out"].copy_(new)
    s["held_out"].copy_(held)
    used, _ = _used(s, new, held)
    s["free_pages"].copy_(_free_list(used))
    return {"block_table": s["table_out"], "held": s["held_out"], "free_pages": s["free_pages"], "n_free": (~used).sum().to(torch.int32).reshape(1),
            "status": torch.zeros(1, dtype=torch.int32, device="cuda"), "k_pages": k, "v_pages": v}


def _plain_compact(s):
    table = s["block_table"].long()
    used, mine = _used(s, table, s["held"].long())
    n_used = used.sum()
    at = torch.arange(s["n_pages"], device="cuda")
    src, dst = (used & (at >= n_used)).nonzero()[:, 0], (~used & (at < n_used)).nonzero()[:, 0]
    to = at.clone()
    to[src] = dst
    s["table_out"].copy_(torch.where(mine, to[table.clamp(min=0)], -1))
    for pool in (s["k_pages"], s["v_pages"]):
        pool[:, dst] = pool[:, src]
    return {"block_table": s["table_out"], "n_used": n_used.to(torch.int32).reshape(1), "k_pages": s["k_pages"], "v_pages": s["v_pages"]}


_PLAIN = {"norm_store": _plain_norm_store, "adjust": _plain_adjust, "accept": _plain_accept, "fork": _plain_fork, "compact": _plain_compact}


def _own(s):
    from paper_2309_04255_amd import binding

    op = s["op"]
    if op == "norm_store":
        N, H, Hkv, Dh = s["N"], s["heads"], s["kv_heads"], s["head_dim"]
        x = s["qkv"].view(N, H + 2 * Hkv, Dh)
        binding.batch_norm_store(s["cfg"], Hkv, 0, x[:, :H], x[:, H:H + Hkv], x[:, H + Hkv:], s["q_gain"], s["k_gain"], s["q_out"], s["k_pages"], s["v_pages"], s["plan"], s["requests"])
        return {"q": s["q_out"], "k_pages": s["k_pages"], "v_pages": s["v_pages"]}
    if op == "adjust":
        binding.batch_adjust(s["cfg"], s["plan"], s["requests"], s["logits"], tokens=s["tokens"], history=s["history"], prompt_len=s["prompt_len"], seen=s["seen"], penalties=s["penalties"],
                             bias=s["bias"], allow=s["allow"], mask_of=s["mask_of"], out=s["out"], greedy=s["greedy"], workspace=s["workspace"])
        return {"greedy": s["greedy"]} if s["out"] is None else {"out": s["out"], "greedy": s["greedy"]}
    if op == "accept":
        binding.batch_accept(s["cfg"], s["plan"], s["requests"], s["tokens"], s["greedy"], s["path"], s["accept_len"], s["next_token"], history=s["history"])
        return {k: s[k] for k in ("path", "accept_len", "next_token", "history")}
    if op == "fork":
        n_free, status = binding.batch_fork(s["cfg"], s["kv_heads"], s["k_pages"], s["v_pages"], s["block_table"], s["held"], s["source"], s["table_out"], s["held_out"], s["free_pages"], s["workspace"])
        return {"block_table": s["table_out"], "held": s["held_out"], "free_pages": s["free_pages"], "n_free": n_free, "status": status, "k_pages": s["k_pages"], "v_pages": s["v_pages"]}
    n_used = binding.batch_compact(s["cfg"], s["kv_heads"], s["k_pages"], s["v_pages"], s["block_table"], s["held"], s["table_out"], s["workspace"])
    return {"block_table": s["table_out"], "n_used": n_used, "k_pages": s["k_pages"], "v_pages": s["v_pages"]}


def run(s):
    return _own(s) if own else _PLAIN[s["op"]](s)


# ------------------------------------------------------------------ 64 bits


def _exact_norm_store(s):
    """Every head as complex numbers, turned by its row's angle."""
    T, H, Hkv, Dh = s["total"], s["heads"], s["kv_heads"], s["head_dim"]
    x = s["qkv"][:T].double().view(T, H + 2 * Hkv, Dh)
    rms = torch.sqrt(torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / Dh + EPS)
    gain = torch.ones(H + 2 * Hkv, Dh, dtype=torch.float64, device="cuda")
    gain[:H], gain[H:H + Hkv] = s["q_gain"].double(), s["k_gain"].double()
    y = (x / rms * gain)[:, :H + Hkv]
    turned = torch.complex(y[..., :Dh // 2], y[..., Dh // 2:]) * torch.view_as_complex(s["rope"][:T].double().contiguous())[:, None]
    turned = torch.cat([turned.real, turned.imag], -1)
    q, k, v = s["q_out"].double(), s["k_pages"].double(), s["v_pages"].double()
    q[:T] = turned[:, :H]
    for i, slot in enumerate(s["slot"][:T].tolist()):
        k[0, slot // PAGE, :, slot % PAGE] = turned[i, H:]
        v[0, slot // PAGE, :, :, slot % PAGE] = x[i, H + Hkv:]
    return {"q": q, "k_pages": k, "v_pages": v}


def _exact_adjust(s):
    """Row by row: the tokens that its sequence holds, one by one with their counts."""
    if s["out"] is None:
        return None
    out, V = s["out"].double(), s["vocab"]
    start, held, prompt = s["row_start"].tolist(), s["held"].tolist(), s["prompt_len"].tolist()
    tokens, history, pen = s["tokens"].tolist(), s["history"].tolist(), s["penalties"].tolist()
    parent = s["parent"].tolist()
    prefix = [32 * i + j for i, w in enumerate(s["seen"].tolist()) for j in range(32) if w >> j & 1]
    mask_of = s["mask_of"].tolist() if s["mask_of"] is not None else [-1] * s["N"]
    for b in range(s["requests"]):
        rho, presence, frequency = pen[b]
        for r in range(start[b], start[b + 1]):
            branch, i = [], r - start[b]
            while i >= 0:
                branch.append(tokens[start[b] + i])
                i = parent[start[b] + i]
            text = history[b][:held[b]] + branch[::-1]
            counts = {}
            for t in text[prompt[b]:]:
                counts[t] = counts.get(t, 0) + 1
            x = s["logits"][r].double()
            hit = _dev(sorted(set(text) | set(prefix)), torch.int64)
            x[hit] = torch.where(x[hit] > 0, x[hit] / rho, x[hit] * rho)
            if counts:
                x[_dev(list(counts), torch.int64)] -= presence + frequency * _dev(list(counts.values()), torch.float64)
            if s["bias"] is not None:
                lo, hi = s["bias"][0][b].item(), s["bias"][0][b + 1].item()
                x.index_add_(0, s["bias"][1][lo:hi].long(), s["bias"][2][lo:hi].double())
            if mask_of[r] >= 0:
                bits = (s["allow"][mask_of[r]].long()[:, None] // 2 ** torch.arange(32, device="cuda")) % 2
                x[bits.view(-1)[:V] == 0] = NINF
            out[r] = x
    return {"out": out, "greedy": None}


def exact(c, seed):
    global own
    if c["op"] not in ("norm_store", "adjust") or sum(_lengths(c)[0]) > 12000:  # (the others compute whole numbers and copy)
        return None
    was, own = own, False
    try:
        s = prepare(c, seed)
    finally:
        own = was
    return {"norm_store": _exact_norm_store, "adjust": _exact_adjust}[c["op"]](s)
