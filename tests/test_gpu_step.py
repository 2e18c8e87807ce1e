"""The operators of a step together, as a server uses them: requests behind one shared prefix of a model that norms its
queries and keys; trees verified under penalties, biases and masks, accepted on the device and rolled back; requests
that fork, change places and end, and a pool that is compacted in between.  Against the same model run on every row's
own text, one after the other in float64, with the adjustment and the walk of oracle/batch.py on the GPU's logits.

Both sides round the same activations to bf16 (queries, keys and values, attention outputs) and sum in other orders, over
two layers: the logits are held to the passes' bar, 2e-2 absolute and 1e-2 in the 2-norm, once for each side."""

import math

import numpy as np
import pytest
import torch

import workloads
from oracle import batch as ob

pytestmark = pytest.mark.gpu

V, P, L, H, HKV, DH = 48, 70, 2, 4, 2, 64
SHAPE = workloads.ModelShape("step", L, H * DH, H, DH, 512, V, seed=1)
EPS, THETA = SHAPE.rms_eps, SHAPE.rope_theta


@pytest.fixture(scope="module")
def binding():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2309_04255_amd import binding

    return binding


class Model:
    def __init__(self, seed=0):
        g = torch.Generator().manual_seed(seed)
        bf = lambda *s, scale: (torch.randn(*s, generator=g) * scale).to(torch.bfloat16)  # noqa: E731
        d = H * DH
        self.embed, self.head = bf(V, d, scale=1.0), bf(V, d, scale=0.08)
        self.layers = [dict(qkv=bf((H + 2 * HKV) * DH, d, scale=0.06), o=bf(d, d, scale=0.05), qg=1 + bf(H, DH, scale=0.2), kg=1 + bf(DH, scale=0.2))
                       for _ in range(L)]

    def to_gpu(self):
        f = lambda t: t.float().cuda()  # noqa: E731
        self.g_embed, self.g_head = f(self.embed), f(self.head)
        self.g_layers = [{k: (f(v) if k in ("qkv", "o") else v.cuda()) for k, v in w.items()} for w in self.layers]

    def forward(self, batch, tokens):
        """A batch's rows on the GPU: logits [N, V]."""
        N = tokens.shape[0]
        x = self.g_embed[tokens.long()]
        q, out = (torch.zeros(N, H, DH, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        for l, w in enumerate(self.g_layers):
            qkv = (x @ w["qkv"].t()).to(torch.bfloat16).view(N, H + 2 * HKV, DH)
            batch.norm_store(l, qkv[:, :H], qkv[:, H:H + HKV], qkv[:, H + HKV:], w["qg"], w["kg"], q)
            batch.attention(l, q, out)
            x = x + out.view(N, -1).float() @ w["o"].t()
        return x @ self.g_head.t()

    def text(self, tokens):
        """One text in float64: (logits [n, V], keys and values of every layer [n, HKV, DH])."""
        r = lambda t: t.to(torch.bfloat16).double()  # noqa: E731
        n = len(tokens)
        x = self.embed[torch.tensor(tokens)].double()
        pos = np.arange(n)[:, None] * THETA ** (-2.0 * np.arange(DH // 2) / DH)
        rope = np.stack([np.cos(pos), np.sin(pos)], -1)
        causal = torch.ones(n, n).tril().bool()
        caches = []
        for w in self.layers:
            qkv = r(x @ w["qkv"].double().t()).view(n, H + 2 * HKV, DH).numpy()
            q = r(torch.from_numpy(ob.turn(ob.norm(qkv[:, :H], w["qg"].double().numpy(), EPS), rope)))
            k = r(torch.from_numpy(ob.turn(ob.norm(qkv[:, H:H + HKV], w["kg"].double().numpy(), EPS), rope)))
            v = torch.from_numpy(qkv[:, H + HKV:])
            caches.append((k, v))
            out = torch.empty(n, H, DH, dtype=torch.float64)
            for h in range(H):
                z = (q[:, h] @ k[:, h // (H // HKV)].t() / math.sqrt(DH)).masked_fill(~causal, -math.inf)
                out[:, h] = torch.softmax(z, -1) @ v[:, h // (H // HKV)]
            x = x + r(out).reshape(n, -1) @ w["o"].double().t()
        return x @ self.head.double().t(), caches


@pytest.fixture(scope="module")
def model():
    return Model()


def _dev(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


class Server:
    """Requests and what a program keeps for them, beside the texts that they should hold."""

    def __init__(self, binding, model, B, N, n_pages, seed):
        model.to_gpu()
        self.rng, self.binding, self.model, self.B, self.N = np.random.default_rng(seed), binding, model, B, N
        self.prefix = self.rng.integers(0, V, P).tolist()
        _, caches = model.text(self.prefix)
        cap = 128
        self.k_cache = torch.zeros(L, HKV, cap, DH, dtype=torch.bfloat16, device="cuda")
        self.v_cache = torch.zeros(L, HKV, DH, cap, dtype=torch.bfloat16, device="cuda")
        for l, (k, v) in enumerate(caches):
            self.k_cache[l, :, :P] = k.to(torch.bfloat16).transpose(0, 1).cuda()
            self.v_cache[l, :, :, :P] = v.to(torch.bfloat16).permute(1, 2, 0).cuda()
        self.batch = binding.Batch(SHAPE, B, N, n_pages=n_pages, max_pages=6, prefix_len=P, k_cache=self.k_cache, v_cache=self.v_cache,
                                   n_kv_heads=HKV)
        self.held = torch.zeros(B, dtype=torch.int32, device="cuda")
        self.history = torch.zeros(B, 300, dtype=torch.int32, device="cuda")
        self.text = [[] for _ in range(B)]
        self.root = self.rng.integers(0, V, B).tolist()  # the token that each request's next tree begins with
        self.prompt_len = np.array([int(self.rng.integers(0, 20)) for _ in range(B)])
        self.seen = sorted(set(self.prefix[:20]))
        self.penalties = np.stack([1 + 0.3 * self.rng.random(B), 0.5 * self.rng.random(B), 0.3 * self.rng.random(B)], -1).astype(np.float32)
        self.penalties[0] = 1, 0, 0
        self.bias = [[(int(t), np.float32(self.rng.normal())) for t in self.rng.integers(0, V, m)] for m in self.rng.integers(0, 6, B)]
        self.allow = [set(np.flatnonzero(self.rng.random(V) < p).tolist()) for p in (0.8, 0.5)]

    def tree(self, b):
        """A tree in which most tokens follow the root somewhere: some path is accepted more often than not."""
        par, tok = [-1], [self.root[b]]
        for t in self.rng.permutation(V)[:int(self.rng.integers(1, 40))]:
            par.append(int(self.rng.choice([0, 0, 0, self.rng.integers(len(par))])))
            tok.append(int(t))
        return par, tok

    def step(self, rows):
        """rows: (parents, tokens) of every request, empty for one that sits out.  Returns the accepted lengths."""
        B, N, b, net = self.B, self.N, self.batch, self.model
        n = [len(p) for p, _ in rows]
        start = np.concatenate([[0], np.cumsum(n)])
        par, tok = np.zeros(N, np.int64), np.zeros(N, np.int64)
        for r, (p, t) in zip(start, rows):
            par[r:r + len(p)], tok[r:r + len(p)] = p, t
        mask_of = self.rng.integers(-1, 2, N)
        b.plan(_dev(start), self.held, _dev(par))
        assert not b.status.any()
        tokens = _dev(tok)
        logits = net.forward(b, tokens)
        b.advance()
        out, greedy = torch.empty_like(logits), torch.full((N,), -7, dtype=torch.int32, device="cuda")
        path, accept = torch.full((N,), -7, dtype=torch.int32, device="cuda"), torch.full((B,), -7, dtype=torch.int32, device="cuda")
        after = _dev(self.root)
        first = np.concatenate([[0], np.cumsum([len(x) for x in self.bias])])
        mask = lambda ts: self.binding.token_mask(_dev(sorted(ts)), V)  # noqa: E731
        b.adjust(logits, tokens, out=out, greedy=greedy, history=self.history, prompt_len=_dev(self.prompt_len), seen=mask(self.seen),
                 penalties=torch.tensor(self.penalties, device="cuda"),
                 bias=(_dev(first), _dev([t for x in self.bias for t, _ in x]), torch.tensor([float(v) for x in self.bias for _, v in x], device="cuda")),
                 allow=torch.stack([mask(s) for s in self.allow]), mask_of=_dev(mask_of))
        b.accept(tokens, greedy, path, accept, after, self.history)
        b.commit(path, accept)
        self.held += accept + 1
        b.trim(self.held)
        # the texts
        ancestors = [[] for _ in range(N)]
        for r, (p, _) in zip(start, rows):
            for i in range(len(p)):
                ancestors[r + i] = (ancestors[r + p[i]] if p[i] >= 0 else []) + [i]
        for r, (p, t), text in zip(start, rows, self.text):
            for i in range(len(p)):
                chain = self.prefix + text + [t[j] for j in ancestors[r + i]]
                want = net.text(chain)[0][-1]
                got = logits[r + i].cpu().double()
                assert float((got - want).abs().max()) <= 4e-2 and float((got - want).norm() / want.norm()) <= 2e-2, (r, i)
        want = ob.adjust(logits.cpu().numpy(), start, [len(t) for t in self.text], ancestors, tok, self.text, self.prompt_len, self.seen,
                         self.penalties, self.bias, self.allow, mask_of)
        np.testing.assert_array_equal(out.cpu().numpy()[:start[B]], want[:start[B]])
        best = [ob.greedy(x) for x in want]
        assert greedy.tolist() == best[:start[B]] + [-7] * (N - start[B])
        for i, (p, t) in enumerate(rows):
            if not p:
                assert int(accept[i]) == -1
                continue
            r = start[i]
            walk, nxt = ob.accept(t, p, best[r:r + len(p)])
            assert path[r:r + len(p)].tolist() == walk + [-1] * (len(p) - len(walk)) and int(accept[i]) == len(walk) - 1
            assert int(after[i]) == nxt
            self.text[i] = self.text[i] + [t[j] for j in walk]
            self.root[i] = max(nxt, 0)  # (no token was allowed: the program goes on with any)
        self.check()
        return accept.tolist()

    def check(self):
        assert self.held.tolist() == [len(t) for t in self.text]
        for b, t in enumerate(self.text):
            assert self.history[b, :len(t)].tolist() == t

    def fork(self, source):
        self.held = self.batch.fork(_dev(source), self.held)
        keep = _dev([max(s, 0) for s in source]).long()
        self.history = self.history[keep].contiguous()
        self.text = [list(self.text[s]) if s >= 0 else [] for s in source]
        self.root = [self.root[s] if s >= 0 else int(self.rng.integers(V)) for s in source]
        self.prompt_len = np.array([self.prompt_len[max(s, 0)] for s in source])
        self.check()


def test_a_server(binding, model):
    s = Server(binding, model, B=4, N=200, n_pages=20, seed=3)
    prompts = [s.rng.integers(0, V, m).tolist() for m in (100, 1, 63, 30)]
    s.root = [p[0] for p in prompts]
    # prompts are chains that are taken in whole: their tokens count as right
    rows = [(list(range(-1, len(p) - 1)), p) for p in prompts]
    n = [len(p) for p in prompts]
    start = np.concatenate([[0], np.cumsum(n)])
    tok = np.zeros(200, np.int64)
    for r, (p, t) in zip(start, rows):
        tok[r:r + len(t)] = t
    s.batch.plan(_dev(start), s.held)
    model.forward(s.batch, _dev(tok))
    s.batch.advance()
    s.held += _dev(n)
    for b, p in enumerate(prompts):
        s.history[b, :len(p)] = _dev(p)
        s.text[b] = list(p)
    accepted = s.step([s.tree(b) for b in range(4)])
    s.fork([0, 0, 2, 2])  # two answers each to two prompts
    accepted += s.step([s.tree(b) for b in range(4)])
    assert s.batch.compact(s.held) + len(s.batch.free_pages) == 20
    accepted += s.step([s.tree(0), ([], []), s.tree(2), s.tree(3)])
    s.fork([1, 0, 3, -1])  # places change, one request ends
    accepted += s.step([s.tree(0), s.tree(1), s.tree(2), ([-1], [s.root[3]])])
    s.batch.release(0)
    s.held[0] = 0
    s.text[0] = []
    s.batch.compact(s.held)
    accepted += s.step([s.tree(b) for b in range(4)])
    assert sum(a > 0 for a in accepted) >= 3  # (drafts were accepted, and rows moved)


def test_a_captured_step(binding, model):
    """Plan to commit in a graph, replayed while the requests grow, eager steps of a second server between: the same
    tables, lengths, texts, next tokens and pages."""
    model.to_gpu()
    B, N = 3, 60
    made = []
    for _ in range(2):
        s = Server(binding, model, B, N, n_pages=18, seed=5)
        work = dict(start=_dev([0, 20, 40, 60]), parent=_dev([0] * N), tokens=_dev([0] * N), free=_dev(range(18)), greedy=_dev([0] * N),
                    path=_dev([0] * N), accept=_dev([0] * B), after=_dev(s.root), held=s.held, history=s.history)
        made.append((s, work))
    kw = dict(seen=binding.token_mask(_dev([1, 2, 3]), V), penalties=torch.tensor(made[0][0].penalties, device="cuda"),
              prompt_len=_dev(made[0][0].prompt_len))

    def step(s, w):
        b = s.batch
        binding.batch_plan(b.cfg, w["start"], w["held"], w["parent"], P, b.block_table, w["free"], b.n_pages, b.plan_buffer, N)
        logits = model.forward(b, w["tokens"])
        b.adjust(logits, w["tokens"], greedy=w["greedy"], history=w["history"], **kw)
        b.accept(w["tokens"], w["greedy"], w["path"], w["accept"], w["after"], w["history"])
        b.commit(w["path"], w["accept"])
        w["held"] += w["accept"] + 1

    (s0, w0), (s1, w1) = made
    keep = {k: v.clone() for k, v in w0.items()}
    table = s0.batch.block_table.clone()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step(s0, w0)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(s0, w0)
    for k, v in keep.items():  # (the warm-up's step is undone)
        w0[k].copy_(v)
    s0.batch.block_table.copy_(table)
    rng = np.random.default_rng(9)
    free = list(range(18))
    for _ in range(4):
        par, tok = [], []
        for b in range(B):
            p = [-1] + [int(rng.choice([0, 0, rng.integers(i)])) for i in range(1, 20)]
            par += p
            tok += [int(w1["after"][b])] + rng.permutation(V)[:19].tolist()
        for w in (w0, w1):
            w["parent"].copy_(_dev(par))
            w["tokens"].copy_(_dev(tok))
            w["free"].copy_(_dev(free + [-1] * (18 - len(free))))
        graph.replay()
        torch.cuda.synchronize()
        step(s1, w1)
        torch.cuda.synchronize()
        for k in w0:
            assert torch.equal(w0[k], w1[k]), k
        assert torch.equal(s0.batch.block_table, s1.batch.block_table)
        assert torch.equal(s0.batch.k_pages, s1.batch.k_pages) and torch.equal(s0.batch.v_pages, s1.batch.v_pages)
        assert not s1.batch.status.any()
        free = free[int(s1.batch.taken):]
    assert int(w1["held"].max()) > 4  # (more than the roots was accepted)
