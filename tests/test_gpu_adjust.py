"""Adjusted logits, greedy tokens and the accept walk against their plain statement (oracle/batch.py).

The operator's steps are single fp32 operations in a stated order, so the adjusted logits are equal, bit for
bit (but for a NaN's payload and the sign of zero), and bf16 ones are their rounding."""

import numpy as np
import pytest
import torch

from oracle import batch as ob
from test_gpu_batch import Case, _cfg, _dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def binding():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2309_04255_amd import binding

    return binding


class Step:
    """A step's logits and all that may adjust them, on the host and on the device."""

    def __init__(self, binding, n, held, V, dtype=torch.float32, pad=0, seed=0, stride=None, masks=3, bias=5, tree=True, free=None,
                 offset=0):
        self.b, self.V = binding, V
        self.c = c = Case(binding, n, held, pad=pad, tree=tree, seed=seed)
        c.cfg = _cfg(binding, c.H, c.Dh, 1, V)
        rng = np.random.default_rng(seed + 1)
        self.views = c.plan(free=free)
        self.want = c.want(free=free)
        N, B = c.N, c.B
        word = lambda *shape: (V * rng.random(shape) ** 2).astype(np.int64)  # noqa: E731
        x = torch.tensor(rng.normal(size=(N, V)) * 3, dtype=torch.float32).to(dtype)
        width = stride or V
        store = torch.zeros(N * width + offset, dtype=dtype, device="cuda")
        self.logits = store[offset:offset + N * width].view(N, width)[:, :V]
        self.logits.copy_(x)
        self.tokens = word(N)
        self.history = word(B, max(max(held), 1))
        self.prompt = np.array([rng.integers(0, h + 2) for h in held])
        self.seen = sorted(set(word(V // 3 + 1).tolist()))
        self.penalties = np.stack([1 + rng.random(B) * 0.5, rng.normal(size=B), rng.normal(size=B) * 0.3], -1).astype(np.float32)
        self.penalties[::4] = 1.0, 0.0, 0.0
        self.biases = [[(int(t), np.float32(v)) for t, v in zip(word(m), rng.normal(size=m) * 5)] for m in rng.integers(0, bias + 1, B)]
        self.allow = [set(np.flatnonzero(rng.random(V) < p).tolist()) for p in (0.5, 0.02, 0.0, 0.99)[:masks]]
        self.mask_of = rng.integers(-1, max(masks, 1), N)

    def kw(self, *names):
        """The binding's arguments for the adjustments named (all of them: none named)."""
        V = self.V
        start = np.concatenate([[0], np.cumsum([len(x) for x in self.biases])])
        mask = lambda ts: self.b.token_mask(_dev(sorted(ts)), V)  # noqa: E731
        a = dict(tokens=_dev(self.tokens), history=_dev(self.history), prompt_len=_dev(self.prompt), seen=mask(self.seen),
                 penalties=torch.tensor(self.penalties, device="cuda"),
                 bias=(_dev(start), _dev([t for x in self.biases for t, _ in x] or [0]),
                       torch.tensor([float(v) for x in self.biases for _, v in x] or [0.0], dtype=torch.float32, device="cuda")),
                 allow=torch.stack([mask(s) for s in self.allow]) if self.allow else None,
                 mask_of=_dev(self.mask_of) if self.allow else None)
        return {k: v for k, v in a.items() if not names or k in names}

    def run(self, out="new", greedy=True, logits=None, **kw):
        c, logits = self.c, self.logits if logits is None else logits
        out = torch.full((c.N, self.V), 5.0, dtype=logits.dtype, device="cuda") if isinstance(out, str) else out
        best = torch.full((c.N,), -7, dtype=torch.int32, device="cuda") if greedy else None
        work = torch.full((self.b.batch_adjust_workspace_bytes(c.cfg, c.N),), 0x5A, dtype=torch.uint8, device="cuda")
        self.b.batch_adjust(c.cfg, c.d_plan, c.B, logits, out=out, greedy=best, workspace=work, **kw)
        torch.cuda.synchronize()
        return out, best

    def oracle(self, *names):
        c = self.c
        use = lambda k, v: v if not names or k in names else None  # noqa: E731
        return ob.adjust(self.logits.float().cpu().numpy(), c.row_start, c.held, self.want["ancestors"], use("tokens", self.tokens),
                         use("history", self.history), use("prompt_len", self.prompt), use("seen", self.seen) or (),
                         use("penalties", self.penalties), use("bias", self.biases), use("allow", self.allow) or None,
                         use("mask_of", self.mask_of))

    def check(self, out, best, want, fill=5.0):
        placed = np.array([len(a) > 0 for a in self.want["ancestors"]])
        want = torch.tensor(want).to(self.logits.dtype)
        if out is not None:
            got = out.cpu()
            same = (got == want) | (got.isnan() & want.isnan())
            assert bool(same[placed].all()), same[placed].logical_not().nonzero()[:5]
            if fill is not None:
                assert bool((got[~placed] == fill).all())
        if best is not None:
            for r in range(self.c.N):
                assert int(best[r]) == (ob.greedy(want[r].float().numpy()) if placed[r] else -7), r


SHAPES = [
    ([1], [0], 1, {}), ([1], [5], 7, {}), ([3], [1], 31, {}), ([2, 2], [64, 0], 32, {}), ([31], [200], 33, {}),
    ([1] * 7, [0, 1, 40, 63, 64, 65, 300], 4095, {"tree": False, "pad": 3}),
    ([5, 0, 12, 1], [100, 7, 0, 1000], 4096, {"pad": 1}), ([9, 9], [33, 500], 4097, {"stride": 4104}),
    ([128, 1], [63, 4000], 9001, {"stride": 9007}), ([4, 3], [10, 20], 8200, {"offset": 3}), ([2], [2000], 20011, {"offset": 1, "stride": 20013}),
]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,held,V,kw", SHAPES)
def test_all_adjustments(binding, n, held, V, kw, dtype):
    s = Step(binding, n, held, V, dtype, seed=V, **kw)
    out, best = s.run(**s.kw())
    s.check(out, best, s.oracle())
    _, alone = s.run(out=None, **s.kw())
    assert torch.equal(alone, best)
    only, _ = s.run(greedy=False, **s.kw())
    assert torch.equal(only, out)
    view = s.logits.clone() if kw.get("offset") is None else s.logits
    same, best2 = s.run(out=view, logits=view, **s.kw())  # in place
    placed = (s.views["slot"] >= 0)
    assert torch.equal(same[placed], out[placed]) and torch.equal(best2, best)


@pytest.mark.parametrize("names", [("mask_of", "allow"), ("bias",), ("penalties", "tokens"), ("penalties", "tokens", "history"),
                                   ("penalties", "tokens", "seen"), ("penalties", "tokens", "history", "prompt_len"), ("history", "seen"),
                                   ("bias", "mask_of", "allow")])
def test_each_alone(binding, names):
    s = Step(binding, [6, 1, 0, 3], [40, 9, 3, 200], 5000, seed=5, pad=2)
    out, best = s.run(**s.kw(*names))
    s.check(out, best, s.oracle(*names))


def test_nothing_is_a_copy(binding):
    s = Step(binding, [4], [6], 1003, torch.bfloat16)
    s.logits[1, 5], s.logits[2, 7], s.logits[3, 0] = float("nan"), float("inf"), float("-inf")
    s.logits[0] = -0.0
    out, best = s.run()
    assert torch.equal(out.view(torch.int16), s.logits.view(torch.int16))
    assert best.tolist()[:3] == [0, -1, 7]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_masks(binding, dtype):
    """A mask that leaves nothing, Inf and NaN in masked places, masks past the last, padding bits of the last word."""
    V = 4100
    s = Step(binding, [6], [3], V, dtype)
    s.allow = [{5, 4099}, set(), set(range(V))]
    s.mask_of = np.array([0, 0, 1, 2, 3, -1])
    s.logits[0, 6], s.logits[0, 4098] = float("nan"), float("inf")
    s.logits[1, 5], s.logits[1, 4099] = float("nan"), 0.0
    s.logits[3, 4097] = float("inf")
    s.logits[5, 3], s.logits[5, 4099] = float("-inf"), 100.0
    kw = s.kw("allow", "mask_of")
    kw["allow"][:, -1] |= -16  # (bits of tokens that are none)
    out, best = s.run(**kw)
    s.check(out, best, s.oracle("allow", "mask_of"))
    assert best.tolist() == [5 if s.logits[0, 5] >= s.logits[0, 4099] else 4099, -1, -1, 4097, -1, 4099]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_ties_go_to_the_lowest_token(binding, dtype):
    V = 9000
    s = Step(binding, [5], [3], V, dtype)
    s.logits.clamp_(max=8.0)
    for r, at in enumerate(([8999, 4096], [4095, 4096], [17, 16, 15], [8000, 100, 4500], [0, 8999])):
        s.logits[r, at] = 9.0
    s.logits[3].fill_(-3.0)
    s.logits[3, [8000, 100]] = torch.tensor([0.0, -0.0], dtype=dtype, device="cuda")
    _, best = s.run()
    assert best.tolist() == [4096, 4095, 15, 100, 0]
    if dtype is torch.bfloat16:  # two values that one rounding makes equal
        s.logits[0].fill_(0.0)
        s.logits[0, [200, 7000]] = torch.tensor([100.0, 100.0], dtype=dtype, device="cuda")
        s.biases = [[(200, np.float32(0.01)), (7000, np.float32(0.02))]]
        out, best = s.run(**s.kw("bias"))
        s.check(out, best, s.oracle("bias"))
        assert int(best[0]) == 200


def test_texts_that_repeat_end_and_lie(binding):
    """One token many times, tokens that are none, a history shorter than the lengths, prompts longer than the text."""
    s = Step(binding, [3, 2, 128, 1], [700, 100, 9, 64], 300, seed=2)
    s.history[0] = 17
    s.history[1, ::2], s.history[1, 1::2] = -1, 300
    s.tokens[0:3] = 17
    s.tokens[5:5 + 128] = np.arange(128) % 3
    s.tokens[5 + 20], s.tokens[5 + 30] = -5, 1 << 30
    s.prompt = np.array([10, 200, 40, 65])  # (the third: rows on both sides of the prompt's end)
    s.penalties[:] = 1.3, 0.7, 0.21
    out, best = s.run(**s.kw())
    s.check(out, best, s.oracle())
    s.history = s.history[:, :50].copy()
    out, best = s.run(**s.kw())
    s.check(out, best, s.oracle())
    s.history = s.history[:, :0].copy()
    out, best = s.run(**s.kw())
    s.check(out, best, s.oracle())


@pytest.mark.parametrize("penalty", [(0.0, 0.0, 0.0), (-1.0, 0.0, 0.0), (1.5, 0.0, float("inf")), (float("inf"), 0.0, 0.0)])
@pytest.mark.parametrize("n,V", [([1, 2], 33), ([1], 1003), ([20, 20], 4099)])
def test_bits_behind_the_vocabulary(binding, n, V, penalty):
    """The last word's bits past the vocabulary are nobody's tokens, whatever the penalties make of them."""
    s = Step(binding, n, [3] * len(n), V, seed=V)
    s.penalties[:] = penalty
    s.seen = []
    s.tokens[:], s.history[:] = -1, -1
    kw = s.kw("tokens", "history", "penalties", "seen", "mask_of", "allow")
    last = -(1 << V % 32)  # bits V % 32 ... 31
    kw["seen"][-1] |= last
    kw["allow"][:, -1] |= last
    out, best = s.run(**kw)
    s.check(out, best, s.oracle("tokens", "history", "penalties", "seen", "mask_of", "allow"))


def test_bias_lists(binding):
    """A token more than once (the last entry counts), tokens that are none, lists that reach past the entries, infinities."""
    s = Step(binding, [2, 2, 2], [1, 1, 1], 4200)
    f = np.float32
    s.biases = [[(7, f(1)), (8, f(2)), (7, f(5)), (4199, f(3)), (7, f(-4))], [(-1, f(9)), (4200, f(9)), (3, f(np.inf))], [(5, f(-np.inf))]]
    out, best = s.run(**s.kw("bias"))
    s.check(out, best, s.oracle("bias"))
    assert best.tolist()[2:4] == [3, 3]
    start, token, value = s.kw("bias")["bias"]
    start = _dev([-3, 5, 900, 9])  # (from before the first to past the last; an empty one)
    out2, _ = s.run(bias=(start, token, value))
    s.biases = [s.biases[0], s.biases[1] + s.biases[2], []]
    s.check(out2, None, s.oracle("bias"))
    out3, _ = s.run(bias=(_dev([0] * 4), token[:0], value[:0]))  # (no entries at all)
    assert torch.equal(out3, s.logits)


def test_a_long_bias_list(binding):
    """More entries than a workgroup has threads, one for most tokens of the vocabulary, some of them twice."""
    s = Step(binding, [2, 1], [3, 0], 6001)
    rng = np.random.default_rng(0)
    s.biases = [[(int(t), np.float32(v)) for t, v in zip(rng.integers(0, 6001, 9000), rng.normal(size=9000))], []]
    out, best = s.run(**s.kw("bias"))
    s.check(out, best, s.oracle("bias"))


def test_long_histories(binding):
    """More tokens than a workgroup sorts (all in one piece, or spread), over several pieces a workgroup."""
    for where, V in (("one", 200003), ("spread", 200003), ("few", 9000)):
        s = Step(binding, [1] * 40, [9000] * 20 + [5000] * 19 + [1], V, torch.bfloat16, seed=4, masks=0, tree=False)
        rng = np.random.default_rng(1)
        s.history[:] = {"one": rng.integers(4096 * 7, 4096 * 7 + 50, s.history.shape), "spread": rng.integers(0, V, s.history.shape),
                        "few": rng.integers(0, 3, s.history.shape)}[where]
        out, best = s.run(**s.kw())
        s.check(out, best, s.oracle())


def test_rows_that_are_not_placed(binding):
    """A request without pages and padding keep their rows; the others are adjusted."""
    s = Step(binding, [1, 70, 70], [60, 0, 0], 500, pad=9, free=[0])
    assert s.views["status"].tolist() == [0, 2, 2]
    out, best = s.run(**s.kw())
    s.check(out, best, s.oracle())
    bad = Step(binding, [70, 3], [0, 0], 500, pad=9)
    bad.views = bad.c.plan(row_start=[0, 200, 3])
    bad.want = dict(bad.want, ancestors=[[]] * bad.c.N)
    out, best = bad.run(**bad.kw())
    bad.check(out, best, bad.logits.float().cpu().numpy())
    out = torch.full((bad.c.N, 500), 5.0, device="cuda")
    work = torch.zeros(bad.b.batch_adjust_workspace_bytes(bad.c.cfg, bad.c.N), dtype=torch.uint8, device="cuda")
    bad.c.plan()
    bad.b.batch_adjust(bad.c.cfg, bad.c.d_plan, 1, bad.logits, out=out, workspace=work)  # (a plan of two requests)
    assert bool((out == 5.0).all())


def test_many_rows_of_few_tokens(binding):
    s = Step(binding, [128] * 30 + [1] * 40, [9] * 70, 50, seed=3, pad=33)
    out, best = s.run(**s.kw())
    s.check(out, best, s.oracle())


def test_a_large_vocabulary(binding):
    """Rows against torch's masked maximum: 250007 tokens, a favourite in every piece."""
    s = Step(binding, [3, 1], [2000, 3], 250007, torch.bfloat16, bias=200, masks=0)
    out, best = s.run(**s.kw())
    s.check(out, best, s.oracle())
    scores = binding.token_scores(out, None, 1)
    assert torch.equal(scores["top_token"][:, 0], best)


def test_a_captured_step(binding):
    """Plan, adjust and accept in a graph, replayed with other lengths and logits, eager work between."""
    s = Step(binding, [20, 1, 41], [50, 3, 700], 9001, seed=9, pad=2)
    c, kw = s.c, s.kw()
    start, held, par, free = _dev(c.row_start), _dev(c.held), _dev(c.parent), _dev(c.free)
    bufs = lambda: [torch.full((c.N, s.V), 5.0, device="cuda"), *(torch.full((m,), -7, dtype=torch.int32, device="cuda") for m in (c.N, c.N, c.B, c.B))]  # noqa: E731
    work = [torch.zeros(binding.batch_adjust_workspace_bytes(c.cfg, c.N), dtype=torch.uint8, device="cuda") for _ in range(2)]

    def step(b, w):
        binding.batch_plan(c.cfg, start, held, par, 0, c.d_table, free, c.n_pages, c.d_plan, c.N)
        binding.batch_adjust(c.cfg, c.d_plan, c.B, s.logits, out=b[0], greedy=b[1], workspace=w, **kw)
        binding.batch_accept(c.cfg, c.d_plan, c.B, kw["tokens"], b[1], b[2], b[3], b[4])

    mine = bufs()
    step(mine, work[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(mine, work[0])
    for i, lengths in enumerate(([50, 3, 700], [49, 0, 650], [0, 64, 0])):
        held.copy_(_dev(lengths))
        s.logits.add_(torch.randn_like(s.logits))
        kw["tokens"].copy_(torch.randint(0, s.V, (c.N,), device="cuda", dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        want = bufs()
        step(want, work[1])
        torch.cuda.synchronize()
        for a, b in zip(mine, want):
            assert torch.equal(a, b)


def test_two_streams_at_once(binding):
    a, b = Step(binding, [31, 3], [500, 20], 32000, seed=1), Step(binding, [1] * 9, [64] * 9, 32000, torch.bfloat16, seed=2)
    want = a.run(**a.kw()), b.run(**b.kw())
    kws = a.kw(), b.kw()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    torch.cuda.synchronize()
    for s, st, kw in zip((a, b), streams, kws):
        c = s.c
        out, best = torch.full((c.N, s.V), 5.0, dtype=s.logits.dtype, device="cuda"), torch.full((c.N,), -7, dtype=torch.int32, device="cuda")
        work = torch.zeros(binding.batch_adjust_workspace_bytes(c.cfg, c.N), dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        for _ in range(20):
            binding.batch_adjust(c.cfg, c.d_plan, c.B, s.logits, out=out, greedy=best, workspace=work, stream=st, **kw)
        got.append((out, best))
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert torch.equal(g[0], w[0]) and torch.equal(g[1], w[1])


# ---------------------------------------------------------------- accept


def _accept(binding, c, tokens, best, history=None):
    path = torch.full((c.N,), -7, dtype=torch.int32, device="cuda")
    length, after = (torch.full((c.B,), -7, dtype=torch.int32, device="cuda") for _ in range(2))
    binding.batch_accept(c.cfg, c.d_plan, c.B, tokens, best, path, length, after, history)
    torch.cuda.synchronize()
    return path.tolist(), length.tolist(), after.tolist()


@pytest.mark.parametrize("n,held,kw", [
    ([1], [0], {}), ([31], [200], {}), ([128], [63], {}), ([128], [0], {"tree": False}), ([64, 65, 33, 32], [1, 2, 3, 4], {}),
    ([5, 0, 128, 1, 77], [64, 999, 128, 0, 3], {"pad": 300}), ([41] * 200, list(range(200)), {"pad": 5}), ([1] * 1024, [3] * 1024, {}),
])
@pytest.mark.parametrize("alphabet", [2, 5, 1000])
def test_accept(binding, n, held, kw, alphabet):
    c = Case(binding, n, held, seed=alphabet, **kw)
    c.plan()
    rng = np.random.default_rng(alphabet)
    tokens, best = rng.integers(0, alphabet, c.N), rng.integers(-1 if alphabet < 10 else 0, alphabet, c.N)
    for b in range(c.B):  # (drafts that are often right)
        for i in range(1, c.n[b]):
            r = c.row_start[b]
            if rng.random() < 0.6 and best[r + c.parent[r + i]] >= 0:
                tokens[r + i] = best[r + c.parent[r + i]]
    width = max(max(held) + 20, 1)
    history = torch.full((c.B, width), -9, dtype=torch.int32, device="cuda")
    path, length, after = _accept(binding, c, _dev(tokens), _dev(best), history)
    want = np.full((c.B, width), -9)
    for b in range(c.B):
        r, m = c.row_start[b], c.n[b]
        if m == 0:
            assert (length[b], after[b]) == (-1, -7)
            continue
        p, t = ob.accept(tokens[r:r + m], c.parent[r:r + m], best[r:r + m])
        assert path[r:r + m] == p + [-1] * (m - len(p)), b
        assert (length[b], after[b]) == (len(p) - 1, t)
        for k, i in enumerate(p):
            if held[b] + k < width:
                want[b, held[b] + k] = tokens[r + i]
    assert path[c.total:] == [-7] * (c.N - c.total)
    np.testing.assert_array_equal(history.cpu().numpy(), want)


def test_accept_of_requests_that_are_not_placed(binding):
    c = Case(binding, [1, 70, 70], [60, 0, 0], pad=2)
    c.plan(free=[0])
    path, length, after = _accept(binding, c, _dev([1] * c.N), _dev([1] * c.N))
    assert length == [0, -1, -1] and after == [1, -7, -7] and path == [0] + [-7] * 142
    c.plan(row_start=[0, 200, 1, 1])
    assert _accept(binding, c, _dev([1] * c.N), _dev([1] * c.N))[1] == [-1] * 3
    c.plan()
    path = torch.full((c.N,), -7, dtype=torch.int32, device="cuda")
    length, after = (torch.full((2,), -7, dtype=torch.int32, device="cuda") for _ in range(2))
    binding.batch_accept(c.cfg, c.d_plan, 2, _dev([1] * c.N), _dev([1] * c.N), path, length, after)
    assert path.tolist() == [-7] * c.N and length.tolist() == [-7] * 2  # (a plan of three requests)


def test_accept_is_the_single_pass_walk(binding):
    """The library's own verification of one tree and this walk on its logits agree."""
    import workloads

    shape = workloads.MODELS["tiny"]
    sess = binding.Session(shape, capacity=128, max_n=64)
    sess.load_weights(workloads.make_weights(shape, "cuda", gain_jitter=0.1))
    prefix = workloads.draw_tokens(20, shape.vocab, seed=1)
    sess.prefill(prefix, 0)
    par = workloads.random_tree(40, 5, seed=4)
    tok = workloads.draw_tokens(40, shape.vocab, seed=6)
    n = sess.verify_tree(20, tok, par)
    logits, _, _, _ = sess.results(n)
    best = logits.argmax(-1).numpy()
    for i in range(1, 40):
        if i % 3:
            tok[i] = best[par[i]]  # (only the walk looks at these: a node's logits change with its branch, so verify again)
    n = sess.verify_tree(20, tok, par)
    logits, path, acc, nxt = sess.results(n)
    batch = binding.Batch(shape, 1, 40, n_pages=2, max_pages=2)
    batch.plan(_dev([0, 40]), _dev([0]), _dev(par))
    mine = torch.full((40,), -7, dtype=torch.int32, device="cuda")
    length, after, best = (torch.full((m,), -7, dtype=torch.int32, device="cuda") for m in (1, 1, 40))
    batch.adjust(logits.cuda(), greedy=best)
    batch.accept(_dev(tok), best, mine, length, after)
    assert (int(length), int(after)) == (acc, nxt) and mine.tolist()[:acc + 1] == path


@pytest.mark.parametrize("change,match", [
    (dict(logits=lambda s: s.logits[:, :-1]), "logits"), (dict(logits=lambda s: s.logits.half()), "logits"),
    (dict(out=lambda s: s.logits.to(torch.bfloat16)), "out"), (dict(tokens=lambda s: _dev([1])), "tokens"),
    (dict(history=lambda s: _dev([[1]])), "history"), (dict(penalties=lambda s: torch.ones(2, 2, device="cuda")), "penalties"),
    (dict(seen=lambda s: _dev([1])), "seen"), (dict(allow=lambda s: _dev([[1]])), "allow"), (dict(mask_of=lambda s: _dev([1])), "mask_of"),
    (dict(greedy=lambda s: torch.zeros(s.c.N, dtype=torch.int64, device="cuda")), "greedy"), (dict(workspace=lambda s: None), "workspace"),
    (dict(tokens=lambda s: torch.zeros(s.c.N, dtype=torch.int32)), "tensors on"),
    (dict(bias=lambda s: (_dev([0, 0, 0]), _dev([1, 2]), torch.ones(1, device="cuda"))), "a value for each"),
])
def test_refusals(binding, change, match):
    s = Step(binding, [3, 2], [0, 5], 500)
    a = dict(logits=s.logits, out=torch.empty(s.c.N, 500, device="cuda"),
             workspace=torch.zeros(binding.batch_adjust_workspace_bytes(s.c.cfg, s.c.N), dtype=torch.uint8, device="cuda"))
    a.update({k: make(s) for k, make in change.items()})
    with pytest.raises(ValueError, match=match):
        binding.batch_adjust(s.c.cfg, s.c.d_plan, s.c.B, a.pop("logits"), **a)
