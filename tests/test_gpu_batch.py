"""The operators for several requests behind one shared prefix against their float64 statement
(oracle/batch.py), through the binding, at the sizes, masks and values where they can go wrong.

Tolerances.  Whole numbers, pages and moves are equal.  The rotary table is computed in 64 bits and
rounded once, but for one fp32 sine (2 ulp) and product: 2^-21.  A turned key or query is a sum of
two fp32 products of bf16 values, rounded to bf16 once: 2^-8 of itself (half a step), and where
the two cancel 2^-20 of the products' size.  The attention's output is rounded once (2^-8 of itself),
each probability at most once to bf16 (2^-8 of sum p |v|), and fp32 sums and scores take 2^-11 of
sum p |v| at the sizes here (128 products of at most about 10 each in a score, an exponential, and up
to 2^13 additions)."""

import numpy as np
import pytest
import torch

from oracle import batch as ob

pytestmark = pytest.mark.gpu

PAGE = 64
THETA = 10000.0


@pytest.fixture(scope="module")
def binding():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2309_04255_amd import binding

    return binding


def _cfg(binding, H, Dh, L=1, V=1000):
    return binding.LlmcadConfig(L, H * Dh, H, Dh, 4 * H * Dh, V, 1e-6, THETA, 16)


def _dev(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


def _np(t):
    return t.float().cpu().numpy().astype(np.float64)


def _random_tree(rng, n):
    return [-1] + [int(rng.integers(max(0, i - 9), i)) for i in range(1, n)]


class Case:
    """A step: requests with counts n and lengths held behind nothing, their trees, tables and free list."""

    def __init__(self, binding, n, held, H=4, Hkv=None, Dh=64, pad=0, tree=True, seed=0, L=1, P=0, spare=3):
        rng = np.random.default_rng(seed)
        self.rng, self.b = rng, binding
        self.n, self.held, self.B = list(n), list(held), len(n)
        self.H, self.Hkv, self.Dh, self.L, self.P = H, Hkv or H, Dh, L, P
        self.cfg = _cfg(binding, H, Dh, L)
        self.row_start = [0]
        for m in n:
            self.row_start.append(self.row_start[-1] + m)
        self.total = self.row_start[-1]
        self.N = max(self.total + pad, 1)
        self.parent = [p for m in n if m for p in (_random_tree(rng, m) if tree else range(-1, m - 1))]
        self.parent += [7] * (self.N - self.total)
        have = [-(-h // PAGE) for h in held]
        want = [-(-(h + m) // PAGE) for h, m in zip(held, n)]
        self.n_pages, self.width = sum(want) + spare, max(want) + 1
        order = rng.permutation(self.n_pages).tolist()
        self.table = np.full((self.B, self.width), -1)
        for b in range(self.B):
            self.table[b, :have[b]] = [order.pop() for _ in range(have[b])]
        self.free = order

    def want(self, free=None, parent="own", row_start=None, held=None, n_pages=None):
        return ob.plan(row_start or self.row_start, held or self.held, self.parent if parent == "own" else parent, self.P,
                       self.table, self.free if free is None else free, n_pages or self.n_pages, self.N, self.Dh, THETA)

    def plan(self, free=None, parent="own", row_start=None, held=None, n_pages=None):
        b = self.b
        self.d_table = _dev(self.table)
        self.d_plan = torch.full((b.batch_plan_bytes(self.cfg, self.B, self.N),), 0x5A, dtype=torch.uint8, device="cuda")
        par = _dev(self.parent) if parent == "own" else None if parent is None else _dev(parent)
        free = _dev(self.free if free is None else free)
        b.batch_plan(self.cfg, _dev(row_start or self.row_start), _dev(held or self.held), par, self.P, self.d_table,
                     free, n_pages or self.n_pages, self.d_plan, self.N)
        torch.cuda.synchronize()
        return b.batch_plan_views(self.cfg, self.B, self.N, self.d_plan)

    def pages(self, fill=None):
        shape = (self.L, self.n_pages, self.Hkv)
        g = torch.Generator(device="cuda").manual_seed(5)
        kp = torch.randn(*shape, PAGE, self.Dh, device="cuda", generator=g).to(torch.bfloat16)
        vp = torch.randn(*shape, self.Dh, PAGE, device="cuda", generator=g).to(torch.bfloat16)
        if fill is not None:  # everything a request's tokens do not cover
            free = torch.ones(self.n_pages, PAGE, dtype=torch.bool, device="cuda")
            table = self.d_table.cpu().numpy()
            for b in range(self.B):
                for t in range(self.held[b] + self.n[b]):
                    free[int(table[b, t // PAGE]), t % PAGE] = False
            kp.masked_fill_(free[None, :, None, :, None], fill)
            vp.masked_fill_(free[None, :, None, None, :], fill)
        return kp, vp


def _check_plan(got, want, table):
    for name in ("slot", "position", "status"):
        np.testing.assert_array_equal(got[name].cpu().numpy(), want[name], err_msg=name)
    assert int(got["taken"].item()) == want["taken"]
    np.testing.assert_array_equal(got["mask"].cpu().numpy().view(np.uint32), ob.mask_words(want["ancestors"]))
    np.testing.assert_array_equal(table.cpu().numpy(), want["block_table"])
    np.testing.assert_allclose(got["rope"].cpu().numpy(), want["rope"], atol=2.0 ** -21, rtol=0)


@pytest.mark.parametrize("n,held,P,kw", [
    ([1], [0], 0, {}),
    ([31], [200], 512, {}),
    ([128], [63], 1, {}),                      # three pages
    ([128, 1, 0, 64, 65], [0, 64, 999, 128, 127], 2048, {"pad": 300}),
    ([3, 0, 0, 5], [1, 0, 64, 0], 7, {"tree": False, "pad": 1}),
    ([0, 0], [5, 0], 3, {"pad": 4}),           # nothing but padding
    ([2] * 1024, list(range(1024)), 100000, {"Dh": 128}),
    ([17, 128, 128, 41], [4000, 64, 1, 2047], 1 << 29, {"Dh": 128}),
])
def test_plan(binding, n, held, P, kw):
    c = Case(binding, n, held, P=P, **kw)
    got = c.plan()
    _check_plan(got, c.want(), c.d_table)
    again = c.d_plan.clone()
    table = c.d_table.clone()
    binding.batch_plan(c.cfg, _dev(c.row_start), _dev(c.held), _dev(c.parent), P, c.d_table, _dev(c.free), c.n_pages,
                       c.d_plan, c.N)
    assert torch.equal(table, c.d_table)  # (the same arguments give the same plan)
    for name, view in binding.batch_plan_views(c.cfg, c.B, c.N, again).items():
        assert torch.equal(view, got[name]), name


def test_plan_chains_without_parents(binding):
    c = Case(binding, [128, 5, 1], [10, 0, 64])
    _check_plan(c.plan(parent=None), c.want(parent=None), c.d_table)


@pytest.mark.parametrize("what", ["free_short", "free_none", "free_bad", "table_bad", "table_narrow", "tree_root", "tree_late",
                                  "falling", "negative_start", "past_rows", "too_many", "negative_held", "huge_held"])
def test_plan_that_cannot_be(binding, what):
    # (bad values reach the kernel only through its own checks; none is used as an index)
    c = Case(binding, [4, 70, 3, 2], [62, 0, 130, 64], pad=2, spare=0)
    kw = {}
    if what == "free_short":
        kw["free"] = c.free[:2]
    elif what == "free_none":
        kw["free"] = []
    elif what == "free_bad":
        kw["free"] = [c.free[0], c.n_pages] + c.free[2:]
    elif what == "table_bad":
        c.table[2, 2] = -5
    elif what == "table_narrow":
        c.table = c.table[:, :2].copy()
    elif what == "tree_root":
        kw["parent"] = [0] + c.parent[1:]
    elif what == "tree_late":
        kw["parent"] = c.parent[:10] + [60] + c.parent[11:]
    elif what == "falling":
        kw["row_start"] = [0, 74, 4, 77, 79]
    elif what == "negative_start":
        kw["row_start"] = [-1, 4, 74, 77, 79]
    elif what == "past_rows":
        kw["row_start"] = [0, 4, 74, 77, c.N + 1]
    elif what == "too_many":
        kw["row_start"] = [0, 0, 0, 0, c.N]
        c2 = Case(binding, [1, 1, 1, 129], [62, 0, 130, 64])
        c = c2
        kw["row_start"] = c.row_start
    elif what == "negative_held":
        kw["held"] = [62, -1, 130, 64]
    elif what == "huge_held":
        kw["held"] = [62, 0, 2 ** 31 - 1, 64]
    want = c.want(**{k: v for k, v in kw.items()})
    assert want["status"].any()
    _check_plan(c.plan(**kw), want, c.d_table)


@pytest.mark.parametrize("P,n,placed", [((1 << 30) - 1, 1, True), ((1 << 30) - 1, 2, False), (1 << 30, 1, False), ((1 << 30) - 2, 2, True)])
def test_plan_at_the_last_position(binding, P, n, placed):
    """Positions up to 2^31 - 1, those behind them refused."""
    held, columns = 1 << 30, (1 << 24) + 1
    cfg = _cfg(binding, 2, 64)
    table = torch.full((1, columns), -1, dtype=torch.int32, device="cuda")
    plan = torch.full((binding.batch_plan_bytes(cfg, 1, n),), 0x5A, dtype=torch.uint8, device="cuda")
    binding.batch_plan(cfg, _dev([0, n]), _dev([held]), None, P, table, _dev([3]), 4, plan, n)
    got = binding.batch_plan_views(cfg, 1, n, plan)
    assert got["status"].tolist() == [binding.PLAN_OK if placed else binding.PLAN_NO_PAGES]
    assert got["position"].tolist() == ([P + held + i for i in range(n)] if placed else [0] * n)
    assert got["slot"].tolist() == ([3 * PAGE + i for i in range(n)] if placed else [-1] * n)
    assert int(table[0, -1]) == (3 if placed else -1)
    if placed:
        ang = np.array(got["position"].tolist(), dtype=np.float64)[:, None] * THETA ** (-2.0 * np.arange(32) / 64)
        np.testing.assert_allclose(got["rope"].cpu().numpy(), np.stack([np.cos(ang), np.sin(ang)], -1), atol=2.0 ** -20, rtol=0)


def _strided(t, gap):
    """A copy of t [N, heads, Dh] whose rows lie `gap` elements further apart."""
    N, h, d = t.shape
    buf = torch.full((N, h * d + gap), 3.0, dtype=t.dtype, device=t.device)
    buf[:, :h * d] = t.reshape(N, -1)
    return buf[:, :h * d].view(N, h, d) if gap == 0 else torch.as_strided(buf, (N, h, d), (h * d + gap, d, 1))


@pytest.mark.parametrize("n,held,kw", [
    ([1], [0], {}),
    ([1] * 8, [0, 1, 7, 8, 63, 64, 65, 300], {"Dh": 128}),
    ([31, 41, 5], [60, 3, 0], {"Dh": 128, "pad": 9}),
    ([128, 128, 128], [0, 4, 61], {"H": 8, "Hkv": 2}),
    ([64, 8, 16, 1], [0, 64, 8, 9], {"H": 6, "Hkv": 3, "pad": 1, "L": 2}),
    ([200 // 2, 0, 100], [1, 2, 3], {"H": 1, "Hkv": 1, "Dh": 128}),
])
@pytest.mark.parametrize("form", ["separate", "fused", "in_place"])
def test_store(binding, n, held, kw, form):
    c = Case(binding, n, held, P=1000, **kw)
    plan = c.plan()
    kp, vp = c.pages()
    k0, v0 = kp.clone(), vp.clone()
    layer = c.L - 1
    g = torch.Generator(device="cuda").manual_seed(9)
    qkv = torch.randn(c.N, c.H + 2 * c.Hkv, c.Dh, device="cuda", generator=g).to(torch.bfloat16)
    q, k, v = qkv[:, :c.H], qkv[:, c.H:c.H + c.Hkv], qkv[:, c.H + c.Hkv:]
    if form == "separate":
        q, k, v = _strided(q, 0), _strided(k, 24), _strided(v, 8)
    if form == "in_place":
        q = q.contiguous()
    q_in, k_in, v_in = _np(q), _np(k), _np(v)
    q_out = q if form == "in_place" else torch.full((c.N, c.H, c.Dh), 77.0, dtype=torch.bfloat16, device="cuda")
    before = _np(q_out)
    binding.batch_store(c.cfg, c.Hkv, layer, q, k, v, q_out, kp, vp, c.d_plan, c.B)
    torch.cuda.synchronize()
    rope = plan["rope"].cpu().numpy().astype(np.float64)
    slot = plan["slot"].cpu().numpy()

    def close(got, want, x):
        half = c.Dh // 2
        size = np.abs(x[..., :half]) + np.abs(x[..., half:])
        assert np.all(np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -20 * np.concatenate([size, size], -1))

    T = c.total
    close(_np(q_out)[:T], ob.turn(q_in, rope)[:T], q_in[:T])
    np.testing.assert_array_equal(_np(q_out)[T:], before[T:])
    rows = np.arange(T)
    got_k = _np(kp)[layer].transpose(0, 2, 1, 3).reshape(-1, c.Hkv, c.Dh)
    got_v = _np(vp)[layer].transpose(0, 3, 1, 2).reshape(-1, c.Hkv, c.Dh)
    close(got_k[slot[rows]], ob.turn(k_in, rope)[:T], k_in[:T])
    np.testing.assert_array_equal(got_v[slot[rows]], v_in[:T])
    # nothing else moved
    other = np.setdiff1d(np.arange(c.n_pages * PAGE), slot[rows])
    old_k = _np(k0)[layer].transpose(0, 2, 1, 3).reshape(-1, c.Hkv, c.Dh)
    old_v = _np(v0)[layer].transpose(0, 3, 1, 2).reshape(-1, c.Hkv, c.Dh)
    np.testing.assert_array_equal(got_k[other], old_k[other])
    np.testing.assert_array_equal(got_v[other], old_v[other])
    if layer:
        assert torch.equal(kp[:layer], k0[:layer]) and torch.equal(vp[:layer], v0[:layer])


def _attend(c, plan, q, kc, vc, kp, vp, layer=0, out=None, table=None):
    b = c.b
    ws = torch.full((b.batch_workspace_bytes(c.cfg, c.Hkv, c.B, c.N),), 0xFF, dtype=torch.uint8, device="cuda")
    out = torch.full((c.N, c.H, c.Dh), 77.0, dtype=torch.bfloat16, device="cuda") if out is None else out
    b.batch_attention(c.cfg, c.Hkv, layer, q, kc, vc, c.P, kp, vp, c.d_table if table is None else table, c.d_plan, out, ws)
    torch.cuda.synchronize()
    return out


def _check_attention(c, q, kc, vc, kp, vp, out, layer=0, table=None):
    pk = np.zeros((c.Hkv, 0, c.Dh)) if kc is None else _np(kc[layer])[:, :c.P]
    pv = pk if vc is None else _np(vc[layer].transpose(1, 2))[:, :c.P]
    anc = c.want()["ancestors"]
    table = c.d_table if table is None else table
    want, size = ob.attention(_np(q), pk, pv, _np(kp[layer]), _np(vp[layer].transpose(2, 3)), table.cpu().numpy(),
                              c.row_start, c.held, anc, c.n_pages)
    got = _np(out)
    T = c.total
    err = np.abs(got[:T] - want[:T])
    tol = 2.0 ** -8 * np.abs(want[:T]) + (2.0 ** -8 + 2.0 ** -11) * size[:T]
    worst = np.unravel_index(np.argmax(err - tol), err.shape) if err.size else None
    assert np.all(err <= tol), (worst, got[:T][worst], want[:T][worst], size[:T][worst])
    assert np.all(got[T:] == 77.0)


def _prefix(c, fill=None, room=0, scale=1.0):
    if c.P == 0:
        return None, None
    cap = (c.P + 63) // 64 * 64 + room
    g = torch.Generator(device="cuda").manual_seed(3)
    kc = (torch.randn(c.L, c.Hkv, cap, c.Dh, device="cuda", generator=g) * scale).to(torch.bfloat16)
    vc = torch.randn(c.L, c.Hkv, c.Dh, cap, device="cuda", generator=g).to(torch.bfloat16)
    if fill is not None:
        kc[:, :, c.P:] = fill
        vc[..., c.P:] = fill
    return kc, vc


def _queries(c, scale=1.5, gap=0):
    g = torch.Generator(device="cuda").manual_seed(4)
    q = (torch.randn(c.N, c.H, c.Dh, device="cuda", generator=g) * scale).to(torch.bfloat16)
    return _strided(q, gap)


CASES = [
    ([1], [0], 0, {}),                                         # a row that sees itself alone
    ([1], [0], 1, {"Dh": 128}),
    ([1], [64], 512, {"Dh": 128, "H": 2}),
    ([1, 1, 1], [0, 31, 32], 31, {}),
    ([2, 1, 3], [33, 64, 127], 33, {"H": 6, "Hkv": 2}),
    ([31], [200], 300, {"Dh": 128, "H": 2}),
    ([128, 41], [63, 0], 65, {"Dh": 128, "H": 2}),
    ([17, 0, 16, 15, 1], [5, 500, 0, 64, 129], 129, {"pad": 5}),
    ([1] * 20, list(range(0, 400, 20)), 700, {"H": 16, "Hkv": 2, "Dh": 128, "tree": False, "pad": 3}),
    ([5, 7], [0, 0], 0, {"H": 8, "Hkv": 1}),
    ([33, 31, 64], [10, 70, 100], 64, {"H": 3, "Hkv": 3}),
    ([9] * 12, [3] * 12, 1500, {"H": 12, "Hkv": 4, "Dh": 128}),
    ([128] * 3, [1, 2, 3], 200, {"H": 4, "Hkv": 1, "Dh": 128}),
    ([1], [3000], 0, {"H": 2, "Dh": 128}),                     # a long request alone
    ([41, 1, 1, 1], [900, 0, 1, 2], 500, {"H": 4, "Hkv": 2}),  # ... and beside short ones
    ([1] * 130, [0] * 130, 40, {"H": 2}),
]


@pytest.mark.parametrize("n,held,P,kw", CASES)
def test_attention(binding, n, held, P, kw):
    c = Case(binding, n, held, P=P, **kw)
    plan = c.plan()
    kp, vp = c.pages()
    kc, vc = _prefix(c, room=64)
    q = _queries(c, gap=16)
    out = _attend(c, plan, q, kc, vc, kp, vp)
    _check_attention(c, q, kc, vc, kp, vp, out)
    assert torch.equal(out, _attend(c, plan, q, kc, vc, kp, vp))  # (the same bits every time)


@pytest.mark.parametrize("n,held,P,kw", [CASES[0], CASES[4], CASES[6], CASES[7], CASES[8], CASES[11], CASES[12]])
@pytest.mark.parametrize("fill", [float("nan"), float("inf"), float("-inf"), torch.finfo(torch.bfloat16).min])
def test_attention_unseen_slots_do_not_matter(binding, n, held, P, kw, fill):
    c = Case(binding, n, held, P=P, **kw)
    c.plan()
    kp, vp = c.pages(fill=fill)
    kc, vc = _prefix(c, fill=fill)
    q = _queries(c)
    out = _attend(c, None, q, kc, vc, kp, vp)
    _check_attention(c, q, kc, vc, torch.nan_to_num(kp, 0, 0, 0), torch.nan_to_num(vp, 0, 0, 0), out)


@pytest.mark.parametrize("fill", [float("nan"), float("inf")])
@pytest.mark.parametrize("Dh,H,Hkv", [(64, 2, 2), (128, 4, 1)])
def test_attention_of_a_sibling_with_bad_values(binding, fill, Dh, H, Hkv):
    # node 2 of the first request holds NaN / Inf: only its own branch may show it
    c = Case(binding, [40, 3], [30, 5], H=H, Hkv=Hkv, Dh=Dh, P=70)
    plan = c.plan()
    anc = c.want()["ancestors"]
    kp, vp = c.pages()
    s = int(plan["slot"][2].item())
    vp[0, s // PAGE, :, :, s % PAGE] = fill
    kc, vc = _prefix(c)
    q = _queries(c)
    out = _np(_attend(c, plan, q, kc, vc, kp, vp))
    clean = vp.clone()
    clean[0, s // PAGE, :, :, s % PAGE] = 0
    ref = _np(_attend(c, plan, q, kc, vc, kp, clean))
    for r in range(c.total):
        if r < 40 and 2 in anc[r]:
            assert not np.isfinite(out[r]).any(), r
        else:
            np.testing.assert_array_equal(out[r], ref[r])


@pytest.mark.parametrize("scale", [0.0, 30.0])
def test_attention_flat_and_sharp(binding, scale):
    # all scores equal; scores of hundreds, where the softmax takes one key
    c = Case(binding, [6, 33], [50, 100], P=257, H=2, Dh=128)
    c.plan()
    kp, vp = c.pages()
    kc, vc = _prefix(c)
    q = _queries(c, scale=scale)
    if scale:  # (one fp32 rounding of a score of 2^9 is 2^-15; 128 of them at most: 2^-8 of a probability)
        out = _np(_attend(c, None, q, kc, vc, kp, vp))
        anc = c.want()["ancestors"]
        want, size = ob.attention(_np(q), _np(kc[0])[:, :c.P], _np(vc[0].transpose(1, 2))[:, :c.P], _np(kp[0]),
                                  _np(vp[0].transpose(2, 3)), c.d_table.cpu().numpy(), c.row_start, c.held, anc, c.n_pages)
        assert np.all(np.abs(out - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -6 * size)
    else:
        _check_attention(c, q, kc, vc, kp, vp, _attend(c, None, q, kc, vc, kp, vp))


def test_attention_absent_pages_and_unplaced_requests(binding):
    c = Case(binding, [3, 20, 2], [130, 70, 64], P=40, H=4, Hkv=2, Dh=64)
    c.plan()
    kp, vp = c.pages()
    kc, vc = _prefix(c)
    q = _queries(c)
    table = c.d_table.clone()
    table[0, 1], table[1, 0] = -1, c.n_pages  # tokens 64..127 of request 0, 0..63 of request 1 are absent
    out = _attend(c, None, q, kc, vc, kp, vp, table=table)
    _check_attention(c, q, kc, vc, kp, vp, out, table=table)
    # request 1 cannot be placed: its rows stay as they were, the others' do not
    c.plan(parent=c.parent[:4] + [3] + c.parent[5:])
    out = _np(_attend(c, None, q, kc, vc, kp, vp))
    assert np.all(out[3:23] == 77.0) and np.all(out[:3] != 77.0) and np.all(out[23:25] != 77.0)


def test_attention_row_that_sees_nothing(binding):
    # every page of the request is absent and there is no prefix: zeros
    c = Case(binding, [5], [64], H=2)
    c.plan()
    kp, vp = c.pages()
    out = _np(_attend(c, None, _queries(c), None, None, kp, vp, table=torch.full_like(c.d_table, -1)))
    assert np.all(out == 0.0)


def test_attention_layers_and_streams(binding):
    c = Case(binding, [7, 7], [20, 90], P=100, H=4, Hkv=2, Dh=64, L=3)
    c.plan()
    kp, vp = c.pages()
    kc, vc = _prefix(c)
    q = _queries(c)
    want = [_attend(c, None, q, kc, vc, kp, vp, layer=l) for l in range(3)]
    for l in range(3):
        _check_attention(c, q, kc, vc, kp, vp, want[l], layer=l)
    assert not torch.equal(want[0], want[1])
    side = torch.cuda.Stream()
    out = torch.full_like(want[0], 77.0)
    ws = torch.zeros(binding.batch_workspace_bytes(c.cfg, c.Hkv, c.B, c.N), dtype=torch.uint8, device="cuda")
    side.wait_stream(torch.cuda.current_stream())
    binding.batch_attention(c.cfg, c.Hkv, 1, q, kc, vc, c.P, kp, vp, c.d_table, c.d_plan, out, ws, stream=side)
    side.synchronize()
    assert torch.equal(out, want[1])


@pytest.mark.parametrize("n,held,P", [
    (128, 83210, 1),    # tiles: runs of 82 pages
    (16, 614401, 100),  # few rows: runs of 76 pages
])
def test_attention_of_long_runs(binding, n, held, P):
    """A request whose pages are cut into runs of more than 64 pages."""
    c = Case(binding, [n], [held], P=P, H=1, Dh=64, tree=True)
    c.plan()
    kp, vp = c.pages()
    kc, vc = _prefix(c)
    q = _queries(c)
    out = _attend(c, None, q, kc, vc, kp, vp)
    ids = c.d_table[0, :-(-(held + n) // PAGE)].long()
    k = torch.cat([kc[0, 0, :P], kp[0, ids, 0].reshape(-1, c.Dh)[:held + n]]).double()
    v = torch.cat([vc[0, 0, :, :P].t(), vp[0, ids, 0].transpose(1, 2).reshape(-1, c.Dh)[:held + n]]).double()
    see = torch.ones(n, P + held + n, dtype=torch.bool)
    see[:, P + held:] = False
    for r, a in enumerate(c.want()["ancestors"]):
        see[r, [P + held + j for j in a]] = True
    z = (q[:n, 0].double() @ k.t()) / 8.0
    w = torch.softmax(z.masked_fill(~see.cuda(), -float("inf")), 1)
    want, size = _np((w @ v).cpu().double()), _np((w @ v.abs()).cpu().double())
    got = _np(out)[:n, 0]
    assert np.all(np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2.0 ** -11) * size)


@pytest.mark.parametrize("n,held,P,kw", [
    ([1, 2, 3, 4] * 256, [(7 * i) % 130 for i in range(1024)], 70, {"H": 2, "Hkv": 1}),      # more rows than kSplitRows
    ([128, 127, 120], [0, 1, 64], 129, {"H": 64}),                                      # one split of the prefix
    ([40, 1, 16, 17, 2], [700, 900, 0, 64, 3], 1000, {"H": 16, "Hkv": 16, "Dh": 128}),      # tiles and few rows side by side
    ([3, 1], [5000, 1], 0, {"H": 48, "Hkv": 48}),                                           # runs joined for many K/V heads
])
def test_attention_of_many(binding, n, held, P, kw):
    c = Case(binding, n, held, P=P, **kw)
    c.plan()
    kp, vp = c.pages()
    kc, vc = _prefix(c)
    q = _queries(c)
    _check_attention(c, q, kc, vc, kp, vp, _attend(c, None, q, kc, vc, kp, vp))


def test_two_steps_at_once(binding):
    """Two steps on two streams, each with its own plan and workspace, over one prefix."""
    cases = [Case(binding, [31, 2, 9], [700, 5, 64], P=700, H=8, Hkv=4, Dh=128, seed=i) for i in range(2)]
    kc, vc = _prefix(cases[0])
    state, want = [], []
    for c in cases:
        c.plan()
        kp, vp = c.pages()
        state.append((c, kp, vp, _queries(c)))
        want.append(_attend(c, None, state[-1][3], kc, vc, kp, vp))
    streams = [torch.cuda.Stream() for _ in cases]
    outs = [torch.empty_like(w) for w in want]
    spaces = [torch.zeros(binding.batch_workspace_bytes(c.cfg, c.Hkv, c.B, c.N), dtype=torch.uint8, device="cuda") for c in cases]
    torch.cuda.synchronize()
    for _ in range(20):
        for i, (c, kp, vp, q) in enumerate(state):
            binding.batch_attention(c.cfg, c.Hkv, 0, q, kc, vc, c.P, kp, vp, c.d_table, c.d_plan, outs[i], spaces[i],
                                    stream=streams[i])
    torch.cuda.synchronize()
    for i, c in enumerate(cases):
        assert torch.equal(outs[i][:c.total], want[i][:c.total])


def test_attention_beyond_32_bit_offsets(binding):
    # a pool of more than 2^32 bytes (and 2^31 elements): the request's pages at its two ends
    c = Case(binding, [3], [100], H=32, Dh=128, P=10)
    c.n_pages = 8300  # 8300 x 32 x 64 x 128 elements = 2.18e9
    c.table[0, :2] = [8299, 1]
    c.d_table = _dev(c.table)
    c.plan()
    kp = torch.zeros(1, c.n_pages, 32, PAGE, 128, dtype=torch.bfloat16, device="cuda")
    vp = torch.zeros(1, c.n_pages, 32, 128, PAGE, dtype=torch.bfloat16, device="cuda")
    kp[0, [8299, 1]] = torch.randn(2, 32, PAGE, 128, device="cuda").to(torch.bfloat16)
    vp[0, [8299, 1]] = torch.randn(2, 32, 128, PAGE, device="cuda").to(torch.bfloat16)
    kc, vc = _prefix(c)
    q = _queries(c)
    out = _attend(c, None, q, kc, vc, kp, vp)
    small = Case(binding, [3], [100], H=32, Dh=128, P=10)
    small.n_pages, small.table[0, :2] = 2, [0, 1]
    small.plan()
    ref = _attend(small, None, q, kc, vc, kp[:, [8299, 1]].contiguous(), vp[:, [8299, 1]].contiguous())
    assert torch.equal(out, ref)
    k = torch.randn(3, 32, 128, device="cuda").to(torch.bfloat16)
    binding.batch_store(c.cfg, 32, 0, q, k, k, torch.empty_like(q), kp, vp, c.d_plan, 1)
    slot = int(binding.batch_plan_views(c.cfg, 1, c.N, c.d_plan)["slot"][0])
    assert slot == 64 + 36 and torch.equal(vp[0, 1, :, :, 36], k[0])


@pytest.mark.parametrize("n,held,kw", [
    ([4], [0], {}),
    ([31, 1, 41, 0, 7], [60, 5, 3, 2, 128], {"Dh": 128, "L": 3, "H": 2}),
    ([128, 128], [1, 63], {"H": 4, "Hkv": 2, "L": 2, "tree": False}),
    ([9] * 200, [(11 * i) % 140 for i in range(200)], {"H": 7, "L": 5}),  # several heads per workgroup, not all of them full
    ([128, 80], [7, 64], {"H": 2, "Dh": 128}),                            # more moves than lanes
])
@pytest.mark.parametrize("kind", ["branch", "shift", "bad", "none"])
def test_commit(binding, n, held, kw, kind):
    c = Case(binding, n, held, **kw)
    plan = c.plan()
    kp, vp = c.pages()
    path, acc = [], []
    anc = c.want()["ancestors"]
    for b, m in enumerate(n):
        r0 = c.row_start[b]
        p = []
        if m:
            p = {"branch": anc[r0 + c.rng.integers(m)], "shift": [0] + list(range(2, m)), "bad": list(range(m)),
                 "none": [0]}[kind]
        if kind == "bad":  # entries out of range, and a path that goes backwards
            p = [x if i % 3 else (m + 5 if i % 2 else -9) for i, x in enumerate(p)][::-1]
        acc.append(len(p) - 1 if kind != "bad" else (m - 1 if b % 2 == 0 else m + 3))
        path += p + [-1] * (m - len(p))
    k0, v0 = kp.clone(), vp.clone()
    binding.batch_commit(c.cfg, c.Hkv, kp, vp, c.d_plan, c.B, _dev(path), _dev(acc))
    torch.cuda.synchronize()
    rows = lambda t: _np(t).reshape(c.L, -1, c.Hkv * c.Dh)  # noqa: E731
    want_k, want_v = ob.commit(c.row_start, plan["slot"].cpu().numpy(), path, acc, rows(k0.transpose(2, 3)),
                               rows(v0.permute(0, 1, 4, 2, 3)))
    np.testing.assert_array_equal(rows(kp.transpose(2, 3)), want_k)
    np.testing.assert_array_equal(rows(vp.permute(0, 1, 4, 2, 3)), want_v)


def test_step_in_a_graph(binding):
    """A captured step (plan, store, attention) replayed while the requests grow, other eager work and
    another captured step on the same workspace between the replays: every replay equals the eager step."""
    n, L = [3, 1, 5], 1
    c = Case(binding, n, [60, 0, 200], P=90, H=4, Hkv=2, Dh=64, pad=4, tree=True)
    B, N = c.B, c.N
    row_start, held, parent = _dev(c.row_start), _dev(c.held), _dev(c.parent)
    width = 8
    table = torch.full((B, width), -1, dtype=torch.int32, device="cuda")
    table[:, :c.width] = _dev(c.table)
    n_pages = 32
    used = set(c.table[c.table >= 0].tolist())
    free = _dev([p for p in range(n_pages) if p not in used])
    g = torch.Generator(device="cuda").manual_seed(8)
    kp = torch.randn(L, n_pages, 2, PAGE, 64, device="cuda", generator=g).to(torch.bfloat16)
    vp = torch.randn(L, n_pages, 2, 64, PAGE, device="cuda", generator=g).to(torch.bfloat16)
    kc, vc = _prefix(c)
    qkv = torch.randn(N, 8, 64, device="cuda", generator=g).to(torch.bfloat16)
    ws = torch.zeros(binding.batch_workspace_bytes(c.cfg, 2, B, N), dtype=torch.uint8, device="cuda")
    plan = torch.zeros(binding.batch_plan_bytes(c.cfg, B, N), dtype=torch.uint8, device="cuda")
    q, out = torch.zeros(N, 4, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(N, 4, 64, dtype=torch.bfloat16, device="cuda")

    def step(plan, table, kp, vp, q, out, ws, heads=slice(0, 4)):
        binding.batch_plan(c.cfg, row_start, held, parent, c.P, table, free, n_pages, plan, N)
        binding.batch_store(c.cfg, 2, 0, qkv[:, :4], qkv[:, 4:6], qkv[:, 6:], q, kp, vp, plan, B)
        binding.batch_attention(c.cfg, 2, 0, q, kc, vc, c.P, kp, vp, table, plan, out, ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    first = (plan, table, kp, vp, q, out)
    second = tuple(x.clone() for x in first)
    with torch.cuda.stream(side):
        graphs = []
        for args in (first, second):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                step(*args, ws)
            graphs.append(graph)
    torch.cuda.current_stream().wait_stream(side)
    for turn in range(4):
        eager = tuple(x.clone() for x in first)
        eager[5].fill_(-1)
        ews = torch.full_like(ws, turn)
        step(*eager, ews)
        torch.cuda.synchronize()
        for graph, args in zip(graphs, (first, second)):
            args[5].fill_(-1)
            graph.replay()
        torch.cuda.synchronize()
        total = c.total
        for args in (first, second):
            assert torch.equal(args[5][:total], eager[5][:total]), turn
            assert torch.equal(args[1], eager[1]) and torch.equal(args[3], eager[3])
        assert int(binding.batch_plan_views(c.cfg, B, N, plan)["status"].sum()) == 0
        held.add_(_dev(n))  # (the requests grow, the first one into a new page)
        qkv.mul_(-1)
        taken = int(binding.batch_plan_views(c.cfg, B, N, plan)["taken"])
        free.copy_(torch.roll(free, -taken))


def test_plan_of_other_sizes_is_not_used(binding):
    """Operators called with other counts than the plan's, or with a buffer that holds none, write nothing."""
    c = Case(binding, [5, 20, 3], [70, 10, 64], P=40, H=4, Hkv=2, Dh=64)
    c.plan()
    kp, vp = c.pages()
    kc, vc = _prefix(c)
    q = _queries(c)
    k0, v0 = kp.clone(), vp.clone()
    path = _dev([0] + list(range(2, c.N + 1)))
    x = torch.randn(c.N, 2, 64, device="cuda").to(torch.bfloat16)
    qo = torch.full_like(q, 5.0)
    good = c.d_plan
    for plan, B in ((good, 2), (torch.zeros_like(good), 3), (torch.full_like(good, 0x5A), 3)):
        c.d_plan = plan
        out = _attend(c, None, q, kc, vc, kp, vp, table=c.d_table[:B].contiguous())
        assert bool((out == 77.0).all())
        binding.batch_store(c.cfg, 2, 0, q, x, x, qo, kp, vp, plan, B)
        binding.batch_commit(c.cfg, 2, kp, vp, plan, B, path, _dev([2] * B))
        torch.cuda.synchronize()
        assert bool((qo == 5.0).all()) and torch.equal(kp, k0) and torch.equal(vp, v0)


def test_attention_with_a_narrower_table_than_the_plans(binding):
    """The plan's runs of pages past the table would have no workgroup: all is left as it was.  A wider table serves."""
    c = Case(binding, [5, 3], [700, 10], P=40, H=4, Hkv=2, Dh=64)
    c.plan()
    kp, vp = c.pages()
    kc, vc = _prefix(c)
    q = _queries(c)
    want = _attend(c, None, q, kc, vc, kp, vp)
    out = _attend(c, None, q, kc, vc, kp, vp, table=c.d_table[:, :4].contiguous())
    assert bool((out == 77.0).all())
    wider = torch.cat([c.d_table, torch.full_like(c.d_table, 1 << 30)], 1)
    assert torch.equal(_attend(c, None, q, kc, vc, kp, vp, table=wider), want)


def test_batch_keeps_its_pages(binding):
    """Many steps whose trees are mostly rejected: trimmed, the pool loses no page; a request that
    cannot be placed is reported."""
    import workloads

    shape = workloads.MODELS["tiny"]
    b = binding.Batch(shape, 3, 96, n_pages=9, max_pages=6)
    held = torch.tensor([0, 60, 100], dtype=torch.int32, device="cuda")
    b.plan(_dev([0, 0, 60, 96]), _dev([0, 0, 65]))
    assert b.status.tolist() == [0, 0, binding.PLAN_NO_PAGES]  # (the page of its 65th token is not in its table)
    with pytest.raises(RuntimeError):
        b.advance()
    b.block_table.fill_(-1)
    b.block_table[1, 0], b.block_table[2, 0], b.block_table[2, 1] = 0, 1, 2
    b.free_pages = _dev(range(3, 9))
    for step in range(12):
        b.plan(_dev([0, 30, 60, 90]), held)
        assert not b.status.any()
        b.advance()
        used = b.block_table[b.block_table >= 0].tolist()
        assert sorted(used + b.free_pages.tolist()) == list(range(9)), step
        held += _dev([1, 2, 3])
        b.trim(held)
        used = b.block_table[b.block_table >= 0].tolist()
        assert sorted(used + b.free_pages.tolist()) == list(range(9)), step
        assert len(used) == sum(-(-int(h) // PAGE) for h in held)
    b.release(2)
    assert len(b.free_pages) == 9 - 1 - 2  # (12 and 84 tokens are held by the others)


def test_refusals_of_the_binding(binding):
    c = Case(binding, [2, 1], [5, 0], P=10, H=2, Dh=128)
    c.plan()
    kp, vp = c.pages()
    kc, vc = _prefix(c)
    q = _queries(c)
    out = torch.empty_like(q)
    ws = torch.zeros(binding.batch_workspace_bytes(c.cfg, 2, 2, c.N), dtype=torch.uint8, device="cuda")

    def attention(**kw):
        a = dict(q=q, kc=kc, vc=vc, P=c.P, kp=kp, vp=vp, table=c.d_table, plan=c.d_plan, out=out, ws=ws, Hkv=2, layer=0)
        a.update(kw)
        binding.batch_attention(c.cfg, a["Hkv"], a["layer"], a["q"], a["kc"], a["vc"], a["P"], a["kp"], a["vp"], a["table"],
                                a["plan"], a["out"], a["ws"])

    attention()
    for kw in (dict(q=q.float()), dict(q=q.transpose(0, 1)), dict(out=out[:, :1]), dict(kp=kp.transpose(3, 4)), dict(vp=kp),
               dict(table=c.d_table.long()), dict(plan=c.d_plan.view(torch.int32)), dict(kc=kc.cpu()), dict(kc=kc[..., :32]),
               dict(q=q[:, :, ::2])):
        with pytest.raises(ValueError):
            attention(**kw)
    for kw, status in ((dict(P=65), binding.ECAPACITY), (dict(kc=None, vc=None), binding.EARG), (dict(ws=ws[:256]), binding.EWORKSPACE),
                       (dict(plan=c.d_plan[:256]), binding.EWORKSPACE), (dict(layer=1), binding.EARG), (dict(P=-1), binding.ECAPACITY)):
        with pytest.raises(binding.LlmcadError) as e:
            attention(**kw)
        assert e.value.status == status, kw
