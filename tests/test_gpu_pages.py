"""Forked requests and compacted pools against their plain statement (oracle/batch.py): tables, lengths, free
lists and every page's bits."""

import numpy as np
import pytest
import torch

from oracle import batch as ob
from test_gpu_batch import PAGE, _cfg, _dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def binding():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2309_04255_amd import binding

    return binding


class Pool:
    def __init__(self, binding, held, spare=5, L=2, Hkv=2, Dh=64, H=None, width=None, seed=0, n_pages=None):
        rng = np.random.default_rng(seed)
        self.rng, self.b, self.held, self.B = rng, binding, list(held), len(held)
        have = [-(-h // PAGE) for h in held]
        self.n_pages = n_pages or sum(have) + spare
        self.table = np.full((self.B, width or max(max(have), 1) + 1), -1)
        order = rng.permutation(self.n_pages).tolist()
        for b in range(self.B):
            self.table[b, :have[b]] = [order.pop() for _ in range(have[b])]
        self.cfg, self.Hkv = _cfg(binding, H or Hkv, Dh, L), Hkv
        g = torch.Generator(device="cuda").manual_seed(seed)
        shape = (L, self.n_pages, Hkv)
        self.k = torch.randint(-2**15, 2**15, (*shape, PAGE, Dh), device="cuda", generator=g, dtype=torch.int16).view(torch.bfloat16)
        self.v = torch.randint(-2**15, 2**15, (*shape, Dh, PAGE), device="cuda", generator=g, dtype=torch.int16).view(torch.bfloat16)
        self.work = torch.full((binding.batch_pages_workspace_bytes(self.B, self.n_pages),), 0x5A, dtype=torch.uint8, device="cuda")

    def moved(self, copies):
        """The pages' bits after (page, new page, tokens) copies."""
        k, v = self.k.view(torch.int16).clone(), self.v.view(torch.int16).clone()
        if copies:
            src, dst = (torch.tensor([int(c[i]) for c in copies], device="cuda") for i in (0, 1))
            filled = torch.arange(PAGE, device="cuda") < torch.tensor([c[2] for c in copies], device="cuda")[:, None]
            k[:, dst] = torch.where(filled[None, :, None, :, None], k[:, src], k[:, dst])
            v[:, dst] = torch.where(filled[None, :, None, None, :], v[:, src], v[:, dst])
        return k, v

    def fork(self, source, held=None, stream=None):
        held = self.held if held is None else held
        table, lengths = torch.full_like(_dev(self.table), -7), torch.full((self.B,), -7, dtype=torch.int32, device="cuda")
        free = torch.full((self.n_pages,), -7, dtype=torch.int32, device="cuda")
        n_free, status = self.b.batch_fork(self.cfg, self.Hkv, self.k, self.v, _dev(self.table), _dev(held), _dev(source), table,
                                           lengths, free, self.work, stream=stream)
        torch.cuda.synchronize()
        return table.cpu().numpy(), lengths.tolist(), free.tolist(), int(n_free), int(status)

    def check_fork(self, source, held=None):
        want = ob.fork(self.table, self.held if held is None else held, source, self.n_pages)
        k, v = self.moved(want["copies"] if want["status"] == 0 else [])
        table, lengths, free, n_free, status = self.fork(source, held)
        assert status == want["status"]
        np.testing.assert_array_equal(table, want["block_table"])
        assert lengths == list(want["held"])
        assert n_free == len(want["free"]) and free == want["free"] + [-1] * (self.n_pages - n_free)
        assert torch.equal(self.k.view(torch.int16), k) and torch.equal(self.v.view(torch.int16), v)
        return want


@pytest.mark.parametrize("held,source,kw", [
    ([5], [0], {}), ([0], [0], {}), ([70], [-1], {}),
    ([150, 0, 0, 0], [0, 0, 0, 0], {}),                              # four answers to one prompt
    ([128, 0, 0], [0, 0, 0], {}),                                    # full pages alone: nothing is copied
    ([1, 63, 64, 65], [1, 0, 3, 2], {}),                             # two pairs change places
    ([130, 131, 132, 133], [1, 2, 3, 0], {"Dh": 128}),               # all of them
    ([130, 131, 132, 133], [3, 3, 3, 2], {"Dh": 128, "Hkv": 3}),     # beams: two end, one goes on twice
    ([200, 7, 90], [-1, 0, 0], {}),                                  # the first to come takes the page over
    ([9, 9, 9, 9], [-1, -1, -1, -1], {}),
    ([0, 0, 100], [2, 1, -5], {}),
    ([77] * 8, [0, 0, 0, 0, 4, 4, 4, 4], {"H": 8, "Hkv": 1, "L": 5}),
    ([33, 700, 1, 64], [1, 1, 0, 0], {"width": 3000}),               # a wide table
])
def test_fork(binding, held, source, kw):
    Pool(binding, held, **kw).check_fork(source)


@pytest.mark.parametrize("r", list(range(1, 64, 3)) + [63])
def test_fork_copies_what_the_page_holds(binding, r):
    """Every number of tokens in the last page; what lies behind them in the new one stays."""
    Pool(binding, [64 + r, 0], Dh=64 if r % 2 else 128, seed=r).check_fork([0, 0])


@pytest.mark.parametrize("seed", range(6))
def test_random_forks(binding, seed):
    rng = np.random.default_rng(seed)
    B = [1, 7, 64, 200, 1024, 300][seed]
    held = rng.integers(0, [500, 500, 300, 200, 100, 1][seed] + 1, B).tolist()
    source = np.where(rng.random(B) < 0.1, -1, np.where(rng.random(B) < 0.5, np.arange(B), rng.integers(0, B, B))).tolist()
    pool = Pool(binding, held, spare=B, L=1, Hkv=1, seed=seed)
    want = pool.check_fork(source)
    assert seed in (0, 5) or want["copies"]


def test_fork_without_room(binding):
    pool = Pool(binding, [100, 3, 0, 0], spare=1)
    assert pool.check_fork([0, 1, 0, 0])["status"] == ob.NO_PAGES
    assert pool.check_fork([0, 1, 0, 3])["status"] == ob.OK
    # pages of requests that end are free after the call, not for it
    pool = Pool(binding, [100, 130, 0], spare=0)
    assert pool.check_fork([0, -1, 0])["status"] == ob.NO_PAGES


@pytest.mark.parametrize("held,source", [([5, -1], [0, 1]), ([5, 1000], [0, 1]), ([5, 6], [0, 2]), ([5, 2**31 - 1], [0, 0])])
def test_fork_of_bad_lengths_or_sources(binding, held, source):
    pool = Pool(binding, [5, 6])
    assert pool.check_fork(source, held)["status"] == ob.BAD_LENGTHS


def test_entries_that_are_no_pages(binding):
    """Absent entries are passed on and copy nothing."""
    pool = Pool(binding, [200, 100, 0])
    pool.table[0, 1], pool.table[1, 1] = -1, pool.n_pages
    want = pool.check_fork([0, 0, 1])
    assert len(want["copies"]) == 1
    out, n_used, moves = ob.compact(pool.table, pool.held, pool.n_pages)
    _check_compact(pool)


def _check_compact(pool, held=None):
    held = pool.held if held is None else held
    want, n_used, moves = ob.compact(pool.table, held, pool.n_pages)
    k, v = pool.moved([(a, b, PAGE) for a, b in moves])
    table = torch.full_like(_dev(pool.table), -7)
    got = pool.b.batch_compact(pool.cfg, pool.Hkv, pool.k, pool.v, _dev(pool.table), _dev(held), table, pool.work)
    torch.cuda.synchronize()
    assert int(got) == n_used
    np.testing.assert_array_equal(table.cpu().numpy(), want)
    assert torch.equal(pool.k.view(torch.int16), k) and torch.equal(pool.v.view(torch.int16), v)
    return moves


@pytest.mark.parametrize("held,kw", [
    ([5], {}), ([0], {}), ([0, 0], {"spare": 1}), ([64], {"spare": 0}), ([65, 300], {"spare": 40}), ([1] * 9, {"spare": 200}),
    ([100, 0, 700, 64], {"spare": 11, "Dh": 128, "Hkv": 3}), ([1000] * 5, {"spare": 3, "L": 5, "H": 4, "Hkv": 1}),
    ([10] * 1024, {"spare": 5000, "L": 1, "Hkv": 1}), ([40, 90], {"width": 5000, "spare": 9}), ([31] * 20, {"n_pages": 32}), ([31] * 20, {"n_pages": 33}),
    ([130] * 11, {"n_pages": 64}), ([130] * 300, {"n_pages": 8191, "L": 1, "Hkv": 1}),
])
def test_compact(binding, held, kw):
    for seed in range(2):
        _check_compact(Pool(binding, held, seed=seed, **kw))


def test_compact_of_odd_lengths_and_shared_pages(binding):
    pool = Pool(binding, [100, 200, 300], spare=20)
    pool.table[1, :2] = pool.table[2, :2]  # (a prompt that two requests share)
    _check_compact(pool)
    _check_compact(pool, [-5, 1, 2**31 - 1])
    pool = Pool(binding, [100, 200, 300], spare=20, seed=3)
    _check_compact(pool, [64, 65, 0])  # (pages past the lengths are free)


def test_the_largest_pool(binding):
    """2^18 pages, the most that is taken; tables of a few requests all over it."""
    big = binding.MAX_POOL
    cfg = _cfg(binding, 1, 64, 1)
    k = torch.zeros(1, big, 1, PAGE, 64, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros(1, big, 1, 64, PAGE, dtype=torch.bfloat16, device="cuda")
    rng = np.random.default_rng(5)
    held = [64 * 1500, 64 * 700 + 5, 0, 1]
    pages = rng.permutation(big)[:1500 + 701 + 1]
    table = np.full((4, 1600), -1)
    table[0, :1500], table[1, :701], table[3, 0] = pages[:1500], pages[1500:2201], pages[2201]
    k[0, torch.tensor(pages.copy()).cuda()] = torch.arange(1, len(pages) + 1, device="cuda").to(torch.bfloat16)[:, None, None, None]
    work = torch.empty(binding.batch_pages_workspace_bytes(4, big), dtype=torch.uint8, device="cuda")
    out, lengths, free = torch.empty_like(_dev(table)), torch.empty(4, dtype=torch.int32, device="cuda"), torch.empty(big, dtype=torch.int32, device="cuda")
    want = ob.fork(table, held, [0, 1, 1, 0], big)
    before = k.clone()
    n_free, status = binding.batch_fork(cfg, 1, k, v, _dev(table), _dev(held), _dev([0, 1, 1, 0]), out, lengths, free, work)
    assert int(status) == 0 and int(n_free) == len(want["free"])
    np.testing.assert_array_equal(out.cpu().numpy(), want["block_table"])
    np.testing.assert_array_equal(free.cpu().numpy()[:int(n_free)], want["free"])
    for src, dst, rows in want["copies"]:
        before[:, dst, :, :rows] = before[:, src, :, :rows]
    assert torch.equal(k, before)
    want, n_used, moves = ob.compact(table, held, big)
    got = binding.batch_compact(cfg, 1, k, v, _dev(table), _dev(held), out, work)
    assert int(got) == n_used and len(moves) > 2000
    np.testing.assert_array_equal(out.cpu().numpy(), want)
    src, dst = (torch.tensor([int(m[i]) for m in moves], device="cuda") for i in (0, 1))
    before[:, dst] = before[:, src]
    assert torch.equal(k, before)


def test_on_another_stream_and_in_a_graph(binding):
    pool = Pool(binding, [100, 0, 0, 65], spare=6, Dh=128)
    want = ob.fork(pool.table, pool.held, [0, 0, 0, 3], pool.n_pages)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    table, lengths, _, n_free, status = pool.fork([0, 0, 0, 3], stream=st)
    np.testing.assert_array_equal(table, want["block_table"])
    assert (n_free, status) == (len(want["free"]), 0) and lengths == want["held"]
    # a captured fork and compaction follow their lengths and sources
    d_table, held, source = _dev(pool.table), _dev(pool.held), _dev([0, 1, 2, 3])
    out, after, packed = torch.empty_like(d_table), torch.empty_like(held), torch.empty_like(d_table)
    free = torch.empty(pool.n_pages, dtype=torch.int32, device="cuda")
    work = pool.work.clone()

    def step():
        n_free, status = binding.batch_fork(pool.cfg, pool.Hkv, pool.k, pool.v, d_table, held, source, out, after, free, pool.work)
        return n_free, status, binding.batch_compact(pool.cfg, pool.Hkv, pool.k, pool.v, out, after, packed, work)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        n_free, status, n_used = step()
    for src, lengths in (([0, 1, 2, 3], [100, 0, 0, 65]), ([0, 0, 3, 3], [99, 0, 0, 65]), ([3, -1, 0, 0], [64, 0, 0, 10])):
        source.copy_(_dev(src))
        held.copy_(_dev(lengths))
        pool.k.view(torch.int16).add_(1)
        torch.cuda.synchronize()
        want = ob.fork(pool.table, lengths, src, pool.n_pages)
        k, v = pool.moved(want["copies"])
        tight, used, moves = ob.compact(want["block_table"], want["held"], pool.n_pages)
        keep, pool.k, pool.v = (pool.k, pool.v), k.view(torch.bfloat16), v.view(torch.bfloat16)
        k, v = pool.moved([(a, b, PAGE) for a, b in moves])
        pool.k, pool.v = keep
        graph.replay()
        torch.cuda.synchronize()
        assert (int(status), int(n_free), int(n_used)) == (want["status"], len(want["free"]), used)
        np.testing.assert_array_equal(out.cpu().numpy(), want["block_table"])
        np.testing.assert_array_equal(packed.cpu().numpy(), tight)
        assert torch.equal(pool.k.view(torch.int16), k) and torch.equal(pool.v.view(torch.int16), v)


@pytest.mark.parametrize("name,make,match", [
    ("held", lambda p: _dev([1]), "held"), ("source", lambda p: _dev([1]), "source"), ("table_out", lambda p: _dev([[1]]), "table_out"),
    ("free_pages", lambda p: _dev([1]), "free_pages"), ("held_out", lambda p: torch.zeros(2, dtype=torch.int32), "tensors on"),
])
def test_refusals(binding, name, make, match):
    pool = Pool(binding, [3, 4])
    a = dict(held=_dev(pool.held), source=_dev([0, 1]), table_out=_dev(pool.table), held_out=_dev([0, 0]),
             free_pages=torch.empty(pool.n_pages, dtype=torch.int32, device="cuda"))
    a[name] = make(pool)
    with pytest.raises(ValueError, match=match):
        binding.batch_fork(pool.cfg, pool.Hkv, pool.k, pool.v, _dev(pool.table), workspace=pool.work, **a)
    with pytest.raises(binding.LlmcadError):  # (tables in place)
        t = _dev(pool.table)
        binding.batch_compact(pool.cfg, pool.Hkv, pool.k, pool.v, t, _dev(pool.held), t, pool.work)


def test_a_plan_that_would_write_into_a_shared_page(binding):
    """After a fork, a request rolled back into a page that another one holds: no request is placed, nothing is
    written, in a captured plan too; a request that ends on the page's border goes on."""
    import workloads

    shape = workloads.MODELS["tiny"]
    b = binding.Batch(shape, 2, 140, n_pages=8, max_pages=4)
    b.plan(_dev([0, 128, 128]), _dev([0, 0]))
    b.advance()
    b.k_pages.normal_()
    b.v_pages.normal_()
    held = b.fork(_dev([0, 0]), _dev([128, 0]))
    assert held.tolist() == [128, 128] and torch.equal(b.block_table[0], b.block_table[1])
    before = b.k_pages.clone(), b.v_pages.clone(), b.block_table.clone(), b.free_pages.clone()
    H, Dh = shape.n_heads, shape.head_dim
    q = torch.randn(140, H, Dh, device="cuda").to(torch.bfloat16)

    def untouched():
        torch.cuda.synchronize()
        b.store(0, q, q, q, torch.empty_like(q))
        for now, old in zip((b.k_pages, b.v_pages, b.block_table, b.free_pages), before):
            assert torch.equal(now, old)

    start, held = _dev([0, 0, 5]), _dev([128, 100])
    b.plan(start, held)
    assert b.status.tolist() == [binding.PLAN_BAD_LENGTHS] * 2
    untouched()
    with pytest.raises(RuntimeError, match="not placed"):
        b.advance()
    assert held.tolist() == [128, 100]
    with pytest.raises(ValueError, match="another one holds"):
        b.fork(_dev([0, 1]), held)
    with pytest.raises(ValueError, match="another one holds"):
        b.compact(held)
    untouched()
    b.plan(_dev([0, 5, 5]), held)  # (the one that ends inside has no rows)
    assert not b.status.any() and int(b.taken) == 1
    b.plan(start, _dev([128, 64]))
    assert not b.status.any() and int(b.taken) == 1
    b.block_table.copy_(before[2])  # (as if the last two had not been)
    b.plan(start, held)
    with pytest.raises(RuntimeError, match="not placed"):
        b.advance()
    untouched()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        b.plan(start, held)
    for length, status in ((100, 1), (128, 0), (127, 1), (64, 0), (1, 1)):
        held.copy_(_dev([128, length]))
        b.block_table.copy_(before[2])
        graph.replay()
        torch.cuda.synchronize()
        assert b.status.tolist() == [status] * 2, length
        if status:
            untouched()


@pytest.mark.parametrize("move", ["fork", "compact"])
def test_a_commit_after_its_pages_moved(binding, move):
    """It raises, and what reaches the device with that plan (a captured commit) moves nothing; a captured step that
    plans for itself works on after it."""
    import workloads

    shape = workloads.MODELS["tiny"]
    N, H, Dh = 40, shape.n_heads, shape.head_dim
    b = binding.Batch(shape, 2, N, n_pages=9, max_pages=4)
    q = torch.randn(N, H, Dh, device="cuda").to(torch.bfloat16)
    start, held, parent = _dev([0, 20, 40]), _dev([50, 0]), _dev([-1] + [0] * 19 + [-1] + [0] * 19)
    b.block_table[0, 0] = 8
    b.free_pages = b.free_pages[:8].clone()
    path, accept = _dev([0, 7] + [-1] * 18 + [0, 9] + [-1] * 18), _dev([1, 1])
    b.plan(start, held, parent)
    for layer in range(shape.n_layers):
        b.store(layer, q, q, q, torch.empty_like(q))
    b.advance()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        b.commit(path, accept)
    held += 20
    b.release(0)  # (so that the other's page moves, or somebody else gets this one's)
    held[0] = 0
    if move == "fork":
        held = b.fork(_dev([1, 1]), held)
    else:
        b.compact(held)
    before = b.k_pages.clone(), b.v_pages.clone()
    with pytest.raises(RuntimeError, match="pages moved"):
        b.commit(path, accept)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(b.k_pages, before[0]) and torch.equal(b.v_pages, before[1])
    free = b.free_pages.clone()

    def step():
        binding.batch_plan(b.cfg, start, held, parent, 0, b.block_table, free, b.n_pages, b.plan_buffer, N)
        for layer in range(shape.n_layers):
            b.store(layer, q, q, q, torch.empty_like(q))
        b.commit(path, accept)

    again = torch.cuda.CUDAGraph()
    with torch.cuda.graph(again):
        step()
    table = b.block_table.clone()
    again.replay()
    torch.cuda.synchronize()
    assert not b.status.any()
    once = b.k_pages.clone(), b.v_pages.clone(), b.block_table.clone()
    assert not torch.equal(once[0], before[0])
    b.commit(path, _dev([0, 0]))  # (an eager call after a replayed plan is no refusal)
    for t, old in zip((b.k_pages, b.v_pages, b.block_table), (*before, table)):
        t.copy_(old)
    step()
    torch.cuda.synchronize()
    for t, want in zip((b.k_pages, b.v_pages, b.block_table), once):
        assert torch.equal(t, want)


@pytest.mark.parametrize("held,source,kw", [
    ([33, 700, 1, 64], [1, 1, 0, 0], {"width": 3000, "L": 3, "Hkv": 3}),       # a wide table
    ([130, 70, 0, 65] * 20, [4 * g + i for g in range(20) for i in (3, 0, 0, 1)], {"L": 8, "H": 8, "Hkv": 8}),  # many page heads
])
def test_forks_of_heads_of_128_in_two_launches(binding, held, source, kw):
    want = Pool(binding, held, spare=30, Dh=128, **kw).check_fork(source)  # (20 groups: a copy each)
    assert want["copies"] and want["status"] == ob.OK


@pytest.mark.parametrize("held,kw", [
    ([100, 0, 700, 64], {"width": 5000, "spare": 11, "L": 3, "H": 6, "Hkv": 3}), ([130] * 300, {"n_pages": 1100, "L": 2, "Hkv": 2, "width": 30}),
])
def test_compactions_of_heads_of_128_in_two_launches(binding, held, kw):
    assert _check_compact(Pool(binding, held, Dh=128, **kw))
