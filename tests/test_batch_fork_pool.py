"""Batch's page accounting with forks and compaction on the CPU, its plans, forks and moves made by the oracle:
whatever a program does, no page is on the free list and in a table, none is lost, and every request reads its own
tokens through its table."""

import numpy as np
import pytest
import torch

import workloads
from oracle import batch as ob

PAGE = ob.PAGE


class Pool:
    """A Batch whose pages hold one number per slot (the token), so that what a request reads can be compared."""

    def __init__(self, binding, monkeypatch, n_requests, n_rows, n_pages, max_pages):
        b = self.b = binding.Batch(workloads.MODELS["tiny"], n_requests, n_rows, n_pages=n_pages, max_pages=max_pages, device="cpu")
        self.slots = np.zeros((n_pages, PAGE), dtype=np.int64)
        self.text = [[] for _ in range(n_requests)]
        self.next = 1

        def plan(cfg, row_start, held, parent, prefix_len, block_table, free_pages, n_pages, plan, n_rows, stream=None):
            want = ob.plan(row_start.tolist(), held.tolist(), None if parent is None else parent.tolist(), prefix_len,
                           block_table.numpy(), free_pages.tolist(), n_pages, n_rows, cfg.head_dim, 10000.0)
            block_table.copy_(torch.from_numpy(want["block_table"]))
            b.status.copy_(torch.from_numpy(want["status"]))
            b.slot.copy_(torch.from_numpy(want["slot"]))
            b.taken[0] = want["taken"]

        def fork(cfg, n_kv_heads, k_pages, v_pages, block_table, held, source, table_out, held_out, free_pages, workspace, stream=None):
            want = ob.fork(block_table.numpy(), held.tolist(), source.tolist(), n_pages)
            for src, dst, rows in want["copies"] if want["status"] == 0 else []:
                self.slots[dst, :rows] = self.slots[src, :rows]
            table_out.copy_(torch.from_numpy(want["block_table"]))
            held_out.copy_(torch.tensor(want["held"]))
            free_pages.fill_(-1)
            free_pages[:len(want["free"])] = torch.tensor(want["free"], dtype=torch.int32)
            return torch.tensor([len(want["free"])], dtype=torch.int32), torch.tensor([want["status"]], dtype=torch.int32)

        def compact(cfg, n_kv_heads, k_pages, v_pages, block_table, held, table_out, workspace, stream=None):
            table, used, moves = ob.compact(block_table.numpy(), held.tolist(), n_pages)
            for src, dst in moves:
                self.slots[dst] = self.slots[src]
                self.slots[src] = -1
            table_out.copy_(torch.from_numpy(table))
            return torch.tensor([used], dtype=torch.int32)

        for name, fn in (("batch_plan", plan), ("batch_fork", fork), ("batch_compact", compact)):
            monkeypatch.setattr(binding, name, fn)

    @property
    def held(self):
        return torch.tensor([len(t) for t in self.text], dtype=torch.int32)

    def step(self, n, keep=None):
        """Adds n[b] rows to request b and keeps the first keep[b] of them."""
        start = torch.tensor(np.concatenate([[0], np.cumsum(n)]), dtype=torch.int32)
        self.b.plan(start, self.held)
        if self.b.status.any():
            with pytest.raises(RuntimeError, match="not placed"):
                self.b.advance()
            return False
        self.b.advance()
        for i, (slot, b) in enumerate(zip(self.b.slot.tolist(), np.repeat(np.arange(len(n)), n))):
            self.slots[slot // PAGE, slot % PAGE] = self.next
            if keep is None or i - int(start[b]) < keep[b]:
                self.text[b].append(self.next)
            self.next += 1
        return True

    def fork(self, source):
        held = self.b.fork(torch.tensor(source, dtype=torch.int32), self.held)
        self.text = [list(self.text[s]) if s >= 0 else [] for s in source]
        assert held.tolist() == [len(t) for t in self.text]

    def check(self, exact=False):
        """exact: the tables hold the pages of the lengths and no others (after a fork, trim or compaction)."""
        table = self.b.block_table.numpy()
        used, free = set(table[table >= 0].tolist()), self.b.free_pages.tolist()
        assert len(free) == len(set(free)) and not used & set(free)
        assert used | set(free) == set(range(self.b.n_pages))
        for b, text in enumerate(self.text):
            pages = table[b, :-(-len(text) // PAGE)]
            got = self.slots[pages].reshape(-1)[:len(text)] if len(pages) else []
            assert list(got) == text, b
            if exact:
                assert (table[b, len(pages):] == -1).all()


@pytest.fixture
def pool(monkeypatch):
    from paper_2309_04255_amd import binding

    return lambda *a: Pool(binding, monkeypatch, *a)


def test_answers_to_one_prompt(pool):
    p = pool(4, 400, 16, 4)
    assert p.step([100, 0, 0, 0])
    p.fork([0, 0, 0, 0])
    p.check(exact=True)
    table = p.b.block_table
    assert (table[:, 0] == table[0, 0]).all() and len(set(table[:, 1].tolist())) == 4
    assert p.step([30, 1, 40, 28])
    p.check()
    p.b.release(0)  # (the shared page stays with the others)
    p.text[0] = []
    p.check()
    p.b.release(2)
    p.text[2] = []
    p.b.release(1)
    p.text[1] = []
    p.check()
    p.b.release(3)
    p.text[3] = []
    p.check()
    assert len(p.b.free_pages) == 16


def test_beams_change_places(pool):
    p = pool(3, 300, 9, 3)
    assert p.step([70, 70, 70])
    for source in ([2, 2, 0], [1, 2, 0], [0, 0, 0], [0, -1, 1]):
        p.fork(source)
        p.check(exact=True)
        assert p.step([3, 3, 3] if p.text[1] else [3, 0, 3])
        p.check()


def test_rejected_rows_of_a_shared_prompt_come_back(pool):
    p = pool(2, 260, 8, 4)
    assert p.step([128, 0])
    p.fork([0, 0])
    assert p.step([70, 70], keep=[2, 65])
    p.b.trim(p.held)
    p.check(exact=True)
    p.fork([0, 0])  # (without a trim before it: pages past the lengths come back by themselves)
    assert p.step([70, 1], keep=[1, 1])
    p.fork([0, 1])
    p.check(exact=True)


def test_a_shared_page_is_not_cut(pool):
    p = pool(2, 260, 8, 4)
    assert p.step([128, 0])
    p.fork([0, 0])
    before = p.b.block_table.clone(), p.b.free_pages.clone()
    with pytest.raises(ValueError, match="another one holds"):
        p.b.trim(torch.tensor([128, 100], dtype=torch.int32))
    assert torch.equal(p.b.block_table, before[0]) and torch.equal(p.b.free_pages, before[1])
    p.b.trim(torch.tensor([128, 64], dtype=torch.int32))  # (a whole page less is no cut)
    p.text[1] = p.text[1][:64]
    p.check(exact=True)


def test_no_room_changes_nothing(pool):
    p = pool(3, 200, 3, 3)
    assert p.step([100, 0, 0])
    p.b.trim(p.held)
    before = p.b.block_table.clone(), p.b.free_pages.clone()
    with pytest.raises(RuntimeError, match="not forked"):
        p.fork([0, 0, 0])
    assert torch.equal(p.b.block_table, before[0]) and torch.equal(p.b.free_pages, before[1])
    with pytest.raises(RuntimeError, match="not forked"):
        p.b.fork(torch.tensor([0, 3, 0], dtype=torch.int32), p.held)
    p.check()


@pytest.mark.parametrize("what", ["fork", "compact"])
def test_a_plan_that_was_not_advanced(pool, what):
    p = pool(2, 200, 6, 3)
    assert p.step([10, 5])
    p.b.plan(torch.tensor([0, 1, 2], dtype=torch.int32), p.held)
    with pytest.raises(RuntimeError, match="not advanced"):
        p.fork([0, 1]) if what == "fork" else p.b.compact(p.held)
    p.b.advance()
    p.fork([0, 1]) if what == "fork" else p.b.compact(p.held)
    p.check(exact=True)


def test_compact_keeps_what_is_shared(pool):
    p = pool(4, 600, 20, 6)
    assert p.step([100, 90, 128, 70])
    p.fork([0, 0, 2, 2])
    assert p.step([100, 20, 70, 1])
    p.b.release(0)
    p.text[0] = []
    assert p.b.compact(p.held) == len({x for x in p.b.block_table.reshape(-1).tolist() if x >= 0})
    p.check(exact=True)
    assert p.b.block_table.max() < 20 - len(p.b.free_pages)
    assert p.step([64, 64, 1, 2])
    p.check()


@pytest.mark.parametrize("seed", range(8))
def test_a_random_program(pool, seed):
    rng = np.random.default_rng(seed)
    B = 5
    p = pool(B, B * 128, 40, 8)
    for _ in range(60):
        do = rng.integers(6)
        if do <= 2:
            n = rng.integers(0, [3, 40, 129][rng.integers(3)], B)
            n = [int(m) if len(t) + m <= 500 else 0 for m, t in zip(n, p.text)]
            p.step(n, keep=[int(rng.integers(0, m + 1)) for m in n])
            p.b.trim(p.held)
        elif do == 3:
            try:
                p.fork([int(s) for s in np.where(rng.random(B) < 0.15, -1, np.where(rng.random(B) < 0.5, np.arange(B), rng.integers(0, B, B)))])
            except RuntimeError:
                pass
        elif do == 4:
            b = int(rng.integers(B))
            p.b.release(b)
            p.text[b] = []
        else:
            p.b.compact(p.held)
        p.check()


def _i(v):
    return torch.tensor(v, dtype=torch.int32)


def _shared(pool):
    """Two requests that share two full pages, request 1 rolled back into the second one without a trim."""
    p = pool(2, 260, 8, 4)
    assert p.step([128, 0])
    p.fork([0, 0])
    p.text[1] = p.text[1][:100]
    return p, (p.b.block_table.clone(), p.b.free_pages.clone())


def _unchanged(p, before):
    assert torch.equal(p.b.block_table, before[0]) and torch.equal(p.b.free_pages, before[1])
    p.check()


def test_a_step_does_not_write_into_a_shared_page(pool):
    p, before = _shared(pool)
    assert not p.step([0, 5])  # (rows of request 1 would be tokens 100 to 104 of request 0)
    assert p.b.status.tolist() == [ob.BAD_LENGTHS] * 2 and p.b.slot.max() < 0
    _unchanged(p, before)
    assert p.step([5, 0])  # (the one that ends inside gets no rows)
    p.check()
    p.b.release(0)
    p.text[0] = []
    assert p.step([0, 5])  # (nobody else holds the page any more)
    p.check()


def test_a_step_of_a_request_that_shares_whole_pages_only(pool):
    p, _ = _shared(pool)
    p.text[1] = p.text[1][:64]
    assert p.step([3, 40])
    p.b.trim(p.held)
    p.check(exact=True)
    assert p.step([1, 1])  # (the pages that it ends in are its own)
    p.check()


def test_a_fork_does_not_keep_a_shared_page_that_is_cut(pool):
    p, before = _shared(pool)
    for source in ([0, 1], [1, 0], [1, 0], [0, 1]):
        with pytest.raises(ValueError, match="another one holds"):
            p.fork(source)
        _unchanged(p, before)
    p.fork([0, 0])  # (what request 1 held is given up)
    p.check(exact=True)
    p, _ = _shared(pool)
    p.fork([-1, 1])  # (request 0 ends: the page is request 1's alone)
    assert p.step([3, 5])
    p.check()
    p, _ = _shared(pool)
    p.fork([1, 1])  # (one goes on with the page, the other with a copy)
    assert p.step([3, 5])
    p.check()
    with pytest.raises(RuntimeError, match="not forked"):
        p.b.fork(_i([0, 2]), p.held)


def test_a_compaction_does_not_cut_a_shared_page(pool):
    p, before = _shared(pool)
    with pytest.raises(ValueError, match="another one holds"):
        p.b.compact(p.held)
    _unchanged(p, before)
    p.text[1] = p.text[1][:64]
    p.b.compact(p.held)
    p.check(exact=True)


@pytest.mark.parametrize("seed", range(8))
def test_a_random_program_that_rolls_back(pool, seed):
    """As test_a_random_program, with requests that step back anywhere and nothing trimmed: a call is refused and
    changes nothing, or every request reads its own tokens after it."""
    rng = np.random.default_rng(100 + seed)
    B, refused = 4, 0
    p = pool(B, B * 128, 60, 8)
    assert p.step([128, 100, 0, 0])
    for _ in range(60):
        do = rng.integers(4)
        before = p.b.block_table.clone(), p.b.free_pages.clone()
        if rng.random() < 0.3:
            b = int(rng.integers(B))
            p.text[b] = p.text[b][:int(rng.integers(0, len(p.text[b]) + 1))]
        try:
            if do <= 1:
                n = [int(m) if len(t) + m <= 500 else 0 for m, t in zip(rng.integers(0, 70, B), p.text)]
                ok = p.step(n)
                refused += not ok
            elif do == 2:
                p.fork([int(s) for s in rng.integers(-1 if rng.random() < 0.2 else 0, B, B)])
            else:
                p.b.compact(p.held)
        except (ValueError, RuntimeError):
            refused += 1
            assert torch.equal(p.b.block_table, before[0]) and torch.equal(p.b.free_pages, before[1])
        for b, text in enumerate(p.text):
            pages = p.b.block_table[b, :-(-len(text) // PAGE)].numpy()
            assert list(p.slots[pages].reshape(-1)[:len(text)] if len(pages) else []) == text, b
    assert refused


@pytest.fixture
def calls(monkeypatch):
    """Names of the step's operators that reached the library."""
    from paper_2309_04255_amd import binding

    made = []
    for name in ("store", "norm_store", "attention", "commit"):
        monkeypatch.setattr(binding, f"batch_{name}", lambda *a, name=name: made.append(name))
    return made


def _operators(b):
    x, i = torch.zeros(b.n_rows, 4, 64), _i([0] * b.n_rows)
    return {"store": lambda: b.store(0, x, x, x, x), "norm_store": lambda: b.norm_store(0, x, x, x, None, None, x),
            "attention": lambda: b.attention(0, x, x), "commit": lambda: b.commit(i, _i([0] * b.n_requests))}


@pytest.mark.parametrize("name", ["store", "norm_store", "attention", "commit"])
@pytest.mark.parametrize("move", ["fork", "compact"])
def test_a_plan_from_before_its_pages_moved(pool, calls, name, move):
    from paper_2309_04255_amd import binding

    p = pool(3, 300, 12, 4)
    call = _operators(p.b)[name]
    assert p.step([70, 80, 90])
    call()
    p.b.release(0)
    p.text[0] = []
    p.fork([0, 1, 1]) if move == "fork" else p.b.compact(p.held)
    del calls[:]
    for _ in range(2):
        with pytest.raises(RuntimeError, match="pages moved"):
            call()
    assert not calls and p.b.slot.max() < 0
    p.check(exact=True)
    free = p.b.free_pages.clone()
    with pytest.raises(RuntimeError):
        p.b.advance()  # (no plan: no pages to drop)
    assert torch.equal(p.b.free_pages, free)
    # a plan made without Batch.plan, as a captured step does
    start = _i([0, 1, 2, 3])
    binding.batch_plan(p.b.cfg, start, p.held, None, 0, p.b.block_table, p.b.free_pages, 12, p.b.plan_buffer, 300)
    call()
    p.fork([0, 1, 2]) if move == "fork" else p.b.compact(p.held)
    with pytest.raises(RuntimeError, match="pages moved"):
        call()
    assert p.step([1, 1, 1])
    call()
    assert calls == [name] * 2


@pytest.mark.parametrize("fails", ["no room", "cut", "not advanced"])
def test_a_fork_or_compaction_that_was_refused_leaves_the_plan(pool, calls, fails):
    p = pool(3, 300, 4 if fails == "no room" else 12, 4)
    if fails == "cut":
        assert p.step([128, 0, 0])
        p.fork([0, 0, 0])
        p.text[1] = p.text[1][:100]
        assert p.step([70, 0, 0])
    else:
        assert p.step([70, 80, 0])
    if fails == "not advanced":
        p.b.plan(_i([0, 1, 2, 3]), p.held)
    slot = p.b.slot.clone()
    with pytest.raises((RuntimeError, ValueError)):
        p.fork([0, 1, 1])
    if fails != "no room":
        with pytest.raises((RuntimeError, ValueError)):
            p.b.compact(p.held)
    for call in _operators(p.b).values():
        call()
    assert len(calls) == 4 and torch.equal(p.b.slot, slot)


def test_workspaces_are_made_with_the_batch(pool, monkeypatch):
    """No call takes memory of whatever stream it runs on: adjust, fork and compact find their workspaces made."""
    from paper_2309_04255_amd import binding

    p = pool(2, 40, 6, 3)
    b, seen = p.b, []
    adjust = lambda *a, workspace, **kw: seen.append(workspace)  # noqa: E731
    pages = lambda name, inner: lambda *a, **kw: (seen.append(a[-1]), inner(*a, **kw))[1]  # noqa: E731
    monkeypatch.setattr(binding, "batch_adjust", adjust)
    for name in ("batch_fork", "batch_compact"):
        monkeypatch.setattr(binding, name, pages(name, getattr(binding, name)))
    made = {t.data_ptr(): t.numel() for t in vars(b).values() if isinstance(t, torch.Tensor)}
    b.adjust(torch.zeros(40, b.cfg.vocab), greedy=_i([0] * 40))
    assert p.step([20, 20])
    p.fork([0, 0])
    b.compact(p.held)
    want = [binding.batch_adjust_workspace_bytes(b.cfg, 40)] + [binding.batch_pages_workspace_bytes(2, 6)] * 2
    assert [t.numel() for t in seen] == want
    assert [made.get(t.data_ptr()) for t in seen] == want


def test_lengths_at_the_ends_of_a_table(pool):
    """Full tables that share every page, lengths of zero and below, rows of the tables that were given back."""
    p = pool(4, 260, 16, 2)
    assert p.step([128, 0, 70, 0])
    p.fork([0, 0, 2, 2])
    p.check(exact=True)
    p.b.trim(p.held)
    p.b.compact(p.held)
    p.check(exact=True)
    p.b.release(3)
    p.text[3] = []
    p.b.trim(_i([128, 128, 70, 5]))  # (nothing of the last one's is left)
    assert not p.step([0, 1, 0, 0])  # (no column is left)
    assert p.b.status.tolist() == [0, ob.NO_PAGES, 0, 0]
    p.text[1] = []
    p.b.trim(_i([128, -1, 70, 0]))
    p.check(exact=True)
    assert p.step([0, 100, 1, 9])
    p.check()


def test_a_refused_plan_is_no_plan(pool, calls, monkeypatch):
    from paper_2309_04255_amd import binding

    p = pool(2, 40, 6, 3)
    assert p.step([20, 20])
    p.b.compact(p.held)

    def refuses(*a, **kw):
        raise ValueError("batch_plan: parent")

    with monkeypatch.context() as m:
        m.setattr(binding, "batch_plan", refuses)
        with pytest.raises(ValueError, match="parent"):
            p.b.plan(_i([0, 1, 2]), p.held)
    for call in _operators(p.b).values():
        with pytest.raises(RuntimeError, match="pages moved"):
            call()
    assert p.step([1, 1])
    p.check()
