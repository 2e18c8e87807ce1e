"""Batch's page accounting on the CPU, its plans made by the oracle: whatever a program does after a step that
could not be placed, or between a plan and advance, every page is in one table entry or once on the
free list, and no two requests share one; and its refusals."""

import numpy as np
import pytest
import torch

import workloads
from oracle import batch as ob


@pytest.fixture
def pool(monkeypatch):
    from paper_2309_04255_amd import binding

    def make(n_requests, n_rows, n_pages, max_pages):
        b = binding.Batch(workloads.MODELS["tiny"], n_requests, n_rows, n_pages=n_pages, max_pages=max_pages, device="cpu")

        def plan(cfg, row_start, held, parent, prefix_len, block_table, free_pages, n_pages, plan, n_rows, stream=None):
            want = ob.plan(row_start.tolist(), held.tolist(), None if parent is None else parent.tolist(), prefix_len,
                           block_table.numpy(), free_pages.tolist(), n_pages, n_rows, cfg.head_dim, 10000.0)
            block_table.copy_(torch.from_numpy(want["block_table"]))
            b.status.copy_(torch.from_numpy(want["status"]))
            b.slot.copy_(torch.from_numpy(want["slot"]))
            b.taken[0] = want["taken"]

        monkeypatch.setattr(binding, "batch_plan", plan)
        return b

    return make


def _i(v):
    return torch.tensor(v, dtype=torch.int32)


def _once(b):
    """Every page is in the tables or on the free list, once."""
    used = b.block_table[b.block_table >= 0].tolist()
    assert sorted(used + b.free_pages.tolist()) == list(range(b.n_pages)), (b.block_table.tolist(), b.free_pages.tolist())


def _plan(b, n, held, parent=None):
    b.plan(_i(np.concatenate([[0], np.cumsum(n)]).tolist()), _i(held), parent)


def test_a_step_that_did_not_fit_can_be_tried_again(pool):
    b = pool(3, 140, 3, 4)
    _plan(b, [65, 65, 1], [0, 0, 0])
    assert b.status.tolist() == [0, 2, 2]
    with pytest.raises(RuntimeError, match="not placed"):
        b.advance()
    _once(b)
    b.release(0)
    _once(b)
    _plan(b, [0, 65, 1], [0, 0, 0])
    assert b.status.tolist() == [0, 0, 0]
    b.advance()
    _once(b)
    assert len(b.free_pages) == 0 and b.block_table[0].tolist() == [-1] * 4


def test_release_of_a_victim_after_a_step_that_did_not_fit(pool):
    b = pool(2, 8, 3, 2)
    _plan(b, [1, 1], [0, 0])
    b.advance()
    held = [64, 64]  # (both pages are full, one is free)
    _plan(b, [1, 1], held)
    assert b.status.tolist() == [0, 2]
    with pytest.raises(RuntimeError):
        b.advance()
    b.release(0)
    _once(b)
    _plan(b, [1, 1], [0, 64])
    assert b.status.tolist() == [0, 0]
    b.advance()
    _once(b)


@pytest.mark.parametrize("again", ["release", "trim"])
def test_a_bad_plan_given_up_without_advance(pool, again):
    b = pool(3, 140, 3, 4)
    _plan(b, [65, 65, 1], [0, 0, 0])
    assert b.status.tolist() == [0, 2, 2]
    b.release(0) if again == "release" else b.trim(_i([0, 0, 0]))
    _once(b)
    _plan(b, [0, 65, 1], [0, 0, 0])
    assert b.status.tolist() == [0, 0, 0]
    b.advance()
    _once(b)


def test_release_between_a_plan_and_advance(pool):
    b = pool(3, 200, 9, 3)
    _plan(b, [65, 10, 64], [0, 0, 0])
    b.release(1)  # (the request ends while the step runs)
    kept = b.block_table.clone()
    assert (kept[0, :2] >= 0).all() and kept[2, 0] >= 0
    b.advance()
    _once(b)
    assert torch.equal(b.block_table, kept) and len(b.free_pages) == 6
    _plan(b, [1, 1, 1], [65, 0, 64])
    b.advance()
    _once(b)


@pytest.mark.parametrize("taken", [None, 3])
def test_trim_between_a_plan_and_advance(pool, taken):
    b = pool(2, 200, 9, 3)
    _plan(b, [100, 10], [0, 0])
    b.trim(_i([3, 1]))  # (the step's trees were mostly rejected)
    b.advance(taken)
    _once(b)
    assert len(b.free_pages) == 7


def test_a_plan_replaced_by_another(pool):
    b = pool(3, 200, 9, 3)
    _plan(b, [70, 70, 70], [0, 0, 0])
    _plan(b, [70, 0, 1], [0, 0, 0])  # (another step: a request sits out)
    assert b.block_table[1].tolist() == [-1] * 3
    _plan(b, [70, 0, 1], [0, 0, 0])  # (the same once more)
    b.advance()
    _once(b)
    assert len(b.free_pages) == 6
    b.trim(_i([70, 0, 1]))
    _once(b)
    b.release(0)
    b.release(2)
    _once(b)
    assert len(b.free_pages) == 9


@pytest.mark.parametrize("entry", [-7, 9, 1 << 30])
def test_entries_that_are_no_pages(pool, entry):
    # (such a request's plan fails; the others' pages stay in order)
    b = pool(2, 200, 9, 3)
    b.block_table[1, 0] = entry
    _plan(b, [70, 1], [0, 5])
    assert b.status.tolist() == [0, 2]
    with pytest.raises(RuntimeError):
        b.advance()
    assert b.block_table.tolist() == [[-1] * 3, [entry, -1, -1]] and b.free_pages.tolist() == list(range(9))
    b.free_pages[3] = entry
    _plan(b, [70, 1], [0, 0])
    assert b.status.tolist() == [0, 0]
    b.release(1)
    b.advance()
    assert b.block_table[0].tolist() == [0, 1, -1] and b.free_pages.tolist() == [2, entry, 4, 5, 6, 7, 8]


@pytest.mark.parametrize("rows", [0, 7, 9])
def test_tensors_of_other_row_counts_are_refused(pool, rows):
    # (the kernels would take them for those of another plan and do nothing)
    b = pool(2, 8, 9, 3)
    H, Dh = b.cfg.n_heads, b.cfg.head_dim
    good, bad = torch.zeros(8, H, Dh, dtype=torch.bfloat16), torch.zeros(rows, H, Dh, dtype=torch.bfloat16)
    for i in range(4):
        with pytest.raises(ValueError, match="must have 8 rows"):
            b.store(0, *[bad if j == i else good for j in range(4)])
    for args in ((bad, good), (good, bad)):
        with pytest.raises(ValueError, match="must have 8 rows"):
            b.attention(0, *args)
    for path in (torch.zeros(rows, dtype=torch.int32), torch.tensor(0, dtype=torch.int32)):
        with pytest.raises(ValueError, match="must have 8 rows"):
            b.commit(path, _i([0, 0]))


def _walk(b, seed):
    """Steps of every kind in random order."""
    dev = b.block_table.device
    rng = np.random.default_rng(seed)
    held = [0] * b.n_requests
    for _ in range(60):
        n = [int(x) for x in rng.choice([0, 1, 40, 80], b.n_requests)]
        b.plan(_i(np.concatenate([[0], np.cumsum(n)]).tolist()).to(dev), _i(held).to(dev))
        fits = not b.status.any()
        kind = rng.integers(6)
        if kind == 0:
            continue  # (planned again in the next round)
        if kind == 1 or not fits:
            if not fits and kind != 1:
                with pytest.raises(RuntimeError):
                    b.advance()
                _once(b)
            v = int(rng.integers(b.n_requests))
            b.release(v)
            held[v] = 0
            if not fits:
                _once(b)
                continue
            n[v] = 0
            b.advance()
        else:
            b.advance(int(b.taken) if kind == 2 else None)
            _once(b)
        held = [h + int(rng.integers(m + 1)) for h, m in zip(held, n)]
        b.trim(_i(held).to(dev))
        _once(b)
        for i in range(b.n_requests):
            have = -(-held[i] // 64)
            assert (b.block_table[i, :have] >= 0).all() and (b.block_table[i, have:] == -1).all()


@pytest.mark.parametrize("seed", range(20))
def test_many_steps(pool, seed):
    _walk(pool(4, 4 * 128, 8, 4), seed)


@pytest.mark.gpu
def test_many_steps_of_the_kernel():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2309_04255_amd import binding

    for seed in range(4):
        _walk(binding.Batch(workloads.MODELS["tiny"], 4, 4 * 128, n_pages=8, max_pages=4), seed)
