"""Pins of the oracle's batch operators: hand-worked plans, the tree-masked attention of the model
oracle, torch's log-softmax, and mistakes planted in the oracle that a check has to see."""

import numpy as np
import pytest
import torch

import oracle
import workloads
from oracle import batch


def test_plan_hand_worked():
    # request 0 holds 63 tokens (page 5) and adds a 3-node tree: slots 63, then a new page
    # request 1 adds one token to nothing; request 2 sits out; request 3 holds 64 (a full page)
    table = [[5, -1], [-1, -1], [7, -1], [8, -1]]
    p = batch.plan([0, 3, 4, 4, 5], [63, 0, 10, 64], [-1, 0, 0, -1, -1, 0], 100, table, [2, 9, 4, 6], 10, 6, 4, 100.0)
    assert p["block_table"].tolist() == [[5, 2], [9, -1], [7, -1], [8, 4]]
    assert p["slot"].tolist() == [5 * 64 + 63, 2 * 64, 2 * 64 + 1, 9 * 64, 4 * 64, -1]
    assert p["position"].tolist() == [163, 164, 164, 100, 164, 0]
    assert p["ancestors"] == [[0], [0, 1], [0, 2], [0], [0], []]
    assert p["status"].tolist() == [0, 0, 0, 0] and p["taken"] == 3
    np.testing.assert_allclose(p["rope"][0], [[np.cos(163), np.sin(163)], [np.cos(16.3), np.sin(16.3)]], atol=1e-12)
    assert batch.mask_words(p["ancestors"])[2].tolist() == [5, 0, 0, 0]


def test_plan_statuses():
    table = [[-1], [-1], [-1]]
    p = batch.plan([0, 1, 2, 3], [0, 0, 0], None, 0, table, [1, 0], 2, 3, 4, 100.0)
    assert p["status"].tolist() == [0, 0, batch.NO_PAGES] and p["taken"] == 3 and p["slot"].tolist() == [64, 0, -1]
    assert set(batch.plan([0, 2, 1, 3], [0, 0, 0], None, 0, table, [1], 2, 3, 4, 100.0)["status"]) == {batch.BAD_LENGTHS}
    p = batch.plan([0, 2, 2, 3], [0, 0, 0], [-1, 1, -1], 0, table, [1, 0], 2, 3, 4, 100.0)
    assert p["status"].tolist() == [batch.BAD_TREE, 0, 0] and p["slot"].tolist() == [-1, -1, 0]


def _tree_case(seed=0):
    shape = workloads.MODELS["tiny"]
    rng = np.random.default_rng(seed)
    parent = workloads.complete_tree((2, 2))
    n, H, Dh, P = len(parent), 2, 8, 5
    anc = []
    for i in range(n):
        chain, j = [], i
        while j >= 0:
            chain.append(j)
            j = int(parent[j])
        anc.append(sorted(chain))
    q, k, v = rng.normal(size=(n, H, Dh)), rng.normal(size=(H, P + n, Dh)), rng.normal(size=(H, P + n, Dh))
    return shape, parent, anc, q, k, v, P


def _paged(k, P, held, n):
    """Keys or values [H, P + held + n, Dh] as a prefix and pages (page 1, then page 0)."""
    H, _, Dh = k.shape
    pages = np.zeros((2, H, 64, Dh))
    for t in range(held + n):
        pages[1 - t // 64, :, t % 64] = k[:, P + t]
    return k[:, :P], pages


def test_attention_is_softmax_over_the_branch():
    _, parent, anc, q, k, v, P = _tree_case()
    n, H, Dh = q.shape
    pk, kp = _paged(k, P, 0, n)
    pv, vp = _paged(v, P, 0, n)
    out, size = batch.attention(q, pk, pv, kp, vp, np.array([[1, 0]]), [0, n], [0], anc, 2)
    for i in range(n):
        keys = list(range(P)) + [P + j for j in anc[i]]
        for h in range(H):
            w = torch.softmax(torch.tensor(k[h, keys] @ q[i, h] / np.sqrt(Dh)), -1).numpy()
            np.testing.assert_allclose(out[i, h], w @ v[h, keys], atol=1e-12)
    assert np.all(size >= np.abs(out))


def test_prefix_and_held_are_interchangeable():
    # tokens moved from the prefix into the request's pages change nothing
    _, _, anc, q, k, v, P = _tree_case(1)
    n = len(anc)
    a = batch.attention(q, *_split(k, v, P, 0, n), np.array([[1, 0]]), [0, n], [0], anc, 2)[0]
    b = batch.attention(q, *_split(k, v, P - 3, 3, n), np.array([[1, 0]]), [0, n], [3], anc, 2)[0]
    np.testing.assert_allclose(a, b, atol=1e-12)


def _split(k, v, P, held, n):
    pk, kp = _paged(k, P, held, n)
    pv, vp = _paged(v, P, held, n)
    return pk, pv, kp, vp


@pytest.mark.parametrize("mistake", ["sees_siblings", "without_self", "without_held"])
def test_planted_mistakes_are_seen(mistake):
    _, _, anc, q, k, v, P = _tree_case(2)
    n, held = len(anc), 2
    args = _split(k, v, P - held, held, n)
    good = batch.attention(q, *args, np.array([[1, 0]]), [0, n], [held], anc, 2)[0]
    wrong, h = anc, held
    if mistake == "sees_siblings":
        wrong = [list(range(i + 1)) for i in range(n)]
    elif mistake == "without_self":
        wrong = [a[:-1] for a in anc]
    else:
        h = 0
    bad = batch.attention(q, *args, np.array([[1, 0]]), [0, n], [h], wrong, 2)[0]
    assert np.abs(good - bad).max() > 1e-2


def test_empty_rows_are_zero():
    q = np.ones((1, 1, 4))
    none = np.zeros((1, 0, 4))
    pages = np.ones((1, 1, 64, 4))
    out, _ = batch.attention(q, none, none, pages, pages, np.array([[-1]]), [0, 1], [0], [[0]], 1)
    assert np.all(out == 0)


def test_turn_matches_the_model_oracle():
    x = np.random.default_rng(0).normal(size=(3, 2, 8))
    pos = np.array([0, 5, 977])
    cfg_rope = oracle.rope(x, pos[:, None], 10000.0)
    ang = pos[:, None] * 10000.0 ** (-2.0 * np.arange(4) / 8)
    np.testing.assert_allclose(batch.turn(x, np.stack([np.cos(ang), np.sin(ang)], -1)), cfg_rope, atol=1e-12)


def test_commit_hand_worked():
    rows = np.arange(12.0).reshape(1, 12, 1)
    # request 0: rows 0..3 in slots 4..7, path 0, 2, 3; request 1: accepts nothing; request 2: entry out of range
    k, v = batch.commit([0, 4, 6, 8], [4, 5, 6, 7, 0, 1, 8, 9], [0, 2, 3, -1, 0, -1, 0, 5], [2, 0, 1], rows, -rows)
    assert k[0, :, 0].tolist() == [0, 1, 2, 3, 4, 6, 7, 7, 8, 9, 10, 11]
    assert v[0, :, 0].tolist() == [-x for x in k[0, :, 0]]


def test_scores_match_torch():
    x = np.random.default_rng(4).normal(size=(5, 77)) * 3
    s = batch.token_scores(x, [3, 76, 0, -1, 77], None, 6)
    lp = torch.log_softmax(torch.tensor(x), -1)
    np.testing.assert_allclose(s["logprob"][:3], [lp[0, 3], lp[1, 76], lp[2, 0]], atol=1e-12)
    assert s["logprob"][3] == 0.0 and np.isnan(s["logprob"][4])
    np.testing.assert_allclose(s["entropy"], torch.distributions.Categorical(logits=torch.tensor(x)).entropy(), atol=1e-12)
    top = torch.topk(lp, 6, -1)
    assert s["top_token"].tolist() == top.indices.tolist()
    np.testing.assert_allclose(s["top_logprob"], top.values, atol=1e-12)


def test_scores_ties_and_special_rows():
    inf = np.inf
    x = np.array([[1.0, 2.0, 2.0, 1.0], [-inf] * 4, [0.0, inf, 0.0, 0.0], [-inf, 0.0, -inf, -1.0], [np.nan, 0, 0, 0]])
    s = batch.token_scores(x, [1, 0, 1, 0, 1, 2], [0, 1, 2, 3, 4, 9], 3)
    assert s["top_token"].tolist() == [[1, 2, 0], [-1] * 3, [-1] * 3, [1, 3, -1], [-1] * 3]
    assert s["lse"][1] == -inf and s["entropy"][1] == 0 and np.isnan(s["lse"][2]) and np.isnan(s["top_logprob"][4]).all()
    assert s["logprob"][1] == -inf and np.isnan(s["logprob"][2]) and s["logprob"][3] == -inf and np.isnan(s["logprob"][5])
