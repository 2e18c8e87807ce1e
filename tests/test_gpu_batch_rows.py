"""What a row's attention owes to Inf and NaN that it sees, and to rows that belong to no request.  All
checks are of equal bits."""

import numpy as np
import pytest
import torch

from test_gpu_batch import Case, _attend, _np, _prefix, _queries, binding  # noqa: F401

pytestmark = pytest.mark.gpu

INF = float("inf")

SIZES = [  # rows and held tokens of the requests, prefix, heads: tiles of pages, of the prefix, few rows, both
    ([40, 33], [20, 70], 0, {"H": 2, "Dh": 128}),
    ([1] * 40, [0] * 40, 200, {"H": 2, "Dh": 64, "tree": False}),
    ([31, 2, 9], [100, 5, 64], 130, {"H": 8, "Hkv": 2, "Dh": 128, "pad": 6}),
    ([9, 1], [33, 90], 70, {"H": 2, "Dh": 64}),
]


@pytest.mark.parametrize("n,held,P,kw", SIZES)
@pytest.mark.parametrize("where", ["prefix", "held", "held beside rows"])
def test_infinities_that_every_row_sees(binding, n, held, P, kw, where):  # noqa: F811
    """A token whose value holds +Inf, -Inf and NaN in three dims: those outputs of the rows that see it are
    +Inf, -Inf and NaN, and no other output changes."""
    c = Case(binding, n, held, P=P, **kw)
    plan = c.plan()
    kp, vp = c.pages()
    kc, vc = _prefix(c)
    q = _queries(c, scale=0.5)
    dims = (0, 5, c.Dh - 1)
    if where == "prefix":
        if P == 0:
            pytest.skip("no prefix")
        rows, lines = range(c.total), vc[0][..., 3]
    else:
        b = int(np.argmax(held))  # (a request with enough tokens: its first page, or the page that its rows begin in)
        t = 3 if where == "held" else held[b] - 1
        if held[b] <= 3:
            pytest.skip("nothing held")
        rows = range(c.row_start[b], c.row_start[b + 1])
        lines = vp[0, int(c.d_table[b, t // 64])][..., t % 64]
    lines[:, dims] = 0
    clean = _np(_attend(c, plan, q, kc, vc, kp, vp))
    for dim, value in zip(dims, (INF, -INF, float("nan"))):
        lines[:, dim] = value
    got = _np(_attend(c, plan, q, kc, vc, kp, vp))
    want = clean.copy()
    for r in rows:
        want[r, :, 0], want[r, :, 5], want[r, :, c.Dh - 1] = INF, -INF, np.nan
    np.testing.assert_array_equal(got, want)


@pytest.mark.parametrize("n,held,P,kw", [
    ([1, 3, 2], [30, 0, 64], 600, {"H": 16, "Hkv": 16, "Dh": 128, "pad": 9}),    # few rows
    ([31, 17], [30, 100], 900, {"H": 8, "Hkv": 4, "Dh": 128, "pad": 40}),         # tiles, some of them padding alone
    ([33, 5, 8], [64, 0, 3], 900, {"H": 8, "Hkv": 8, "Dh": 64, "pad": 5}),
    ([2, 1], [5, 0], 700, {"H": 4, "Hkv": 4, "Dh": 64, "pad": 300}),              # most of it padding
])
@pytest.mark.parametrize("unplaced", [False, True])
def test_rows_of_no_request_do_not_matter(binding, n, held, P, kw, unplaced):  # noqa: F811
    """The same bits whatever lies in the queries of padding rows and of a request that was not placed."""
    c = Case(binding, n, held, P=P, **kw)
    if unplaced:  # (the second request's root has a parent)
        parent = list(c.parent)
        parent[c.row_start[1]] = 0
        plan = c.plan(parent=parent)
        assert int(plan["status"][1]) == binding.PLAN_BAD_TREE
    else:
        plan = c.plan()
    nobody = plan["slot"] < 0
    assert int(nobody.sum()) > 0
    kp, vp = c.pages()
    kc, vc = _prefix(c)
    q = _queries(c, scale=0.7)
    outs = []
    for fill in (0.0, 30.0, -INF, float("nan")):
        x = q.clone()
        x[nobody] = fill if fill != 30.0 else fill * torch.randn(
            x[nobody].shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).to(torch.bfloat16)
        outs.append(_attend(c, plan, x, kc, vc, kp, vp))
    for out in outs:
        assert torch.equal(out, outs[0])
        assert bool((out[nobody] == 77.0).all()) and bool((out[~nobody] != 77.0).any())
