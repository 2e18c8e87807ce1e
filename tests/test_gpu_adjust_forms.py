"""The forms of the adjusted logits that large steps take, against their plain statement (oracle/batch.py), equal bit
for bit as in test_gpu_adjust.py: a workgroup with several rows of several requests on every piece of the vocabulary,
and one with more pieces of a row than it sorts the history for."""

import numpy as np
import pytest
import torch

from test_gpu_adjust import Step, binding  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


def _check(s, names=()):
    out, best = s.run(**s.kw(*names))
    s.check(out, best, s.oracle(*names))
    _, alone = s.run(out=None, **s.kw(*names))
    assert torch.equal(alone, best)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("names", [(), ("bias",), ("penalties", "tokens", "history")])
def test_few_rows_of_three_pieces(binding, dtype, names):  # noqa: F811
    """901 rows in threes or fours, 2703 pieces; requests change within a workgroup, one has no rows."""
    _check(Step(binding, [41, 20, 0, 128, 33] * 4, [30, 0, 7, 200, 64] * 4, 9001, dtype, pad=13, seed=6), names)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_sixteen_rows_of_fifteen_pieces(binding, dtype):  # noqa: F811
    """14370 pieces: the most rows a workgroup takes, in requests that begin and end inside it."""
    s = Step(binding, [41, 20, 0, 128, 33, 5, 3, 9] * 4, [30, 0, 7, 200, 64, 1, 2, 300] * 4, 4096 * 14 + 7, dtype, seed=7, masks=0, pad=2)
    s.seen = s.seen[::97]
    _check(s)


def test_rows_of_no_request_between_those_of_others(binding):  # noqa: F811
    """Requests that are not placed (their parents are no trees) lie between the others' rows in a workgroup."""
    s = Step(binding, [41, 20, 3, 128, 33] * 4, [30, 0, 0, 200, 64] * 4, 9001, pad=40, seed=8)
    for b in (1, 2, 7, 8, 18):
        s.c.parent[s.c.row_start[b]] = 0
    s.views, s.want = s.c.plan(), s.c.want()
    assert s.views["status"].tolist() == [3 if b in (1, 2, 7, 8, 18) else 0 for b in range(20)]
    _check(s)


def test_more_pieces_than_a_history_is_sorted_for(binding):  # noqa: F811
    """One workgroup has all 65 pieces of a row."""
    s = Step(binding, [1] * 100, [int(h) for h in np.random.default_rng(0).integers(0, 700, 100)], 4096 * 64 + 77, torch.bfloat16,
             seed=9, masks=0, pad=663, tree=False)
    s.seen = s.seen[::997]
    _check(s)
