"""Token scores (llmcad_token_scores) against their float64 statement (oracle/batch.py).

Tolerances: a logit enters exactly; lse and log probabilities are m + log S (in base 2, where a
product with log2 e takes another half step of the value) with S a sum of fp32 exponentials (each
within 2^-22, the sum of up to 2^18 of them in chains of at most 2^9 additions and 14 joins: 2^-14 at
the worst, 2^-20 in the mean of random roundings), the difference x - m rounded once: 2^-18 absolute
and 2^-22 of the value.  The entropy adds products p (x - m) of size up to about
100: 2^-15."""

import numpy as np
import pytest
import torch

from oracle import batch as ob

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def binding():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2309_04255_amd import binding

    return binding


def _check(binding, logits, tokens, k, row_of=None, **kw):
    dev = lambda a: None if a is None else torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")  # noqa: E731
    got = binding.token_scores(logits, dev(tokens), k, row_of=dev(row_of), **kw)
    torch.cuda.synchronize()
    x = logits.float().cpu().numpy().astype(np.float64)
    want = ob.token_scores(x, [] if tokens is None else tokens, row_of if tokens is not None else [], k)
    np.testing.assert_array_equal(got["top_token"].cpu().numpy(), want["top_token"])
    for name, atol in (("lse", 2.0 ** -18), ("logprob", 2.0 ** -18), ("top_logprob", 2.0 ** -18), ("entropy", 2.0 ** -15)):
        np.testing.assert_allclose(got[name].cpu().numpy(), want[name], rtol=2.0 ** -22, atol=atol, err_msg=name)
    return got


def _logits(n, V, dtype=torch.float32, seed=0, scale=3.0, stride=None, shift=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = (torch.randn(n, V, device="cuda", generator=g) * scale).to(dtype)
    buf = torch.zeros(n * (stride or V) + shift, dtype=dtype, device="cuda")
    view = torch.as_strided(buf, (n, V), (stride or V, 1), shift)
    view.copy_(x)
    return view


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,V,k", [(1, 1, 1), (3, 2, 5), (2, 63, 64), (5, 1000, 7), (31, 1998, 8), (2, 16384, 64), (2, 16385, 1),
                                   (4, 32000, 20), (1, 50257, 0), (2, 131075, 64), (1, 262144, 33)])
def test_scores(binding, dtype, n, V, k):
    rng = np.random.default_rng(V)
    _check(binding, _logits(n, V, dtype), rng.integers(0, V, n), k)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shift,extra", [(1, 3), (3, 5), (7, 1), (0, 9)])
def test_rows_off_any_alignment(binding, dtype, shift, extra):
    V = 4001
    _check(binding, _logits(6, V, dtype, stride=V + extra, shift=shift), np.arange(6) * 100, 16)


@pytest.mark.parametrize("order", ["constant", "rising", "falling", "two_values", "late_peaks"])
@pytest.mark.parametrize("V", [700, 20000, 70000])
def test_orders_and_ties(binding, order, V):
    x = torch.arange(V, dtype=torch.float64, device="cuda")
    x = {"constant": torch.zeros_like(x) + 1.5, "rising": x * (8.0 / V), "falling": -x * (8.0 / V), "two_values": (x % 2),
         "late_peaks": torch.where(x > V - 3000, 5.0 + x / V, torch.sin(x))}[order]
    logits = x.to(torch.float32)[None].repeat(2, 1).contiguous()
    if order == "rising":
        logits = torch.round(logits * 64) / 64  # (long runs of ties)
    _check(binding, logits, [0, V - 1], 64)


def test_special_rows(binding):
    inf, V = float("inf"), 3000
    x = _logits(10, V)
    x[0] = -inf
    x[1, 5:] = -inf
    x[2, 77] = float("nan")
    x[3, 2999] = inf
    x[4] = torch.finfo(torch.float32).min
    x[5, 100:] = torch.finfo(torch.float32).min
    x[6] = float("nan")
    x[7, :] = -inf
    x[7, 2000] = 3.0
    x[8] = 1e30
    x[8, 3] = -1e30
    x[9, ::2] = 0.0
    x[9, 1::2] = -0.0
    _check(binding, x, [0, 4, 3, 1, 9, 99, 0, 2000, 3, 8], 9)


@pytest.mark.parametrize("order", ["constant", "rising", "falling", "late_peaks", "few"])
def test_rows_in_parts(binding, order):
    """Rows long enough to be shared between workgroups, their best in one part or in all."""
    V = 150001
    x = torch.arange(V, dtype=torch.float64, device="cuda")
    x = {"constant": torch.zeros_like(x) - 2.0, "rising": torch.round(x * (512.0 / V)) / 64, "falling": -x * (8.0 / V),
         "late_peaks": torch.where(x > V - 3000, 5.0 + x / V, torch.sin(x)),
         "few": torch.where(x % 17000 == 3, x / V, -float("inf"))}[order]
    _check(binding, x.to(torch.float32)[None].repeat(3, 1).contiguous(), [0, V - 1, 3], 64)


@pytest.mark.parametrize("V", [3001, 120003])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_special_parts(binding, V, dtype):
    """Values in one place of a row only, or everywhere but there."""
    inf, low = float("inf"), torch.finfo(dtype).min
    x = _logits(12, V, dtype, seed=5)
    x[0, : V // 2] = -inf
    x[1, V // 2:] = low
    x[2, V - 1] = float("nan")
    x[3, V - 1] = inf
    x[4] = -inf
    x[4, V - 2] = 1.0
    x[5] = low
    x[5, V - 2] = -3.0e38
    x[6, V // 3] = 3.0e38  # its product with log2 e is no fp32 number
    x[7] = low
    x[8, 1:] = -inf
    x[9] = 3.0e38
    x[10] = -inf
    x[11, : V - 1] = -2.0e37
    tok = [0, V - 1, 5, 5, V - 2, V - 2, V // 3, 1, 0, 7, 7, V - 1]
    got = _check(binding, x, tok, 11)
    assert got["lse"][[2, 3]].isnan().all() and not got["lse"][[0, 1, 4, 5, 6, 7, 8, 9]].isnan().any()


@pytest.mark.parametrize("n", [65, 256, 257, 513])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_row_counts(binding, n, dtype):
    _check(binding, _logits(n, 33001, dtype, stride=33003), np.arange(n) * 64, 20)


def test_parts_in_graphs_that_share_a_workspace(binding):
    V, k = 140000, 9
    x = [_logits(5, V, seed=i) for i in range(2)]
    tok = torch.arange(5, dtype=torch.int32, device="cuda") * 1000
    ws = torch.zeros(binding.token_scores_workspace_bytes(5, V, k), dtype=torch.uint8, device="cuda")
    graphs, got = [], []
    for i in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            got.append(binding.token_scores(x[i], tok, k, workspace=ws))
    for turn in range(3):
        for i in range(2):
            x[i].copy_(_logits(5, V, seed=10 * turn + i + 7))
        for i in (0, 1, 0):
            graphs[i].replay()
        for i in range(2):
            want = binding.token_scores(x[i], tok, k)
            torch.cuda.synchronize()
            for name in want:
                assert torch.equal(got[i][name], want[name]), (turn, i, name)


def test_given_tokens_of_a_tree(binding):
    x = _logits(7, 997)
    _check(binding, x, [5, 996, -1, 0, 3, 900, 997, 5, 5, 1 << 30], 3, row_of=[0, 0, 1, 6, 6, 2, 3, -1, 7, 0])
    _check(binding, x, [1] * 3000, 2, row_of=[i % 8 for i in range(3000)])
    _check(binding, x, None, 4)
    _check(binding, x, [1, 2, 3, 4, 5, 6, -3], 0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,V,m", [(6000, 300, 2048), (6000, 300, 2049), (3, 150001, 5000), (9, 3000, 40000)])
def test_many_tokens_under_rows_of_their_own(binding, dtype, n, V, m):
    """The same bits as a few at a time, whatever the rows hold."""
    x = _logits(n, V, dtype, stride=V + 5)
    x[0] = -float("inf")
    x[1, 7] = float("nan")
    x[2] = torch.finfo(dtype).max  # (whose product with log2 e is no number of these)
    g = torch.Generator(device="cuda").manual_seed(m)
    tok = torch.randint(-2, V + 2, (m,), device="cuda", generator=g, dtype=torch.int32)
    row = torch.randint(-1, n + 1, (m,), device="cuda", generator=g, dtype=torch.int32)
    row[:40] = torch.arange(40, device="cuda", dtype=torch.int32) % 3
    got = binding.token_scores(x, tok, 3, row_of=row)
    parts = [binding.token_scores(x, tok[i:i + 1000].contiguous(), 3, row_of=row[i:i + 1000].contiguous()) for i in range(0, m, 1000)]
    want = torch.cat([p["logprob"] for p in parts])
    assert torch.equal(got["logprob"].isnan(), want.isnan())
    assert torch.equal(got["logprob"].nan_to_num(nan=7.0), want.nan_to_num(nan=7.0))
    for name in ("lse", "entropy", "top_token", "top_logprob"):
        assert torch.equal(got[name].nan_to_num(nan=7.0), parts[0][name].nan_to_num(nan=7.0))


def test_time_of_many_tokens_grows_with_their_number(binding):
    """300000 rows and tokens: within five times the call without row_of (looking through all
    tokens for every row would take a hundred times it)."""
    n, V = 300000, 64
    x = _logits(n, V, torch.bfloat16)
    tok = torch.arange(n, device="cuda", dtype=torch.int32) % V
    row = torch.arange(n, device="cuda", dtype=torch.int32)

    def ms(row_of):
        ev = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
        for i in range(2):  # (the second one counts)
            ev[0].record()
            got = binding.token_scores(x, tok, row_of=row_of)
            ev[1].record()
        torch.cuda.synchronize()
        return ev[0].elapsed_time(ev[1]), got

    (plain, a), (under, b) = ms(None), ms(row)
    assert torch.equal(a["logprob"], b["logprob"])
    assert under <= 5 * plain, (plain, under)


def test_near_certain_row(binding):
    x = torch.full((1, 32000), -30.0, device="cuda")
    x[0, 123] = 10.0
    got = _check(binding, x, [123], 2)
    assert float(got["logprob"][0]) <= 0.0


def test_in_a_graph_and_on_a_stream(binding):
    x = _logits(9, 32000)
    tok = torch.arange(9, dtype=torch.int32, device="cuda")
    ws = torch.zeros(binding.token_scores_workspace_bytes(9, 32000, 5), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = binding.token_scores(x, tok, 5, workspace=ws)
    for turn in range(3):
        x.copy_(_logits(9, 32000, seed=turn + 10))
        want = binding.token_scores(x, tok, 5)
        graph.replay()
        torch.cuda.synchronize()
        for name in want:
            assert torch.equal(got[name], want[name]), (turn, name)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = binding.token_scores(x, tok, 5, stream=side)
    side.synchronize()
    assert torch.equal(other["logprob"], want["logprob"])


def test_refusals(binding):
    x = _logits(2, 100)
    tok = torch.zeros(2, dtype=torch.int32, device="cuda")
    for bad in (x.double(), x[0], x.t(), x.cpu()):
        with pytest.raises(ValueError):
            binding.token_scores(bad, tok)
    for bad in (tok.long(), tok[:1], tok[None]):
        with pytest.raises(ValueError):
            binding.token_scores(x, bad)
    with pytest.raises(ValueError):
        binding.token_scores(x, tok, row_of=tok[:1])
    for k in (-1, 65):
        with pytest.raises((binding.LlmcadError, RuntimeError, ValueError)):
            binding.token_scores(x, tok, k)
    with pytest.raises(binding.LlmcadError):
        binding.token_scores(x, tok, 3, workspace=torch.zeros(8, dtype=torch.uint8, device="cuda"))


def test_a_stream_of_another_gpu_is_refused(binding):
    import types

    x = _logits(2, 100)
    with pytest.raises(ValueError, match="stream"):
        binding.token_scores(x, None, stream=types.SimpleNamespace(device=torch.device("cuda", 1)))
