"""Normed, turned and stored queries and keys against their float64 statement (oracle/batch.py).

Tolerance.  A value is rounded to bf16 once: 2^-8 of itself.  Before that, in fp32: the sum of up to 128
squares (16 in a lane one after the other, then three joins: 19 roundings, halved by the root), mean, eps, root
and quotient (5), scale and gain (2), and the rotation's products and sum (2): at most 2^-24 * 19, under 2^-19,
of the size of the two products that a rotation adds."""

import numpy as np
import pytest
import torch

from oracle import batch as ob
from test_gpu_batch import PAGE, Case, _dev, _np

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def binding():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2309_04255_amd import binding

    return binding


def _inputs(c, seed=0, scale=2.0, extra=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    width = (c.H + 2 * c.Hkv) * c.Dh
    x = (torch.randn(c.N, width + extra, device="cuda", generator=g) * scale).to(torch.bfloat16)[:, :width]
    return x, [t.unflatten(-1, (-1, c.Dh)) for t in x.split([c.H * c.Dh, c.Hkv * c.Dh, c.Hkv * c.Dh], -1)]


def _gains(c, kind, seed=3):
    g = torch.Generator(device="cuda").manual_seed(seed)
    if kind == "none":
        return None, None
    one = lambda h: (1 + 0.3 * torch.randn(*((h, c.Dh) if kind == "heads" else (c.Dh,)), device="cuda", generator=g)).to(torch.bfloat16)  # noqa: E731
    return one(c.H), one(c.Hkv)


def _check(c, rope, slots, q, k, v, gains, eps, q_out, kp, vp, before):
    rope = rope.cpu().numpy().astype(np.float64)
    for x, gain, got in ((q, gains[0], "q"), (k, gains[1], "k")):
        y = ob.norm(_np(x), None if gain is None else _np(gain), eps)
        want = ob.turn(y, rope)
        size = ob.turn(np.abs(y), np.stack([np.abs(rope[..., 0]), -np.abs(rope[..., 1])], -1))
        half = c.Dh // 2
        size[..., half:] = np.abs(y[..., half:]) * np.abs(rope[:, None, :, 0]) + np.abs(y[..., :half]) * np.abs(rope[:, None, :, 1])
        tol = 2.0 ** -8 * np.abs(want) + 2.0 ** -19 * size + 1e-38
        for r in range(c.N):
            if slots[r] < 0:
                if got == "q":
                    assert torch.equal(q_out[r], before[0][r])
                continue
            mine = _np(q_out[r]) if got == "q" else _np(kp[0, slots[r] // PAGE, :, slots[r] % PAGE])
            assert (np.abs(mine - want[r]) <= tol[r]).all(), (got, r)
    kw, vw = before[1].clone(), before[2].clone()
    for r in range(c.N):
        if slots[r] >= 0:
            kw[0, slots[r] // PAGE, :, slots[r] % PAGE] = kp[0, slots[r] // PAGE, :, slots[r] % PAGE]
            vw[0, slots[r] // PAGE, :, :, slots[r] % PAGE] = v[r]
    assert torch.equal(kp, kw) and torch.equal(vp, vw)  # (nothing else is written)


@pytest.mark.parametrize("n,held,kw,kind", [
    ([1], [0], {}, "one"),
    ([1], [63], {"H": 1, "Hkv": 1}, "heads"),
    ([1] * 9, [0, 1, 62, 63, 64, 65, 127, 128, 700], {"H": 8, "Hkv": 2, "Dh": 128, "tree": False}, "one"),
    ([31], [200], {"H": 4, "Dh": 128}, "heads"),
    ([128, 0, 3, 65], [63, 5, 64, 1], {"H": 6, "Hkv": 3, "pad": 40}, "none"),
    ([41] * 7, [10 * i for i in range(7)], {"H": 5, "Hkv": 5, "Dh": 128, "pad": 1}, "heads"),
    ([3] * 100, [7 * i for i in range(100)], {"H": 24, "Hkv": 8, "P": 1000}, "one"),
])
@pytest.mark.parametrize("extra", [0, 24])
def test_norm_store(binding, n, held, kw, kind, extra):
    c = Case(binding, n, held, **kw)
    got = c.plan()
    _, (q, k, v) = _inputs(c, extra=extra)
    gains = _gains(c, kind)
    kp, vp = c.pages()
    q_out = torch.full((c.N, c.H, c.Dh), 7.0, dtype=torch.bfloat16, device="cuda")
    before = q_out.clone(), kp.clone(), vp.clone()
    binding.batch_norm_store(c.cfg, c.Hkv, 0, q, k, v, *gains, q_out, kp, vp, c.d_plan, c.B)
    torch.cuda.synchronize()
    _check(c, got["rope"], got["slot"].tolist(), q, k, v, gains, 1e-6, q_out, kp, vp, before)


def test_small_zero_and_large_heads(binding):
    """Heads of zeros stay zeros, tiny ones are divided by the root of eps, large ones come to the norm's size."""
    c = Case(binding, [4], [9], H=4, Dh=64)
    c.cfg.rms_eps = 1e-3
    got = c.plan()
    _, (q, k, v) = _inputs(c)
    q = q.contiguous().clone()
    q[0], q[1], q[2, 0] = 0.0, q[1] * 1e-20, q[2, 0] * 1e15
    gains = _gains(c, "one")
    kp, vp = c.pages()
    q_out = torch.zeros(c.N, c.H, c.Dh, dtype=torch.bfloat16, device="cuda")
    before = q_out.clone(), kp.clone(), vp.clone()
    binding.batch_norm_store(c.cfg, c.Hkv, 0, q, k, v, *gains, q_out, kp, vp, c.d_plan, c.B)
    assert not q_out[0].any()
    _check(c, got["rope"], got["slot"].tolist(), q, k, v, gains, 1e-3, q_out, kp, vp, before)


def test_a_nan_stays_in_its_head(binding):
    c = Case(binding, [5], [9], H=4, Dh=128)
    got = c.plan()
    _, (q, k, v) = _inputs(c)
    q = q.contiguous().clone()
    gains = _gains(c, "one")
    out = []
    for bad in (0.0, float("nan"), float("inf")):
        q[2, 1, 77] = bad
        kp, vp = c.pages()
        q_out = torch.zeros(c.N, c.H, c.Dh, dtype=torch.bfloat16, device="cuda")
        binding.batch_norm_store(c.cfg, c.Hkv, 0, q, k, v, *gains, q_out, kp, vp, c.d_plan, c.B)
        out.append((q_out, kp, vp))
    for q_out, kp, vp in out[1:]:
        assert torch.equal(kp, out[0][1]) and torch.equal(vp, out[0][2])
        other = torch.ones(c.N, c.H, dtype=torch.bool)
        other[2, 1] = False
        assert torch.equal(q_out[other.cuda()], out[0][0][other.cuda()])
    assert got["slot"][0] >= 0


def test_in_place_layers_and_gains_of_a_wider_tensor(binding):
    """q_out may be q; layers are apart; gains may be rows of a larger tensor."""
    c = Case(binding, [17, 5], [60, 0], H=4, Hkv=2, Dh=64, L=3)
    got = c.plan()
    _, (q, k, v) = _inputs(c)
    wide = torch.randn(4, 2, 64, device="cuda").to(torch.bfloat16)
    gains = wide[:, 1], wide[:2, 0]
    kp, vp = c.pages()
    before = kp.clone(), vp.clone()
    q = q.contiguous()
    want = torch.empty_like(q)
    binding.batch_norm_store(c.cfg, c.Hkv, 1, q, k, v, gains[0], gains[1], want, kp, vp, c.d_plan, c.B)
    assert torch.equal(kp[0], before[0][0]) and torch.equal(kp[2], before[0][2]) and torch.equal(vp[0], before[1][0])
    k1, v1 = kp[1:2].clone(), vp[1:2].clone()
    kp2, vp2 = before[0].clone(), before[1].clone()
    mine = q.clone()
    binding.batch_norm_store(c.cfg, c.Hkv, 1, mine, k, v, gains[0].contiguous(), gains[1].contiguous(), mine, kp2, vp2, c.d_plan, c.B)
    assert torch.equal(mine, want) and torch.equal(kp2, kp) and torch.equal(vp2, vp)
    c.L = 1
    _check(c, got["rope"], got["slot"].tolist(), q, k, v, [g.contiguous() for g in gains], 1e-6, want, k1, v1, (want.clone(), before[0][1:2], before[1][1:2]))


def test_a_plan_of_other_sizes_writes_nothing(binding):
    c = Case(binding, [5, 3], [9, 0], pad=4)
    c.plan()
    _, (q, k, v) = _inputs(c)
    kp, vp = c.pages()
    before = kp.clone(), vp.clone()
    q_out = torch.zeros(c.N, c.H, c.Dh, dtype=torch.bfloat16, device="cuda")
    binding.batch_norm_store(c.cfg, c.Hkv, 0, q, k, v, None, None, q_out, kp, vp, c.d_plan, c.B - 1)
    binding.batch_norm_store(c.cfg, c.Hkv, 0, q[:-1], k[:-1], v[:-1], None, None, q_out[:-1], kp, vp, c.d_plan, c.B)
    assert not q_out.any() and torch.equal(kp, before[0]) and torch.equal(vp, before[1])


def test_a_captured_store_follows_its_plan(binding):
    """Plan, normed store and attention in one graph, replayed with other lengths, eager work between."""
    c = Case(binding, [7, 1, 30], [10, 64, 3], H=4, Hkv=2, Dh=128)
    c.plan()
    _, (q, k, v) = _inputs(c)
    gains = _gains(c, "heads")
    kp, vp = c.pages()
    q_out = torch.zeros(c.N, c.H, c.Dh, dtype=torch.bfloat16, device="cuda")
    start, held, par, free = _dev(c.row_start), _dev(c.held), _dev(c.parent), _dev(c.free)

    def step(q_out, kp, vp):
        binding.batch_plan(c.cfg, start, held, par, 0, c.d_table, free, c.n_pages, c.d_plan, c.N)
        binding.batch_norm_store(c.cfg, c.Hkv, 0, q, k, v, *gains, q_out, kp, vp, c.d_plan, c.B)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step(q_out, kp, vp)
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(q_out, kp, vp)
    for lengths in ([10, 64, 3], [9, 60, 40], [0, 1, 2]):
        held.copy_(_dev(lengths))
        clean = c.pages()
        kp.copy_(clean[0])
        vp.copy_(clean[1])
        q_out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        want = torch.zeros_like(q_out), *(t.clone() for t in clean)
        step(*want)
        torch.cuda.synchronize()
        assert torch.equal(q_out, want[0]) and torch.equal(kp, want[1]) and torch.equal(vp, want[2])


@pytest.mark.parametrize("change,match", [
    (dict(q_gain=lambda c: torch.ones(c.Dh, device="cuda")), "q_gain"),
    (dict(q_gain=lambda c: torch.ones(c.H + 1, c.Dh, dtype=torch.bfloat16, device="cuda")), "q_gain"),
    (dict(k_gain=lambda c: torch.ones(c.Dh + 1, dtype=torch.bfloat16, device="cuda")), "k_gain"),
    (dict(k_gain=lambda c: torch.ones(c.Dh, dtype=torch.bfloat16)), "cuda"),
    (dict(q=lambda c: torch.zeros(c.N, c.H, c.Dh, device="cuda")), "q must be"),
])
def test_refusals(binding, change, match):
    c = Case(binding, [3], [0])
    c.plan()
    _, (q, k, v) = _inputs(c)
    kp, vp = c.pages()
    a = dict(q=q, k=k, v=v, q_gain=None, k_gain=None, q_out=torch.empty(c.N, c.H, c.Dh, dtype=torch.bfloat16, device="cuda"))
    a.update({name: make(c) for name, make in change.items()})
    with pytest.raises(ValueError, match=match):
        binding.batch_norm_store(c.cfg, c.Hkv, 0, a["q"], a["k"], a["v"], a["q_gain"], a["k_gain"], a["q_out"], kp, vp, c.d_plan, c.B)
