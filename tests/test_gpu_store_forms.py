"""The forms of the store that steps of many rows take, plain and normed, against their float64 statement
(oracle/batch.py): several heads a workgroup, four of them loaded ahead, with the last group of queries reaching into
the keys; a head's values by one, two or four workgroups.

Tolerances as in test_gpu_norm_store.py: one rounding to bf16 (2^-8 of the value), and before it under 2^-19 of the
size of the two products that a rotation adds (without the norm, fewer operations)."""

import numpy as np
import pytest
import torch

from oracle import batch as ob
from test_gpu_batch import PAGE, Case, _np

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def binding():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2309_04255_amd import binding

    return binding


def _rows(total, seed):
    """Requests of 0 to 41 rows, `total` in all, and what they hold."""
    rng = np.random.default_rng(seed)
    n = []
    while sum(n) < total:
        n.append(min(int(rng.integers(0, 42)), total - sum(n)))
    return n, rng.integers(0, 200, len(n)).tolist()


# (a workgroup turns 256 / (Dh / 16) rows of (their number of such blocks) (H + Hkv) / 128 heads, up to eight; values:
# (64-row blocks) Hkv workgroups, doubled until there are 256)
FORMS = [
    pytest.param(_rows(751, 1), {"H": 30, "Hkv": 10, "Dh": 128, "pad": 9}, id="7 heads, values by 4"),
    pytest.param(_rows(990, 2), {"H": 30, "Hkv": 10, "Dh": 128, "pad": 33}, id="8 heads, values by 2"),
    pytest.param(_rows(1000, 3), {"H": 20, "Hkv": 20, "Dh": 128, "pad": 1}, id="8 heads, values whole"),
    pytest.param(([128] * 8, [64 * i for i in range(8)]), {"H": 20, "Hkv": 20, "Dh": 128, "tree": False}, id="whole pieces"),
    pytest.param(([128] * 8, [64 * i for i in range(8)]), {"H": 12, "Hkv": 6, "Dh": 128, "tree": False}, id="whole pieces by 4"),
    pytest.param(_rows(2100, 4), {"H": 16, "Hkv": 4, "Dh": 64, "pad": 5}, id="5 heads of 64, values by 2"),
    pytest.param(_rows(4200, 5), {"H": 9, "Hkv": 3, "Dh": 64, "pad": 2}, id="6 heads of 64, values by 2"),
    pytest.param(_rows(6200, 6), {"H": 9, "Hkv": 3, "Dh": 64}, id="8 heads of 64, values whole"),
]


@pytest.mark.parametrize("rows,kw", FORMS)
@pytest.mark.parametrize("gains", ["plain", "none", "one", "heads"])
def test_store(binding, rows, kw, gains):
    c = Case(binding, *rows, P=300, **kw)
    plan = c.plan()
    kp, vp = c.pages()
    k0, v0 = kp.clone(), vp.clone()
    g = torch.Generator(device="cuda").manual_seed(9)
    qkv = (torch.randn(c.N, c.H + 2 * c.Hkv, c.Dh, device="cuda", generator=g) * 2).to(torch.bfloat16)
    q, k, v = qkv[:, :c.H], qkv[:, c.H:c.H + c.Hkv], qkv[:, c.H + c.Hkv:]
    q_out = torch.full((c.N, c.H, c.Dh), 77.0, dtype=torch.bfloat16, device="cuda")
    shape = {"one": lambda h: (c.Dh,), "heads": lambda h: (h, c.Dh)}.get(gains)
    gain = [1 + 0.3 * torch.randn(*shape(h), device="cuda", generator=g) for h in (c.H, c.Hkv)] if shape else [None] * 2
    gain = [None if x is None else x.to(torch.bfloat16) for x in gain]
    if gains == "plain":
        binding.batch_store(c.cfg, c.Hkv, 0, q, k, v, q_out, kp, vp, c.d_plan, c.B)
    else:
        binding.batch_norm_store(c.cfg, c.Hkv, 0, q, k, v, *gain, q_out, kp, vp, c.d_plan, c.B)
    torch.cuda.synchronize()
    slot = torch.tensor(c.want()["slot"], device="cuda")
    assert torch.equal(plan["slot"].long(), slot)
    T = c.total
    assert bool((slot[:T] >= 0).all()) and bool((slot[T:] < 0).all())
    page, at = slot[:T] // PAGE, slot[:T] % PAGE
    rope = plan["rope"][:T].cpu().numpy().astype(np.float64)
    half = c.Dh // 2
    for x, w, got in ((q, gain[0], q_out[:T]), (k, gain[1], kp[0, page, :, at])):
        y = _np(x[:T])
        if gains != "plain":
            y = ob.norm(y, None if w is None else _np(w), 1e-6)
        want, (co, si) = ob.turn(y, rope), (np.abs(rope[:, None, :, i]) for i in range(2))
        a, b = np.abs(y[..., :half]), np.abs(y[..., half:])
        size = np.concatenate([a * co + b * si, b * co + a * si], -1)
        wrong = np.abs(_np(got) - want) > 2.0 ** -8 * np.abs(want) + 2.0 ** -19 * size
        assert not wrong.any(), np.argwhere(wrong)[:5]
    assert bool((q_out[T:] == 77.0).all())
    k0[0, page, :, at] = kp[0, page, :, at]
    v0[0, page, :, :, at] = v[:T]
    assert torch.equal(kp, k0) and torch.equal(vp, v0)  # (the values' bits, and nothing else is written)
