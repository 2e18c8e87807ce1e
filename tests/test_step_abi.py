"""Refusals of the operators around a step's attention (normed store, adjusted logits, accept walk, forks and
compaction) on the CPU: every bad argument is turned down on the host, before anything reaches a device; the
sizes they report; and token masks."""

import ctypes

import pytest
import torch

import workloads

FAKE = 0x10000  # (aligned; never dereferenced: every case below fails a host check)
FAR = 0x40000000


@pytest.fixture(scope="module")
def binding():
    from paper_2309_04255_amd import binding

    return binding


@pytest.fixture(scope="module")
def cfg(binding):
    return binding.make_config(workloads.MODELS["llama7b"])


def _call(binding, name, cfg, order, defaults, kw):
    a = {**defaults, **kw}
    return getattr(binding.lib(), name)(None if a.get("cfg", 1) is None else ctypes.byref(cfg), *(a[k] for k in order), None)


STORE = dict(Hkv=32, layer=0, q=FAKE, qs=12288, k=FAKE, ks=12288, v=FAKE, vs=12288, qg=FAKE, qgs=0, kg=None, kgs=128, out=FAKE,
             kp=FAKE, vp=FAKE, n_pages=9, plan=FAKE, bytes=1 << 30, B=4, N=10)


@pytest.mark.parametrize("kw,status", [
    (dict(cfg=None), "EARG"), (dict(Hkv=0), "EARG"), (dict(Hkv=7), "ESHAPE"), (dict(layer=-1), "EARG"), (dict(layer=32), "EARG"), (dict(q=None), "EARG"),
    (dict(v=None), "EARG"), (dict(out=None), "EARG"), (dict(kp=None), "EARG"), (dict(q=FAKE + 2), "EARG"), (dict(vp=FAKE + 8), "EARG"),
    (dict(qs=4088), "ESHAPE"), (dict(vs=-8), "ESHAPE"), (dict(ks=4100), "EARG"), (dict(n_pages=0), "EARG"), (dict(bytes=64), "EWORKSPACE"),
    (dict(B=0), "EARG"), (dict(N=0), "EARG"), (dict(qg=FAKE + 2), "EARG"), (dict(kg=FAKE + 8), "EARG"), (dict(qgs=129), "EARG"), (dict(kgs=4), "EARG"),
    (dict(qgs=120), "ESHAPE"), (dict(kgs=-128), "ESHAPE"),
])
def test_norm_store(binding, cfg, kw, status):
    assert _call(binding, "llmcad_batch_norm_store", cfg, STORE, STORE, kw) == getattr(binding, status)


BY = dict(tokens=FAKE, history=FAKE, history_stride=100, prompt_len=FAKE, seen=FAKE, penalties=FAKE, bias_start=FAKE, bias_token=FAKE,
          bias_value=FAKE, n_bias=4, allow=FAKE, n_masks=3, mask_of=FAKE)
ADJUST = dict(plan=FAKE, bytes=1 << 30, B=4, N=10, logits=FAKE, bits=32, stride=32000, by=BY, out=FAR, out_stride=32000, greedy=FAKE, ws=FAKE,
              ws_bytes=1 << 30)


@pytest.mark.parametrize("kw,status", [
    (dict(cfg=None), "EARG"), (dict(plan=None), "EARG"), (dict(plan=FAKE + 4), "EARG"), (dict(logits=None), "EARG"), (dict(bits=8), "EARG"), (dict(by=None), "EARG"),
    (dict(out=None, greedy=None), "EARG"), (dict(ws=None), "EARG"), (dict(ws=FAKE + 8), "EARG"), (dict(logits=FAKE + 2), "EARG"),
    (dict(logits=FAKE + 1, bits=16), "EARG"), (dict(out=FAR + 2), "EARG"), (dict(greedy=FAKE + 1), "EARG"), (dict(stride=31999), "ESHAPE"),
    (dict(out_stride=31999), "ESHAPE"), (dict(bytes=100), "EWORKSPACE"), (dict(ws_bytes=100), "EWORKSPACE"), (dict(B=0), "EARG"), (dict(N=0), "EARG"),
    (dict(B=1025), "EARG"), (dict(out=FAKE, out_stride=32008), "EARG"), (dict(out=FAKE + 4), "EARG"), (dict(out=FAKE + 9 * 128000 + 127996), "EARG"),
    (dict(by=dict(tokens=None)), "EARG"), (dict(by=dict(history_stride=-1)), "EARG"), (dict(by=dict(bias_token=None)), "EARG"),
    (dict(by=dict(bias_value=None)), "EARG"), (dict(by=dict(n_bias=-1)), "EARG"), (dict(by=dict(n_masks=0)), "EARG"), (dict(by=dict(mask_of=None)), "EARG"),
    (dict(by=dict(allow=None)), "EARG"),
    *((dict(by={k: FAKE + 2}), "EARG") for k in BY if isinstance(BY[k], int) and BY[k] == FAKE),
])
def test_adjust(binding, cfg, kw, status):
    if "by" in kw and kw["by"] is not None:
        kw = dict(kw, by={**BY, **kw["by"]})
    a = {**ADJUST, **kw}
    by = None if a["by"] is None else ctypes.byref(binding.LlmcadAdjustments(*(a["by"][k] for k, _ in binding.LlmcadAdjustments._fields_)))
    assert _call(binding, "llmcad_batch_adjust", cfg, ADJUST, {**a, "by": by}, {k: v for k, v in kw.items() if k == "cfg"}) == getattr(binding, status)


ACCEPT = dict(plan=FAKE, bytes=1 << 30, B=4, N=10, tokens=FAKE, greedy=FAKE, path=FAKE, length=FAKE, after=FAKE, history=None, stride=0)


@pytest.mark.parametrize("kw,status", [
    (dict(cfg=None), "EARG"), (dict(plan=None), "EARG"), (dict(plan=FAKE + 8), "EARG"), (dict(bytes=64), "EWORKSPACE"), (dict(B=0), "EARG"), (dict(N=-1), "EARG"),
    (dict(tokens=None), "EARG"), (dict(greedy=None), "EARG"), (dict(path=None), "EARG"), (dict(length=None), "EARG"), (dict(after=None), "EARG"),
    (dict(history=FAKE, stride=-1), "EARG"), (dict(tokens=FAKE + 2), "EARG"), (dict(history=FAKE + 1, stride=5), "EARG"), (dict(path=FAKE + 3), "EARG"),
])
def test_accept(binding, cfg, kw, status):
    assert _call(binding, "llmcad_batch_accept", cfg, ACCEPT, ACCEPT, kw) == getattr(binding, status)


@pytest.mark.parametrize("out", ["path", "length", "after", "history"])
@pytest.mark.parametrize("at", [0, 36, 4096, 4132])  # (the first and the last of the tokens and of the greedy ones)
def test_accept_writes_apart_from_what_it_reads(binding, cfg, out, at):
    apart = dict(tokens=FAKE, greedy=FAKE + 4096, path=FAR, length=FAR + 4096, after=FAR + 8192, history=FAR + 12288, stride=5)
    a = {**ACCEPT, **apart, out: FAKE + at}
    assert _call(binding, "llmcad_batch_accept", cfg, ACCEPT, a, {}) == binding.EARG


FORK = dict(Hkv=32, kp=FAKE, vp=FAKE, n_pages=9, B=4, table=FAKE, max_pages=3, held=FAKE, source=FAKE, table_out=FAR, held_out=FAR + 4096,
            free=FAR + 8192, n_free=FAR + 9000, status=FAR + 9004, ws=FAKE, ws_bytes=1 << 20)


@pytest.mark.parametrize("kw,status", [
    (dict(cfg=None), "EARG"), (dict(Hkv=0), "EARG"), (dict(Hkv=3), "ESHAPE"), (dict(kp=None), "EARG"), (dict(vp=FAKE + 8), "EARG"), (dict(n_pages=0), "EARG"),
    (dict(n_pages=(1 << 18) + 1), "EARG"), (dict(B=0), "EARG"), (dict(B=1025), "EARG"), (dict(table=None), "EARG"), (dict(max_pages=0), "EARG"),
    (dict(max_pages=(1 << 18) + 1), "EARG"), (dict(held=None), "EARG"), (dict(source=None), "EARG"), (dict(table_out=None), "EARG"),
    (dict(held_out=None), "EARG"), (dict(free=None), "EARG"), (dict(n_free=None), "EARG"), (dict(status=None), "EARG"), (dict(ws=None), "EARG"),
    (dict(ws=FAKE + 4), "EARG"), (dict(ws_bytes=256), "EWORKSPACE"), (dict(table=FAKE + 2), "EARG"), (dict(status=FAKE + 1), "EARG"),
    (dict(table_out=FAKE), "EARG"), (dict(table_out=FAKE + 44), "EARG"), (dict(held_out=FAKE), "EARG"), (dict(held_out=FAKE + 12), "EARG"),
    (dict(table=FAR + 4100), "EARG"), (dict(free=FAKE + 40), "EARG"), (dict(n_free=FAKE), "EARG"), (dict(status=FAKE + 8), "EARG"),
])
def test_fork(binding, cfg, kw, status):
    assert _call(binding, "llmcad_batch_fork", cfg, FORK, FORK, kw) == getattr(binding, status)


COMPACT = dict(Hkv=32, kp=FAKE, vp=FAKE, n_pages=9, B=4, table=FAKE, max_pages=3, held=FAKE, table_out=FAR, n_used=FAR + 9000, ws=FAKE, ws_bytes=1 << 20)


@pytest.mark.parametrize("kw,status", [
    (dict(cfg=None), "EARG"), (dict(Hkv=5), "ESHAPE"), (dict(kp=FAKE + 2), "EARG"), (dict(n_pages=(1 << 18) + 1), "EARG"), (dict(n_used=None), "EARG"),
    (dict(n_used=FAR + 2), "EARG"), (dict(n_used=FAKE + 44), "EARG"), (dict(table_out=FAKE + 4), "EARG"), (dict(ws_bytes=100), "EWORKSPACE"), (dict(held=None), "EARG"),
])
def test_compact(binding, cfg, kw, status):
    assert _call(binding, "llmcad_batch_compact", cfg, COMPACT, COMPACT, kw) == getattr(binding, status)


def test_workspace_sizes(binding, cfg):
    assert binding.batch_adjust_workspace_bytes(cfg, 10) >= 10 * 8 * 8  # (32000 tokens are eight pieces)
    assert binding.batch_adjust_workspace_bytes(cfg, 0) == 0
    for bad in ((0, 5), (1025, 5), (1, 0), (1, (1 << 18) + 1)):
        assert binding.batch_pages_workspace_bytes(*bad) == 0
    assert binding.batch_pages_workspace_bytes(1024, 2) >= 256 + 12 * 1024
    assert binding.batch_pages_workspace_bytes(1, 1 << 18) >= 256 + 12 * (1 << 17)


def test_token_mask(binding):
    t = torch.tensor([[0, 31, 32], [70, -1, 71]], dtype=torch.int32)
    words = binding.token_mask(t, 71).tolist()
    assert [w & 0xFFFFFFFF for w in words] == [1 | 1 << 31, 1, 1 << 6]
    assert binding.token_mask(torch.arange(64), 64).tolist() == [-1, -1]
    assert binding.token_mask(torch.tensor([], dtype=torch.int64), 5).tolist() == [0]


@pytest.mark.parametrize("call", ["norm_store", "adjust", "accept", "fork", "compact"])
def test_tensors_must_be_on_a_gpu(binding, cfg, call):
    i = torch.zeros(1, dtype=torch.int32)
    t = torch.zeros(1, 1, dtype=torch.int32)
    x = torch.zeros(1, 32, 128, dtype=torch.bfloat16)
    k = torch.zeros(32, 1, 32, 64, 128, dtype=torch.bfloat16)
    p = torch.zeros(64, dtype=torch.uint8)
    with pytest.raises(ValueError, match="GPU"):
        if call == "norm_store":
            binding.batch_norm_store(cfg, 32, 0, x, x, x, None, None, x, k, k.transpose(3, 4).contiguous(), p, 1)
        elif call == "adjust":
            binding.batch_adjust(cfg, p, 1, torch.zeros(1, 32000), greedy=i, workspace=p)
        elif call == "accept":
            binding.batch_accept(cfg, p, 1, i, i, i, i, i)
        elif call == "fork":
            binding.batch_fork(cfg, 32, k, k, t, i, i, t, i, i, p)
        else:
            binding.batch_compact(cfg, 32, k, k, t, i, t, p)
