"""Refusals of the batch operators and the token scores on the CPU: every bad argument is turned down
on the host, before anything reaches a device; and the sizes they report."""

import ctypes

import pytest

import workloads

FAKE = 0x10000  # (aligned; never dereferenced: every case below fails a host check)


@pytest.fixture(scope="module")
def binding():
    from paper_2309_04255_amd import binding

    return binding


@pytest.fixture(scope="module")
def cfg(binding):
    return binding.make_config(workloads.MODELS["llama7b"])


def test_plan_sizes(binding, cfg):
    for B, N in ((1, 1), (7, 300), (1024, 262144)):
        total, regions = binding.batch_plan_bytes(cfg, B, N), []
        for which, want in enumerate((4 * N, 4 * N, 16 * N, 512 * N, 4 * B, 4)):
            off, size = ctypes.c_size_t(), ctypes.c_size_t()
            assert binding.lib().llmcad_batch_plan_region(ctypes.byref(cfg), B, N, which, ctypes.byref(off),
                                                          ctypes.byref(size)) == binding.OK
            assert size.value == want and off.value % 4 == 0 and off.value + want <= total
            regions.append((off.value, off.value + want))
        regions.sort()
        assert all(a[1] <= b[0] for a, b in zip(regions, regions[1:]))
    for B, N in ((0, 1), (1, 0), (1025, 10), (1, 262145), (-1, 5)):
        assert binding.batch_plan_bytes(cfg, B, N) == 0
    off = ctypes.c_size_t()
    assert binding.lib().llmcad_batch_plan_region(ctypes.byref(cfg), 1, 1, 6, ctypes.byref(off), ctypes.byref(off)) == binding.EARG
    assert binding.lib().llmcad_batch_plan_region(ctypes.byref(cfg), 1, 1, 0, None, ctypes.byref(off)) == binding.EARG


def test_workspace_sizes(binding, cfg):
    sizes = [binding.batch_workspace_bytes(cfg, 32, 8, n) for n in (1, 31, 500, 2000, 100000)]
    assert all(s > 0 for s in sizes) and sizes[-1] > sizes[-2]
    assert binding.batch_workspace_bytes(cfg, 5, 8, 31) == 0   # (32 heads are no multiple of 5)
    assert binding.batch_workspace_bytes(cfg, 0, 8, 31) == 0
    assert binding.token_scores_workspace_bytes(1, 32000, 64) > 0
    for bad in ((0, 5, 1), (1, 0, 1), (1, 5, 65), (1, 5, -1)):
        assert binding.token_scores_workspace_bytes(*bad) == 0


PLAN = dict(B=4, N=10, row_start=FAKE, held=FAKE, parent=FAKE, prefix=5, table=FAKE, max_pages=3, free=FAKE, n_free=2,
            n_pages=9, plan=FAKE, bytes=1 << 30)


def _plan(binding, cfg, **kw):
    a = {**PLAN, **kw}
    return binding.lib().llmcad_batch_plan(ctypes.byref(cfg), a["B"], a["N"], a["row_start"], a["held"], a["parent"], a["prefix"],
                                           a["table"], a["max_pages"], a["free"], a["n_free"], a["n_pages"], a["plan"],
                                           a["bytes"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(B=0), "EARG"), (dict(B=1025), "EARG"), (dict(N=0), "EARG"), (dict(N=1 << 30), "EARG"), (dict(row_start=None), "EARG"),
    (dict(held=None), "EARG"), (dict(table=None), "EARG"), (dict(plan=None), "EARG"), (dict(plan=FAKE + 4), "EARG"),
    (dict(max_pages=0), "EARG"), (dict(n_pages=0), "EARG"), (dict(n_pages=1 << 25), "EARG"), (dict(n_free=-1), "EARG"),
    (dict(free=None), "EARG"), (dict(prefix=-1), "ECAPACITY"), (dict(prefix=(1 << 30) + 1), "ECAPACITY"),
    (dict(bytes=100), "EWORKSPACE"),
])
def test_plan_refusals(binding, cfg, kw, status):
    assert _plan(binding, cfg, **kw) == getattr(binding, status)


STORE = dict(Hkv=32, layer=0, q=FAKE, qs=12288, k=FAKE, ks=12288, v=FAKE, vs=12288, out=FAKE, kp=FAKE, vp=FAKE, n_pages=9,
             plan=FAKE, bytes=1 << 30, B=4, N=10)


def _store(binding, cfg, **kw):
    a = {**STORE, **kw}
    return binding.lib().llmcad_batch_store(ctypes.byref(cfg), a["Hkv"], a["layer"], a["q"], a["qs"], a["k"], a["ks"], a["v"],
                                            a["vs"], a["out"], a["kp"], a["vp"], a["n_pages"], a["plan"], a["bytes"], a["B"],
                                            a["N"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(Hkv=0), "EARG"), (dict(Hkv=7), "ESHAPE"), (dict(Hkv=64), "ESHAPE"), (dict(layer=-1), "EARG"), (dict(layer=32), "EARG"),
    (dict(q=None), "EARG"), (dict(v=None), "EARG"), (dict(out=None), "EARG"), (dict(kp=None), "EARG"), (dict(q=FAKE + 2), "EARG"),
    (dict(vp=FAKE + 8), "EARG"), (dict(qs=4095), "ESHAPE"), (dict(ks=100), "ESHAPE"), (dict(vs=-8), "ESHAPE"),
    (dict(qs=12289), "EARG"), (dict(ks=4100), "EARG"), (dict(n_pages=0), "EARG"), (dict(bytes=64), "EWORKSPACE"),
    (dict(B=0), "EARG"), (dict(N=0), "EARG"),
])
def test_store_refusals(binding, cfg, kw, status):
    assert _store(binding, cfg, **kw) == getattr(binding, status)


ATTENTION = dict(Hkv=32, layer=0, q=FAKE, qs=4096, kc=FAKE, vc=FAKE, cap=128, prefix=100, kp=FAKE, vp=FAKE, n_pages=9, table=FAKE,
                 max_pages=3, plan=FAKE, bytes=1 << 30, B=4, N=10, out=FAKE, ws=FAKE, ws_bytes=1 << 34)


def _attention(binding, cfg, **kw):
    a = {**ATTENTION, **kw}
    return binding.lib().llmcad_batch_attention(
        ctypes.byref(cfg), a["Hkv"], a["layer"], a["q"], a["qs"], a["kc"], a["vc"], a["cap"], a["prefix"], a["kp"], a["vp"],
        a["n_pages"], a["table"], a["max_pages"], a["plan"], a["bytes"], a["B"], a["N"], a["out"], a["ws"], a["ws_bytes"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(Hkv=3), "ESHAPE"), (dict(layer=32), "EARG"), (dict(q=None), "EARG"), (dict(qs=4088), "ESHAPE"), (dict(qs=4100), "EARG"),
    (dict(kc=None), "EARG"), (dict(vc=FAKE + 2), "EARG"), (dict(cap=100), "ECAPACITY"), (dict(cap=64), "ECAPACITY"), (dict(cap=(1 << 24) + 64), "ECAPACITY"),
    (dict(prefix=-1), "ECAPACITY"), (dict(prefix=129), "ECAPACITY"), (dict(kp=None), "EARG"), (dict(table=None), "EARG"),
    (dict(max_pages=0), "EARG"), (dict(out=FAKE + 4), "EARG"), (dict(ws=None), "EARG"), (dict(ws_bytes=1000), "EWORKSPACE"),
    (dict(bytes=1000), "EWORKSPACE"), (dict(B=2000), "EARG"), (dict(N=-1), "EARG"),
])
def test_attention_refusals(binding, cfg, kw, status):
    assert _attention(binding, cfg, **kw) == getattr(binding, status)


COMMIT = dict(Hkv=32, kp=FAKE, vp=FAKE, n_pages=9, plan=FAKE, bytes=1 << 30, B=4, N=10, path=FAKE, acc=FAKE)


def _commit(binding, cfg, **kw):
    a = {**COMMIT, **kw}
    return binding.lib().llmcad_batch_commit(ctypes.byref(cfg), a["Hkv"], a["kp"], a["vp"], a["n_pages"], a["plan"], a["bytes"],
                                             a["B"], a["N"], a["path"], a["acc"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(Hkv=-1), "EARG"), (dict(Hkv=31), "ESHAPE"), (dict(kp=None), "EARG"), (dict(vp=FAKE + 2), "EARG"), (dict(path=None), "EARG"),
    (dict(acc=None), "EARG"), (dict(plan=None), "EARG"), (dict(n_pages=-4), "EARG"), (dict(bytes=0), "EWORKSPACE"), (dict(N=0), "EARG"),
])
def test_commit_refusals(binding, cfg, kw, status):
    assert _commit(binding, cfg, **kw) == getattr(binding, status)


SCORES = dict(x=FAKE, bits=32, stride=1000, n=3, V=1000, tok=FAKE, row_of=None, m=3, lp=FAKE, ent=FAKE, lse=FAKE, k=4, tt=FAKE,
              tl=FAKE, ws=FAKE, ws_bytes=1 << 20)


def _scores(binding, **kw):
    a = {**SCORES, **kw}
    return binding.lib().llmcad_token_scores(a["x"], a["bits"], a["stride"], a["n"], a["V"], a["tok"], a["row_of"], a["m"], a["lp"],
                                             a["ent"], a["lse"], a["k"], a["tt"], a["tl"], a["ws"], a["ws_bytes"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), "EARG"), (dict(x=FAKE + 2), "EARG"), (dict(bits=16, x=FAKE + 1), "EARG"), (dict(bits=8), "EARG"), (dict(n=0), "EARG"),
    (dict(V=0, stride=0), "EARG"), (dict(V=(1 << 24) + 1, stride=1 << 25), "ESHAPE"), (dict(stride=999), "ESHAPE"),
    (dict(tok=None), "EARG"), (dict(lp=None), "EARG"), (dict(m=2), "EARG"), (dict(m=-1), "EARG"), (dict(k=65), "EARG"),
    (dict(k=-1), "EARG"), (dict(tt=None), "EARG"), (dict(ent=None), "EARG"), (dict(lse=None), "EARG"), (dict(ws=None), "EARG"),
    (dict(ws_bytes=1), "EWORKSPACE"), (dict(tok=FAKE + 2), "EARG"),
])
def test_scores_refusals(binding, kw, status):
    assert _scores(binding, **kw) == getattr(binding, status)


@pytest.mark.parametrize("kw", [dict(n=1 << 24, m=1 << 24), dict(m=(1 << 30) + 1, row_of=FAKE), dict(m=(1 << 31) - 1, row_of=FAKE)])
def test_scores_of_too_many(binding, kw):
    # (2^31 - 1 tokens: the count of the last step past them would turn negative, and an index with it)
    assert _scores(binding, **kw) == binding.EARG
    assert binding.token_scores_workspace_bytes((1 << 24) - 1, 5, 1) > 0 and binding.token_scores_workspace_bytes(1 << 24, 5, 1) == 0


@pytest.mark.parametrize("call,names", [(_plan, ("row_start", "held", "parent", "table", "free")), (_attention, ("table",)),
                                        (_commit, ("path", "acc")), (_scores, ("row_of", "lp", "ent", "lse", "tt", "tl"))])
def test_unaligned_words(binding, cfg, call, names):
    for name in names:
        for off in (1, 2, 3):
            args = (binding,) if call is _scores else (binding, cfg)
            assert call(*args, **{name: FAKE + off}) == binding.EARG, (name, off)


def test_bad_configurations(binding):
    bad = binding.make_config(workloads.MODELS["llama7b"])
    bad.head_dim = 96
    assert binding.batch_plan_bytes(bad, 1, 1) == 0 and binding.batch_workspace_bytes(bad, 32, 1, 1) == 0
    for call in (_plan, _store, _attention, _commit):
        assert call(binding, bad) == binding.ESHAPE
    assert binding.lib().llmcad_batch_plan_bytes(None, 1, 1) == 0


def test_wrappers_refuse_host_tensors(binding, cfg):
    import torch

    t = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError):
        binding.batch_plan(cfg, t, t[:3], None, 0, t[None], t, 9, t, 3)
    with pytest.raises(ValueError):
        binding.token_scores(torch.zeros(2, 5), t[:2])


def test_streams_of_another_gpu_are_refused(binding, monkeypatch):
    import types

    import torch

    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    ran = []
    stream = lambda i: types.SimpleNamespace(device=torch.device("cuda", i), cuda_stream=77 + i)  # noqa: E731
    with pytest.raises(ValueError, match="stream"):
        binding._enqueue(lambda *a: ran.append(a), 0, stream(1), (1, 2))
    assert not ran
    binding._enqueue(lambda *a: ran.append(a), 0, stream(0), (1, 2))
    assert ran == [(1, 2, 77)]
