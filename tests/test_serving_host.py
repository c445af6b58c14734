"""Refusals of the serving entry points (no GPU: they come before any launch),
and of their Python binding."""
import ctypes
from types import SimpleNamespace

import pytest
import torch

from paper_2607_12789_amd import avq

OK, INVALID, UNSUPPORTED = avq.AVQ_OK, avq.AVQ_ERR_INVALID_ARG, avq.AVQ_ERR_UNSUPPORTED
F32, BF16 = avq.AVQ_F32, avq.AVQ_BF16
FAKE, ODD = ctypes.c_void_p(16), ctypes.c_void_p(24)  # never dereferenced


@pytest.fixture(scope="module")
def L():
    return avq.lib()


def prompt(L, dtype=BF16, S=2, Tq=8, Tk=8, Hq=4, Hkv=2, d=64, scale=1.0, causal=1, qs=256, ks=128,
           vs=128, Q=FAKE, K=FAKE, V=FAKE, cu_q=FAKE, cu_k=FAKE, Y=FAKE, lse=None, ws=None, ws_bytes=0):
    return L.avq_prompt_attention_fwd(dtype, S, Tq, Tk, Hq, Hkv, d, scale, causal, Q, qs, K, ks, V,
                                      vs, cu_q, cu_k, Y, lse, ws, ws_bytes, None)


def append(L, dtype=BF16, fmt=1, S=2, T=8, Hq=4, Hkv=2, d=64, n_pages=4, ps=16, max_pages=2, rot=0,
           n_pos=0, inter=0, Q=None, qs=256, K=FAKE, ks=128, V=FAKE, vs=128, cu=FAKE, start=FAKE,
           table=FAKE, cos=None, sin=None, cache=FAKE, Qo=None, Ko=None):
    return L.avq_cache_append(dtype, fmt, S, T, Hq, Hkv, d, n_pages, ps, max_pages, rot, n_pos,
                              inter, Q, qs, K, ks, V, vs, cu, start, table, cos, sin, cache, Qo, Ko,
                              None)


def gather(L, dtype=BF16, fmt=1, S=2, T=8, Hkv=2, d=64, n_pages=4, ps=16, max_pages=2, cache=FAKE,
           cu=FAKE, start=FAKE, table=FAKE, K=FAKE, V=FAKE):
    return L.avq_cache_gather(dtype, fmt, S, T, Hkv, d, n_pages, ps, max_pages, cache, cu, start,
                              table, K, V, None)


def cached(L, dtype=BF16, fmt=1, S=2, n_q=1, Hq=4, Hkv=2, d=64, n_pages=4, ps=16, max_pages=2,
           scale=1.0, Q=FAKE, qs=256, cache=FAKE, lens=FAKE, table=FAKE, Y=FAKE, lse=None, ws=FAKE,
           ws_bytes=1 << 40):
    return L.avq_cache_attention_fwd(dtype, fmt, S, n_q, Hq, Hkv, d, n_pages, ps, max_pages, scale,
                                     Q, qs, cache, lens, table, Y, lse, ws, ws_bytes, None)


HEADS = [(dict(dtype=5), INVALID), (dict(S=0), INVALID), (dict(S=1 << 21), UNSUPPORTED),
         (dict(Hkv=0), INVALID), (dict(d=96, qs=384, ks=192, vs=192), UNSUPPORTED)]
CACHE = [(dict(fmt=2), INVALID), (dict(n_pages=0), INVALID), (dict(max_pages=0), INVALID),
         (dict(ps=8), UNSUPPORTED), (dict(ps=48), UNSUPPORTED), (dict(ps=512), UNSUPPORTED),
         (dict(ps=256, max_pages=(1 << 22) + 1), UNSUPPORTED)]
INF, NAN = float("inf"), float("nan")
CASES = {
    prompt: HEADS + [
        (dict(Hq=3), INVALID), (dict(Hq=2048, qs=131072), UNSUPPORTED),
        (dict(Tq=-1), INVALID), (dict(Tk=-1), INVALID), (dict(Tq=(1 << 24) + 1), UNSUPPORTED),
        (dict(causal=2), INVALID), (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID),
        (dict(scale=INF), INVALID), (dict(scale=NAN), INVALID),
        (dict(qs=255), INVALID), (dict(qs=248), INVALID), (dict(ks=132), INVALID),
        (dict(vs=(1 << 22) + 8), UNSUPPORTED),
        (dict(Q=None), INVALID), (dict(K=None), INVALID), (dict(V=None), INVALID),
        (dict(cu_q=None), INVALID), (dict(cu_k=None), INVALID), (dict(Y=None), INVALID),
        (dict(Q=ODD), INVALID), (dict(V=ODD), INVALID), (dict(lse=ODD), INVALID),
        (dict(cu_k=ODD), INVALID), (dict(ws=ODD), INVALID),
        (dict(Tk=1 << 20), INVALID), (dict(Tk=1 << 20, ws=FAKE, ws_bytes=1000), INVALID),
        (dict(S=1 << 20, Hq=16, Hkv=16, qs=1024, ks=1024, vs=1024), UNSUPPORTED),
        (dict(Tq=0, Q=None, Y=None), OK)],
    append: HEADS + CACHE + [
        (dict(T=-1), INVALID), (dict(T=(1 << 24) + 1), UNSUPPORTED), (dict(cu=None), INVALID),
        (dict(rot=8), INVALID), (dict(rot=80), INVALID), (dict(rot=-16), INVALID),
        (dict(rot=16), INVALID), (dict(rot=16, cos=FAKE, sin=FAKE), INVALID),
        (dict(rot=16, cos=FAKE, n_pos=4), INVALID), (dict(inter=2), INVALID),
        (dict(Q=FAKE), INVALID), (dict(Qo=FAKE), INVALID), (dict(Q=FAKE, Qo=FAKE, Hq=3), INVALID),
        (dict(Q=FAKE, Qo=FAKE, qs=100), INVALID), (dict(K=None), INVALID), (dict(V=None), INVALID),
        (dict(start=None), INVALID), (dict(table=None), INVALID), (dict(cache=None), INVALID),
        (dict(cache=ODD), INVALID), (dict(Ko=ODD), INVALID), (dict(ks=100), INVALID),
        (dict(T=0, K=None, V=None), OK)],
    gather: HEADS + CACHE + [
        (dict(T=-1), INVALID), (dict(T=(1 << 24) + 1), UNSUPPORTED), (dict(cu=None), INVALID),
        (dict(start=None), INVALID), (dict(table=None), INVALID), (dict(cache=None), INVALID),
        (dict(K=None), INVALID), (dict(V=ODD), INVALID), (dict(T=0, K=None, V=None), OK)],
    cached: HEADS + CACHE + [
        (dict(n_q=0), INVALID), (dict(n_q=17), UNSUPPORTED), (dict(Hq=3), INVALID),
        (dict(scale=0.0), INVALID), (dict(scale=NAN), INVALID), (dict(qs=100), INVALID),
        (dict(Q=None), INVALID), (dict(cache=None), INVALID), (dict(lens=None), INVALID),
        (dict(table=None), INVALID), (dict(Y=None), INVALID),
        (dict(ws=None, max_pages=33), INVALID),
        (dict(ws_bytes=64), INVALID), (dict(Y=ODD), INVALID), (dict(ws=ODD), INVALID),
        (dict(S=1024, ps=256, max_pages=1 << 20), UNSUPPORTED),
        (dict(S=1 << 20, Hq=16, Hkv=16, qs=16 * 64), UNSUPPORTED)],
}


@pytest.mark.parametrize("fn,kw,status", [(f, kw, st) for f, v in CASES.items() for kw, st in v])
def test_refusals(L, fn, kw, status):
    if fn is gather:
        kw = {k: v for k, v in kw.items() if k not in ("qs", "ks", "vs")}
    if fn is cached:
        kw = {k: v for k, v in kw.items() if k not in ("ks", "vs")}
    assert fn(L, **kw) == status, avq.lib().avq_last_error()
    assert (L.avq_last_error().decode() != "") == (status != OK)


def test_page_bytes(L):
    assert L.avq_cache_page_bytes(BF16, 0, 64, 128) == 2 * 64 * 128 * 2
    assert L.avq_cache_page_bytes(F32, 0, 16, 64) == 2 * 16 * 64 * 4
    for dt in (F32, BF16):  # 4.25 bits per element
        assert L.avq_cache_page_bytes(dt, 1, 32, 128) * 8 == 2 * 32 * 128 * 4.25
    for bad in ((9, 0, 64, 128), (BF16, 2, 64, 128), (BF16, 0, 8, 128), (BF16, 0, 48, 128),
                (BF16, 0, 64, 96)):
        assert L.avq_cache_page_bytes(*bad) == -1
    with pytest.raises(ValueError):
        avq.cache_page_bytes(torch.float16, 64, 128)
    with pytest.raises(ValueError):
        avq.cache_page_bytes(torch.bfloat16, 24, 128)


def test_workspace_bytes(L):
    assert avq.prompt_attention_workspace(torch.bfloat16, 4, 1 << 16, 1 << 16, 16, 128) == 0
    assert avq.prompt_attention_workspace(torch.bfloat16, 1, 300, 1 << 16, 4, 128) > 0
    assert avq.prompt_attention_workspace(torch.bfloat16, 1, 300, 300, 4, 128) == 0
    for bad in ((9, 1, 8, 8, 4, 64, 1), (BF16, 0, 8, 8, 4, 64, 1), (BF16, 1, -1, 8, 4, 64, 1),
                (BF16, 1, 8, 8, 4, 96, 1), (BF16, 1, 8, 8, 4, 64, 2),
                (BF16, 1 << 20, 8, 8, 16, 64, 1)):
        assert L.avq_prompt_attention_workspace(*bad) == -1
    small = avq.cache_attention_workspace(1, 1, 8, 8, 64)
    assert 0 < small < avq.cache_attention_workspace(4096, 16, 32, 8, 64)
    for bad in ((0, 1, 8, 8, 64), (1, 17, 8, 8, 64), (1, 1, 8, 3, 64), (1, 1, 8, 8, 80),
                (1 << 20, 1, 16, 16, 64)):
        assert L.avq_cache_attention_workspace(*bad) == -1


def test_binding_refuses_cpu_tensors():
    x, i = torch.zeros(4, 2, 64, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    cache = torch.zeros(2, 2, 16 * 64 * 4, dtype=torch.uint8)
    table = torch.zeros(2, 1, dtype=torch.int32)
    with pytest.raises(ValueError):
        avq.prompt_attention_fwd(x, x, x, i, i, 1.0)
    with pytest.raises(ValueError):
        avq.cache_append(x, x, cache, table, i[:2], 16, cu=i)
    with pytest.raises(ValueError):
        avq.cache_gather(cache, table, i[:2], i, 4, 16, torch.bfloat16, 64)
    with pytest.raises(ValueError):
        avq.cache_attention_fwd(x[None], cache, table, i[:2], 16, 1.0)


def test_binding_refuses_another_device(monkeypatch):
    """The library launches on the current device: tensors or streams of
    another one are refused."""
    dev = torch.device("cuda", 1)
    stream = SimpleNamespace(device=dev, cuda_stream=0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda i: 77, raising=False)
    for s in (None, stream):
        with pytest.raises(ValueError):
            avq._launch_stream(s, dev)
    with pytest.raises(ValueError):
        avq._launch_stream(stream, torch.device("cuda", 0))
    assert avq._launch_stream(None, torch.device("cuda", 0)) == 77
    a, b = SimpleNamespace(device=dev), SimpleNamespace(device=torch.device("cuda", 0))
    with pytest.raises(ValueError):
        avq._same_device(a, other=b)


@pytest.mark.parametrize("fn", [prompt, cached])
@pytest.mark.parametrize("scale", [2.4e38, 2.9e38])
def test_scales_that_overflow_are_refused(L, fn, scale):
    """scale log2(e), by which the kernels multiply, has to be finite."""
    assert fn(L, scale=scale) == INVALID
    assert "scale" in L.avq_last_error().decode()


def test_binding_without_the_raw_stream(monkeypatch):
    """A torch that does not give out the raw handle: the public Stream's."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: SimpleNamespace(cuda_stream=55))
    assert avq._launch_stream(None, torch.device("cuda", 0)) == 55
