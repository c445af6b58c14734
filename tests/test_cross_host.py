"""Refusals of the rotation, cross attention and shared-prefix entry points (no GPU:
they come before any launch), of their binding, and the reference's gradients."""
import ctypes
import math

import pytest
import torch

from paper_2607_12789_amd import avq
from tests.cross_reference import about, backward64, check_backward_of, forward64

OK, INVALID, UNSUPPORTED = avq.AVQ_OK, avq.AVQ_ERR_INVALID_ARG, avq.AVQ_ERR_UNSUPPORTED
F32, BF16 = avq.AVQ_F32, avq.AVQ_BF16
FAKE, ODD = ctypes.c_void_p(16), ctypes.c_void_p(24)  # never dereferenced
INF, NAN = float("inf"), float("nan")
AXES = bytes([0, 1] * 16)


@pytest.fixture(scope="module")
def L():
    return avq.lib()


def rotate(L, dtype=BF16, T=8, Hq=4, Hkv=2, d=64, rot=64, n_axes=2, axis=AXES, n_pos=9, inter=0,
           inv=0, Q=FAKE, qs=256, K=FAKE, ks=128, pos=FAKE, cos=FAKE, sin=FAKE, Qo=FAKE, Ko=FAKE):
    return L.avq_rotate_axes(dtype, T, Hq, Hkv, d, rot, n_axes, axis, n_pos, inter, inv, Q, qs, K, ks,
                             pos, cos, sin, Qo, Ko, None)


def cross(L, dtype=BF16, S=2, Tq=8, Tk=8, Hq=4, Hkv=2, d=64, scale=1.0, Q=FAKE, qs=256, K=FAKE,
          ks=128, V=FAKE, vs=128, cu_q=FAKE, cu_k=FAKE, mask=None, Y=FAKE, lse=None, ws=FAKE,
          ws_bytes=1 << 40):
    return L.avq_cross_attention_fwd(dtype, S, Tq, Tk, Hq, Hkv, d, scale, Q, qs, K, ks, V, vs, cu_q,
                                     cu_k, mask, Y, lse, ws, ws_bytes, None)


def back(L, dtype=BF16, S=2, Tq=8, Tk=8, Hq=4, Hkv=2, d=64, scale=1.0, dY=FAKE, ds=256, Q=FAKE,
         qs=256, K=FAKE, ks=128, V=FAKE, vs=128, Y=FAKE, lse=FAKE, cu_q=FAKE, cu_k=FAKE, mask=None,
         dQ=FAKE, dK=FAKE, dV=FAKE, ws=FAKE, ws_bytes=1 << 40):
    return L.avq_cross_attention_bwd(dtype, S, Tq, Tk, Hq, Hkv, d, scale, dY, ds, Q, qs, K, ks, V, vs,
                                     Y, lse, cu_q, cu_k, mask, dQ, dK, dV, ws, ws_bytes, None)


def prefix(L, dtype=BF16, fmt=1, S=2, Ng=1, n_q=1, Hq=4, Hkv=2, d=64, n_pages=4, ps=16, max_pages=2,
           scale=1.0, Q=FAKE, qs=256, cache=FAKE, lens=FAKE, table=FAKE, cu=FAKE, shared=FAKE, Y=FAKE,
           lse=None, ws=FAKE, ws_bytes=1 << 40):
    return L.avq_cache_prefix_attention_fwd(dtype, fmt, S, Ng, n_q, Hq, Hkv, d, n_pages, ps, max_pages,
                                            scale, Q, qs, cache, lens, table, cu, shared, Y, lse, ws,
                                            ws_bytes, None)


HEADS = [(dict(dtype=5), INVALID), (dict(Hkv=0), INVALID), (dict(Hq=3), INVALID),
         (dict(Hq=2048, qs=131072), UNSUPPORTED), (dict(qs=255), INVALID), (dict(qs=248), INVALID),
         (dict(qs=(1 << 22) + 8), UNSUPPORTED), (dict(Q=None), INVALID), (dict(Q=ODD), INVALID)]
PACKED = HEADS + [
    (dict(S=0), INVALID), (dict(S=1 << 21), UNSUPPORTED), (dict(Tq=-1), INVALID),
    (dict(Tk=-1), INVALID), (dict(Tq=(1 << 24) + 1), UNSUPPORTED), (dict(ks=132), INVALID),
    (dict(d=96, qs=384, ks=192, vs=192), UNSUPPORTED), (dict(vs=120), INVALID),
    (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID), (dict(scale=INF), INVALID),
    (dict(scale=NAN), INVALID), (dict(scale=3e38), INVALID), (dict(K=None), INVALID),
    (dict(V=None), INVALID), (dict(cu_q=None), INVALID), (dict(cu_k=None), INVALID),
    (dict(Y=None), INVALID), (dict(V=ODD), INVALID), (dict(cu_k=ODD), INVALID),
    (dict(lse=ODD), INVALID), (dict(ws=ODD), INVALID), (dict(Y=ODD), INVALID),
    (dict(S=1 << 20, Hq=16, Hkv=16, qs=1024, ks=1024, vs=1024), UNSUPPORTED),
    (dict(Tq=1 << 24, Hq=1024, Hkv=1, qs=65536), UNSUPPORTED)]
CASES = {
    rotate: HEADS + [
        (dict(T=-1), INVALID), (dict(T=(1 << 24) + 1), UNSUPPORTED), (dict(ks=132), INVALID),
        (dict(d=96, qs=384, ks=192), UNSUPPORTED), (dict(rot=0), INVALID), (dict(rot=8), INVALID),
        (dict(rot=80), INVALID), (dict(rot=24), INVALID), (dict(n_axes=0), INVALID),
        (dict(n_axes=5), INVALID), (dict(n_axes=1), INVALID), (dict(n_pos=0), INVALID),
        (dict(inter=2), INVALID), (dict(inv=-1), INVALID), (dict(axis=None), INVALID),
        (dict(axis=bytes([0] * 31 + [2])), INVALID), (dict(pos=None), INVALID),
        (dict(cos=None), INVALID), (dict(sin=None), INVALID), (dict(Qo=None), INVALID),
        (dict(K=None), INVALID), (dict(Ko=None), INVALID), (dict(Ko=ODD), INVALID),
        (dict(pos=ODD), INVALID), (dict(T=0), OK), (dict(T=0, Q=None, Qo=None, pos=None), OK),
        (dict(T=0, K=None, Ko=None, Hkv=3, ks=0), OK)],
    cross: PACKED + [
        (dict(Tk=1 << 16, ws=None), INVALID), (dict(Tk=1 << 16, ws_bytes=1000), INVALID),
        (dict(Tq=0, Q=None, Y=None), OK)],
    back: PACKED + [
        (dict(dY=None), INVALID), (dict(dY=ODD), INVALID), (dict(ds=0), INVALID),
        (dict(ds=100), INVALID), (dict(lse=None), INVALID), (dict(dQ=None), INVALID),
        (dict(dK=None), INVALID), (dict(dV=None), INVALID), (dict(dQ=ODD), INVALID),
        (dict(dV=ODD), INVALID), (dict(ws=None), INVALID), (dict(ws_bytes=64), INVALID),
        (dict(Tq=0, Tk=0, Q=None, K=None, V=None, Y=None, dY=None, dQ=None, dK=None, dV=None,
              lse=None, ws=None), OK)],
    prefix: HEADS + [
        (dict(fmt=2), INVALID), (dict(n_pages=0), INVALID), (dict(max_pages=0), INVALID),
        (dict(ps=8), UNSUPPORTED), (dict(ps=48), UNSUPPORTED), (dict(d=96, qs=384), UNSUPPORTED),
        (dict(S=0), INVALID), (dict(n_q=0), INVALID), (dict(n_q=17), UNSUPPORTED),
        (dict(Ng=0), INVALID), (dict(Ng=-1), INVALID), (dict(Ng=1 << 21), UNSUPPORTED),
        (dict(Ng=1 << 20, Hq=16, Hkv=16, qs=1024), UNSUPPORTED), (dict(scale=0.0), INVALID),
        (dict(scale=NAN), INVALID), (dict(cache=None), INVALID), (dict(lens=None), INVALID),
        (dict(table=None), INVALID), (dict(cu=None), INVALID), (dict(shared=None), INVALID),
        (dict(Y=None), INVALID), (dict(cu=ODD), INVALID), (dict(shared=ODD), INVALID),
        (dict(lse=ODD), INVALID), (dict(ws=None, max_pages=33), INVALID),
        (dict(ws=ODD), INVALID), (dict(ws_bytes=64), INVALID), (dict(S=1024, ps=256, max_pages=1 << 20), UNSUPPORTED)],
}


@pytest.mark.parametrize("fn,kw,status", [(f, kw, st) for f, v in CASES.items() for kw, st in v])
def test_refusals(L, fn, kw, status):
    assert fn(L, **kw) == status, L.avq_last_error()
    assert (L.avq_last_error().decode() != "") == (status != OK)


def test_workspaces(L):
    # as many tiles as fill the device: nothing is divided
    assert avq.cross_attention_workspace(torch.bfloat16, 4, 1 << 16, 1 << 16, 16, 4, 128) == 0
    assert avq.cross_attention_workspace(torch.float32, 1, 1, 1 << 16, 16, 4, 128) > 0
    assert avq.cross_attention_workspace(torch.float32, 1, 1, 40, 16, 4, 128) == 0
    # one fp32 per query and head at least
    assert avq.cross_attention_workspace(torch.bfloat16, 4, 1 << 16, 1 << 16, 16, 4, 128, True) >= 4 * 16 << 16
    assert (avq.cache_prefix_attention_workspace(64, 1, 1, 16, 4, 128)
            > avq.cache_attention_workspace(64, 1, 16, 4, 128))
    for bad in ((0, 8, 8, 4, 2, 64), (1, -1, 8, 4, 2, 64), (1, 8, 8, 4, 3, 64), (1, 8, 8, 4, 2, 96),
                (1 << 20, 8, 8, 16, 16, 64), (1, 1 << 24, 8, 1024, 1, 64)):
        assert L.avq_cross_attention_workspace(BF16, *bad) == -1
        assert L.avq_cross_attention_bwd_workspace(F32, *bad) == -1
        with pytest.raises(ValueError):
            avq.cross_attention_workspace(torch.bfloat16, *bad)
    assert L.avq_cross_attention_workspace(7, 1, 8, 8, 4, 2, 64) == -1
    with pytest.raises(ValueError):
        avq.cross_attention_workspace(torch.float16, 1, 8, 8, 4, 2, 64)
    for bad in ((0, 1, 1, 4, 2, 64), (2, 0, 1, 4, 2, 64), (2, 1, 17, 4, 2, 64), (2, 1, 1, 4, 3, 64),
                (2, 1, 1, 4, 2, 96), (2, 1 << 21, 1, 4, 2, 64)):
        assert L.avq_cache_prefix_attention_workspace(*bad) == -1
        with pytest.raises(ValueError):
            avq.cache_prefix_attention_workspace(*bad)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("d", [64, 128])
def test_no_queries_need_no_workspace(L, dtype, d):
    """Without queries nothing is launched, however many states there are to divide."""
    for S, Tk, Hq, Hkv in ((1, 1 << 16, 4, 2), (3, 40, 4, 1), (1, 1 << 24, 1, 1)):
        assert L.avq_cross_attention_workspace(dtype, S, 0, Tk, Hq, Hkv, d) == 0
        kw = dict(dtype=dtype, S=S, Tq=0, Tk=Tk, Hq=Hq, Hkv=Hkv, d=d, qs=Hq * d, ks=Hkv * d,
                  vs=Hkv * d)
        assert cross(L, Q=None, Y=None, ws=None, ws_bytes=0, **kw) == OK, L.avq_last_error()


def test_binding_refuses_host_tensors():
    x, c = torch.zeros(4, 2, 64), torch.zeros(2, dtype=torch.int32)
    for call in (lambda: avq.rotate_axes(x, x, c[:, None], x[0], x[0], (0,) * 32),
                 lambda: avq.cross_attention_fwd(x, x, x, c, c, 1.0),
                 lambda: avq.cross_attention_bwd(x, x, x, x, x, x, c, c, 1.0),
                 lambda: avq.cache_prefix_attention_fwd(x[None], x, c, c, c, c, 16, 1.0)):
        with pytest.raises(ValueError, match="on the GPU"):
            call()


def test_reference_gradients():
    """The 64-bit gradients that the kernels are compared with, against central
    differences: the error of those is of the order e^2, a third at e of what the
    steps e and 2 e differ by."""
    g = torch.Generator().manual_seed(3)
    lens_q, lens_k, scale = [3, 0, 2], [5, 4, 6], 0.3
    Q = torch.randn(5, 4, 8, generator=g).double()
    K, V = (torch.randn(15, 2, 8, generator=g).double() for _ in "kv")
    dY = torch.randn(5, 4, 8, generator=g).double()
    mask = torch.rand(15, generator=g) < 0.7
    mask[9:] = torch.tensor([False, True, True, False, True, False])
    # the bounds are defined for the storage types; only the values are used here
    want = backward64(*(t.float() for t in (dY, Q, K, V)), lens_q, lens_k, scale, mask)[0]
    x = [t.float().double() for t in (Q, K, V)]
    dY = dY.float().double()
    for i in range(3):
        u = torch.randn(x[i].shape, generator=g).double()

        def loss(e):
            z = list(x)
            z[i] = x[i] + e * u
            return (forward64(*z, lens_q, lens_k, scale, mask)[0] * dY).sum().item()

        near, far = (loss(1e-4) - loss(-1e-4)) / 2e-4, (loss(2e-4) - loss(-2e-4)) / 4e-4
        # differences of losses of order 1 at steps of 1e-4: rounding 1e-12
        assert abs((want[i] * u).sum().item() - near) <= abs(near - far) + 1e-10
    assert (want[1][~mask] == 0).all() and (want[2][~mask] == 0).all()
    assert not math.isnan(sum(t.sum().item() for t in want))


def test_bounds_tell_a_mended_delta():
    """The bounds on gradients from a Y that is off by its own rounding, against the
    kernels' steps with their roundings to bf16: kept with the mended delta, not without."""
    g = torch.Generator().manual_seed(4)
    lens_q, lens_k, scale, h16 = [9], [70], 0.2, torch.bfloat16
    Q, K, V, dY = (torch.randn(n, 1, 64, generator=g).to(h16) for n in (9, 70, 70, 9))
    K, V = about(K, 1.0, 0.3), about(V, 4.0, 0.1)

    def rounded(x):
        return x.to(h16).double()

    q, k, v, dy = (x[:, 0].double() for x in (Q, K, V, dY))
    S = scale * q @ k.T
    p = torch.exp(S - S.amax(1, keepdim=True))
    y = rounded(rounded(p) @ v / p.sum(1, keepdim=True))
    lse = torch.logsumexp(S, 1).float().double()
    P = torch.exp(S - lse[:, None])
    dP, delta = dy @ v.T, (dy * y).sum(1, keepdim=True)
    dS = P * (dP - delta)
    taken = rounded(dS)
    mended = rounded(P * (dP - delta - dS.sum(1, keepdim=True)))
    dV = rounded(P).T @ dy
    one = [scale * taken @ k, scale * taken.T @ q, dV]
    other = [scale * (taken @ k - taken.sum(1, keepdim=True) * (rounded(P) @ k)), scale * mended.T @ q,
             dV]
    args = (dY, Q, K, V, y.to(h16)[:, None], lse.float()[:, None], lens_q, lens_k, scale)
    check_backward_of([x.to(h16)[:, None] for x in other], *args)
    for i, name in enumerate(("dQ", "dK")):
        mixed = list(other)
        mixed[i] = one[i]
        with pytest.raises(AssertionError, match=name):
            check_backward_of([x.to(h16)[:, None] for x in mixed], *args)
