"""rotate_axes against 64 bits (MI355X). Each result is two products and a sum in
fp32, rounded once to the type: off by at most 3 2^-24 (|a cos| + |b sin|) and half a
step of the type."""
import pytest
import torch

from paper_2607_12789_amd import avq
from tests.serving_reference import HALF_STEP

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def make(T, Hq, Hkv, d, rot, n_axes, n_pos, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    Q = torch.randn(T, Hq, d, generator=g).to(dtype)
    K = torch.randn(T, Hkv, d, generator=g).to(dtype)
    pos = torch.randint(0, n_pos, (T, n_axes), generator=g, dtype=torch.int32)
    angle = 100 * torch.randn(n_pos, rot // 2, generator=g)
    return Q, K, pos, angle.cos(), angle.sin()


def reference(x, pos, cos, sin, axis, interleaved, inverse):
    half = cos.shape[1]
    at = pos.long()[:, torch.tensor(axis)]
    i = torch.arange(half)
    c, s = cos.double()[at, i][:, None], sin.double()[at, i][:, None]
    if inverse:
        s = -s
    y, err = x.double().clone(), torch.zeros(x.shape).double()
    ia, ib = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    a, b = x.double()[..., ia], x.double()[..., ib]
    y[..., ia], y[..., ib] = a * c - b * s, b * c + a * s
    err[..., ia] = 3 * 2.0 ** -24 * ((a * c).abs() + (b * s).abs())
    err[..., ib] = 3 * 2.0 ** -24 * ((b * c).abs() + (a * s).abs())
    return y, err


def check(out, x, *how):
    y, err = reference(x, *how)
    tol = err + HALF_STEP[x.dtype] * (y.abs() + err)
    tol[..., 2 * how[1].shape[1]:] = 0  # copied
    d = (out.cpu().double() - y).abs()
    assert (d <= tol).all(), f"off by {(d / tol.clamp(min=1e-30)).max():.3g} times the bound"


def blocked(half, n):
    return tuple(min(n - 1, i * n // half) for i in range(half))


def mixed(half, n):
    return tuple(i % n for i in range(half))


def uneven(half, n):
    """Sections that begin inside a group of four pairs."""
    return tuple(0 if i < 3 else min(n - 1, 1 + (i - 3) // max(1, half // 3)) for i in range(half))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("axes", [blocked, mixed, uneven])
@pytest.mark.parametrize("d,rot,n_axes", [(64, 64, 3), (64, 16, 1), (128, 128, 4), (128, 96, 2),
                                          (128, 32, 3)])
def test_rotation(d, rot, n_axes, axes, interleaved, dtype):
    axis = axes(rot // 2, n_axes)
    Q, K, pos, cos, sin = make(29, 6, 2, d, rot, n_axes, 50, dtype)
    for inverse in (False, True):
        q, k = avq.rotate_axes(Q.cuda(), K.cuda(), pos.cuda(), cos.cuda(), sin.cuda(), axis,
                               interleaved=interleaved, inverse=inverse)
        check(q, Q, pos, cos, sin, axis, interleaved, inverse)
        check(k, K, pos, cos, sin, axis, interleaved, inverse)


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (3, 1), (12, 12), (32, 8), (50, 5)])
@pytest.mark.parametrize("T", [0, 1, 3, 257])
def test_heads_and_tokens(T, Hq, Hkv):
    axis = blocked(32, 3)
    Q, K, pos, cos, sin = make(T, Hq, Hkv, 64, 64, 3, 9, BF16, 1)
    q, k = avq.rotate_axes(Q.cuda(), K.cuda(), pos.cuda(), cos.cuda(), sin.cuda(), axis)
    check(q, Q, pos, cos, sin, axis, False, False)
    check(k, K, pos, cos, sin, axis, False, False)
    q2, none = avq.rotate_axes(Q.cuda(), None, pos.cuda(), cos.cuda(), sin.cuda(), axis)
    assert none is None and torch.equal(q, q2)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("interleaved", [False, True])
def test_in_place_and_slices(interleaved, dtype):
    axis = mixed(24, 3)
    Q, K, pos, cos, sin = make(40, 4, 2, 64, 48, 3, 9, dtype, 2)
    fused = torch.cat((Q.flatten(1), K.flatten(1)), 1).cuda()
    q, k = (x.unflatten(1, (-1, 64)) for x in fused.split([256, 128], 1))
    q1, k1 = avq.rotate_axes(q, k, pos.cuda(), cos.cuda(), sin.cuda(), axis, interleaved=interleaved)
    check(q1, Q, pos, cos, sin, axis, interleaved, False)
    q, k = Q.cuda(), K.cuda()
    q2, k2 = avq.rotate_axes(q, k, pos.cuda(), cos.cuda(), sin.cuda(), axis, interleaved=interleaved,
                             Q_out=q, K_out=k)
    assert q2 is q and k2 is k and torch.equal(q, q1) and torch.equal(k, k1)


def test_positions_outside_the_tables():
    """A token with such a position is not written; the others are."""
    axis = blocked(32, 2)
    Q, K, pos, cos, sin = make(7, 2, 2, 64, 64, 2, 9, BF16, 3)
    bad = pos.clone()
    bad[1, 0], bad[3, 1], bad[6, 0] = 9, -1, 2 ** 31 - 1
    out = [torch.full_like(x, 5).cuda() for x in (Q, K)]
    avq.rotate_axes(Q.cuda(), K.cuda(), bad.cuda(), cos.cuda(), sin.cuda(), axis, Q_out=out[0],
                    K_out=out[1])
    good = [0, 2, 4, 5]
    for x, o in zip((Q, K), out):
        assert (o[[1, 3, 6]] == 5).all()
        check(o[good], x[good], pos[good], cos, sin, axis, False, False)


@pytest.mark.parametrize("interleaved", [False, True])
def test_gradient(interleaved):
    """Of the loss sum rotate(Q) G it is G rotated back: against differences along a
    direction. The rotation is linear, so a difference of two losses is exact but for
    their roundings: each fp32 result is off by at most 4 2^-24 (|a| + |b|)."""
    axis = mixed(32, 2)
    Q, K, pos, cos, sin = make(11, 3, 3, 64, 64, 2, 9, F32, 4)
    g, back = avq.rotate_axes(K.cuda(), K.cuda(), pos.cuda(), cos.cuda(), sin.cuda(), axis,
                              interleaved=interleaved, inverse=True)
    assert torch.equal(g, back)
    u = Q  # the direction; loss(u) - loss(0) = loss(u)
    turned = avq.rotate_axes(u.cuda(), None, pos.cuda(), cos.cuda(), sin.cuda(), axis,
                             interleaved=interleaved)[0]
    along, change = (g.cpu().double() * u).sum(), (turned.cpu().double() * K).sum()
    bound = 16 * 2.0 ** -24 * (u.double().norm(dim=-1) * K.double().norm(dim=-1)).sum()
    assert (along - change).abs() <= bound


def test_refusals_on_the_gpu():
    axis = blocked(32, 2)
    Q, K, pos, cos, sin = (x.cuda() for x in make(7, 2, 2, 64, 64, 2, 9, BF16, 3))
    for change in (dict(pos=pos[:6]), dict(pos=pos.long()), dict(cos=cos[:, :16].contiguous()),
                   dict(axis=axis[:5]), dict(axis=(300,) * 32), dict(axis=(-1,) * 32),
                   dict(K=K[:6]), dict(K=K.float()), dict(K=None, K_out=K), dict(Q_out=Q.float()),
                   dict(pos=pos.cpu())):
        kw = dict(Q=Q, K=K, pos=pos, cos=cos, sin=sin, axis=axis)
        kw.update(change)
        with pytest.raises(ValueError):
            avq.rotate_axes(**kw)
    with pytest.raises(avq.AvqError):
        avq.rotate_axes(Q, K, pos, cos, sin, (2,) * 32)
    with pytest.raises(avq.AvqError):
        avq.rotate_axes(Q, K, pos, cos[:, :12].contiguous(), sin[:, :12].contiguous(), axis[:12])


def test_graph_and_stream():
    axis = blocked(32, 2)
    Q, K, pos, cos, sin = (x.cuda() for x in make(33, 4, 2, 64, 64, 2, 9, BF16, 5))
    want = avq.rotate_axes(Q, K, pos, cos, sin, axis)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    got = avq.rotate_axes(Q, K, pos, cos, sin, axis, stream=st)
    st.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = avq.rotate_axes(Q, K, pos, cos, sin, axis)
    for i in range(3):
        pos.copy_((pos + 1) % 9)
        graph.replay()
        torch.cuda.synchronize()
        now = avq.rotate_axes(Q, K, pos, cos, sin, axis)
        assert torch.equal(out[0], now[0]) and torch.equal(out[1], now[1])


def test_rows_past_32_bits():
    axis, T = blocked(64, 2), 1_100_000
    Q, K, pos, cos, sin = make(50, 16, 1, 128, 128, 2, 9, BF16, 6)
    big = torch.zeros(T, 16, 128, dtype=BF16, device="cuda")
    big[T - 50:] = Q.cuda()
    at = torch.zeros(T, 2, dtype=torch.int32, device="cuda")
    at[T - 50:] = pos.cuda()
    q, _ = avq.rotate_axes(big, None, at, cos.cuda(), sin.cuda(), axis)
    check(q[T - 50:], Q, pos, cos, sin, axis, False, False)
    assert (q[:T - 50] == 0).all()


def test_unaligned_rows_are_refused():
    Q, K, pos, cos, sin = (x.cuda() for x in make(7, 2, 2, 64, 64, 2, 9, BF16, 3))
    odd = torch.empty(7 * 128 + 1, dtype=BF16, device="cuda")[1:].view(7, 2, 64)
    with pytest.raises(avq.AvqError):
        avq.rotate_axes(odd, K, pos, cos, sin, blocked(32, 2))
    with pytest.raises(avq.AvqError):
        avq.rotate_axes(Q, K, pos, cos, sin, blocked(32, 2), K_out=odd)
