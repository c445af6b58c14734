"""cross_attention_fwd and cross_attention_bwd against the 64-bit reference (MI355X)."""
import math

import pytest
import torch

from paper_2607_12789_amd import avq
from tests.cross_reference import (HALF_STEP, about, check_backward, check_backward_of, check_forward,
                                   forward64)

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def cu(lens):
    t = torch.zeros(len(lens) + 1, dtype=torch.int32)
    t[1:] = torch.tensor(lens).cumsum(0)
    return t.cuda()


def make(lens_q, lens_k, Hq, Hkv, d, dtype, seed=0, q_scale=2.0):
    g = torch.Generator().manual_seed(seed)
    Q = (q_scale * torch.randn(sum(lens_q), Hq, d, generator=g)).to(dtype)
    K = torch.randn(sum(lens_k), Hkv, d, generator=g).to(dtype)
    V = torch.randn(sum(lens_k), Hkv, d, generator=g).to(dtype)
    dY = torch.randn(sum(lens_q), Hq, d, generator=g).to(dtype)
    return Q, K, V, dY


def gpu(x):
    return None if x is None else x.cuda()


def fwd(Q, K, V, lens_q, lens_k, scale, mask=None, **kw):
    Y, lse = avq.cross_attention_fwd(gpu(Q), gpu(K), gpu(V), cu(lens_q), cu(lens_k), scale,
                                     mask=gpu(mask), with_lse=True, **kw)
    torch.cuda.synchronize()
    return Y, lse


def both(Q, K, V, dY, lens_q, lens_k, scale, mask=None):
    """Forward, then backward on what it stored; checks all of it."""
    Y, lse = fwd(Q, K, V, lens_q, lens_k, scale, mask)
    check_forward(Y.cpu(), lse.cpu(), Q, K, V, lens_q, lens_k, scale, mask)
    # the bounds on the gradients take Y and lse as the rounded exact ones
    y64, l64 = forward64(Q, K, V, lens_q, lens_k, scale, mask)
    got = avq.cross_attention_bwd(gpu(dY), gpu(Q), gpu(K), gpu(V), gpu(y64.to(Q.dtype)),
                                  gpu(l64.float()), cu(lens_q), cu(lens_k), scale, mask=gpu(mask))
    torch.cuda.synchronize()
    check_backward([x.cpu() for x in got], dY, Q, K, V, lens_q, lens_k, scale, mask)
    return Y, lse, got


LENS = [
    ([1], [1]), ([37], [33]), ([64], [31]), ([1], [700]), ([300], [1]), ([127, 128, 129], [32, 64, 65]),
    ([0, 3, 5, 0, 70], [10, 0, 129, 0, 1]), ([5] * 20, [100] * 20), ([1] * 70, [3] * 70),
    ([513, 2], [40, 1100]),
]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens_q,lens_k", LENS)
def test_lengths(lens_q, lens_k, d, dtype):
    Q, K, V, dY = make(lens_q, lens_k, 4, 2, d, dtype)
    both(Q, K, V, dY, lens_q, lens_k, 1 / math.sqrt(d))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("S", [63, 64, 65])
@pytest.mark.parametrize("long", ["states", "queries"])
def test_sources_of_all_lengths(long, S, dtype):
    """As many sources as a wave has lanes, one less and one more, whose states (or
    queries) are shared out over several workgroups, some of no length."""
    few, many = [i * 7 % 13 for i in range(S)], [i * 331 % 400 if i % 9 else 0 for i in range(S)]
    lens_q, lens_k = (few, many) if long == "states" else (many, few)
    Q, K, V, dY = make(lens_q, lens_k, 2, 1, 64, dtype, 6)
    both(Q, K, V, dY, lens_q, lens_k, 0.2)


@pytest.mark.parametrize("dtype,d", [(BF16, 64), (BF16, 128), (F32, 64), (F32, 128)])
@pytest.mark.parametrize("rows", [20, 900])
@pytest.mark.parametrize("bad", [math.inf, math.nan])
def test_bad_gradients_and_hidden_states(bad, rows, d, dtype):
    """States that take no part get gradients of 0, whatever the others' are; queries that
    see no state too."""
    lens_q, lens_k = [rows, 9], [130, 40]
    Q, K, V, dY = make(lens_q, lens_k, 2, 1, d, dtype, 8)
    mask = torch.arange(170) % 3 > 0
    mask[130:] = False
    dY[7] = dY[rows + 3] = bad
    Y, lse = fwd(Q, K, V, lens_q, lens_k, 0.2, mask)
    dQ, dK, dV = avq.cross_attention_bwd(gpu(dY), gpu(Q), gpu(K), gpu(V), Y, lse, cu(lens_q),
                                         cu(lens_k), 0.2, mask=gpu(mask))
    hidden = ~gpu(mask)
    assert not dK[hidden].any() and not dV[hidden].any() and not dQ[rows:].any()
    assert not dV[~hidden].isfinite().any() and not dQ[7].isfinite().any()
    assert dQ[:7].isfinite().all() and dQ[8:].isfinite().all()


@pytest.mark.parametrize("dtype,d", [(BF16, 64), (BF16, 128), (F32, 64), (F32, 128)])
@pytest.mark.parametrize("S", [2, 5, 16, 17])
def test_uneven_sources(S, d, dtype):
    """One source holds most of the work; both its rows and its states are shared out."""
    lens_q, lens_k = [33 + i * 7 for i in range(S)], [40 + i * 11 for i in range(S)]
    lens_q[S // 2], lens_k[S // 2] = 700, 1500
    Q, K, V, dY = make(lens_q, lens_k, 2, 1, d, dtype, 7)
    both(Q, K, V, dY, lens_q, lens_k, 1 / math.sqrt(d))


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (7, 1), (6, 6), (8, 2), (24, 8), (5, 5), (33, 1)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_heads(Hq, Hkv, dtype):
    lens_q, lens_k = [19, 50], [90, 41]
    Q, K, V, dY = make(lens_q, lens_k, Hq, Hkv, 64, dtype, 3)
    both(Q, K, V, dY, lens_q, lens_k, 0.2)


MASKS = ["none", "all", "one", "tail", "head", "random", "tiles"]


def mask_of(kind, n, g):
    m = torch.ones(n, dtype=torch.bool)
    if kind == "none":
        m[:] = False
    elif kind == "one":
        m[:] = False
        m[n // 2] = True
    elif kind == "tail":
        m[n // 3:] = False
    elif kind == "head":
        m[:2 * n // 3] = False
    elif kind == "random":
        m = torch.rand(n, generator=g) < 0.5
    elif kind == "tiles":
        m[32:96] = False
    return m


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bad", [None, math.inf, -math.inf, math.nan, "lowest"])
def test_masks(bad, d, dtype):
    """Every kind of mask, a source each; what the hidden states hold has no effect."""
    g = torch.Generator().manual_seed(5)
    lens_q, lens_k = [9] * len(MASKS), [130, 77, 40, 201, 65, 140, 128]
    Q, K, V, dY = make(lens_q, lens_k, 4, 2, d, dtype, 1)
    mask = torch.cat([mask_of(m, n, g) for m, n in zip(MASKS, lens_k)])
    if bad is not None:
        K[~mask] = V[~mask] = torch.finfo(dtype).min if bad == "lowest" else bad
    both(Q, K, V, dY, lens_q, lens_k, 1 / math.sqrt(d), mask)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_long_masked(dtype):
    """Divided states and rows, whole parts of them hidden."""
    lens_q, lens_k = [3, 400], [1500, 900]
    Q, K, V, dY = make(lens_q, lens_k, 2, 1, 64, dtype, 2)
    mask = torch.ones(2400, dtype=torch.uint8)
    mask[300:1200] = 0
    mask[1500:2390] = 0
    both(Q, K, V, dY, lens_q, lens_k, 0.3, mask)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("q_scale", [0.0, 30.0])
def test_flat_and_peaked(dtype, q_scale):
    """Equal logits (a plain mean), and logits of hundreds that grow along the states."""
    lens_q, lens_k = [70], [260]
    Q, K, V, dY = make(lens_q, lens_k, 2, 1, 128, dtype, 5, q_scale)
    if q_scale:
        K = (K.float() * torch.linspace(0.1, 3, 260)[:, None, None]).to(dtype)
    both(Q, K, V, dY, lens_q, lens_k, 0.5)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_slices_of_fused_projections(dtype):
    lens_q, lens_k, Hq, Hkv, d = [70, 130], [33, 64], 4, 2, 64
    g = torch.Generator().manual_seed(1)
    fused = torch.randn(200, (2 * Hq) * d, generator=g).to(dtype).cuda()
    kv = torch.randn(97, (2 * Hkv + 1) * d, generator=g).to(dtype).cuda()
    dY, q = (x.unflatten(1, (Hq, d)) for x in fused.split(Hq * d, 1))
    k, v = kv[:, :Hkv * d].unflatten(1, (Hkv, d)), kv[:, (Hkv + 1) * d:].unflatten(1, (Hkv, d))
    Y, lse = avq.cross_attention_fwd(q, k, v, cu(lens_q), cu(lens_k), 0.3, with_lse=True)
    got = avq.cross_attention_bwd(dY, q, k, v, Y, lse, cu(lens_q), cu(lens_k), 0.3)
    again = avq.cross_attention_bwd(dY.contiguous(), q.contiguous(), k.contiguous(), v.contiguous(),
                                    Y, lse, cu(lens_q), cu(lens_k), 0.3)
    check_forward(Y.cpu(), lse.cpu(), q.cpu(), k.cpu(), v.cpu(), lens_q, lens_k, 0.3)
    for x, y in zip(got, again):
        assert torch.equal(x, y)


def test_rows_of_no_source_stay():
    lens_q, lens_k = [40, 10], [20, 33]
    Q, K, V, dY = (x.cuda() for x in make([70], [90], 2, 2, 64, BF16))
    Y, lse = torch.full_like(Q, 7), torch.full((70, 2), 7.0, device="cuda")
    avq.cross_attention_fwd(Q, K, V, cu(lens_q), cu(lens_k), 0.3, Y=Y, with_lse=True, lse=lse)
    assert (Y[50:] == 7).all() and (lse[50:] == 7).all()
    check_forward(Y[:50].cpu(), lse[:50].cpu(), Q.cpu(), K.cpu(), V.cpu(), lens_q, lens_k, 0.3)
    out = [torch.full_like(x, 7) for x in (Q, K, V)]
    avq.cross_attention_bwd(dY, Q, K, V, Y, lse, cu(lens_q), cu(lens_k), 0.3, dQ=out[0], dK=out[1],
                            dV=out[2])
    assert (out[0][50:] == 7).all() and (out[1][53:] == 7).all() and (out[2][53:] == 7).all()
    assert not (out[0][:50] == 7).all(-1).any() and not (out[1][:53] == 7).all(-1).any()


def test_bounds_outside_the_rows():
    """Bounds past the rows are taken as their end, negative ones as 0."""
    Q, K, V, dY = make([60], [60], 1, 1, 64, BF16)
    c = torch.tensor([-5, 20, 500], dtype=torch.int32, device="cuda")
    Y, lse = avq.cross_attention_fwd(Q.cuda(), K.cuda(), V.cuda(), c, c, 0.3, with_lse=True)
    check_forward(Y.cpu(), lse.cpu(), Q, K, V, [20, 40], [20, 40], 0.3)
    got = avq.cross_attention_bwd(dY.cuda(), Q.cuda(), K.cuda(), V.cuda(), Y, lse, c, c, 0.3)
    want = avq.cross_attention_bwd(dY.cuda(), Q.cuda(), K.cuda(), V.cuda(), Y, lse, cu([20, 40]),
                                   cu([20, 40]), 0.3)
    for x, y in zip(got, want):
        assert torch.equal(x, y)


@pytest.mark.parametrize("bad", [math.inf, math.nan])
def test_bad_values_stay_in_their_source(bad):
    lens_q, lens_k = [40, 30, 50], [65, 64, 70]
    Q, K, V, dY = make(lens_q, lens_k, 2, 1, 64, BF16, 4)
    clean = [x.cpu() for x in both(Q, K, V, dY, lens_q, lens_k, 0.3)[2]]
    Q[50], K[70], V[80], dY[45] = bad, bad, bad, bad
    Y, lse = fwd(Q, K, V, lens_q, lens_k, 0.3)
    got = avq.cross_attention_bwd(dY.cuda(), Q.cuda(), K.cuda(), V.cuda(), Y, lse, cu(lens_q),
                                  cu(lens_k), 0.3)
    for name, x, own in zip("QKV", got, (slice(40, 70), slice(65, 129), slice(65, 129))):
        assert torch.isfinite(torch.cat((x[:own.start], x[own.stop:]))).all(), name


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_same_bits_again(dtype):
    """The sums have one order: the same bits at every call, on any workspace."""
    lens_q, lens_k = [300, 1, 90], [900, 700, 3]
    Q, K, V, dY = (x.cuda() for x in make(lens_q, lens_k, 4, 1, 128, dtype, 6))
    Y, lse = avq.cross_attention_fwd(Q, K, V, cu(lens_q), cu(lens_k), 0.1, with_lse=True)
    first = avq.cross_attention_bwd(dY, Q, K, V, Y, lse, cu(lens_q), cu(lens_k), 0.1)
    n = avq.cross_attention_workspace(dtype, 3, 391, 1603, 4, 1, 128, backward=True)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    for _ in range(3):
        again = avq.cross_attention_bwd(dY, Q, K, V, Y, lse, cu(lens_q), cu(lens_k), 0.1,
                                        workspace=ws)
        for x, y in zip(first, again):
            assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_differences(dtype):
    """The gradient along random directions against central differences of the loss
    sum Y dY in 64 bits. The differences at steps e and 2 e bound their own error:
    it is of the order e^2, so at e a third of what they differ by."""
    lens_q, lens_k, scale = [6, 1], [50, 35], 0.3
    Q, K, V, dY = make(lens_q, lens_k, 4, 2, 64, dtype, 8)
    mask = torch.rand(85, generator=torch.Generator().manual_seed(2)) < 0.7
    Y, lse, got = both(Q, K, V, dY, lens_q, lens_k, scale, mask)
    from tests.cross_reference import HALF_STEP, backward64
    want, tol = backward64(dY, Q, K, V, lens_q, lens_k, scale, mask)
    g = torch.Generator().manual_seed(9)
    for i in range(3):
        x = [Q.double(), K.double(), V.double()]
        u = torch.randn(x[i].shape, generator=g).double()

        def loss(e):
            z = list(x)
            z[i] = x[i] + e * u
            return (forward64(*z, lens_q, lens_k, scale, mask)[0] * dY.double()).sum()

        near = (loss(1e-4) - loss(-1e-4)) / 2e-4
        far = (loss(2e-4) - loss(-2e-4)) / 4e-4
        bound = ((tol[i] * (1 + 2.0 ** -6) + HALF_STEP[dtype] * (want[i].abs() + tol[i]))
                 * u.abs()).sum()
        along = (got[i].cpu().double() * u).sum()
        assert (along - near).abs() <= bound + (near - far).abs() + 1e-8 * near.abs()


def test_nothing_to_do():
    Q, K, V, dY = (x.cuda() for x in make([8], [8], 2, 1, 64, BF16))
    none = Q[:0]
    Y, lse = avq.cross_attention_fwd(none, K, V, cu([0]), cu([8]), 0.3, with_lse=True)
    assert Y.shape == (0, 2, 64)
    dQ, dK, dV = avq.cross_attention_bwd(none, none, K, V, Y, lse, cu([0]), cu([8]), 0.3)
    assert (dK == 0).all() and (dV == 0).all()
    Y, lse = avq.cross_attention_fwd(Q, K[:0], V[:0], cu([8]), cu([0]), 0.3, with_lse=True)
    assert (Y == 0).all() and (lse == -math.inf).all()
    dQ, dK, dV = avq.cross_attention_bwd(dY, Q, K[:0], V[:0], Y, lse, cu([8]), cu([0]), 0.3)
    assert (dQ == 0).all() and dK.shape == (0, 1, 64)


def test_refusals_on_the_gpu():
    Q, K, V, dY = (x.cuda() for x in make([8], [8], 2, 1, 64, BF16))
    c = cu([8])
    Y, lse = avq.cross_attention_fwd(Q, K, V, c, c, 0.3, with_lse=True)
    bad = torch.ones(8, device="cuda")
    for kw in (dict(mask=bad), dict(mask=bad[:7].bool()), dict(mask=torch.ones(8).bool()),
               dict(Y=Y.float()), dict(lse=lse.half())):
        with pytest.raises(ValueError):
            avq.cross_attention_fwd(Q, K, V, c, c, 0.3, **kw)
    with pytest.raises(ValueError):
        avq.cross_attention_fwd(Q, K, V.float(), c, c, 0.3)
    with pytest.raises(ValueError):
        avq.cross_attention_bwd(dY[:7], Q, K, V, Y, lse, c, c, 0.3)
    with pytest.raises(ValueError):
        avq.cross_attention_bwd(dY, Q, K, V, Y, lse[:7], c, c, 0.3)
    with pytest.raises(avq.AvqError):  # one row for all tokens
        avq.cross_attention_bwd(dY[:1].expand(8, 2, 64), Q, K, V, Y, lse, c, c, 0.3)
    with pytest.raises(avq.AvqError):
        avq.cross_attention_bwd(dY, Q, K, V, Y, lse, c, c, 0.3,
                                workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))


def test_graph():
    """Forward and backward captured once, replayed with new inputs."""
    lens_q, lens_k = [40, 3], [200, 700]
    x = [t.cuda() for t in make(lens_q, lens_k, 4, 2, 64, BF16, 11)]
    mask = torch.ones(900, dtype=torch.bool, device="cuda")
    cq, ck = cu(lens_q), cu(lens_k)

    def step():
        Y, lse = avq.cross_attention_fwd(x[0], x[1], x[2], cq, ck, 0.2, mask=mask, with_lse=True)
        return (Y, lse) + avq.cross_attention_bwd(x[3], x[0], x[1], x[2], Y, lse, cq, ck, 0.2,
                                                  mask=mask)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for seed in (12, 13, 14):
        for t, n in zip(x, make(lens_q, lens_k, 4, 2, 64, BF16, seed)):
            t.copy_(n.cuda())
        mask.copy_(torch.rand(900, device="cuda") < 0.8)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, step()):
            assert torch.equal(a, b)


def test_two_streams():
    """Calls at once on two streams, each with its own workspace."""
    lens_q, lens_k = [200], [1200]
    sets = [[t.cuda() for t in make(lens_q, lens_k, 4, 2, 64, BF16, s)] for s in (20, 21)]
    c, k = cu(lens_q), cu(lens_k)
    want = []
    for Q, K, V, dY in sets:
        Y, lse = avq.cross_attention_fwd(Q, K, V, c, k, 0.2, with_lse=True)
        want.append((Y, lse) + avq.cross_attention_bwd(dY, Q, K, V, Y, lse, c, k, 0.2))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    got = []
    for st, (Q, K, V, dY) in zip(streams, sets):
        Y, lse = avq.cross_attention_fwd(Q, K, V, c, k, 0.2, with_lse=True, stream=st)
        got.append((Y, lse) + avq.cross_attention_bwd(dY, Q, K, V, Y, lse, c, k, 0.2, stream=st))
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        for x, y in zip(a, b):
            assert torch.equal(x, y)


def test_rows_past_32_bits():
    """Elements past 2^31: the last source of a long packed array."""
    T, Hq, Hkv, d = 1_100_000, 16, 16, 128
    lens_q, lens_k, n = [T - 70, 70], [T - 100, 100], 100
    Q, K, V, dY = make([n], [n], Hq, Hkv, d, BF16, 15)
    big = [torch.zeros(T, 16, d, dtype=BF16, device="cuda") for _ in range(4)]
    for x, y in zip(big, (Q, K, V, dY)):
        x[T - n:] = y.cuda()
    mask = torch.ones(T, dtype=torch.bool, device="cuda")
    mask[:T - 100] = False  # the first source sees nothing
    c, k = cu(lens_q), cu(lens_k)
    Y, lse = avq.cross_attention_fwd(*big[:3], c, k, 0.1, mask=mask, with_lse=True)
    check_forward(Y[T - 70:].cpu(), lse[T - 70:].cpu(), Q[30:], K, V, [70], [100], 0.1)
    assert (Y[:T - 70] == 0).all() and (lse[:T - 70] == -math.inf).all()
    y64, l64 = forward64(Q[30:], K, V, [70], [100], 0.1)
    Y[T - 70:], lse[T - 70:] = y64.to(BF16).cuda(), l64.float().cuda()
    got = avq.cross_attention_bwd(big[3], *big[:3], Y, lse, c, k, 0.1, mask=mask)
    check_backward([got[0][T - 70:].cpu(), got[1][T - 100:].cpu(), got[2][T - 100:].cpu()], dY[30:],
                   Q[30:], K, V, [70], [100], 0.1)
    for x, m in zip(got, (70, 100, 100)):
        assert (x[:T - m] == 0).all()


def test_many_sources_of_few_states():
    """More sources than a wave has lanes, of all lengths, some without queries, states or
    visible ones."""
    g = torch.Generator().manual_seed(30)
    lens_q = torch.randint(0, 5, (150,), generator=g).tolist()
    lens_k = (torch.randint(0, 70, (150,), generator=g) * (torch.rand(150, generator=g) < 0.8)).tolist()
    Q, K, V, dY = make(lens_q, lens_k, 2, 1, 64, BF16, 31)
    mask = torch.rand(sum(lens_k), generator=g) < 0.3
    both(Q, K, V, dY, lens_q, lens_k, 0.2, mask)


def test_unaligned_rows_are_refused():
    Q, K, V, dY = (x.cuda() for x in make([8], [8], 2, 1, 64, BF16))
    odd = torch.empty(8 * 128 + 1, dtype=BF16, device="cuda")[1:].view(8, 2, 64)
    with pytest.raises(avq.AvqError):
        avq.cross_attention_fwd(odd, K, V, cu([8]), cu([8]), 0.3)
    Y, lse = avq.cross_attention_fwd(Q, K, V, cu([8]), cu([8]), 0.3, with_lse=True)
    with pytest.raises(avq.AvqError):
        avq.cross_attention_bwd(odd, Q, K, V, Y, lse, cu([8]), cu([8]), 0.3)


def test_two_graphs():
    """Two captured graphs, replayed in turn and at once on two streams."""
    lens_q, lens_k = [40, 3], [200, 700]
    c, k = cu(lens_q), cu(lens_k)
    graphs, inputs = [], []
    for seed in (1, 2):
        x = [t.cuda() for t in make(lens_q, lens_k, 4, 2, 64, BF16, seed)]

        def step(x=x):
            Y, lse = avq.cross_attention_fwd(*x[:3], c, k, 0.2, with_lse=True)
            return (Y, lse) + avq.cross_attention_bwd(x[3], *x[:3], Y, lse, c, k, 0.2)

        want = step()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = step()
        graphs.append((g, out, want, torch.cuda.Stream()))
        inputs.append(x)  # a graph reads them where they are
    for at_once in (False, True):
        for _ in range(3):
            for _, out, _, _ in graphs:
                for t in out:
                    t.zero_()
            torch.cuda.synchronize()
            for g, _, _, st in graphs:
                with torch.cuda.stream(st):
                    g.replay()
                if not at_once:
                    torch.cuda.synchronize()
            torch.cuda.synchronize()
            for _, out, want, _ in graphs:
                for a, b in zip(out, want):
                    assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("close", [False, True])
@pytest.mark.parametrize("lens_q,lens_k", [([37], [33]), ([300, 1], [90, 700]), ([3], [2000]),
                                           ([513, 2, 0, 70], [40, 1100, 9, 0]),
                                           ([5] * 20, [100] * 20), ([1] * 70, [3] * 70)])
def test_gradients_of_what_the_forward_call_stored(lens_q, lens_k, close, d, dtype):
    """The pair as a training step calls it: the backward pass is handed the forward
    kernel's own Y and lse. close: keys and values that lie close together, where what
    delta is off by through Y's rounding counts most. Some states are hidden."""
    Q, K, V, dY = make(lens_q, lens_k, 4, 2, d, dtype, 40)
    if close:
        K, V = about(K, 1.0, 0.3), about(V, 4.0, 0.1)
    mask = torch.rand(sum(lens_k), generator=torch.Generator().manual_seed(41)) < 0.8
    scale = 1 / math.sqrt(d)
    Y, lse = fwd(Q, K, V, lens_q, lens_k, scale, mask)
    check_forward(Y.cpu(), lse.cpu(), Q, K, V, lens_q, lens_k, scale, mask)
    got = avq.cross_attention_bwd(gpu(dY), gpu(Q), gpu(K), gpu(V), Y, lse, cu(lens_q), cu(lens_k),
                                  scale, mask=gpu(mask))
    check_backward_of([x.cpu() for x in got], dY, Q, K, V, Y.cpu(), lse.cpu(), lens_q, lens_k, scale,
                      mask)


def huge(lens_k, at, Hq, Hkv, d, dtype):
    """Two sources of 34 queries; states `at` of the first are 2^40. Query 0 of each sees
    equal logits, query 1 sees the huge ones, the others see them with the other sign."""
    Q, K, V, _ = make([34, 34], lens_k, Hq, Hkv, d, dtype, 42)
    Q = -Q.abs()
    Q[0] = Q[34] = 0
    Q[1] = Q[35] = 1
    K[at] = 2.0 ** 40
    return Q, K, V


@pytest.mark.parametrize("dtype,d", [(BF16, 64), (BF16, 128), (F32, 64), (F32, 128)])
@pytest.mark.parametrize("n,at,divided", [(60, [40], False), (88, [0], False), (60, [59], False),
                                          (88, [10, 87], False), (300, [200], True),
                                          (3000, [0], True), (3000, [1500, 2999], True)])
@pytest.mark.parametrize("masked", [False, True])
def test_one_huge_state_among_ordinary_ones(masked, n, at, divided, d, dtype):
    """Logits of 2^43 and more take the softmax's second form, maximum first, in some
    parts of the states and not in others."""
    Hq, Hkv, lens_q, lens_k = 2, 1, [34, 34], [n, 40]
    Q, K, V = huge(lens_k, at, Hq, Hkv, d, dtype)
    mask = None
    if masked:  # a huge one more, which is hidden, and ordinary ones
        mask = torch.arange(n + 40) % 7 != 3
        mask[at] = True
        K[3] = 2.0 ** 41
        assert not mask[3]
    assert (avq.cross_attention_workspace(dtype, 2, 68, n + 40, Hq, Hkv, d) > 0) == divided
    Y, lse = (x.cpu() for x in fwd(Q, K, V, lens_q, lens_k, 0.125, mask))
    seen = torch.ones(n, dtype=torch.bool) if mask is None else mask[:n]
    check_forward(Y[:1], lse[:1], Q[:1], K[:n], V[:n], [1], [n], 0.125, seen)
    # the mean of the huge ones' values: their sum and its quotient rounded in fp32, then
    # to the type
    v = V[at, 0].double()
    tol = HALF_STEP[dtype] * v.mean(0).abs() + 3 * 2.0 ** -24 * v.abs().sum(0)
    if len(at) == 1:
        tol = torch.zeros_like(tol)
    assert ((Y[1].double() - v.mean(0)).abs() <= tol).all()
    # the maximum is exact; log2(e), its product, ln 2 and theirs are rounded
    assert ((lse[1].double() / (0.125 * d * 2.0 ** 40) - 1).abs() <= 5 * 2.0 ** -24).all()
    rest = seen.clone()
    rest[at] = False
    check_forward(Y[2:34], lse[2:34], Q[2:34], K[:n], V[:n], [32], [n], 0.125, rest)
    check_forward(Y[34:], lse[34:], Q[34:], K[n:], V[n:], [34], [40], 0.125,
                  None if mask is None else mask[n:])
