"""prompt_attention_fwd against the 64-bit reference (MI355X)."""
import math

import pytest
import torch

from paper_2607_12789_amd import avq
from tests.serving_reference import check_attention, check_prompt, seen_of

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
    return Q, K, V


def run(Q, K, V, lens_q, lens_k, scale, causal, **kw):
    Y, lse = avq.prompt_attention_fwd(Q.cuda(), K.cuda(), V.cuda(), cu(lens_q), cu(lens_k), scale,
                                      causal=causal, with_lse=True, **kw)
    torch.cuda.synchronize()
    return Y.cpu(), lse.cpu()


LENS = [
    ([1], None), ([37], None), ([64], None), ([65], None), ([127, 128, 129], None),
    ([300, 1, 0, 0, 77], None), ([0, 0, 5, 0], None), ([513, 31, 33], None),
    # queries at the end of longer keys, and more queries than keys (the first
    # see nothing under the causal mask), and no keys at all
    ([16, 130], [400, 131]), ([1, 1, 1], [1, 70, 513]), ([5, 140, 3], [0, 100, 64]),
    ([2] * 90, [3] * 90),
]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens_q,lens_k", LENS)
def test_lengths(lens_q, lens_k, causal, d, dtype):
    lens_k = lens_k or lens_q
    Q, K, V = make(lens_q, lens_k, 4, 2, d, dtype)
    Y, lse = run(Q, K, V, lens_q, lens_k, 1 / math.sqrt(d), causal)
    check_prompt(Y, lse, Q, K, V, lens_q, lens_k, 1 / math.sqrt(d), causal)


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (7, 1), (6, 6), (8, 2), (24, 8), (5, 5)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_heads(Hq, Hkv, dtype):
    lens = [90, 201]
    Q, K, V = make(lens, lens, Hq, Hkv, 64, dtype, 3)
    Y, lse = run(Q, K, V, lens, lens, 0.2, True)
    check_prompt(Y, lse, Q, K, V, lens, lens, 0.2, True)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("q_scale", [0.0, 40.0])
def test_flat_and_peaked(dtype, q_scale):
    """Equal logits (a plain mean), and logits of hundreds that grow along the
    keys, so that the running maximum moves all the time."""
    lens = [260]
    Q, K, V = make(lens, lens, 2, 1, 128, dtype, 5, q_scale)
    if q_scale:
        K = (K.float() * torch.linspace(0.1, 3, 260)[:, None, None]).to(dtype)
    Y, lse = run(Q, K, V, lens, lens, 0.5, True)
    check_prompt(Y, lse, Q, K, V, lens, lens, 0.5, True)


def test_negative_logits():
    """Every logit far below zero: the first maximum is not zero's."""
    Q = torch.full((150, 1, 64), 8.0, dtype=BF16)
    K = torch.full((150, 1, 64), -8.0, dtype=BF16)
    V = make([150], [150], 1, 1, 64, BF16)[2]
    Y, lse = run(Q, K, V, [150], [150], 1.0, True)
    check_prompt(Y, lse, Q, K, V, [150], [150], 1.0, True)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_slices_of_a_fused_projection(dtype):
    lens, Hq, Hkv, d = [70, 130], 4, 2, 64
    g = torch.Generator().manual_seed(1)
    fused = torch.randn(200, (Hq + 2 * Hkv) * d, generator=g).to(dtype).cuda()
    q, k, v = fused.split([Hq * d, Hkv * d, Hkv * d], 1)
    q, k, v = (x.unflatten(1, (-1, d)) for x in (q, k, v))
    assert not q.is_contiguous()
    Y, lse = avq.prompt_attention_fwd(q, k, v, cu(lens), cu(lens), 0.3, with_lse=True)
    check_prompt(Y.cpu(), lse.cpu(), q.cpu(), k.cpu(), v.cpu(), lens, lens, 0.3, True)


def test_rows_behind_the_last_sequence_stay():
    lens = [40, 10]
    Q, K, V = make([70], [70], 2, 2, 64, BF16)
    Y = torch.full((70, 2, 64), 7.0, dtype=BF16, device="cuda")
    lse = torch.full((70, 2), 7.0, device="cuda")
    avq.prompt_attention_fwd(Q.cuda(), K.cuda(), V.cuda(), cu(lens), cu(lens), 0.3, Y=Y,
                             with_lse=True, lse=lse)
    assert (Y[50:] == 7).all() and (lse[50:] == 7).all()
    check_prompt(Y[:50].cpu(), lse[:50].cpu(), Q, K, V, lens, lens, 0.3, True)


def test_cu_outside_the_rows():
    """Sequence bounds past the rows are taken as their end, negative ones as 0."""
    Q, K, V = make([60], [60], 1, 1, 64, BF16)
    c = torch.tensor([-5, 20, 500], dtype=torch.int32, device="cuda")
    Y, lse = avq.prompt_attention_fwd(Q.cuda(), K.cuda(), V.cuda(), c, c, 0.3, with_lse=True)
    check_prompt(Y.cpu(), lse.cpu(), Q, K, V, [20, 40], [20, 40], 0.3, True)


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_bad_values_stay_in_their_sequence(bad, dtype):
    lens = [50, 30, 129, 64]
    Q, K, V = make(lens, lens, 2, 1, 64, dtype, 9)
    want = run(Q, K, V, lens, lens, 0.3, True)
    for x in (Q, K, V):
        x[50:80] = bad
    Y, lse = run(Q, K, V, lens, lens, 0.3, True)
    for a, b in ((0, 50), (80, 273)):
        assert torch.equal(Y[a:b], want[0][a:b]) and torch.equal(lse[a:b], want[1][a:b])


def test_the_same_call_twice_gives_the_same_bits():
    lens = [700, 45, 300]
    Q, K, V = make(lens, lens, 8, 2, 128, BF16, 2)
    a, b = (run(Q, K, V, lens, lens, 0.1, True) for _ in range(2))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_one_long_sequence():
    """Thousands of keys: some rows of one head against the reference."""
    n, d = 9001, 128
    Q, K, V = make([n], [n], 2, 1, d, BF16, 4)
    Y, lse = run(Q, K, V, [n], [n], 1 / math.sqrt(d), True)
    at = torch.tensor([0, 1, 63, 64, 4095, 4096, 8191, 8999, 9000])
    for h in range(2):
        check_attention(Y[at, h], lse[at, h], Q[at, h], K[:, 0], V[:, 0], 1 / math.sqrt(d), at + 1)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d,Hq,causal", [(64, 2, True), (128, 7, False), (128, 1, True)])
@pytest.mark.parametrize("lens_q,lens_k", [([5], [3000]), ([130, 1], [3100, 2700]),
                                           ([300, 0, 0, 4, 0], [290, 9000, 0, 6000, 0])])
def test_few_queries_many_keys(lens_q, lens_k, d, Hq, causal, dtype):
    """Tiles whose keys several workgroups share (rows without keys among them,
    and sequences without queries)."""
    scale = 1 / math.sqrt(d)
    n = avq.prompt_attention_workspace(dtype, len(lens_q), sum(lens_q), sum(lens_k), Hq, d, causal)
    assert n > 0
    Q, K, V = make(lens_q, lens_k, Hq, 1, d, dtype, 7)
    Y, lse = run(Q, K, V, lens_q, lens_k, scale, causal)
    check_prompt(Y, lse, Q, K, V, lens_q, lens_k, scale, causal)


@pytest.mark.parametrize("S", [64, 70, 130])
def test_many_sequences_with_many_keys(S):
    """Shared tiles of more sequences than lanes."""
    lens_q, lens_k = [s % 3 for s in range(S)], [2600 + 17 * (s % 40) for s in range(S)]
    assert avq.prompt_attention_workspace(BF16, S, sum(lens_q), sum(lens_k), 1, 64) > 0
    Q, K, V = make(lens_q, lens_k, 1, 1, 64, BF16, 13)
    Y, lse = run(Q, K, V, lens_q, lens_k, 0.2, True)
    check_prompt(Y, lse, Q, K, V, lens_q, lens_k, 0.2, True)


def test_shared_tiles_captured_with_one_workspace():
    """Two graphs with one workspace, replayed in turn with eager calls between,
    for lengths that change."""
    g = torch.Generator().manual_seed(8)
    Q = torch.randn(200, 4, 64, generator=g).to(BF16).cuda()
    K, V = (torch.randn(9000, 2, 64, generator=g).to(BF16).cuda() for _ in range(2))
    cq, ck = cu([100, 100]), cu([4500, 4500])
    n = avq.prompt_attention_workspace(BF16, 2, 200, 9000, 4, 64)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    outs = [torch.empty(200, 4, 64, dtype=BF16, device="cuda") for _ in range(2)]
    avq.prompt_attention_fwd(Q, K, V, cq, ck, 0.3, Y=outs[0], workspace=ws)
    torch.cuda.synchronize()
    graphs = []
    for Y in outs:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            avq.prompt_attention_fwd(Q, K, V, cq, ck, 0.3, Y=Y, workspace=ws)
    for i, (a, b) in enumerate([([100, 100], [4500, 4500]), ([1, 199], [8000, 1000]),
                                ([128, 72], [0, 9000]), ([0, 200], [3000, 6000])] * 2):
        cq.copy_(cu(a)), ck.copy_(cu(b))
        want = avq.prompt_attention_fwd(Q, K, V, cq, ck, 0.3)
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[i % 2], want), i


@pytest.mark.parametrize("S", [63, 64, 65, 300])
def test_many_sequences(S):
    """One sequence per lane and more: both orders of the tiles."""
    lens = [1 + 37 * s % 300 if s % 3 else 0 for s in range(S)]
    Q, K, V = make(lens, lens, 1, 1, 64, BF16, 12)
    Y, lse = run(Q, K, V, lens, lens, 0.2, True)
    check_prompt(Y, lse, Q, K, V, lens, lens, 0.2, True)


def test_offsets_past_32_bits():
    """Token rows 2^22 elements apart: 700 of them span 5.9 GB."""
    n, stride = 700, 1 << 22
    big = torch.empty(n, stride, dtype=BF16, device="cuda")
    Q, K, V = make([n], [n], 1, 1, 64, BF16, 6)
    k, v = big[:, 64:128].unflatten(1, (1, 64)), big[:, 256:320].unflatten(1, (1, 64))
    k.copy_(K), v.copy_(V)
    Y, lse = avq.prompt_attention_fwd(Q.cuda(), k, v, cu([n]), cu([n]), 0.3, with_lse=True)
    check_prompt(Y.cpu(), lse.cpu(), Q, K, V, [n], [n], 0.3, True)


def test_another_stream():
    lens = [200, 100]
    Q, K, V = (x.cuda() for x in make(lens, lens, 4, 4, 64, BF16))
    c = cu(lens)
    want = avq.prompt_attention_fwd(Q, K, V, c, c, 0.3)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = [avq.prompt_attention_fwd(Q, K, V, c, c, 0.3, stream=s) for _ in range(3)]
    s.synchronize()
    assert all(torch.equal(x, want) for x in got)


def test_captured_and_replayed():
    """Lengths are read on the device: one graph serves other lengths."""
    n, S = 300, 3
    g = torch.Generator().manual_seed(8)
    Q, K, V = (torch.randn(n, 2, 64, generator=g).to(BF16).cuda() for _ in range(3))
    c = cu([100, 100, 100])
    Y, lse = avq.prompt_attention_fwd(Q, K, V, c, c, 0.3, with_lse=True)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        avq.prompt_attention_fwd(Q, K, V, c, c, 0.3, Y=Y, with_lse=True, lse=lse)
    for lens in ([100, 100, 100], [1, 298, 1], [0, 0, 300], [150, 100, 20]):
        c.copy_(cu(lens))
        want = avq.prompt_attention_fwd(Q, K, V, c, c, 0.3, with_lse=True)
        graph.replay()
        torch.cuda.synchronize()
        m = sum(lens)
        assert torch.equal(Y[:m], want[0][:m]) and torch.equal(lse[:m], want[1][:m])


def test_no_tokens():
    e = torch.empty(0, 2, 64, dtype=BF16, device="cuda")
    Y = avq.prompt_attention_fwd(e, e, e, cu([0]), cu([0]), 0.3)
    assert Y.shape == (0, 2, 64)
    Q, K, _ = make([4], [4], 2, 2, 64, BF16)
    Y, lse = avq.prompt_attention_fwd(Q.cuda(), e, e, cu([4]), cu([0]), 0.3, with_lse=True)
    assert (Y == 0).all() and (lse == -math.inf).all()


def test_refusals():
    Q, K, V = (x.cuda() for x in make([8], [8], 2, 2, 64, BF16))
    c = cu([8])
    bad = [dict(K=K[:, :, :32]), dict(K=K.float()), dict(V=V[:5]), dict(cu_q=c.long()),
           dict(cu_k=cu([4, 4])), dict(Y=torch.empty(8, 2, 64, device="cuda")),
           dict(lse=torch.empty(8, device="cuda")), dict(Q=Q.transpose(0, 1)),
           dict(Q=Q.transpose(1, 2)), dict(cu_q=c[:1], cu_k=c[:1])]
    for kw in bad:
        a = dict(Q=Q, K=K, V=V, cu_q=c, cu_k=c, scale=1.0) | kw
        with pytest.raises(ValueError):
            avq.prompt_attention_fwd(**a)
    with pytest.raises(avq.AvqError):
        avq.prompt_attention_fwd(Q, K, V, c, c, -1.0)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_equal_logits_of_any_size(dtype):
    """Equal logits give the mean of the values, however far from 0 they lie."""
    for n, size in ((70, 1e15), (70, -1e15), (3000, -1e15)):
        Q = torch.full((2, 1, 64), 1e17).to(dtype)
        K = torch.full((n, 1, 64), size).to(dtype)
        V = make([1], [n], 1, 1, 64, dtype)[2]
        Y, _ = run(Q, K, V, [2], [n], 1.0, False)
        half = 2.0 ** -8 if dtype == BF16 else n * 2.0 ** -24
        mean, size_ = V[:, 0].double().mean(0), V[:, 0].double().abs().mean(0)
        assert ((Y[:, 0].double() - mean).abs() <= half * (mean.abs() + size_)).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n", [300, 3000])
def test_one_huge_key_among_ordinary_ones(n, dtype):
    """A wave with a row of equal logits, one that sees a huge logit, and ones
    that see it with the other sign (weight 0) among ordinary ones."""
    Q, K, V = make([34], [n], 1, 1, 64, dtype, 9)
    Q = -Q.abs()
    Q[0], Q[1] = 0, 1
    K[200] = 2.0 ** 40
    Y, lse = run(Q, K, V, [34], [n], 0.125, False)
    check_attention(Y[:1, 0], lse[:1, 0], Q[:1, 0], K[:, 0], V[:, 0], 0.125, seen_of(1, n, False))
    assert torch.equal(Y[1, 0], V[200, 0])
    rest = torch.arange(n) != 200
    check_attention(Y[2:, 0], lse[2:, 0], Q[2:, 0], K[rest, 0], V[rest, 0], 0.125,
                    seen_of(32, n - 1, False))


def test_equal_runs_on_two_streams_at_once():
    d, Lk = 128, 6000
    sets = [[x.cuda() for x in make([200], [Lk], 8, 2, d, BF16, s)] for s in range(2)]
    c, ck = cu([200]), cu([Lk])
    assert avq.prompt_attention_workspace(BF16, 1, 200, Lk, 8, d) > 0
    want = [avq.prompt_attention_fwd(*x, c, ck, 0.1) for x in sets]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(10):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(avq.prompt_attention_fwd(*sets[i], c, ck, 0.1))
    torch.cuda.synchronize()
    assert all(torch.equal(y, want[i]) for i in range(2) for y in got[i])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens_q,lens_k,Hq", [([32], [1024], 4), ([31, 75, 9], [357, 2209, 125], 4),
                                              ([130, 1, 0], [2000, 1500, 1700], 6)])
def test_parts_of_few_tiles(lens_q, lens_k, Hq, d, dtype):
    """Tiles of few rows, in a few runs of one tile each or less."""
    Q, K, V = make(lens_q, lens_k, Hq, 2, d, dtype, 21)
    n = avq.prompt_attention_workspace(dtype, len(lens_q), sum(lens_q), sum(lens_k), Hq, d)
    assert n > 0
    Y, lse = run(Q, K, V, lens_q, lens_k, 1 / math.sqrt(d), True)
    check_prompt(Y, lse, Q, K, V, lens_q, lens_k, 1 / math.sqrt(d), True)


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d,Hq", [(64, 4), (128, 16)])
def test_bad_values_stay_in_their_sequence_in_parts(d, Hq, dtype, bad):
    """The same where workgroups go from one sequence's tiles to the next and
    leave parts that a second launch joins."""
    lens_q, lens_k = [130, 5, 40], [3100, 2700, 4000]
    assert avq.prompt_attention_workspace(dtype, 3, sum(lens_q), sum(lens_k), Hq, d, True) > 0
    Q, K, V = make(lens_q, lens_k, Hq, 2, d, dtype, 9)
    want = run(Q, K, V, lens_q, lens_k, 0.3, True)
    Q[130:135], K[3100:5800], V[3100:5800] = bad, bad, bad
    Y, lse = run(Q, K, V, lens_q, lens_k, 0.3, True)
    for a, b in ((0, 130), (135, 175)):
        assert torch.equal(Y[a:b], want[0][a:b]) and torch.equal(lse[a:b], want[1][a:b])
