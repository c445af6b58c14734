"""The paged cache (append, gather, attention) against the 64-bit reference
(MI355X)."""
import math

import pytest
import torch

from paper_2607_12789_amd import avq
from tests.serving_reference import (HALF_STEP, check_attention, check_fp4, check_prompt, decode,
                                     read_cache, rotate64, views)

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def cu(lens):
    t = torch.zeros(len(lens) + 1, dtype=torch.int32)
    t[1:] = torch.tensor(lens).cumsum(0)
    return t


def angles(n, rot):
    f = 10000.0 ** (-torch.arange(rot // 2).double() / max(1, rot // 2))
    a = torch.arange(n).double()[:, None] * f
    return a.cos().float(), a.sin().float()


def tables(lens, ps, seed=0, extra=1):
    """Pages in random order for the given lengths; returns (table, n_pages)."""
    held = [max(1, -(-n // ps)) for n in lens]
    n_pages = sum(held) + extra
    order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed))
    table = torch.full((len(lens), max(held)), -7, dtype=torch.int32)
    at = 0
    for i, n in enumerate(held):
        table[i, :n] = order[at:at + n].int()
        at += n
    return table, n_pages


def garbage(n_pages, Hkv, E, seed=1):
    """Bytes left from anything: as bf16 or fp32 also infinities and NaN."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randint(0, 256, (n_pages, Hkv, E), generator=g, dtype=torch.uint8)
    x.view(-1)[::3] = 0xff
    return x


class Setup:
    def __init__(self, new, old, Hq, Hkv, d, dtype, fp4, ps, rot=0, inter=False, seed=0):
        self.__dict__.update(new=new, old=old, Hq=Hq, Hkv=Hkv, d=d, dtype=dtype, fp4=fp4, ps=ps)
        g = torch.Generator().manual_seed(seed)
        self.S, self.T, self.lens = len(new), sum(new), [a + b for a, b in zip(new, old)]
        self.table, self.n_pages = tables(self.lens, ps, seed)
        self.E = avq.cache_page_bytes(dtype, ps, d, fp4)
        self.cache = garbage(self.n_pages, Hkv, self.E)
        self.Q = torch.randn(self.T, Hq, d, generator=g).to(dtype)
        wide = torch.exp(torch.randn(Hkv, d, generator=g))
        self.K = (wide * torch.randn(self.T, Hkv, d, generator=g)).to(dtype)
        self.V = torch.randn(self.T, Hkv, d, generator=g).to(dtype)
        self.cos, self.sin = angles(max(self.lens) + 1, rot) if rot else (None, None)
        self.inter = inter
        self.start = torch.tensor(old, dtype=torch.int32)

    def append(self, **kw):
        """Appends on the GPU; self.cache becomes the new cache."""
        dev = {n: None if getattr(self, n) is None else getattr(self, n).cuda()
               for n in ("K", "V", "cache", "table", "start", "Q", "cos", "sin")}
        out = avq.cache_append(dev["K"], dev["V"], dev["cache"], dev["table"], dev["start"], self.ps,
                               cu=cu(self.new).cuda(), Q=dev["Q"], cos=dev["cos"], sin=dev["sin"],
                               interleaved=self.inter, fp4=self.fp4, with_K=True, **kw)
        torch.cuda.synchronize()
        self.before, self.cache = self.cache, dev["cache"].cpu()
        return [x.cpu() for x in out]

    def places(self):
        """(row, sequence, position) of every token."""
        r = 0
        for s, (n, o) in enumerate(zip(self.new, self.old)):
            for i in range(n):
                yield r, s, o + i
                r += 1


APPEND = [  # new, cached before
    ([5], [0]), ([1], [7]), ([8, 8], [0, 8]), ([100, 3, 0, 17], [13, 255, 4, 0]),
    ([33, 1, 0, 0, 64], [31, 16, 0, 9, 64]), ([1] * 70, list(range(70))),
]


@pytest.mark.parametrize("new,old", APPEND)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("d,Hkv,rot,inter,ps", [(64, 3, 64, False, 16), (128, 2, 48, True, 64),
                                                (128, 1, 128, False, 32), (64, 2, 0, False, 256)])
def test_append(new, old, dtype, fp4, d, Hkv, rot, inter, ps):
    t = Setup(new, old, 2 * Hkv, Hkv, d, dtype, fp4, ps, rot, inter)
    Qo, Ko = t.append()
    pos = torch.tensor([p for _, _, p in t.places()])
    q, qe = rotate64(t.Q, pos, t.cos, t.sin, inter)
    k, ke = rotate64(t.K, pos, t.cos, t.sin, inter)
    half = HALF_STEP[dtype]
    assert ((Qo.double() - q).abs() <= half * q.abs() + 1.01 * qe).all()
    assert ((Ko.double() - k).abs() <= half * k.abs() + 1.01 * ke).all()
    # the cache: the new positions hold the rows, every other byte is as it was
    w, expect = views(t.cache, dtype, fp4, ps, d), t.before.clone()
    e = views(expect, dtype, fp4, ps, d)
    for r, s, p in t.places():
        page, slot = int(t.table[s, p // ps]), p % ps
        o, j = slot // 8, slot % 8
        if fp4:
            kd, ku = decode(w["Kc"][page, :, slot], w["Ks"][page, :, slot])
            vd, vu = decode(w["Vc"][page, :, o, :, j], w["Vs"][page, :, o, :, j])
            check_fp4(kd, ku, k[r], 1.01 * ke[r])
            check_fp4(vd, vu, t.V[r].double(), 0)
            for n in ("Kc", "Ks"):
                e[n][page, :, slot] = w[n][page, :, slot]
            for n in ("Vc", "Vs"):
                e[n][page, :, o, :, j] = w[n][page, :, o, :, j]
        else:
            assert torch.equal(w["K"][page, :, slot], Ko[r])
            assert torch.equal(w["V"][page, :, o, :, j], t.V[r])
            e["K"][page, :, slot], e["V"][page, :, o, :, j] = Ko[r], t.V[r]
    assert torch.equal(t.cache, expect), "a byte outside the new positions changed"


def test_fp4_codes():
    """Every border between two codes, zeros, the smallest and largest values."""
    d = 128
    x = torch.zeros(16, 1, d, dtype=F32)
    grid = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    ties = torch.cat((grid, -grid, torch.nextafter(grid, torch.tensor(0.)),
                      torch.nextafter(grid, torch.tensor(9.))))
    for r, s in enumerate((1.0, 2.0 ** -20, 2.0 ** 60, 2.0 ** -100)):
        x[r, 0, :28], x[r, 0, 28] = ties * s, 6.0 * s
    x[4, 0, 0], x[5, 0, 0], x[6, 0, 0] = 6.0, torch.nextafter(torch.tensor(6.), torch.tensor(9.)), 7.9
    x[7, 0], x[8, 0] = 3.0e38, 1e-45
    x[9, 0, 40] = 2.0 ** -126
    cache = torch.zeros(1, 1, avq.cache_page_bytes(F32, 16, d, True), dtype=torch.uint8).cuda()
    table, start = torch.zeros(1, 1, dtype=torch.int32).cuda(), torch.zeros(1, dtype=torch.int32).cuda()
    xd = x.cuda()
    avq.cache_append(xd, xd, cache, table, start, 16, cu=cu([16]).cuda(), fp4=True)
    K, V, _ = read_cache(cache.cpu(), table.cpu(), 0, 16, F32, True, 16, d)
    assert torch.equal(K, V)
    want = torch.tensor([0, 1, 1, 2, 2, 4, 4.], dtype=torch.float64)  # ties to the even code
    for r, s in enumerate((1.0, 2.0 ** -20, 2.0 ** 60, 2.0 ** -100)):
        assert torch.equal(K[0, r, :7] / s, want) and torch.equal(K[0, r, 7:14] / s, -want)
    assert K[0, 4, 0] == 6 and K[0, 5, 0] == 6 and K[0, 6, 0] == 8  # 7.9 at a scale of 2
    w = views(cache.cpu(), F32, True, 16, d)
    kd, ku = decode(w["Kc"][0, :, :10], w["Ks"][0, :, :10])
    check_fp4(kd, ku, x[:10].double().transpose(0, 1), 2.0 ** -126)
    assert (K[0, 10:] == 0).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("d,ps", [(64, 16), (128, 64)])
def test_gather(dtype, fp4, d, ps):
    t = Setup([60, 1, 0, 200], [0, 18, 5, 7], 3, 3, d, dtype, fp4, ps)
    t.append()
    # ranges that begin and end inside pages, an empty one, rows behind the last
    start, n = torch.tensor([3, 0, 2, 150], dtype=torch.int32), [50, 19, 0, 57]
    K = torch.full((sum(n) + 4, 3, d), 5.0, dtype=dtype, device="cuda")
    V = K.clone()
    avq.cache_gather(t.cache.cuda(), t.table.cuda(), start.cuda(), cu(n).cuda(), len(K), ps, dtype, d,
                     fp4=fp4, K=K, V=V)
    assert (K[-4:] == 5).all() and (V[-4:] == 5).all()
    r = 0
    for s, m in enumerate(n):
        k, v, _ = read_cache(t.cache, t.table, s, int(start[s]) + m, dtype, fp4, ps, d)
        for got, x in ((K, k), (V, v)):
            got, x = got[r:r + m].cpu().double(), x[:, int(start[s]):].transpose(0, 1)
            written = max(0, t.old[s] - int(start[s]))  # the rows before hold anything
            assert torch.equal(got[written:], x[written:])
        r += m


CACHED = [  # n_q, lengths
    (1, [1]), (1, [0, 5, 128, 129]), (1, [300, 31, 32, 33, 1000]), (1, [2600]),
    (4, [4, 2, 0, 130, 515]), (16, [16, 700]),
]


def fill(t):
    """Every position of the sequences' pages within the lengths, by the kernel
    that appends; what lies behind stays garbage."""
    t.append()
    return t.cache.cuda(), t.table.cuda(), torch.tensor(t.lens, dtype=torch.int32).cuda()


def check_cached(Y, lse, Q, t, lens, scale, rows=None):
    n_q = Q.shape[1]
    G = Q.shape[2] // t.Hkv
    for s, n in enumerate(lens):
        if rows is not None and s not in rows:
            continue
        K, V, ok = read_cache(t.cache, t.table, s, n, t.dtype, t.fp4, t.ps, t.d)
        seen = (torch.arange(n_q) + n - n_q + 1).clamp(0, n)
        for h in range(Q.shape[2]):
            check_attention(Y[s, :, h], None if lse is None else lse[s, :, h], Q[s, :, h], K[h // G],
                            V[h // G], scale, seen, f"sequence {s} head {h}")


@pytest.mark.parametrize("n_q,lens", CACHED)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("d,Hq,Hkv,ps", [(64, 4, 4, 16), (128, 8, 2, 64), (128, 7, 1, 256)])
def test_cached(n_q, lens, dtype, fp4, d, Hq, Hkv, ps):
    t = Setup(lens, [0] * len(lens), Hkv, Hkv, d, dtype, fp4, ps)
    cache, table, n = fill(t)
    Q = (2 * torch.randn(len(lens), n_q, Hq, d, generator=torch.Generator().manual_seed(3))).to(dtype)
    Y, lse = avq.cache_attention_fwd(Q.cuda(), cache, table, n, ps, 1 / math.sqrt(d), fp4=fp4,
                                     with_lse=True)
    check_cached(Y.cpu(), lse.cpu(), Q, t, lens, 1 / math.sqrt(d))


@pytest.mark.parametrize("S", [255, 257, 600])
def test_many_sequences(S):
    lens = [17 + s % 5 for s in range(S)]
    t = Setup(lens, [0] * S, 2, 2, 64, BF16, True, 16)
    cache, table, n = fill(t)
    Q = torch.randn(S, 1, 4, 64, generator=torch.Generator().manual_seed(3)).to(BF16)
    Y, lse = avq.cache_attention_fwd(Q.cuda(), cache, table, n, 16, 0.3, fp4=True, with_lse=True)
    check_cached(Y.cpu(), lse.cpu(), Q, t, lens, 0.3, rows={0, 1, 150, 254, 255, 256, 511, S - 1})


@pytest.mark.parametrize("Hq,Hkv", [(32, 1), (40, 2), (3, 3), (48, 8)])
def test_cached_heads(Hq, Hkv):
    t = Setup([200, 77], [0, 0], Hkv, Hkv, 64, BF16, True, 32)
    cache, table, n = fill(t)
    Q = torch.randn(2, 3, Hq, 64, generator=torch.Generator().manual_seed(3)).to(BF16)
    Y, lse = avq.cache_attention_fwd(Q.cuda(), cache, table, n, 32, 0.4, fp4=True, with_lse=True)
    check_cached(Y.cpu(), lse.cpu(), Q, t, [200, 77], 0.4)


@pytest.mark.parametrize("fp4", [False, True])
def test_bad_pages(fp4):
    """Entries outside the pool, and positions past the table: not written, read
    as 0, no part in the attention."""
    ps, d, lens = 16, 64, [100, 60]
    t = Setup(lens, [0, 0], 2, 2, d, BF16, fp4, ps)
    t.table[0, 2], t.table[1, 0] = t.n_pages, -1
    t.table = t.table[:, :5].contiguous()  # sequence 0 has 80 of its 100 positions
    t.append()
    spare = set(range(t.n_pages)) - set(t.table[t.table >= 0].tolist())
    for p in spare:
        assert torch.equal(t.cache[p], t.before[p])
    K, V = avq.cache_gather(t.cache.cuda(), t.table.cuda(), torch.zeros(2, dtype=torch.int32).cuda(),
                            cu(lens).cuda(), 160, ps, BF16, d, fp4=fp4)
    Q = torch.randn(2, 1, 4, d, generator=torch.Generator().manual_seed(3)).to(BF16)
    Y = avq.cache_attention_fwd(Q.cuda(), t.cache.cuda(), t.table.cuda(),
                                torch.tensor(lens, dtype=torch.int32).cuda(), ps, 0.4, fp4=fp4).cpu()
    for s, n in enumerate(lens):
        k, v, ok = read_cache(t.cache, t.table, s, n, BF16, fp4, ps, d)
        assert not ok.all()
        a = sum(lens[:s])
        assert torch.equal(K[a:a + n].cpu().double(), k.transpose(0, 1))
        assert torch.equal(V[a:a + n].cpu().double(), v.transpose(0, 1))
        kk, vv = k[:, ok], v[:, ok]
        for h in range(4):
            check_attention(Y[s, :, h], None, Q[s, :, h], kk[h // 2], vv[h // 2], 0.4,
                            torch.tensor([kk.shape[1]]), f"sequence {s}")


def test_lengths_outside_the_cache():
    """A negative length is 0, one past the table's positions is their number; a
    negative start and positions outside the angles are not written."""
    t = Setup([64], [0], 1, 1, 64, BF16, False, 16)
    t.append()
    Q = torch.randn(1, 1, 1, 64).to(BF16)
    args = (Q.cuda(), t.cache.cuda(), t.table.cuda())
    one = lambda n: torch.tensor([n], dtype=torch.int32).cuda()
    full = avq.cache_attention_fwd(*args, one(64), 16, 0.4)
    assert torch.equal(avq.cache_attention_fwd(*args, one(1 << 30), 16, 0.4), full)
    assert (avq.cache_attention_fwd(*args, one(-3), 16, 0.4) == 0).all()
    for start, rot in ((-1, False), (-(1 << 31), False), ((1 << 31) - 1, False), (1000, False),
                       (10, True)):
        cos, sin = angles(10, 64)
        c = t.cache.cuda()
        q = torch.full((64, 1, 64), 3.0, dtype=BF16, device="cuda")
        avq.cache_append(t.K.cuda(), t.V.cuda(), c, t.table.cuda(), one(start), 16,
                         cu=cu([64]).cuda(), Q=t.Q.cuda(), cos=cos.cuda() if rot else None,
                         sin=sin.cuda() if rot else None, Q_out=q)
        assert torch.equal(c.cpu(), t.cache)
        if start < 0 or rot:  # without angles a position past the table only lacks a page
            assert (q == 3).all()


def test_in_place_rotation():
    for inter in (False, True):
        t = Setup([70, 9], [3, 0], 4, 2, 128, BF16, True, 16, 96, inter)
        Qo, Ko = t.append()
        Q, K = t.Q.cuda(), t.K.cuda()
        avq.cache_append(K, t.V.cuda(), t.cache.cuda(), t.table.cuda(), t.start.cuda(), 16,
                         cu=cu(t.new).cuda(), Q=Q, cos=t.cos.cuda(), sin=t.sin.cuda(),
                         interleaved=inter, fp4=True, Q_out=Q, K_out=K)
        assert torch.equal(Q.cpu(), Qo) and torch.equal(K.cpu(), Ko)


def test_one_token_each_equals_the_packed_form():
    t = Setup([1] * 5, [0, 7, 8, 300, 15], 6, 2, 64, BF16, True, 16, 64)
    Qo, _ = t.append()
    c = t.before.cuda()
    q, none = avq.cache_append(t.K.cuda(), t.V.cuda(), c, t.table.cuda(), t.start.cuda(), 16,
                               Q=t.Q.cuda(), cos=t.cos.cuda(), sin=t.sin.cuda(), fp4=True)
    assert none is None and torch.equal(q.cpu(), Qo) and torch.equal(c.cpu(), t.cache)


@pytest.mark.parametrize("fp4", [False, True])
def test_pool_past_32_bits(fp4):
    """Pages more than 4 GiB into the pool."""
    ps, d, Hkv = 256, 128, 8
    E = avq.cache_page_bytes(BF16, ps, d, fp4)
    n_pages = (5 << 30) // (Hkv * E) + 2
    cache = torch.empty(n_pages, Hkv, E, dtype=torch.uint8, device="cuda")
    t = Setup([300, 40], [0, 100], 8, Hkv, d, BF16, fp4, ps)
    t.append()
    far = t.table.clone()
    far[t.table >= 0] += n_pages - t.n_pages
    Qd, Kd, Vd = t.Q.cuda(), t.K.cuda(), t.V.cuda()
    cache[n_pages - t.n_pages:] = t.before.cuda()
    avq.cache_append(Kd, Vd, cache, far.cuda(), t.start.cuda(), ps, cu=cu(t.new).cuda(), Q=Qd,
                     fp4=fp4)
    assert torch.equal(cache[n_pages - t.n_pages:].cpu(), t.cache)
    Q = torch.randn(2, 1, 16, d).to(BF16).cuda()
    lens = torch.tensor([300, 0], dtype=torch.int32).cuda()
    small = avq.cache_attention_fwd(Q, t.cache.cuda(), t.table.cuda(), lens, ps, 0.3, fp4=fp4)
    assert torch.equal(avq.cache_attention_fwd(Q, cache, far.cuda(), lens, ps, 0.3, fp4=fp4), small)
    z, c = torch.zeros(2, dtype=torch.int32).cuda(), cu([300, 0]).cuda()
    for x, y in zip(avq.cache_gather(cache, far.cuda(), z, c, 300, ps, BF16, d, fp4=fp4),
                    avq.cache_gather(t.cache.cuda(), t.table.cuda(), z, c, 300, ps, BF16, d, fp4=fp4)):
        assert torch.equal(x, y)


def test_long_context():
    """20000 positions in many parts, next to short sequences."""
    lens = [20000, 1, 130, 0, 4097]
    t = Setup(lens, [0] * 5, 1, 1, 128, BF16, True, 64)
    cache, table, n = fill(t)
    Q = (2 * torch.randn(5, 1, 4, 128, generator=torch.Generator().manual_seed(3))).to(BF16)
    Y, lse = avq.cache_attention_fwd(Q.cuda(), cache, table, n, 64, 0.1, fp4=True, with_lse=True)
    check_cached(Y.cpu(), lse.cpu(), Q, t, lens, 0.1)


def test_captured_steps_share_a_workspace():
    """Two graphs of a step (append, attention) with one workspace, replayed in
    turn with eager work between, as the sequences grow."""
    S, Hq, Hkv, d, ps, rot = 3, 8, 2, 64, 16, 64
    n0 = [5, 127, 300]
    t = Setup(n0, [0] * S, Hkv, Hkv, d, BF16, True, ps)
    t.lens = [n + 40 for n in n0]
    t.table, t.n_pages = tables(t.lens, ps)
    t.cache = garbage(t.n_pages, Hkv, t.E)
    t.append()
    cache, table = t.cache.cuda(), t.table.cuda()
    cos, sin = (x.cuda() for x in angles(400, rot))
    ws = torch.empty(avq.cache_attention_workspace(S, 1, Hq, Hkv, d), dtype=torch.uint8, device="cuda")
    Q, K, V = (torch.zeros(S, h, d, dtype=BF16, device="cuda") for h in (Hq, Hkv, Hkv))
    start, lens = torch.tensor(n0, dtype=torch.int32).cuda(), torch.tensor(n0, dtype=torch.int32).cuda()

    def step(cache, Qo, Y, ws):
        avq.cache_append(K, V, cache, table, start, ps, Q=Q, cos=cos, sin=sin, fp4=True, Q_out=Qo)
        avq.cache_attention_fwd(Qo[:, None], cache, table, lens, ps, 0.3, fp4=True, Y=Y, workspace=ws)

    bufs = [(torch.empty_like(Q), torch.empty(S, 1, Hq, d, dtype=BF16, device="cuda"))
            for _ in range(3)]
    step(cache.clone(), *bufs[2], ws)
    torch.cuda.synchronize()
    graphs = []
    for i in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            step(cache, *bufs[i], ws)
    other = cache.clone()
    for i in range(8):
        g = torch.Generator().manual_seed(i)
        for x in (Q, K, V):
            x.copy_(torch.randn(x.shape, generator=g).to(BF16))
        lens.copy_(start + 1)
        step(other, *bufs[2], torch.empty_like(ws))
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        assert torch.equal(bufs[i % 2][1], bufs[2][1]) and torch.equal(cache, other), i
        start.add_(1)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("fp4", [False, True])
def test_serving_run(dtype, fp4):
    """As a server uses them: a prompt (rotate, cache, attend), a chunk behind
    it (append, gather, attend), then single tokens (append, attend over the
    cache), each against attention over everything cached so far."""
    S, Hq, Hkv, d, ps, scale = 2, 4, 2, 64, 16, 0.25
    g = torch.Generator().manual_seed(11)
    plan = [[50, 7], [20, 33], [1, 1], [1, 1], [1, 1]]
    total = [sum(p[s] for p in plan) for s in range(S)]
    table, n_pages = tables(total, ps)
    E = avq.cache_page_bytes(dtype, ps, d, fp4)
    cache = garbage(n_pages, Hkv, E).cuda()
    cos, sin = (x.cuda() for x in angles(100, d))
    table_d, done = table.cuda(), [0] * S
    for step, new in enumerate(plan):
        T = sum(new)
        Q, K, V = (torch.randn(T, h, d, generator=g).to(dtype).cuda() for h in (Hq, Hkv, Hkv))
        start, c = torch.tensor(done, dtype=torch.int32).cuda(), cu(new).cuda()
        Qr, Kr = avq.cache_append(K, V, cache, table_d, start, ps, cu=c, Q=Q, cos=cos, sin=sin,
                                  fp4=fp4, with_K=True)
        pos = torch.cat([torch.arange(o, o + n) for o, n in zip(done, new)])
        want, err = rotate64(Q.cpu(), pos, cos.cpu(), sin.cpu(), False)
        assert ((Qr.cpu().double() - want).abs() <= HALF_STEP[dtype] * want.abs() + 1.01 * err).all()
        done = [a + b for a, b in zip(done, new)]
        rows = [read_cache(cache.cpu(), table, s, done[s], dtype, fp4, ps, d) for s in range(S)]
        Kc = torch.cat([r[0].transpose(0, 1) for r in rows])
        Vc = torch.cat([r[1].transpose(0, 1) for r in rows])
        if step == 0:  # the prompt itself, not yet rounded to 4 bits
            Y, lse = avq.prompt_attention_fwd(Qr, Kr, V, c, c, scale, with_lse=True)
            check_prompt(Y.cpu(), lse.cpu(), Qr.cpu(), Kr.cpu(), V.cpu(), new, new, scale, True)
        elif step == 1:
            k, v = avq.cache_gather(cache, table_d, torch.zeros_like(start), cu(done).cuda(),
                                    sum(done), ps, dtype, d, fp4=fp4)
            Y, lse = avq.prompt_attention_fwd(Qr, k, v, c, cu(done).cuda(), scale, with_lse=True)
            check_prompt(Y.cpu(), lse.cpu(), Qr.cpu(), Kc, Vc, new, done, scale, True)
        else:
            lens = torch.tensor(done, dtype=torch.int32).cuda()
            Y, lse = avq.cache_attention_fwd(Qr[:, None], cache, table_d, lens, ps, scale, fp4=fp4,
                                             with_lse=True)
            check_prompt(Y[:, 0].cpu(), lse[:, 0].cpu(), Qr.cpu(), Kc, Vc, new, done, scale, True)


def test_refusals():
    t = Setup([8], [0], 2, 2, 64, BF16, True, 16, 64)
    dev = {n: getattr(t, n).cuda() for n in ("K", "V", "cache", "table", "start", "Q", "cos", "sin")}
    base = dict(K=dev["K"], V=dev["V"], cache=dev["cache"], block_table=dev["table"],
                start=dev["start"], page_size=16, cu=cu([8]).cuda(), Q=dev["Q"], cos=dev["cos"],
                sin=dev["sin"], fp4=True)
    for kw in (dict(fp4=False), dict(page_size=32), dict(page_size=24), dict(cos=None),
               dict(start=dev["start"].long()), dict(block_table=dev["table"][0]),
               dict(cache=dev["cache"][:, :1].contiguous()), dict(cu=cu([4, 4]).cuda()),
               dict(V=dev["V"][:4]), dict(Q=dev["Q"][:4]), dict(Q=None, Q_out=dev["Q"]),
               dict(cos=dev["cos"][:, :0], sin=dev["sin"][:, :0]), dict(K_out=dev["K"].float())):
        with pytest.raises(ValueError):
            avq.cache_append(**(base | kw))
    for kw in (dict(cu=None), dict(cos=dev["cos"][:, :4].contiguous(), sin=dev["sin"][:, :4].contiguous())):
        with pytest.raises(avq.AvqError):
            avq.cache_append(**(base | kw))
    Q = torch.zeros(1, 1, 2, 64, dtype=BF16, device="cuda")
    base = dict(Q=Q, cache=dev["cache"], block_table=dev["table"], lens=dev["start"], page_size=16,
                scale=1.0, fp4=True)
    for kw in (dict(Q=Q[0]), dict(Q=Q.float(), fp4=False), dict(lens=dev["start"].long()),
               dict(Y=Q[0]), dict(Q=torch.zeros(1, 17, 2, 64, dtype=BF16, device="cuda"))):
        with pytest.raises(ValueError):
            avq.cache_attention_fwd(**(base | kw))
    for kw in (dict(scale=0.0), dict(workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(avq.AvqError):
            avq.cache_attention_fwd(**(base | kw))


def test_query_strides():
    """Queries as a slice of a fused projection; tokens must be evenly spaced."""
    t = Setup([60, 33, 5], [0, 0, 0], 2, 2, 64, BF16, True, 16)
    cache, table, n = fill(t)
    for n_q in (1, 3):
        fused = torch.randn(3, n_q, 6, 64, generator=torch.Generator().manual_seed(3)).to(BF16).cuda()
        Q = fused[:, :, :4]
        assert not Q.is_contiguous()
        Y = avq.cache_attention_fwd(Q, cache, table, n, 16, 0.3, fp4=True)
        assert torch.equal(Y, avq.cache_attention_fwd(Q.contiguous(), cache, table, n, 16, 0.3, fp4=True))
    with pytest.raises(ValueError):
        avq.cache_attention_fwd(fused[:, :2, :4], cache, table, n, 16, 0.3, fp4=True)
    with pytest.raises(ValueError):
        avq.cache_attention_fwd(fused.transpose(1, 2)[:, :4], cache, table, n, 16, 0.3, fp4=True)


@pytest.mark.parametrize("fp4", [False, True])
def test_equal_logits_of_any_size(fp4):
    for n, size in ((70, 2.0 ** 50), (700, -(2.0 ** 50))):
        t = Setup([n], [0], 1, 1, 64, F32, fp4, 16)
        t.K = torch.full((n, 1, 64), size)
        cache, table, lens = fill(t)
        Q = torch.full((1, 1, 1, 64), 2.0 ** 56).cuda()
        Y = avq.cache_attention_fwd(Q, cache, table, lens, 16, 1.0, fp4=fp4).cpu()
        v = read_cache(t.cache, t.table, 0, n, F32, fp4, 16, 64)[1][0]
        assert ((Y[0, 0, 0].double() - v.mean(0)).abs() <= n * 2.0 ** -24 * 2 * v.abs().mean(0)).all()


def test_the_most_tokens_of_one_call():
    """2^24 packed tokens: their launch has more than one row of workgroups."""
    lens, T, ps = [(1 << 24) - 100, 60, 40], 1 << 24, 64
    K = torch.zeros(T, 1, 64, dtype=BF16, device="cuda")
    V = torch.zeros(T, 1, 64, dtype=BF16, device="cuda")
    K[-1000:], V[-1000:] = torch.randn(2, 1000, 1, 64, device="cuda").to(BF16)
    c = torch.tensor([0, lens[0], T - 40, T], dtype=torch.int32, device="cuda")
    start = torch.zeros(3, dtype=torch.int32, device="cuda")
    table = torch.full((3, T // ps), -1, dtype=torch.int32)
    first = (lens[0] - 500) // ps  # the long sequence: its last pages
    table[0, first:(lens[0] + ps - 1) // ps] = torch.arange((lens[0] + ps - 1) // ps - first)
    table[1, 0], table[2, 0] = 20, 21
    table = table.cuda()
    cache = torch.zeros(22, 1, avq.cache_page_bytes(BF16, ps, 64), dtype=torch.uint8, device="cuda")
    avq.cache_append(K, V, cache, table, start, ps, cu=c)
    K2, V2 = avq.cache_gather(cache, table, start, c, T, ps, BF16, 64)
    n = lens[0] - first * ps + 100  # positions before them have no page and read as 0
    for a, b in ((K, K2), (V, V2)):
        assert torch.equal(a[-n:], b[-n:])
        assert not b[:-n].any()


@pytest.mark.parametrize("dtype,fp4", [(BF16, True), (BF16, False), (F32, True)])
def test_shared_pages(dtype, fp4):
    """Sequences that read the same pages (a common prompt), and one that names
    a page twice."""
    lens, ps = [200, 230, 96], 32
    t = Setup(lens, [0] * 3, 2, 2, 64, dtype, fp4, ps)
    cache, _, n = fill(t)
    t.table[1, :5] = t.table[0, :5]
    t.table[2, 2] = t.table[2, 0]
    Q = torch.randn(3, 2, 4, 64, generator=torch.Generator().manual_seed(3)).to(dtype)
    table = t.table.cuda()
    Y, lse = avq.cache_attention_fwd(Q.cuda(), cache, table, n, ps, 0.3, fp4=fp4, with_lse=True)
    check_cached(Y.cpu(), lse.cpu(), Q, t, lens, 0.3)
    K, V = avq.cache_gather(cache, table, torch.zeros_like(n), cu(lens).cuda(), sum(lens), ps, dtype,
                            64, fp4=fp4)
    assert torch.equal(K[:160], K[200:360]) and torch.equal(V[:160], V[200:360])
    assert torch.equal(K[430:462], K[494:526]) and torch.equal(V[430:462], V[494:526])


@pytest.mark.parametrize("Hq,n_q,fp4", [(1024, 16, True), (1024, 1, False), (31, 11, True)])
def test_many_rows_per_head(Hq, n_q, fp4):
    lens = [700, 20]
    t = Setup(lens, [0, 0], 1, 1, 128, BF16, fp4, 64)
    cache, table, n = fill(t)
    Q = torch.randn(2, n_q, Hq, 128, generator=torch.Generator().manual_seed(3)).to(BF16)
    Y, lse = avq.cache_attention_fwd(Q.cuda(), cache, table, n, 64, 0.1, fp4=fp4, with_lse=True)
    Y, lse = Y.cpu(), lse.cpu()
    for s in range(2):
        K, V, _ = read_cache(t.cache, t.table, s, lens[s], BF16, fp4, 64, 128)
        seen = (torch.arange(n_q) + lens[s] - n_q + 1).clamp(0, lens[s]).repeat_interleave(Hq)
        check_attention(Y[s].reshape(-1, 128), lse[s].reshape(-1), Q[s].reshape(-1, 128), K[0], V[0],
                        0.1, seen)


def test_two_streams_at_once():
    """Calls on two streams, each with its own workspace, over one cache."""
    lens, ps = [3000, 500, 64], 64
    t = Setup(lens, [0] * 3, 2, 2, 128, BF16, True, ps)
    cache, table, n = fill(t)
    g = torch.Generator().manual_seed(3)
    Q = [torch.randn(3, 4, 8, 128, generator=g).to(BF16).cuda() for _ in range(2)]
    P = [torch.randn(300, 8, 128, generator=g).to(BF16).cuda() for _ in range(2)]
    c, ck = cu([100, 150, 50]).cuda(), cu(lens).cuda()

    def work(i):
        y = avq.cache_attention_fwd(Q[i], cache, table, n, ps, 0.1, fp4=True)
        k, v = avq.cache_gather(cache, table, torch.zeros_like(n), ck, sum(lens), ps, BF16, 128,
                                fp4=True)
        return y, k, v, avq.prompt_attention_fwd(P[i], k, v, c, ck, 0.1)

    want = [work(i) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(10):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(work(i))
    torch.cuda.synchronize()
    for i in range(2):
        for r in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(r, want[i]))


def test_undivided_needs_no_workspace():
    """Up to 512 positions of room: no workspace, and the same result with one."""
    lens, ps = [512, 3, 400], 16
    t = Setup(lens, [0] * 3, 2, 2, 64, BF16, True, ps)
    cache, table, n = fill(t)
    assert table.shape[1] * ps == avq.CACHE_UNDIVIDED
    Q = torch.randn(3, 2, 4, 64, generator=torch.Generator().manual_seed(3)).to(BF16).cuda()
    Y = avq.cache_attention_fwd(Q, cache, table, n, ps, 0.3, fp4=True)
    check_cached(Y.cpu(), None, Q.cpu(), t, lens, 0.3)
    ws = torch.zeros(avq.cache_attention_workspace(3, 2, 4, 2, 64), dtype=torch.uint8, device="cuda")
    assert torch.equal(Y, avq.cache_attention_fwd(Q, cache, table, n, ps, 0.3, fp4=True, workspace=ws))
    assert not ws.any()


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_gathered_starts_without_a_place(dtype, fp4):
    """Keys and values of positions that no page can hold (before 0, past the
    table, past 2^31) both read as 0; positions with a page beside them are read."""
    ps, d, lens = 16, 64, [40, 24, 9, 30, 17]
    t = Setup(lens, [0] * 5, 2, 2, d, dtype, fp4, ps)
    t.append()
    top = (1 << 31) - 1
    start = torch.tensor([0, -1, top - 3, -(1 << 31), top - 24], dtype=torch.int32)
    K = torch.full((sum(lens) + 3, 2, d), 5.0, dtype=dtype, device="cuda")
    V = K.clone()
    avq.cache_gather(t.cache.cuda(), t.table.cuda(), start.cuda(), cu(lens).cuda(), len(K), ps, dtype,
                     d, fp4=fp4, K=K, V=V)
    k, v, _ = read_cache(t.cache, t.table, 0, lens[0], dtype, fp4, ps, d)
    for got, x in ((K, k), (V, v)):
        assert torch.equal(got[:40].cpu().double(), x.transpose(0, 1))
        assert (got[40:-3] == 0).all() and (got[-3:] == 5).all()


def test_appended_starts_without_a_place():
    """Tokens past 2^31 have no page, but their queries and keys are given out
    like those of any position without one; a negative start takes no part."""
    top, d = (1 << 31) - 1, 64
    t = Setup([20, 20, 5], [0, 0, 0], 2, 2, d, BF16, True, 16)
    t.start = torch.tensor([top - 7, -1, 0], dtype=torch.int32)
    Qo, Ko = (torch.full((45, 2, d), 3.0, dtype=BF16, device="cuda") for _ in range(2))
    t.append(Q_out=Qo, K_out=Ko)
    for got, x in ((Qo.cpu(), t.Q), (Ko.cpu(), t.K)):
        assert torch.equal(got[:20], x[:20]) and torch.equal(got[40:], x[40:])
        assert (got[20:40] == 3).all()
    changed = (t.cache != t.before).flatten(1).any(1).nonzero().flatten().tolist()
    assert set(changed) <= {int(t.table[2, 0])}


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_the_largest_values_in_4_bits_are_read_as_finite(dtype):
    """Magnitudes above 3.5 2^126 take code 4 at a scale of 2^126, which is
    2^128: read as the largest finite value."""
    d, top = 64, torch.finfo(dtype).max
    x = torch.zeros(16, 1, d, dtype=dtype)
    x[0], x[1], x[2, 0, 5], x[2, 0, 6] = 3.0e38, -3.0e38, top, -2.0e38
    x[3], x[4, 0, 33] = 2.9e38, 2.0 ** 127
    cache = torch.zeros(1, 1, avq.cache_page_bytes(dtype, 16, d, True), dtype=torch.uint8).cuda()
    table, start = torch.zeros(1, 1, dtype=torch.int32).cuda(), torch.zeros(1, dtype=torch.int32).cuda()
    avq.cache_append(x.cuda(), x.cuda(), cache, table, start, 16, cu=cu([16]).cuda(), fp4=True)
    k64 = read_cache(cache.cpu(), table.cpu(), 0, 16, dtype, True, 16, d)[0].transpose(0, 1)
    assert (k64.abs() == 2.0 ** 128).sum() == 2 * d + 1  # rows 0 and 1, and one of row 2
    for y in avq.cache_gather(cache, table, start, cu([16]).cuda(), 16, 16, dtype, d, fp4=True):
        assert torch.isfinite(y).all()
        assert torch.equal(y.cpu().double(), k64.clamp(-top, top))


@pytest.mark.parametrize("bad", [math.inf, math.nan])
@pytest.mark.parametrize("dtype,fp4", [(BF16, False), (BF16, True), (F32, False), (F32, True)])
def test_bad_values_stay_in_their_sequence(bad, dtype, fp4):
    """Infinities and NaN in one sequence's queries, keys and values, where
    workgroups go from one sequence to the next and leave parts (1248
    units of 128 keys): the others' results keep their bits."""
    lens, ps, Hkv, d = [2900, 300, 1500, 3], 64, 32, 64
    t = Setup(lens, [0] * 4, Hkv, Hkv, d, dtype, fp4, ps)
    assert t.table.shape[1] * ps > avq.CACHE_UNDIVIDED
    cache, table, n = fill(t)
    Q = torch.randn(4, 4, 2 * Hkv, d, generator=torch.Generator().manual_seed(3)).to(dtype).cuda()
    want = avq.cache_attention_fwd(Q, cache, table, n, ps, 0.1, fp4=fp4, with_lse=True)
    t.K[2900:3200] = t.V[2900:3200] = bad
    t.cache = t.before
    cache, table, n = fill(t)
    if fp4:  # in 4 bits the codes hold neither: scales of 2^128, infinite in both types
        for p in t.table[1, :4].tolist():
            cache[p, :, ps * d:] = 0xff
    Q[1] = bad
    got = avq.cache_attention_fwd(Q, cache, table, n, ps, 0.1, fp4=fp4, with_lse=True)
    for a, b in zip(got, want):
        for s in (0, 2, 3):
            assert torch.equal(a[s], b[s]), f"sequence {s}"


@pytest.mark.parametrize("fp4", [False, True])
def test_many_sequences_in_parts(fp4):
    """More sequences than threads of a workgroup (several per thread), among
    them long ones whose keys are divided."""
    S, ps, far = 600, 64, {0: 1500, 255: 700, 256: 2000, 511: 3, 599: 1100}
    lens = [far.get(s, s % 90) for s in range(S)]
    t = Setup(lens, [0] * S, 2, 2, 64, BF16, fp4, ps)
    assert t.table.shape[1] * ps > avq.CACHE_UNDIVIDED
    cache, table, n = fill(t)
    Q = torch.randn(S, 2, 6, 64, generator=torch.Generator().manual_seed(3)).to(BF16)
    Y, lse = avq.cache_attention_fwd(Q.cuda(), cache, table, n, ps, 0.3, fp4=fp4, with_lse=True)
    check_cached(Y.cpu(), lse.cpu(), Q, t, lens, 0.3, rows=set(far) | {1, 2, 90, 254, 257, 598})


@pytest.mark.parametrize("dtype,fp4", [(BF16, False), (BF16, True), (F32, True)])
def test_drafted_tokens_after_a_prompt(dtype, fp4):
    """Drafted tokens as a server tries them: a prompt is appended, then rounds
    of n_q tokens per sequence (append with cu, attention of the rotated
    queries), of which some are kept: the next round's start overwrites the
    rest."""
    S, Hq, Hkv, d, ps, scale, n_q = 3, 4, 2, 64, 16, 0.25, 4
    g = torch.Generator().manual_seed(17)
    done, kept = [600, 14, 0], [[1, 4, 2], [3, 2, 4], [4, 1, 1]]
    table, n_pages = tables([n + 4 * n_q for n in done], ps)
    cache = garbage(n_pages, Hkv, avq.cache_page_bytes(dtype, ps, d, fp4)).cuda()
    cos, sin = (x.cuda() for x in angles(700, d))
    table_d = table.cuda()
    K, V = (torch.randn(sum(done), Hkv, d, generator=g).to(dtype).cuda() for _ in range(2))
    avq.cache_append(K, V, cache, table_d, torch.zeros(S, dtype=torch.int32).cuda(), ps,
                     cu=cu(done).cuda(), cos=cos, sin=sin, fp4=fp4)
    for keep in kept:
        Q, K, V = (torch.randn(S * n_q, h, d, generator=g).to(dtype).cuda() for h in (Hq, Hkv, Hkv))
        start = torch.tensor(done, dtype=torch.int32).cuda()
        Qr, _ = avq.cache_append(K, V, cache, table_d, start, ps, cu=cu([n_q] * S).cuda(), Q=Q,
                                 cos=cos, sin=sin, fp4=fp4)
        pos = torch.cat([torch.arange(o, o + n_q) for o in done])
        want, err = rotate64(Q.cpu(), pos, cos.cpu(), sin.cpu(), False)
        assert ((Qr.cpu().double() - want).abs() <= HALF_STEP[dtype] * want.abs() + 1.01 * err).all()
        lens = [n + n_q for n in done]
        Y, lse = avq.cache_attention_fwd(Qr.view(S, n_q, Hq, d), cache, table_d, start + n_q, ps, scale,
                                         fp4=fp4, with_lse=True)
        rows = [read_cache(cache.cpu(), table, s, lens[s], dtype, fp4, ps, d) for s in range(S)]
        check_prompt(Y.flatten(0, 1).cpu(), lse.flatten(0, 1).cpu(), Qr.cpu(),
                     torch.cat([r[0].transpose(0, 1) for r in rows]),
                     torch.cat([r[1].transpose(0, 1) for r in rows]), [n_q] * S, lens, scale, True)
        done = [a + b for a, b in zip(done, keep)]
