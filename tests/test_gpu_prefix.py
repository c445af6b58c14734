"""cache_prefix_attention_fwd against the 64-bit reference, every sequence over its own
pages (MI355X)."""
import math

import pytest
import torch

from paper_2607_12789_amd import avq
from tests.serving_reference import check_attention, read_cache, views

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


class Setup:
    """groups: (shared positions, lengths of the group's sequences); a sequence's
    shared positions are those it has of them. Slots behind the lengths hold anything.
    The tables have room for `room` positions (nothing is shared up to 512)."""

    def __init__(self, groups, Hq, Hkv, d, dtype, fp4=False, ps=16, n_q=1, seed=0, room=513):
        self.__dict__.update(Hq=Hq, Hkv=Hkv, d=d, dtype=dtype, fp4=fp4, ps=ps, n_q=n_q)
        g = torch.Generator().manual_seed(seed)
        self.lens = [n for _, lens in groups for n in lens]
        self.S = len(self.lens)
        rows, copies, next_page = [], [], 0
        for shared, lens in groups:
            whole = []
            holder, held = None, 0
            for n in lens:
                common = min(n, shared)
                row = []
                for j in range(-(-n // ps)):
                    if (j + 1) * ps <= common:
                        if j == len(whole):
                            whole.append(next_page)
                            next_page += 1
                        row.append(whole[j])
                    else:
                        row.append(next_page)
                        next_page += 1
                rows.append(row)
                # positions of a page that the sequences share only in part
                for j, page in enumerate(row):
                    part = min(min(common, held) - j * ps, ps)
                    if part > 0 and holder is not None and j < len(holder) and page != holder[j]:
                        copies.append((holder[j], page, part))
                if holder is None or len(row) > len(holder):
                    holder, held = row, n
        self.n_pages = next_page + 2
        order = torch.randperm(self.n_pages, generator=g).tolist()
        columns = max(1, -(-room // ps), max(map(len, rows)))
        self.table = torch.full((self.S, columns), -7, dtype=torch.int32)
        for i, row in enumerate(rows):
            self.table[i, :len(row)] = torch.tensor([order[p] for p in row], dtype=torch.int32)
        E = avq.cache_page_bytes(dtype, ps, d, fp4)
        self.cache = torch.randint(0, 256, (self.n_pages, Hkv, E), generator=g, dtype=torch.uint8)
        self.cache.view(-1)[::3] = 0xff  # as bf16 or fp32 also infinities and NaN
        self.names = [("Kc", "Ks"), ("Vc", "Vs")] if fp4 else [("K",), ("V",)]
        w = self.views()
        for row, n in zip(rows, self.lens):
            for j, page in enumerate(row):
                slots = torch.arange(min(n - j * ps, ps))
                for name, x in w.items():
                    at = self.at(x, order[page], slots, name)
                    if name in ("Ks", "Vs"):
                        v = torch.randint(124, 128, at.shape, generator=g, dtype=torch.uint8)
                    elif fp4:
                        v = torch.randint(0, 256, at.shape, generator=g, dtype=torch.uint8)
                    else:
                        v = torch.randn(at.shape, generator=g).to(dtype)
                    self.put(x, order[page], slots, name, v)
        for a, b, n in copies:
            slots = torch.arange(n)
            for name, x in w.items():
                self.put(x, order[b], slots, name, self.at(x, order[a], slots, name))
        self.Q = torch.randn(self.S, n_q, Hq, d, generator=g).to(dtype)
        self.cu = torch.tensor([0] + [len(x) for _, x in groups]).cumsum(0).int()
        self.shared = torch.tensor([n for n, _ in groups], dtype=torch.int32)

    def views(self):
        return views(self.cache, self.dtype, self.fp4, self.ps, self.d)

    @staticmethod
    def at(x, page, slots, name):
        return x[page, :, slots] if name[0] == "K" else x[page, :, slots // 8, :, slots % 8]

    @staticmethod
    def put(x, page, slots, name, v):
        if name[0] == "K":
            x[page, :, slots] = v
        else:
            x[page, :, slots // 8, :, slots % 8] = v

    def run(self, scale=0.2, **kw):
        dev = [x.cuda() for x in (self.Q, self.cache, self.table,
                                  torch.tensor(self.lens, dtype=torch.int32), self.cu, self.shared)]
        Y, lse = avq.cache_prefix_attention_fwd(*dev, self.ps, scale, fp4=self.fp4, with_lse=True,
                                                **kw)
        torch.cuda.synchronize()
        return Y.cpu(), lse.cpu()

    def check(self, Y, lse, scale=0.2, lens=None):
        for s, n in enumerate(lens or self.lens):
            n = min(max(n, 0), self.table.shape[1] * self.ps)
            K, V, ok = read_cache(self.cache, self.table, s, n, self.dtype, self.fp4, self.ps,
                                  self.d)
            for i in range(self.n_q):
                seen = max(0, n - (self.n_q - 1 - i))
                keep = ok.clone()
                keep[seen:] = False
                for h in range(self.Hq):
                    k = h // (self.Hq // self.Hkv)
                    check_attention(Y[s, i, h][None], lse[s, i, h][None], self.Q[s, i, h][None],
                                    K[k, keep], V[k, keep], scale, torch.tensor([int(keep.sum())]),
                                    f"sequence {s} token {i} head {h}")


GROUPS = [
    [(40, [41, 45, 70])],                               # ends inside a page, and an octet
    [(64, [65, 200, 64, 80])],                          # one sequence has nothing else
    [(33, [40, 90]), (0, [7, 30]), (128, [129, 300, 150])],
    [(100, [101]), (50, [60, 61])],                     # one sequence alone shares nothing
    [(3, [4, 5, 9]), (8, [9, 8])],
    [(300, [301, 20, 0, 310])],                         # shorter than the shared positions, idle
    [(300, [0, 310, 320])],                             # the first one is idle
    [(500, [200, 510, 700])],                           # the first one holds only some of them
    [(1000, [1001, 1100, 1300])],                       # divided
]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("groups", GROUPS)
def test_groups(groups, d, fp4, dtype):
    s = Setup(groups, 4, 2, d, dtype, fp4, 16)
    s.check(*s.run())


@pytest.mark.parametrize("fp4", [False, True])
def test_room_for_few_positions(fp4):
    """Up to 512 positions nothing is shared: no workspace, the same bits as without
    groups."""
    s = Setup([(100, [101, 160, 0]), (30, [40, 41])], 4, 2, 64, BF16, fp4, 16, room=512)
    Y, lse = s.run()
    s.check(Y, lse)
    y, l = avq.cache_attention_fwd(*(x.cuda() for x in (s.Q, s.cache, s.table, torch.tensor(
        s.lens, dtype=torch.int32))), 16, 0.2, fp4=fp4, with_lse=True)
    assert torch.equal(y.cpu(), Y) and torch.equal(l.cpu(), lse)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("ps", [16, 32, 64, 256])
def test_pages(ps, fp4, dtype):
    s = Setup([(130, [131, 200, 300]), (257, [260, 259])], 2, 1, 64, dtype, fp4, ps, seed=1)
    s.check(*s.run())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("Hq,Hkv,n_q", [(1, 1, 1), (7, 1, 3), (6, 6, 2), (8, 1, 5), (12, 4, 16),
                                        (32, 1, 4), (16, 2, 3)])
def test_heads_and_drafts(Hq, Hkv, n_q, fp4, dtype):
    """Up to 128 rows a sequence, several row tiles; tokens see up to their own place,
    also where that lies in the shared positions."""
    s = Setup([(90, [91, 95, 140]), (40, [40, 41, 60])], Hq, Hkv, 64, dtype, fp4, 16, n_q, seed=2)
    s.check(*s.run())


@pytest.mark.parametrize("fp4", [False, True])
def test_many_sequences(fp4):
    """More rows than a tile holds, in one group; groups that begin inside a tile."""
    groups = [(70, [71 + i % 5 for i in range(50)]), (33, [34 + i for i in range(9)]),
              (16, [17] * 40)]
    s = Setup(groups, 4, 1, 64, BF16, fp4, 16, seed=3)
    s.check(*s.run())


def test_more_groups_than_fit_in_lds():
    groups = [(20 + i % 3, [24 + i % 7, 25]) for i in range(300)]
    s = Setup(groups, 1, 1, 64, BF16, False, 16, seed=4)
    s.check(*s.run())


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_sequences_of_no_group(dtype):
    """Before the first group, behind the last, and empty groups between them."""
    s = Setup([(40, [41, 50]), (64, [70, 80, 90]), (30, [33, 35])], 2, 1, 64, dtype, False, 16,
              seed=5)
    s.cu = torch.tensor([2, 2, 5, 5, 5], dtype=torch.int32)
    s.shared = torch.tensor([10 ** 9, 64, 77, -4], dtype=torch.int32)
    s.check(*s.run())


def test_bounds_outside_the_batch():
    s = Setup([(40, [41, 50]), (64, [70, 80, 90])], 2, 1, 64, BF16, False, 16, seed=6)
    s.cu = torch.tensor([-3, 2, 1000], dtype=torch.int32)
    s.shared = torch.tensor([40, 64], dtype=torch.int32)
    s.check(*s.run())
    s.shared = torch.tensor([-5, -1], dtype=torch.int32)
    s.check(*s.run())


@pytest.mark.parametrize("fp4", [False, True])
def test_positions_without_a_page(fp4):
    """A shared page that is none takes no part, for any sequence; lengths beyond the
    table are taken as its end, and negative ones as 0."""
    s = Setup([(96, [100, 120, 110])], 4, 2, 64, BF16, fp4, 16, seed=7)
    s.table[:, 1], s.table[:, 4] = 10 ** 6, -1
    s.check(*s.run())
    for longest in (128, 640):  # not shared and shared
        s = Setup([(96, [longest, 120, 110])], 4, 2, 64, BF16, fp4, 16, seed=8, room=0)
        s.lens = [10 ** 9, 120, -5]
        Y, lse = s.run()
        s.check(Y, lse, lens=[longest, 120, 0])


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_large_logits(dtype, fp4):
    """Logits of hundreds: one part outweighs the other."""
    s = Setup([(200, [230, 260, 201])], 4, 2, 128, dtype, fp4, 64, seed=9)
    s.check(*s.run(scale=8.0), scale=8.0)


def test_same_as_without_groups():
    """Against cache_attention_fwd on the same arguments: each within the bounds, and
    for groups of one sequence the same bits."""
    s = Setup([(0, [50, 300, 0, 700])], 4, 2, 64, BF16, False, 16, seed=10)
    lens = torch.tensor(s.lens, dtype=torch.int32).cuda()
    args = [x.cuda() for x in (s.Q, s.cache, s.table)]
    s.cu, s.shared = torch.arange(5).int(), torch.full((4,), 30, dtype=torch.int32)
    Y, lse = s.run()
    y, l = avq.cache_attention_fwd(*args, lens, 16, 0.2, with_lse=True)
    s.check(y.cpu(), l.cpu())
    s.check(Y, lse)


def test_strided_queries_and_untouched_cache():
    s = Setup([(90, [91, 95, 140])], 4, 2, 64, BF16, False, 16, 2, seed=11)
    wide = torch.randn(3, 2, 6, 64).to(BF16).cuda()
    wide[:, :, :4] = s.Q.cuda()
    cache = s.cache.cuda()
    lens = torch.tensor(s.lens, dtype=torch.int32).cuda()
    Y, lse = avq.cache_prefix_attention_fwd(wide[:, :, :4], cache, s.table.cuda(), lens, s.cu.cuda(),
                                            s.shared.cuda(), 16, 0.2, with_lse=True)
    s.check(Y.cpu(), lse.cpu())
    assert torch.equal(cache.cpu(), s.cache)


def test_refusals_on_the_gpu():
    s = Setup([(40, [41, 50])], 2, 1, 64, BF16)
    assert s.table.shape[1] * 16 > 512
    lens = torch.tensor(s.lens, dtype=torch.int32)
    names = ("Q", "cache", "block_table", "lens", "cu_groups", "shared")
    good = dict(zip(names, (x.cuda() for x in (s.Q, s.cache, s.table, lens, s.cu, s.shared))))
    for change in (dict(Q=s.Q.cuda()[0]), dict(lens=lens), dict(shared=s.shared.cuda().long()),
                   dict(cu_groups=s.cu.cuda()[:1]), dict(shared=s.shared.cuda()[None]),
                   dict(Y=torch.empty(1, device="cuda")), dict(lens=lens.cuda()[:1])):
        with pytest.raises(ValueError):
            avq.cache_prefix_attention_fwd(**{**good, **change}, page_size=16, scale=0.2)
    for kw in (dict(workspace=torch.empty(64, dtype=torch.uint8, device="cuda")),
               dict(scale=-1.0)):
        with pytest.raises(avq.AvqError):
            avq.cache_prefix_attention_fwd(**good, page_size=16, **{"scale": 0.2, **kw})


def test_graph():
    """Captured once, replayed while the sequences grow."""
    s = Setup([(300, [340, 600, 350]), (64, [90, 100])], 4, 2, 64, BF16, False, 16, seed=12)
    dev = [x.cuda() for x in (s.Q, s.cache, s.table)]
    lens = torch.tensor([301, 305, 302, 65, 70], dtype=torch.int32, device="cuda")
    groups = [s.cu.cuda(), s.shared.cuda()]
    call = lambda: avq.cache_prefix_attention_fwd(*dev, lens, *groups, 16, 0.2, with_lse=True)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    for n in range(4):
        lens += 5
        graph.replay()
        torch.cuda.synchronize()
        s.check(out[0].cpu(), out[1].cpu(), lens=lens.tolist())
        eager = call()
        assert torch.equal(out[0], eager[0]) and torch.equal(out[1], eager[1])


def test_two_streams():
    sets = [Setup([(300, [340, 600, 350])], 4, 2, 64, BF16, fp4, 16, seed=13) for fp4 in (0, 1)]
    want = [s.run() for s in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    dev = [[x.cuda() for x in (s.Q, s.cache, s.table, torch.tensor(s.lens, dtype=torch.int32), s.cu,
                               s.shared)] for s in sets]
    torch.cuda.synchronize()
    got = [avq.cache_prefix_attention_fwd(*x, 16, 0.2, fp4=s.fp4, with_lse=True, stream=st)
           for s, x, st in zip(sets, dev, streams)]
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a[0], b[0].cpu()) and torch.equal(a[1], b[1].cpu())


@pytest.mark.parametrize("fp4", [False, True])
def test_pages_past_32_bits(fp4):
    """Pages that lie past 2^32 bytes of the pool."""
    s = Setup([(300, [310, 600, 305])], 4, 2, 128, BF16, fp4, 64, seed=14)
    E, n = s.cache.shape[2], s.n_pages
    far = (5 << 30) // (2 * E)
    pool = torch.zeros(far + n, 2, E, dtype=torch.uint8, device="cuda")
    pool[far:] = s.cache.cuda()
    table = torch.where(s.table >= 0, s.table + far, s.table)
    lens = torch.tensor(s.lens, dtype=torch.int32)
    Y, lse = avq.cache_prefix_attention_fwd(
        s.Q.cuda(), pool, *(x.cuda() for x in (table.int(), lens, s.cu, s.shared)), 64, 0.2, fp4=fp4,
        with_lse=True)
    s.check(Y.cpu(), lse.cpu())


def test_bad_queries_stay_in_their_sequence():
    """An infinity or NaN in one sequence's queries leaves the others of its group."""
    s = Setup([(300, [340, 600, 350, 301])], 4, 2, 64, BF16, False, 16, seed=15)
    s.Q[1] = math.inf
    s.Q[2, 0, 1] = math.nan
    Y, lse = s.run()
    for i in (0, 3):
        t = Setup.__new__(Setup)
        t.__dict__.update(s.__dict__)
        t.Q, t.table, t.lens = s.Q[i:i + 1], s.table[i:i + 1], s.lens[i:i + 1]
        t.check(Y[i:i + 1], lse[i:i + 1])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("fp4", [False, True])
def test_bad_values_behind_a_shorter_sequence(fp4, dtype):
    """A value that is not finite, of shared positions behind the end of one sequence,
    is nothing to that one."""
    s = Setup([(300, [310, 100, 640, 150])], 4, 2, 64, dtype, fp4, 16, seed=14)
    page, slot = int(s.table[0, 200 // 16]), torch.tensor([200 % 16])
    assert page == int(s.table[2, 200 // 16])
    x = s.views()["Vs" if fp4 else "V"]
    s.put(x, page, slot, "V", 0xff if fp4 else math.nan)
    Y, lse = s.run()
    assert not Y[[0, 2]].isfinite().any() and lse.isfinite().all()
    for i in (1, 3):
        K, V, ok = read_cache(s.cache, s.table, i, s.lens[i], dtype, fp4, 16, 64)
        for h in range(4):
            check_attention(Y[i, :, h], lse[i, :, h], s.Q[i, :, h], K[h // 2, ok], V[h // 2, ok],
                            0.2, torch.tensor([int(ok.sum())]), f"sequence {i} head {h}")


def test_long_shared_positions_in_many_runs():
    """Every run of several tiles, rows of several tiles, lengths that end anywhere."""
    s = Setup([(2500, [2501, 2530, 2600] * 4), (1900, [1901, 2000])], 8, 1, 64, BF16, False, 64,
              n_q=4, seed=16)
    s.check(*s.run())


def huge(s, page, slot):
    """The key at a place becomes 2^40 in all dimensions."""
    w, slots = s.views(), torch.tensor([slot])
    if s.fp4:
        s.put(w["Kc"], page, slots, "Kc", 0x22)  # 1 and 1
        s.put(w["Ks"], page, slots, "Ks", 127 + 40)
    else:
        s.put(w["K"], page, slots, "K", 2.0 ** 40)


@pytest.mark.parametrize("dtype,d", [(BF16, 64), (BF16, 128), (F32, 64), (F32, 128)])
@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("where", ["shared", "own", "both", "last"])
@pytest.mark.parametrize("groups", [[(600, [640, 700, 612, 330])], [(2, [2, 600, 700, 4])]])
@pytest.mark.parametrize("scale", [0.125, 8.0])
def test_one_huge_key_among_ordinary_ones(scale, groups, where, fp4, d, dtype):
    """Logits of 2^43 and more take the softmax's second form, maximum first, in the
    shared positions, in a sequence's own, or in both, where they weigh the same. Head 0
    sees equal logits, head 1 sees the huge ones, the others with the other sign. Early
    drafts do not see the last position ("last"), and those of a sequence of two positions
    see none."""
    Hq, n_q, ps = 4, 4, 16
    s = Setup(groups, Hq, 1, d, dtype, fp4, ps, n_q, seed=20)
    s.Q = -s.Q.abs()
    s.Q[:, :, 0], s.Q[:, :, 1] = 0, 1
    P = groups[0][0]
    places = {"shared": [1], "own": [595 if P < 500 else 605], "last": [s.lens[1] - 1]}
    places["both"] = places["shared"] + places["own"]
    for at in places[where]:  # as sequence 1 reads it
        huge(s, int(s.table[1, at // ps]), at % ps)
        if at < P and P % ps > at % ps and int(s.table[1, at // ps]) != int(s.table[0, at // ps]):
            for i in range(s.S):  # a copy of the page for each sequence
                if s.lens[i] > at:
                    huge(s, int(s.table[i, at // ps]), at % ps)
    Y, lse = s.run(scale)
    for i, n in enumerate(s.lens):
        K, V, ok = read_cache(s.cache, s.table, i, n, dtype, fp4, ps, d)
        assert ok.all()
        big = K[0, :, 0] == 2.0 ** 40
        for t in range(n_q):
            seen = torch.arange(n) <= n - n_q + t
            here = seen & big
            for h in range(Hq):
                what = f"sequence {i} token {t} head {h}"
                y, l = Y[i, t, h], lse[i, t, h]
                if h != 1 or not here.any():
                    keep = seen if h < 2 else seen & ~big
                    check_attention(y[None], l[None], s.Q[i, t, h][None], K[0, keep], V[0, keep],
                                    scale, torch.tensor([int(keep.sum())]), what)
                    continue
                # the mean of their values, as summed and divided in fp32 and rounded; the
                # maximum is exact, log2(e), its product, ln 2 and theirs are rounded
                v = V[0, here]
                tol = 2.0 ** -8 if dtype == BF16 else 2.0 ** -24
                tol = tol * v.mean(0).abs() + 3 * 2.0 ** -24 * v.abs().sum(0)
                assert ((y.double() - v.mean(0)).abs() <= tol).all(), what
                assert abs(l.item() / (scale * d * 2.0 ** 40) - 1) <= 5 * 2.0 ** -24, what


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("n", [16, 17, 20, 64, 65, 80])
def test_many_groups_in_many_runs(n, fp4):
    """16 groups and more, which are looked at 64 at a time: shared positions of all lengths
    from none to 63 tiles, whose runs are several for some and one for others, also behind
    the 64th group."""
    shared = [(i * 613) % 400 if i % 6 else (i * 977) % 2000 for i in range(n)]
    shared[1], shared[n - 1] = 2000, 1990
    groups = [(m, [m + 1 + i % 9, m + 4]) for i, m in enumerate(shared)]
    s = Setup(groups, 2, 1, 64, BF16, fp4, 64, seed=21)
    Y, lse = s.run()
    few = sorted({0, 1, 2, 5, 6, 12, 15, n // 2, n - 2, n - 1} | set(range(63, n)))
    for g in few:
        t = Setup.__new__(Setup)
        t.__dict__.update(s.__dict__)
        own = slice(2 * g, 2 * g + 2)
        t.Q, t.table, t.lens = s.Q[own], s.table[own], s.lens[own]
        t.check(Y[own], lse[own])
