"""Performance cases of rotary positions with several axes, of cross attention
(with its gradient), and of decoding behind shared prefixes.

A case is one pass through the entry points of ``paper_2607_12789_amd.avq`` on
inputs resident in device memory:

* ``rotate``  ``rotate_axes``: queries and keys of packed tokens rotated by
              their positions on several axes, or gradients rotated back;
* ``cross``   ``cross_attention_fwd``: packed queries read the states of their
              source, some of which a mask may hide;
* ``train``   the same, then ``cross_attention_bwd``: gradients of queries,
              keys and values;
* ``prefix``  ``cache_prefix_attention_fwd``: the newest tokens of every
              sequence over the paged cache, whose groups of sequences share
              their first positions.

The layout of a page (see ``include/avq.h``), per page and key-value head:
native: K [page][d], V [page/8][d][8] in the inputs' type; 4 bits: K codes
[page][d/2], V codes [page/8][d/2][8], K scales [page][d/32], V scales
[page/8][d/32][8], all bytes; a code byte holds dimensions 2i (low) and 2i+1.

With ``own`` the framework's operators run, without it their plain forms in
elementary 32-bit torch operations. ``exact`` is the same pass in 64 bits.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _text(v):
    return ",".join(str(x) for x in v)


def _ints(t):
    return [int(x) for x in t.split(",")] if t else []


def _rotate(name, T, Hq, Hkv, d, dtype, rot, sections, n_pos, *, mixed=False, interleaved=False,
            inverse=False):
    """sections: pairs of each axis, one after the other, or with mixed dealt
    out in turn; n_pos: rows of the angle tables."""
    return {"name": name, "path": "rotate", "T": T, "Hq": Hq, "Hkv": Hkv, "d": d, "dtype": dtype,
            "rot": rot, "sections": sections, "n_pos": n_pos, "mixed": mixed,
            "interleaved": interleaved, "inverse": inverse}


def _cross(name, path, lq, lk, Hq, Hkv, d, dtype, *, mask="", hide=0.0):
    """lq, lk: queries and states of each source. mask: "", "tail" (the last
    part of every source's states is padding) or "drop" (states left out at
    random); hide: which part of them."""
    return {"name": name, "path": path, "lq": lq, "lk": lk, "Hq": Hq, "Hkv": Hkv, "d": d,
            "dtype": dtype, "mask": mask, "hide": hide}


def _prefix(name, members, shared, rest, Hq, Hkv, d, dtype, *, n_q=1, fp4=False, page=64):
    """members: sequences of each group; shared: positions they have in
    common; rest: each sequence's positions behind them, its n_q newest ones
    among them (-1: an idle entry of the batch)."""
    return {"name": name, "path": "prefix", "members": members, "shared": shared, "rest": rest,
            "Hq": Hq, "Hkv": Hkv, "d": d, "dtype": dtype, "n_q": n_q, "fp4": fp4, "page": page}


def listed():
    return [
        # the next tokens of a few videos' captions: launch latency
        _rotate("rotate-8", 8, 12, 12, 64, "bf16", 64, "16,8,8", 1024),
        # an fp32 encoder of 28x28 image patches, the gradients' way back
        _rotate("rotate-patches-back", 8 * 784, 12, 12, 64, "f32", 64, "16,16", 28, inverse=True),
        # a clip of 16 frames of 32x32 patches, grouped heads
        _rotate("rotate-clip", 16384, 32, 8, 128, "bf16", 128, "16,24,24", 64),
        # an odd number of tokens, half of each head rotated, axes in turn, adjacent pairs
        _rotate("rotate-mixed", 20003, 14, 2, 128, "bf16", 64, "12,10,10", 2048, mixed=True,
                interleaved=True),
        # five answers about each of eight images: a decoding step
        _cross("cross-step", "cross", _text([5] * 8), _text([784] * 8), 12, 12, 64, "bf16"),
        # one token for each of 32 documents of all lengths, padding behind them
        _cross("cross-documents", "cross", _text([1] * 32),
               _text([(i * 2741) % 8000 + 190 for i in range(32)]), 32, 8, 128, "bf16", mask="tail",
               hide=0.1),
        # fp32 training, ragged, a source without states and one without queries
        _cross("train-f32-ragged", "train", "300,1,64,0,517", "90,700,0,33,1025", 8, 2, 64, "f32",
               mask="drop", hide=0.25),
        # image tokens that read short texts: few states, many rows
        _cross("train-texts", "train", _text([4096] * 4), "77,31,128,77", 12, 12, 64, "bf16",
               mask="tail", hide=0.3),
        # as many queries as states, grouped heads, the largest products
        _cross("train-4k", "train", "4096,4096", "4096,4000", 16, 4, 128, "bf16"),
        # the first tokens of four short answers to one question: launch latency
        _prefix("prefix-4-short", "4", "300", "1,9,30,2", 12, 12, 64, "bf16", page=16),
        # 64 answers to one long question
        _prefix("prefix-64", "64", "16000", _text([(i * 331) % 1400 + 40 for i in range(64)]), 16, 4,
                128, "bf16"),
        # questions about several documents, two drafted tokens, 4-bit cache, an idle entry
        _prefix("prefix-groups-fp4", "24,1,9,40,6", "8000,3001,12345,600,0",
                _text([(i * 577) % 900 + 2 for i in range(79)] + [-1]), 32, 8, 128, "bf16", n_q=2,
                fp4=True),
    ]


def _lens(c):
    """(queries, states) of each source."""
    return list(zip(_ints(c["lq"]), _ints(c["lk"])))


def _sequences(c):
    """(group, cached length) of each sequence."""
    out, rest = [], iter(_ints(c["rest"]))
    for g, (m, n) in enumerate(zip(_ints(c["members"]), _ints(c["shared"]))):
        for _ in range(m):
            r = next(rest)
            out.append((g, 0 if r < 0 else n + r))
    return out


def work(c):
    e = 4 if c["dtype"] == "f32" else 2
    Hq, Hkv, d = c["Hq"], c["Hkv"], c["d"]
    if c["path"] == "rotate":
        table = 4 * c["rot"] * c["n_pos"]
        axes = len(_ints(c["sections"]))
        return {"bytes": 2 * c["T"] * (Hq + Hkv) * d * e + 4 * c["T"] * axes + table,
                "flops": 3 * c["T"] * (Hq + Hkv) * c["rot"]}
    if c["path"] == "prefix":
        row = d // 2 + d // 32 if c["fp4"] else d * e
        seqs = _sequences(c)
        shared, n_q = _ints(c["shared"]), c["n_q"]
        own_rows = sum(max(0, n - shared[g]) for g, n in seqs)
        once = sum(shared[g] for g in {g for g, n in seqs if n})
        seen = sum(n * n_q - n_q * (n_q - 1) // 2 for _, n in seqs if n)
        return {"bytes": 2 * len(seqs) * n_q * Hq * d * e + 2 * (own_rows + once) * Hkv * row,
                "flops": 4 * d * Hq * seen}
    lens = _lens(c)
    Tq, Tk = sum(a for a, _ in lens), sum(b for _, b in lens)
    keep = 1 - c["hide"] if c["mask"] else 1.0
    pairs = Hq * sum(a * max(1, int(b * keep)) for a, b in lens)
    q, kv = Tq * Hq * d * e, Tk * Hkv * d * e
    mask = Tk if c["mask"] else 0
    if c["path"] == "cross":
        return {"bytes": 2 * q + 2 * kv + mask, "flops": 4 * d * pairs}
    return {"bytes": 6 * q + 6 * kv + mask, "flops": 14 * d * pairs}


_MOST = {"bytes": 1.0e9, "flops": 9e11}


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        path = rng.choice(["rotate"] * 2 + ["cross"] * 2 + ["train"] * 3 + ["prefix"] * 4)
        dtype = "f32" if rng.random() < 0.25 else "bf16"
        d = rng.choice([64, 128])
        Hkv = rng.choice([1, 2, 4, 6, 8])
        Hq = Hkv * rng.choice([1, 1, 2, 3, 4, 7, 8])
        if path == "rotate":
            rot = rng.choice([16, 32, d // 2, d, d])
            axes = rng.randint(1, 4)
            cuts = sorted(rng.randint(0, rot // 2) for _ in range(axes - 1))
            sections = [b - a for a, b in zip([0] + cuts, cuts + [rot // 2])]
            c = _rotate("", log_int(1, 40000), Hq, Hkv, d, dtype, rot, _text(sections),
                        log_int(4, 8192), mixed=rng.random() < 0.3,
                        interleaved=rng.random() < 0.3, inverse=rng.random() < 0.5)
        elif path in ("cross", "train"):
            S = log_int(1, 32)
            few = path == "cross" and rng.random() < 0.6
            top_q, top_k = log_int(1, 16 if few else 6000), log_int(16, 8192)
            lq = [rng.choice([top_q, top_q, rng.randint(0, top_q)]) for _ in range(S)]
            lk = [rng.choice([top_k, rng.randint(0, top_k), log_int(1, top_k)]) for _ in range(S)]
            mask = rng.choice(["", "tail", "drop"])
            c = _cross("", path, _text(lq), _text(lk), Hq, Hkv, d, dtype, mask=mask,
                       hide=round(rng.uniform(0.05, 0.6), 2) if mask else 0.0)
            if sum(lq) == 0 or sum(lk) == 0 or S * Hq * max(lq) * max(lk) > 6e8:
                continue  # the plain form's logits
        else:
            groups, n_q = log_int(1, 8), rng.choice([1, 1, 1, 2, 4, 5])
            members = [log_int(1, 64) for _ in range(groups)]
            shared = [rng.choice([0, log_int(16, 32768), log_int(256, 32768)]) for _ in range(groups)]
            top = log_int(8, 2000)
            rest = [-1 if rng.random() < 0.05 else n_q + rng.choice([0, rng.randint(0, top)])
                    for _ in range(sum(members))]
            c = _prefix("", _text(members), _text(shared), _text(rest), Hq, Hkv, d, dtype, n_q=n_q,
                        fp4=rng.random() < 0.5, page=rng.choice([16, 32, 64, 64, 128, 256]))
            if max(rest) < 0:
                continue
            if max(members) * n_q * Hq * (max(shared) + max(rest)) > 6e8:
                continue
        del c["name"]
        w = work(c)
        cost = w["flops"] * (10 if dtype == "f32" else 1)
        if w["bytes"] <= _MOST["bytes"] and cost <= _MOST["flops"]:
            return c


# ---- inputs -----------------------------------------------------------------

def _axis(c):
    """The axis of each pair."""
    left = _ints(c["sections"])
    if not c["mixed"]:
        return tuple(a for a, n in enumerate(left) for _ in range(n))
    out = []
    while len(out) < c["rot"] // 2:
        for a in range(len(left)):
            if left[a]:
                out.append(a)
                left[a] -= 1
    return tuple(out)


def _views(s):
    """The arrays of the cache's pages: K, V (native), or K codes, V codes, K
    scales, V scales (4 bits)."""
    c, pool = s["case"], s["cache"]
    n, H, ps, d = pool.shape[0], c["Hkv"], c["page"], c["d"]
    if not c["fp4"]:
        p = pool.view(DTYPES[c["dtype"]])
        return p[..., :ps * d].view(n, H, ps, d), p[..., ps * d:].view(n, H, ps // 8, d, 8)
    a, b = ps * d // 2, ps * d // 32
    return (pool[..., :a].view(n, H, ps, d // 2), pool[..., a:2 * a].view(n, H, ps // 8, d // 2, 8),
            pool[..., 2 * a:2 * a + b].view(n, H, ps, d // 32),
            pool[..., 2 * a + b:].view(n, H, ps // 8, d // 32, 8))


def _to_fp4(x):
    """fp32 [..., d] to codes [..., d/2] and scales [..., d/32] (bytes): the
    smallest power of two with no value above 6, ties to the even code."""
    x = x.unflatten(-1, (-1, 32))
    m, ex = torch.frexp(x.abs().amax(-1))
    e = ex - 3 + (m > 0.75)
    e = torch.where(m == 0, -126, e).clamp(-126, 127)
    y = torch.ldexp(x, -e[..., None])
    a = y.abs()
    code = ((a > 0.25).int() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5)
            + (a > 5) + 8 * (y < 0))
    code = code.flatten(-2)
    return (code[..., 0::2] + 16 * code[..., 1::2]).to(torch.uint8), (e + 127).to(torch.uint8)


def _cu(lens):
    return torch.tensor([0] + lens, dtype=torch.int64).cumsum(0).to(torch.int32).cuda()


def prepare(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt, Hq, Hkv, d = DTYPES[c["dtype"]], c["Hq"], c["Hkv"], c["d"]

    def randn(*shape):
        return torch.randn(*shape, device="cuda", generator=g)

    s = {"case": c}
    # keys with a few strong dimensions; logits of a few units
    strong = 1 + 3 * (torch.rand(Hkv, d, device="cuda", generator=g) < 0.03)
    if c["path"] == "rotate":
        T, half, axis = c["T"], c["rot"] // 2, _axis(c)
        s["Q"], s["K"] = (2 * randn(T, Hq, d)).to(dt), (strong * randn(T, Hkv, d)).to(dt)
        s["pos"] = torch.randint(0, c["n_pos"], (T, len(_ints(c["sections"]))), device="cuda",
                                 generator=g, dtype=torch.int32)
        freq = 10000.0 ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)
        angle = torch.arange(c["n_pos"], dtype=torch.float64, device="cuda")[:, None] * freq
        s["cos"], s["sin"], s["axis"] = angle.cos().float(), angle.sin().float(), axis
        s["of_pair"] = torch.tensor(axis, dtype=torch.int64, device="cuda")
        return s
    s["scale"] = 1 / math.sqrt(d)
    if c["path"] != "prefix":
        lens = _lens(c)
        lq, lk = [a for a, _ in lens], [b for _, b in lens]
        s["Q"] = (2 * randn(sum(lq), Hq, d)).to(dt)
        s["K"], s["V"] = (strong * randn(sum(lk), Hkv, d)).to(dt), randn(sum(lk), Hkv, d).to(dt)
        if c["path"] == "train":
            s["dY"] = randn(sum(lq), Hq, d).to(dt)
        s["cu_q"], s["cu_k"], s["Lq"], s["Lk"] = _cu(lq), _cu(lk), max(lq), max(lk)
        s["mask"] = None
        if c["mask"] == "tail":
            s["mask"] = torch.cat([torch.arange(n, device="cuda") < n - int(n * c["hide"])
                                   for n in lk])
        elif c["mask"] == "drop":
            s["mask"] = torch.rand(sum(lk), device="cuda", generator=g) >= c["hide"]
        return s
    # the cache: pages in random order; a group's sequences name the same pages
    # for the whole ones of their shared positions, the one that these end in is
    # each sequence's own copy; what lies behind a length is left from earlier use
    ps, n_q, seqs, shared = c["page"], c["n_q"], _sequences(c), _ints(c["shared"])
    S = len(seqs)
    n_pages = 3 + sum(n // ps for n in shared) + sum(
        max(0, -(-n // ps) - shared[g] // ps) for g, n in seqs)
    order = iter(torch.randperm(n_pages, generator=g, device="cuda").tolist())
    common = [[next(order) for _ in range(n // ps)] for n in shared]
    rows, copies, first = [], [], {}
    for i, (gr, n) in enumerate(seqs):
        row = (common[gr] + [next(order) for _ in range(-(-n // ps) - shared[gr] // ps)]) if n else []
        if n and shared[gr] % ps:
            here = row[shared[gr] // ps]
            copies.append((first.setdefault(gr, here), here, shared[gr] % ps))
        rows.append(row)
    table = torch.zeros(S, max(1, max(map(len, rows))), dtype=torch.int32)
    for i, row in enumerate(rows):
        table[i, :len(row)] = torch.tensor(row, dtype=torch.int32)
    s["table"] = table.cuda()
    row = d // 2 + d // 32 if c["fp4"] else d * dt.itemsize
    s["cache"] = torch.empty(n_pages, Hkv, 2 * ps * row, dtype=torch.uint8, device="cuda")
    views = _views(s)
    step = max(1, (1 << 27) // (Hkv * ps * d))
    for a in range(0, n_pages, step):
        b = min(n_pages, a + step)
        k, v = strong[None, :, None] * randn(b - a, Hkv, ps, d), randn(b - a, Hkv, ps, d)
        octets = (lambda x: x.unflatten(2, (ps // 8, 8)).transpose(3, 4))
        if c["fp4"]:
            kc, ks = _to_fp4(k)
            vc, vs = _to_fp4(v)
            for to, x in zip(views, (kc, octets(vc), ks, octets(vs))):
                to[a:b] = x
        else:
            views[0][a:b] = k.to(dt)
            views[1][a:b] = octets(v.to(dt))
    for source, to, n in copies:
        if source == to:
            continue
        slot = torch.arange(n, device="cuda")
        for j, x in enumerate(views):
            if j % 2 == 0:
                x[to, :, :n] = x[source, :, :n]
            else:
                x[to, :, slot // 8, :, slot % 8] = x[source, :, slot // 8, :, slot % 8]
    s["Q"] = (2 * randn(S, n_q, Hq, d)).to(dt)
    s["lens"] = torch.tensor([n for _, n in seqs], dtype=torch.int32, device="cuda")
    s["cu_groups"] = _cu(_ints(c["members"]))
    s["shared"] = torch.tensor(shared, dtype=torch.int32, device="cuda")
    return s


# ---- the plain forms, 32 bits -----------------------------------------------

def _rotate_plain(s):
    c = s["case"]
    half, r = c["rot"] // 2, c["rot"]
    at = s["pos"].long()[:, s["of_pair"]]
    i = torch.arange(half, device=at.device)
    cos, sin = s["cos"][at, i][:, None], s["sin"][at, i][:, None]
    if c["inverse"]:
        sin = -sin
    out = {}
    for name in "QK":
        x = s[name].float()
        if c["interleaved"]:
            a, b = x[..., 0:r:2], x[..., 1:r:2]
            t = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
        else:
            a, b = x[..., :half], x[..., half:r]
            t = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
        out[name] = torch.cat((t, x[..., r:]), -1).to(s[name].dtype)
    return out


def _padded(x, cu, L):
    """Rows of packed x as [S, L, ...] in 32 bits, and which are a source's own."""
    i = torch.arange(L, device=x.device)
    own_row = i < (cu[1:] - cu[:-1])[:, None]
    rows = torch.where(own_row, cu[:-1, None] + i, 0).long()
    return x[rows].float(), own_row, rows


def _per_head(x, Hkv):
    """[S, Lq, Hq, d] as [S, Hkv, G Lq, d]."""
    S, L, Hq, d = x.shape
    return x.unflatten(2, (Hkv, Hq // Hkv)).permute(0, 2, 3, 1, 4).reshape(S, Hkv, -1, d)


def _per_token(x, Hq, L):
    """The other way."""
    S, Hkv, _, d = x.shape
    return x.view(S, Hkv, Hq // Hkv, L, d).permute(0, 3, 1, 2, 4).reshape(S, L, Hq, d)


def _weights(q, k, see, scale):
    """softmax(scale q k^T) over the keys that see leaves, its largest logits
    and its sums; rows without keys are 0."""
    p = torch.matmul(q, k.transpose(-1, -2).contiguous())
    p.mul_(scale).masked_fill_(~see, -math.inf)
    m = p.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    p.sub_(m).exp_()
    z = p.sum(-1, keepdim=True)
    return p, m, z


def _cross_plain(s):
    c = s["case"]
    Hq, Hkv, Lq, dt = c["Hq"], c["Hkv"], s["Lq"], s["Q"].dtype
    q, q_own, _ = _padded(s["Q"], s["cu_q"], Lq)
    k, k_own, k_rows = _padded(s["K"], s["cu_k"], s["Lk"])
    v, _, _ = _padded(s["V"], s["cu_k"], s["Lk"])
    see = k_own if s["mask"] is None else k_own & s["mask"][k_rows]
    q, k, v = _per_head(q, Hkv), k.transpose(1, 2).contiguous(), v.transpose(1, 2).contiguous()
    p, m, z = _weights(q, k, see[:, None, None], s["scale"])
    p.div_(torch.where(z > 0, z, 1.0))
    y = _per_token(torch.matmul(p, v), Hq, Lq)[q_own].to(dt)
    lse = _per_token(m + z.log(), Hq, Lq)[q_own][..., 0]
    out = {"Y": y, "lse": lse}
    if c["path"] == "cross":
        return out
    dy = _per_head(_padded(s["dY"], s["cu_q"], Lq)[0] * q_own[..., None, None], Hkv)
    dv = torch.matmul(p.transpose(-1, -2).contiguous(), dy)
    ds = torch.matmul(dy, v.transpose(-1, -2).contiguous())
    ds.sub_((p * ds).sum(-1, keepdim=True)).mul_(p).mul_(s["scale"])
    out["dQ"] = _per_token(torch.matmul(ds, k), Hq, Lq)[q_own].to(dt)
    dk = torch.matmul(ds.transpose(-1, -2).contiguous(), q)
    out["dK"], out["dV"] = dk.transpose(1, 2)[k_own].to(dt), dv.transpose(1, 2)[k_own].to(dt)
    return out


def _from_fp4(code, scale):
    """codes [..., d/2] and scales [..., d/32] to fp32 [..., d]."""
    lut = torch.tensor(E2M1 + tuple(-x for x in E2M1), device=code.device)
    x = torch.stack((lut[(code & 15).long()], lut[(code >> 4).long()]), -1).flatten(-2)
    return torch.ldexp(x.unflatten(-1, (-1, 32)), scale.int()[..., None] - 127).flatten(-2)


def _read_plain(s, page, slot):
    """The cached rows at (page, slot), fp32 [..., Hkv, d]."""
    views = _views(s)
    if not s["case"]["fp4"]:
        return (views[0][page, :, slot].float(),
                views[1][page, :, slot // 8, :, slot % 8].float())
    kc, vc, ks, vs = views
    return (_from_fp4(kc[page, :, slot], ks[page, :, slot]),
            _from_fp4(vc[page, :, slot // 8, :, slot % 8], vs[page, :, slot // 8, :, slot % 8]))


def _cached_rows(s, table, pos):
    """Keys and values at positions pos of the sequences of table, as
    [sequences, Hkv, positions, d]."""
    ps = s["case"]["page"]
    column = (pos // ps).clamp(max=table.shape[1] - 1)
    page = torch.gather(table.long(), 1, column.expand(table.shape[0], -1))
    k, v = _read_plain(s, page, (pos % ps).expand_as(page))
    return k.transpose(1, 2).contiguous(), v.transpose(1, 2).contiguous()


def _prefix_plain(s):
    """Group by group: the logits against the shared positions once for all
    its sequences, those against their own positions beside them."""
    c = s["case"]
    Hq, Hkv, d, n_q = c["Hq"], c["Hkv"], c["d"], c["n_q"]
    y = torch.zeros(s["Q"].shape, device="cuda")
    lse = torch.full(s["Q"].shape[:-1], -math.inf, device="cuda")
    at, seqs = 0, _sequences(c)
    for m, P in zip(_ints(c["members"]), _ints(c["shared"])):
        live = [i for i in range(at, at + m) if seqs[i][1] > 0]
        at += m
        if not live:
            continue
        G, n = Hq // Hkv, len(live)
        rows = slice(live[0], live[-1] + 1) if live[-1] - live[0] + 1 == n else live
        last = s["lens"][rows][:, None] - n_q + 1 + torch.arange(n_q, device="cuda")
        last = last[:, None, None, :, None]
        q = s["Q"][rows].float().unflatten(2, (Hkv, G)).permute(0, 2, 3, 1, 4).contiguous()
        L = max(seqs[i][1] for i in live) - P
        pos = torch.arange(P, device="cuda")
        k0, v0 = _cached_rows(s, s["table"][live[0]:live[0] + 1], pos)
        k1, v1 = _cached_rows(s, s["table"][rows], P + torch.arange(L, device="cuda"))
        # [Hkv, all rows, d] against the shared keys; [n, Hkv, rows, d] against the others
        x0 = torch.matmul(q.transpose(0, 1).reshape(Hkv, -1, d), k0[0].transpose(-1, -2).contiguous())
        x0 = x0.view(Hkv, n, G, n_q, P).transpose(0, 1)
        x1 = torch.matmul(q.view(n, Hkv, G * n_q, d), k1.transpose(-1, -2).contiguous())
        x = torch.cat((x0, x1.view(n, Hkv, G, n_q, L)), -1).mul_(s["scale"])
        x.masked_fill_(torch.arange(P + L, device="cuda") >= last, -math.inf)
        top = x.amax(-1, keepdim=True)
        top = torch.where(top == -math.inf, 0.0, top)
        x.sub_(top).exp_()
        z = x.sum(-1, keepdim=True)
        p0 = x[..., :P].transpose(0, 1).reshape(Hkv, n * G * n_q, P)
        p1 = x[..., P:].reshape(n, Hkv, G * n_q, L)
        o = torch.matmul(p0, v0[0]).view(Hkv, n, G, n_q, d).transpose(0, 1)
        o = o + torch.matmul(p1, v1).view(n, Hkv, G, n_q, d)
        o = torch.where(z > 0, o / z, 0.0)
        y[rows] = o.permute(0, 3, 1, 2, 4).flatten(2, 3)
        lse[rows] = (top + z.log())[..., 0].permute(0, 3, 1, 2).flatten(2, 3)
    return {"Y": y.to(s["Q"].dtype), "lse": lse}


# ---- the framework's operators ----------------------------------------------

def run(s):
    c = s["case"]
    if not own:
        if c["path"] == "rotate":
            return _rotate_plain(s)
        return _prefix_plain(s) if c["path"] == "prefix" else _cross_plain(s)
    from paper_2607_12789_amd import avq
    if c["path"] == "rotate":
        q, k = avq.rotate_axes(s["Q"], s["K"], s["pos"], s["cos"], s["sin"], s["axis"],
                               interleaved=c["interleaved"], inverse=c["inverse"])
        return {"Q": q, "K": k}
    if c["path"] == "prefix":
        y, lse = avq.cache_prefix_attention_fwd(
            s["Q"], s["cache"], s["table"], s["lens"], s["cu_groups"], s["shared"], c["page"],
            s["scale"], fp4=c["fp4"], with_lse=True)
        return {"Y": y, "lse": lse}
    y, lse = avq.cross_attention_fwd(s["Q"], s["K"], s["V"], s["cu_q"], s["cu_k"], s["scale"],
                                     mask=s["mask"], with_lse=True)
    out = {"Y": y, "lse": lse}
    if c["path"] == "train":
        out["dQ"], out["dK"], out["dV"] = avq.cross_attention_bwd(
            s["dY"], s["Q"], s["K"], s["V"], y, lse, s["cu_q"], s["cu_k"], s["scale"],
            mask=s["mask"])
    return out


# ---- the same pass in 64 bits -----------------------------------------------

def _turned64(x, s):
    """x [T, H, d] as complex numbers times unit ones, pair by pair."""
    c = s["case"]
    r, x = c["rot"], x.double().clone()
    unit = torch.empty(c["T"], 1, r // 2, dtype=torch.complex128, device=x.device)
    for i, a in enumerate(s["axis"]):
        at = s["pos"][:, a].long()
        unit[:, 0, i] = torch.complex(s["cos"][:, i].double()[at], s["sin"][:, i].double()[at])
    if c["inverse"]:
        unit = unit.conj()
    if c["interleaved"]:
        z = torch.view_as_complex(x[..., :r].unflatten(-1, (-1, 2)).contiguous()) * unit
        x[..., :r] = torch.view_as_real(z).flatten(-2)
    else:
        z = torch.complex(x[..., :r // 2].contiguous(), x[..., r // 2:r].contiguous()) * unit
        x[..., :r] = torch.cat((z.real, z.imag), -1)
    return x


def _cross64(s):
    """Head by head of every source."""
    c = s["case"]
    Hq, G = c["Hq"], c["Hq"] // c["Hkv"]
    f = {n: s[n].double() for n in ("Q", "K", "V", "dY") if n in s}
    names = ("Y", "dQ", "dK", "dV") if c["path"] == "train" else ("Y",)
    out = {n: torch.zeros_like(f[{"Y": "Q"}.get(n, n[1:])]) for n in names}
    out["lse"] = torch.full((len(f["Q"]), Hq), -math.inf, dtype=torch.float64, device="cuda")
    a = b = 0
    for lq, lk in _lens(c):
        qi, ki = slice(a, a + lq), torch.arange(b, b + lk, device="cuda")
        a, b = a + lq, b + lk
        if s["mask"] is not None:
            ki = ki[s["mask"][ki]]
        if not lq or not len(ki):
            continue
        for h in range(Hq):
            q, k, v = f["Q"][qi, h], f["K"][ki, h // G], f["V"][ki, h // G]
            x = s["scale"] * (q @ k.T)
            lse = torch.logsumexp(x, 1, keepdim=True)
            w = torch.exp(x - lse)
            out["lse"][qi, h], out["Y"][qi, h] = lse[:, 0], w @ v
            if c["path"] == "train":
                dy = f["dY"][qi, h]
                out["dV"][ki, h // G] += w.T @ dy
                g = dy @ v.T
                g = s["scale"] * w * (g - (w * g).sum(1, keepdim=True))
                out["dQ"][qi, h] = g @ k
                out["dK"][ki, h // G] += g.T @ q
    return out


def _rows64(s, i, n):
    """The first n cached rows of sequence i, as [Hkv, n, d]."""
    c = s["case"]
    ps, d, Hkv = c["page"], c["d"], c["Hkv"]
    pages = s["cache"][s["table"][i, :-(-n // ps)].long()]
    m = pages.shape[0]
    if not c["fp4"]:
        x = pages.view(s["Q"].dtype).double().view(m, Hkv, 2, ps * d)
        k = x[:, :, 0].view(m, Hkv, ps, d)
        v = x[:, :, 1].view(m, Hkv, ps // 8, d, 8).transpose(3, 4).reshape(m, Hkv, ps, d)
    else:
        body = ps * d // 2

        def decode(code, scale):
            lo, hi = code.int() % 16, code.int() // 16
            code = torch.stack((lo, hi), -1).reshape(m, Hkv, ps, d // 32, 32)
            mag = code % 8
            val = torch.where(mag < 2, mag * 0.5, (2 + mag % 2) * torch.exp2((mag // 2 - 2).double()))
            val = torch.where(code >= 8, -val, val)
            return (val * torch.exp2(scale.double() - 127)[..., None]).reshape(m, Hkv, ps, d)

        kc, vc, sc = pages[..., :body], pages[..., body:2 * body], pages[..., 2 * body:]
        ks, vs = sc[..., :ps * d // 32], sc[..., ps * d // 32:]
        k = decode(kc.reshape(m, Hkv, ps, d // 2), ks.reshape(m, Hkv, ps, d // 32))
        v = decode(vc.reshape(m, Hkv, ps // 8, d // 2, 8).transpose(3, 4).reshape(m, Hkv, ps, d // 2),
                   vs.reshape(m, Hkv, ps // 8, d // 32, 8).transpose(3, 4).reshape(
                       m, Hkv, ps, d // 32))
    return (k.transpose(0, 1).reshape(Hkv, m * ps, d)[:, :n],
            v.transpose(0, 1).reshape(Hkv, m * ps, d)[:, :n])


def _prefix64(s):
    """Sequence by sequence, each over all its own positions."""
    c = s["case"]
    Hq, n_q, G = c["Hq"], c["n_q"], c["Hq"] // c["Hkv"]
    y = torch.zeros(s["Q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["Q"].shape[:-1], -math.inf, dtype=torch.float64, device="cuda")
    for i, (_, n) in enumerate(_sequences(c)):
        if n == 0:
            continue
        k, v = _rows64(s, i, n)
        k, v = k.repeat_interleave(G, 0), v.repeat_interleave(G, 0)
        for t in range(n_q):
            e = n - (n_q - 1 - t)
            if e <= 0:
                continue
            x = s["scale"] * (k[:, :e] * s["Q"][i, t].double()[:, None]).sum(-1)
            lse[i, t] = torch.logsumexp(x, 1)
            y[i, t] = (torch.exp(x - lse[i, t][:, None])[..., None] * v[:, :e]).sum(1)
    return {"Y": y, "lse": lse}


def exact(c, seed):
    s = prepare(c, seed)
    if c["path"] == "rotate":
        return {"Q": _turned64(s["Q"], s), "K": _turned64(s["K"], s)}
    return _prefix64(s) if c["path"] == "prefix" else _cross64(s)
