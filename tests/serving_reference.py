"""Plain 64-bit implementations of the serving operators (CPU), and the error
bounds the kernels are held to.

Bounds, per element of Y = sum p v / sum p with a = sum p |v| / sum p and
A = the largest scale sum |q_i k_i| of the row:
  * an fp32 logit is off by at most (d + 8) 2^-24 A (d products, the scale, the
    maximum taken off), as is, relatively, its weight; both sums run over at
    most n + d terms, and their quotient and the exponential add a few
    roundings: delta = 2 ((d + 8) A + n + 64) 2^-24, on a;
  * bf16: a weight and the result are rounded once each, by at most 2^-8
    relatively: 2^-8 a + 2^-8 |Y|.
The logarithm of the sum is off by delta and its own rounding.
"""
import math

import torch

HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
E2M1 = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)


def attention64(q, k, v, scale, seen):
    """One head. q [Lq, d], k, v [Lk, d], seen [Lq] (keys each query sees, the
    first ones). Returns Y, lse, and the bounds on both."""
    q, k, v = q.double(), k.double(), v.double()
    Lq, d = q.shape
    Lk = k.shape[0]
    y, a = torch.zeros(Lq, v.shape[1]).double(), torch.zeros(Lq, v.shape[1]).double()
    lse = torch.full((Lq,), -math.inf).double()
    delta = torch.zeros(Lq).double()
    if Lk:
        see = torch.arange(Lk) < seen[:, None]
        x = (scale * q @ k.T).masked_fill(~see, -math.inf)
        rows = seen > 0
        lse[rows] = torch.logsumexp(x[rows], 1)
        w = torch.where(see, torch.exp(x - torch.where(rows, lse, 0.0)[:, None]), 0.0)
        vz = torch.nan_to_num(v)
        y, a = w @ vz, w @ vz.abs()
        big = (scale * q.abs() @ k.abs().T).masked_fill(~see, 0.0).amax(1)
        delta = 2 * ((d + 8) * big + Lk + 64) * 2.0 ** -24
    return y, lse, a * delta[:, None], a, delta + 4 * HALF_STEP[torch.float32] * lse.abs().nan_to_num(0, 0, 0)


def check_attention(Y, lse, q, k, v, scale, seen, what=""):
    """One head's output against the reference, within the bounds."""
    y, l, tol, a, ltol = attention64(q, k, v, scale, seen)
    half = HALF_STEP[Y.dtype]
    tol = tol + half * y.abs() + (half * a if Y.dtype == torch.bfloat16 else 0) + 1e-30
    err = (Y.double() - y).abs()
    assert torch.isfinite(Y).all(), f"{what}: not finite"
    assert (err <= tol).all(), f"{what}: off by {(err / tol).max():.3g} times the bound"
    if lse is not None:
        empty = l == -math.inf
        assert torch.equal(lse.double() == -math.inf, empty), f"{what}: rows without keys"
        e = (lse.double() - l).abs()[~empty]
        assert (e <= ltol[~empty]).all(), f"{what}: lse off by {(e / ltol[~empty]).max():.3g} bounds"


def seen_of(Lq, Lk, causal):
    i = torch.arange(Lq)
    return (i + Lk - Lq + 1).clamp(0, Lk) if causal else torch.full((Lq,), Lk)


def check_prompt(Y, lse, Q, K, V, lens_q, lens_k, scale, causal):
    G = Q.shape[1] // K.shape[1]
    a = b = 0
    for s, (Lq, Lk) in enumerate(zip(lens_q, lens_k)):
        for h in range(Q.shape[1]):
            check_attention(Y[a:a + Lq, h], None if lse is None else lse[a:a + Lq, h],
                            Q[a:a + Lq, h], K[b:b + Lk, h // G], V[b:b + Lk, h // G], scale,
                            seen_of(Lq, Lk, causal), f"sequence {s} head {h}")
        a, b = a + Lq, b + Lk


def rotate64(x, pos, cos, sin, interleaved):
    """x [n, H, d] rotated to positions pos, and a bound on the fp32 error."""
    x = x.double().clone()
    err = torch.zeros_like(x)
    if cos is None:
        return x, err
    half = cos.shape[1]
    c, s = cos.double()[pos][:, None], sin.double()[pos][:, None]
    i = torch.arange(half)
    ia, ib = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    a, b = x[..., ia], x[..., ib]
    x[..., ia], x[..., ib] = a * c - b * s, b * c + a * s
    # two products and a sum, each rounded
    err[..., ia] = 3 * 2.0 ** -24 * ((a * c).abs() + (b * s).abs())
    err[..., ib] = 3 * 2.0 ** -24 * ((b * c).abs() + (a * s).abs())
    return x, err


def views(cache, dtype, fp4, ps, d):
    """The arrays of a cache's pages (as include/avq.h lays them out)."""
    n, H, _ = cache.shape
    if not fp4:
        p = cache.view(dtype)
        return {"K": p[..., :ps * d].view(n, H, ps, d),
                "V": p[..., ps * d:].view(n, H, ps // 8, d, 8)}
    a, b = ps * d // 2, ps * d // 32
    return {"Kc": cache[..., :a].view(n, H, ps, d // 2),
            "Vc": cache[..., a:2 * a].view(n, H, ps // 8, d // 2, 8),
            "Ks": cache[..., 2 * a:2 * a + b].view(n, H, ps, d // 32),
            "Vs": cache[..., 2 * a + b:].view(n, H, ps // 8, d // 32, 8)}


def decode(code, scale):
    """codes [..., d/2], scales [..., d/32] to values, and the scales per value."""
    c = torch.stack((code % 16, code // 16), -1).flatten(-2).long()
    val = E2M1[c % 8] * torch.where(c >= 8, -1.0, 1.0).double()
    unit = torch.exp2(scale.double() - 127).repeat_interleave(32, -1)
    return val * unit, unit


def read_cache(cache, table, s, n, dtype, fp4, ps, d):
    """The first n cached positions of sequence s: K, V [Hkv, n, d] in 64 bits
    (positions without a page: 0), and which positions have a page."""
    w = views(cache, dtype, fp4, ps, d)
    H = cache.shape[1]
    K, V = torch.zeros(H, n, d).double(), torch.zeros(H, n, d).double()
    ok = torch.zeros(n, dtype=torch.bool)
    for j in range(n):
        if j // ps >= table.shape[1]:
            continue
        page, slot = int(table[s, j // ps]), j % ps
        if not 0 <= page < cache.shape[0]:
            continue
        ok[j] = True
        if fp4:
            K[:, j], _ = decode(w["Kc"][page, :, slot], w["Ks"][page, :, slot])
            V[:, j], _ = decode(w["Vc"][page, :, slot // 8, :, slot % 8],
                                w["Vs"][page, :, slot // 8, :, slot % 8])
        else:
            K[:, j], V[:, j] = w["K"][page, :, slot], w["V"][page, :, slot // 8, :, slot % 8]
    return K, V, ok


def check_fp4(dec, unit, x, err):
    """Decoded values against x (known to within err): the scale is the
    smallest power of two with no magnitude above 6, each value the nearest."""
    top = x.abs().unflatten(-1, (-1, 32)).amax(-1).repeat_interleave(32, -1)
    slack = 1 + 2.0 ** -20
    tiny = 2.0 ** -126
    assert (top <= 6 * unit * slack).all(), "a value above 6"
    assert ((3 * unit <= top * slack) | (unit == tiny)).all(), "the scale is too large"
    r = (x / unit).abs()
    step = torch.where(r < 2, 0.5, torch.where(r < 4, 1.0, 2.0)) * unit
    assert ((dec - x).abs() <= step / 2 * slack + err).all(), "not the nearest value"
