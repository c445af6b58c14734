"""Plain 64-bit cross attention and its gradients (CPU), and the error bounds the
kernels are held to.

Forward: the bounds of ``tests.serving_reference`` over the states that take part.

Backward, given lse and Y as the forward pass stores them (lse rounded to fp32, Y to
the type, by at most half a step h). With u = 2^-24, A_i the largest scale
sum |q_i k_j| of a row, B_ij = sum_d |dY_id v_jd|, C_i = sum_d |dY_id Y_id|:
  * a logit is off by at most (d + 8) u A_i (d products, the scale and log2(e)),
    lse as stored and times log2(e) by 4 u |lse_i|, their difference and the
    exponential by a few roundings: P_ij is off relatively by at most
    eP_i = ((d + 12) A_i + 4 |lse_i| + 16) u;
  * dP_ij by (d + 1) u B_ij, delta_i by (d + 1) u C_i and, Y being rounded, h C_i;
  * fp32: dS_ij = P_ij (dP_ij - delta_i) by
    eS_ij = P_ij ((eP_i + 3 u) (|dP_ij| + |delta_i|) + (d + 1) u (B_ij + C_i) + h C_i);
  * bf16: delta_i is mended by rest_i = sum_j dS_ij, which is 0 for the exact one. With
    e_ij = eS_ij without h C_i, and n states, rest_i is off by E_i = sum_j e_ij +
    (n + 64) u sum_j |dS_ij|, and so is delta_i. What h C_i was leaves two products of
    it with a rounding to bf16: of the dS it is in and of the P it is taken off with.
    So eS_ij = e_ij + P_ij (E_i + 2 h h C_i). dQ takes rest_i from the dS as rounded
    to bf16: P_ij h sum_j |dS_ij| more;
  * bf16: P and dS are rounded once more before their products: h |P|, h |dS|;
  * a sum of n products is off by (n + 64) u times the sum of their magnitudes, and a
    result by its own rounding.
Products of these errors are covered by a factor 1 + 2^-6 on the whole.
"""
import math

import torch

from tests.serving_reference import HALF_STEP, check_attention

U = 2.0 ** -24


def split(lens):
    ends = torch.tensor([0] + list(lens)).cumsum(0).tolist()
    return list(zip(ends[:-1], ends[1:]))


def forward64(Q, K, V, lens_q, lens_k, scale, mask=None):
    """Y and lse in 64 bits; rows without states are 0 and -inf."""
    Hq, G = Q.shape[1], Q.shape[1] // K.shape[1]
    Y = torch.zeros(Q.shape, dtype=torch.float64)
    lse = torch.full(Q.shape[:2], -math.inf, dtype=torch.float64)
    for (a, b), (c, d) in zip(split(lens_q), split(lens_k)):
        keep = torch.arange(c, d)
        if mask is not None:
            keep = keep[mask[c:d].bool()]
        if not len(keep) or a == b:
            continue
        for h in range(Hq):
            x = scale * Q[a:b, h].double() @ K[keep, h // G].double().T
            lse[a:b, h] = torch.logsumexp(x, 1)
            Y[a:b, h] = torch.exp(x - lse[a:b, h, None]) @ V[keep, h // G].double()
    return Y, lse


def backward64(dY, Q, K, V, lens_q, lens_k, scale, mask=None):
    """(dQ, dK, dV) and the bounds on them without the results' own rounding."""
    Hq, G, d = Q.shape[1], Q.shape[1] // K.shape[1], Q.shape[2]
    half = HALF_STEP[Q.dtype]
    rounds = half if Q.dtype == torch.bfloat16 else 0.0
    Y, lse = forward64(Q, K, V, lens_q, lens_k, scale, mask)
    out = [torch.zeros(x.shape, dtype=torch.float64) for x in (Q, K, V)]
    tol = [torch.zeros(x.shape, dtype=torch.float64) for x in (Q, K, V)]
    for (a, b), (c, e) in zip(split(lens_q), split(lens_k)):
        keep = torch.arange(c, e)
        if mask is not None:
            keep = keep[mask[c:e].bool()]
        if not len(keep) or a == b:
            continue
        rows, n = (b - a) * G, len(keep)
        for h in range(Hq):
            q, k, v, g = (Q[a:b, h].double(), K[keep, h // G].double(), V[keep, h // G].double(),
                          dY[a:b, h].double())
            P = torch.exp(scale * q @ k.T - lse[a:b, h, None])
            dP, delta = g @ v.T, (g * Y[a:b, h]).sum(1, keepdim=True)
            dS = P * (dP - delta)
            A = (scale * q.abs() @ k.abs().T).amax(1, keepdim=True)
            B, C = g.abs() @ v.abs().T, (g * Y[a:b, h]).abs().sum(1, keepdim=True)
            eP = ((d + 12) * A + 4 * lse[a:b, h, None].abs() + 16) * U
            eS = P * ((eP + 3 * U) * (dP.abs() + delta.abs()) + (d + 1) * U * (B + C))
            if rounds:
                E = (eS + (n + 64) * U * dS.abs()).sum(1, keepdim=True)
                eS = eS + P * (E + 2 * half * half * C)
            else:
                eS = eS + P * half * C
            eS = eS + (rounds + (n + 64) * U) * dS.abs()
            out[0][a:b, h] = scale * dS @ k
            eQ = eS + P * rounds * dS.abs().sum(1, keepdim=True)
            tol[0][a:b, h] = scale * eQ @ k.abs()
            eS = eS + (rows + 64) * U * dS.abs()
            out[1][keep, h // G] += scale * dS.T @ q
            tol[1][keep, h // G] += scale * eS.T @ q.abs()
            out[2][keep, h // G] += P.T @ g
            tol[2][keep, h // G] += (P * (eP + rounds + (rows + 64) * U)).T @ g.abs()
    return out, tol


def check_forward(Y, lse, Q, K, V, lens_q, lens_k, scale, mask=None):
    G = Q.shape[1] // K.shape[1]
    for s, ((a, b), (c, d)) in enumerate(zip(split(lens_q), split(lens_k))):
        keep = torch.arange(c, d)
        if mask is not None:
            keep = keep[mask[c:d].bool()]
        for h in range(Q.shape[1]):
            check_attention(Y[a:b, h], None if lse is None else lse[a:b, h], Q[a:b, h],
                            K[keep, h // G], V[keep, h // G], scale,
                            torch.full((b - a,), len(keep)), f"source {s} head {h}")


def check_backward(got, dY, Q, K, V, lens_q, lens_k, scale, mask=None):
    """got: (dQ, dK, dV) of the kernels, given the forward pass's Y and lse."""
    want, tol = backward64(dY, Q, K, V, lens_q, lens_k, scale, mask)
    for name, x, y, t in zip(("dQ", "dK", "dV"), got, want, tol):
        assert torch.isfinite(x).all(), f"{name}: not finite"
        t = t * (1 + 2.0 ** -6) + HALF_STEP[x.dtype] * (y.abs() + t) + 1e-30
        err = (x.double() - y).abs()
        assert (err <= t).all(), f"{name}: off by {(err / t).max():.3g} times the bound"


def backward_of(dY, Q, K, V, Y, lse, lens_q, lens_k, scale, mask=None):
    """(dQ, dK, dV) and the bounds on them without the results' own rounding, where the
    backward pass is handed any Y and lse, those that the forward kernel stored say.

    As above, but for what these two are off by, which is known: lse by l_i, delta_i by
    eta_i = dY_i . (Y_i - the exact one).
      * P_ij is off relatively by l_i more: eP_i = ((d + 12) A_i + 4 |lse_i| + 16) u + l_i;
      * C_i is taken of the Y handed over, and e_ij = P_ij ((eP_i + 3 u) (|dP_ij| +
        |delta_i|) + (d + 1) u (B_ij + C_i));
      * fp32: eS_ij = e_ij + P_ij |eta_i|;
      * bf16: the sum of dS is -eta_i, as far as the P sum to 1 (off by eP_i): E_i = sum_j
        (e_ij + (n + 64) u |dS_ij|) + |eta_i| (eP_i + (n + 64) u), and eS_ij = e_ij + P_ij
        E_i;
      * bf16, dQ: the dS rounded there hold P_ij eta_i, and so do the P that it is taken
        off with, and rest_i as the sum of the former: P_ij h (sum_j |dS_ij| + 3 |eta_i|)
        more.
    """
    Hq, G, d = Q.shape[1], Q.shape[1] // K.shape[1], Q.shape[2]
    h16 = HALF_STEP[Q.dtype] if Q.dtype == torch.bfloat16 else 0.0
    Y64, lse64 = forward64(Q, K, V, lens_q, lens_k, scale, mask)
    out = [torch.zeros(x.shape, dtype=torch.float64) for x in (Q, K, V)]
    tol = [torch.zeros(x.shape, dtype=torch.float64) for x in (Q, K, V)]
    for (a, b), (c, e) in zip(split(lens_q), split(lens_k)):
        keep = torch.arange(c, e)
        if mask is not None:
            keep = keep[mask[c:e].bool()]
        if not len(keep) or a == b:
            continue
        rows, n = (b - a) * G, len(keep)
        for h in range(Hq):
            q, k, v, g = (Q[a:b, h].double(), K[keep, h // G].double(), V[keep, h // G].double(),
                          dY[a:b, h].double())
            y, y64, l64 = Y[a:b, h].double(), Y64[a:b, h], lse64[a:b, h, None]
            P = torch.exp(scale * q @ k.T - l64)
            dP, delta = g @ v.T, (g * y64).sum(1, keepdim=True)
            dS = P * (dP - delta)
            eta = (g * (y - y64)).sum(1, keepdim=True).abs()
            A = (scale * q.abs() @ k.abs().T).amax(1, keepdim=True)
            B, C = g.abs() @ v.abs().T, (g * y).abs().sum(1, keepdim=True)
            eP = ((d + 12) * A + 4 * l64.abs() + 16) * U + (lse[a:b, h, None].double() - l64).abs()
            eS = P * ((eP + 3 * U) * (dP.abs() + delta.abs()) + (d + 1) * U * (B + C))
            if h16:
                E = (eS + (n + 64) * U * dS.abs()).sum(1, keepdim=True) + eta * (eP + (n + 64) * U)
                eS = eS + P * E
            else:
                eS = eS + P * eta
            eS = eS + (h16 + (n + 64) * U) * dS.abs()
            out[0][a:b, h] = scale * dS @ k
            eQ = eS + P * h16 * (dS.abs().sum(1, keepdim=True) + 3 * eta)
            tol[0][a:b, h] = scale * eQ @ k.abs()
            eS = eS + (rows + 64) * U * dS.abs()
            out[1][keep, h // G] += scale * dS.T @ q
            tol[1][keep, h // G] += scale * eS.T @ q.abs()
            out[2][keep, h // G] += P.T @ g
            tol[2][keep, h // G] += (P * (eP + h16 + (rows + 64) * U)).T @ g.abs()
    return out, tol


def check_backward_of(got, dY, Q, K, V, Y, lse, lens_q, lens_k, scale, mask=None):
    """got: (dQ, dK, dV) of the kernels, given this Y and lse."""
    want, tol = backward_of(dY, Q, K, V, Y, lse, lens_q, lens_k, scale, mask)
    for name, x, y, t in zip(("dQ", "dK", "dV"), got, want, tol):
        assert torch.isfinite(x).all(), f"{name}: not finite"
        t = t * (1 + 2.0 ** -6) + HALF_STEP[x.dtype] * (y.abs() + t) + 1e-30
        err = (x.double() - y).abs()
        assert (err <= t).all(), f"{name}: off by {(err / t).max():.3g} times the bound"


def about(x, mean, spread):
    """x scaled to `spread` around `mean`: values that lie close together, where what
    delta is off by counts most (dS is small, the sums of P k are not)."""
    return (mean + spread * x.float()).to(x.dtype)
