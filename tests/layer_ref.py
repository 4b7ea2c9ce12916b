"""64-bit references of the layer operators (CPU, torch float64) with elementwise error bounds.

Each function returns the exact results and, for each, how far a correct kernel may be off: fp32
arithmetic (u = 2^-24 per operation, sums counted by their longest chain of additions) plus the
roundings to the element type (half a step, h = eps / 2, and half of its smallest subnormal number).
"""
import math

import torch

U = 2.0 ** -24
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
TINY = {torch.float32: 2.0 ** -150, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}


def half_step(dtype) -> float:
    return torch.finfo(dtype).eps / 2


def assert_within(name, got, want, bound):
    """Elementwise |got - want| <= bound; infinities have to be equal, and a NaN in got never passes."""
    got, want = got.detach().double().cpu(), want.double()
    assert got.shape == want.shape, f"{name}: shape {tuple(got.shape)}, expected {tuple(want.shape)}"
    same = got == want
    bad = ~(same | ((got - want).abs() <= bound))
    if bad.any():
        i = tuple(int(x) for x in bad.nonzero()[0])
        off = torch.where(bad, (got - want).abs() / bound.expand_as(want).clamp_min(1e-300), torch.zeros_like(want))
        raise AssertionError(f"{name}: {int(bad.sum())} of {bad.numel()} values off by up to {float(off.max()):.3g} bounds; "
                             f"first at {i}: got {float(got[i]):.9g}, expected {float(want[i]):.9g}")


def up(x):
    return None if x is None else x.detach().cpu().double()


# ---------------------------------------------------------------- layer norm


def layernorm(x, weight=None, bias=None, residual=None, eps=1e-5, grad_out=None, grad_sum=None):
    """{name: (value, bound)} of every result for x [rows, C]."""
    h, tiny = half_step(x.dtype), TINY[x.dtype]
    C = x.shape[1]
    w = up(weight) if weight is not None else torch.ones(C, dtype=torch.float64)
    b = up(bias) if bias is not None else torch.zeros(C, dtype=torch.float64)
    s = up(x) if residual is None else up(x) + up(residual)
    mean = s.mean(1, keepdim=True)
    c = s - mean
    var = (c * c).mean(1, keepdim=True)
    rstd = (var + eps).rsqrt()
    xh = c * rstd
    # a sum over a row: 16 elements per lane, 6 steps within a wave, 16 waves, and the division
    chain = 40 * U
    d_mean = chain * s.abs().mean(1, keepdim=True) + U * mean.abs()
    d_c = U * (s.abs() + c.abs()) + d_mean
    d_rstd = chain + 8 * U + d_c.amax(1, keepdim=True) * rstd  # relative
    d_xh = rstd * d_c + xh.abs() * (d_rstd + 2 * U)
    out = xh * w + b
    res = {"out": (out, w.abs() * d_xh + 4 * U * ((xh * w).abs() + b.abs()) + h * out.abs() * 1.01 + tiny),
           "mean": (mean[:, 0], d_mean[:, 0]), "rstd": (rstd[:, 0], (rstd * d_rstd)[:, 0] + U * rstd[:, 0]),
           "sum": (s, (h + U) * s.abs() * 1.01 + tiny)}
    if grad_out is not None:
        go = up(grad_out)
        g = go * w
        m0, m1 = g.mean(1, keepdim=True), (g * xh).mean(1, keepdim=True)
        gx = rstd * (g - m0 - xh * m1)
        d_m0 = (chain + U) * g.abs().mean(1, keepdim=True)
        d_m1 = (chain + 2 * U) * (g * xh).abs().mean(1, keepdim=True) + (g.abs() * d_xh).mean(1, keepdim=True)
        parts = g.abs() + m0.abs() + (xh * m1).abs()
        d = rstd * (4 * U * parts + d_m0 + xh.abs() * d_m1 + d_xh * m1.abs()) + gx.abs() * d_rstd
        total = gx if grad_sum is None else gx + up(grad_sum)
        res["grad_x"] = (total, d + 2 * U * (gx.abs() + total.abs()) + h * total.abs() * 1.01 + tiny)
        rows = x.shape[0]
        adds = (math.ceil(rows / 1024) + 80) * U  # rows of a lane, of a workgroup, and of the workgroups
        res["grad_weight"] = ((go * xh).sum(0), adds * (go * xh).abs().sum(0) + (go.abs() * d_xh).sum(0))
        res["grad_bias"] = (go.sum(0), adds * go.abs().sum(0))
    return res


# ---------------------------------------------------------------- rotary positions


def rotary(x, pos, freqs, interleaved, sign=1.0):
    """(value, bound) of x [N, T, M, D] turned by sign * pos . freqs."""
    h, tiny = half_step(x.dtype), TINY[x.dtype]
    R = freqs.shape[1]
    xs, p, f = up(x), up(pos), up(freqs)
    angle = (p[..., :, None] * f).sum(-2)
    c, s = torch.cos(angle)[..., None, :], sign * torch.sin(angle)[..., None, :]
    a, b = (slice(0, 2 * R, 2), slice(1, 2 * R, 2)) if interleaved else (slice(0, R), slice(R, 2 * R))
    y, bound = xs.clone(), torch.zeros_like(xs)
    y[..., a] = xs[..., a] * c - xs[..., b] * s
    y[..., b] = xs[..., a] * s + xs[..., b] * c
    # cosine and sine to 6 u (the angle's remainder in fp32, four multiply-adds), two products and a sum;
    # the fp64 angle is off by 4 * 2^-53 of the sum's terms
    d = 9 * U + 2.0 ** -51 * (p.abs()[..., :, None] * f.abs()).sum(-2)[..., None, :]
    both = d * (xs[..., a].abs() + xs[..., b].abs())
    bound[..., a] = both + h * y[..., a].abs() * 1.01 + tiny
    bound[..., b] = both + h * y[..., b].abs() * 1.01 + tiny
    return y, bound  # channels beyond the pairs are copied: a bound of 0


# ---------------------------------------------------------------- attention


def seen_pairs(N, Lq, Lk, q_doc=None, k_doc=None, prefix=None, causal=False):
    """[N, Lq, Lk]: whether query i sees key j, pair by pair from the rules."""
    i, j = torch.arange(Lq)[:, None], torch.arange(Lk)[None]
    seen = torch.ones(N, Lq, Lk, dtype=torch.bool)
    for n in range(N):
        first = j < (int(prefix[n]) if prefix is not None else 0)
        if causal:
            seen[n] &= (j <= i + Lk - Lq) | first
        if q_doc is not None:
            a, b = q_doc[n].cpu()[:, None], k_doc[n].cpu()[None]
            seen[n] &= (a >= 0) & (b >= 0) & ((a == b) | first)
    return seen


def attention(q, k, v, scale=None, softcap=0.0, slopes=None, q_pos=None, k_pos=None, q_doc=None, k_doc=None, prefix=None,
              causal=False, grad_out=None, few_keys=False, carried=False):
    """{name: (value, bound)} of out, lse and, with grad_out, grad_q, grad_k and grad_v. What a query does not see
    is left out of every sum, whatever it holds. few_keys: every row has so few that its delta is not that of the
    rounded out, but mended by sum_j P (dP - delta). carried: fp16 gradients of scores are rounded with a power of two that
    holds the largest of a row (for grad_q) or key (grad_k) at 2^10 or more, so that half of fp16's smallest number, 2^-25, is
    2^-35 of that, and its probabilities (of a row's largest in the forward) with one of 2^11."""
    dt = q.dtype
    h, tiny = half_step(dt), TINY[dt]
    hp = 0.0 if dt == torch.float32 else h           # probabilities and dS go through the element type
    tp = 2.0 ** -25 if dt == torch.float16 else 0.0  # half of fp16's smallest number
    N, Lq, M, D = q.shape
    Lk, Mkv = k.shape[1], k.shape[2]
    scale = D ** -0.5 if scale is None else scale
    seen = seen_pairs(N, Lq, Lk, q_doc, k_doc, prefix, causal)[:, None]

    def heads(x, to=None):
        y = torch.nan_to_num(up(x), 0.0, 0.0, 0.0).transpose(1, 2)  # what is seen is finite in these tests
        return y if to is None else y.repeat_interleave(to // y.shape[1], dim=1)

    Q, K, V = heads(q), heads(k, M), heads(v, M)
    raw = Q @ K.transpose(2, 3) * scale
    dz = (D + 6) * U * (Q.abs() @ K.abs().transpose(2, 3)) * scale
    slack = torch.ones_like(raw)
    z = raw
    if softcap:
        t = torch.tanh(raw / softcap)
        z, slack = softcap * t, 1 - t * t
        dz = dz + 6 * U * softcap
    if slopes is not None:
        d = up(q_pos)[:, :, None, :] - up(k_pos)[:, None, :, :]
        far = up(slopes)[:, None, None] * (d * d).sum(-1).sqrt()[:, None]
        far = torch.nan_to_num(far, 0.0, 0.0, 0.0)
        z = z - far
        dz = dz + 8 * U * far
    neg = torch.full((), -math.inf, dtype=torch.float64)
    zm = torch.where(seen, z, neg)
    any_seen = seen.any(-1, keepdim=True).expand(N, M, Lq, 1)
    lse = torch.logsumexp(torch.where(any_seen, zm, torch.zeros_like(zm)), -1, keepdim=True)
    P = torch.where(seen & any_seen, torch.exp(z - lse), torch.zeros_like(z))
    zero = torch.zeros_like(P)
    top = torch.where(seen, z.abs(), zero).amax(-1, keepdim=True)
    # the exponent in units of log 2: a product and a difference, of values up to the largest score
    rho = torch.where(seen, dz, zero).amax(-1, keepdim=True) + 8 * U * (top + 1)
    out = P @ V
    A = P @ V.abs()
    spread = seen.double().expand(N, M, Lq, Lk) @ V.abs()
    d_out = (2 * rho + hp + (2 * Lk + 8) * U) * A + (tp * 2.0 ** -11 if carried else tp) * spread
    d_lse = rho + (Lk + 4) * U + 6 * U * lse.abs()
    flat = lambda x: x.transpose(1, 2)  # noqa: E731
    res = {"out": (flat(out), flat(d_out * 1.02 + h * out.abs() * 1.01 + tiny)),
           "lse": (torch.where(any_seen, lse, neg)[..., 0], d_lse[..., 0])}
    if grad_out is None:
        return res
    G = heads(grad_out)
    dP = G @ V.transpose(2, 3)
    delta = (G * out).sum(-1, keepdim=True)
    E = torch.where(seen, dP - delta, zero)
    dS = P * E * slack
    rho2 = rho + d_lse + 8 * U * (lse.abs() + 1)
    d_dP = (D + 4) * U * (G.abs() @ V.abs().transpose(2, 3))
    d_delta = (G.abs() * (d_out + h * out.abs() + tiny)).sum(-1, keepdim=True) + (D + 8) * U * (G * out).abs().sum(-1, keepdim=True)
    if few_keys:  # delta + sum P (dP - delta): the errors of the sum, and what 1 - sum P leaves of delta's own
        d_delta = (P * (d_dP + (rho2 + (Lk + 12) * U) * (E.abs() + d_delta))).sum(-1, keepdim=True)
        d_delta = d_delta + 2 * U * delta.abs()
    d_dS = P * ((rho2 + 12 * U) * E.abs() + d_dP + d_delta) + hp * dS.abs()
    lost_q = lost_k = torch.full((), tp, dtype=torch.float64)
    if carried:
        lost_q = dS.abs().amax(-1, keepdim=True) * (tp * 2.0 ** -10)
        lost_k = dS.abs().reshape(N, Mkv, M // Mkv, Lq, Lk).amax((2, 3), keepdim=True).expand(N, Mkv, M // Mkv, 1, Lk)
        lost_k = lost_k.reshape(N, M, 1, Lk) * (tp * 2.0 ** -10)
    d_q, d_dS = (torch.where(seen, d_dS * 1.02 + lost, zero) for lost in (lost_q, lost_k))
    groups = lambda x: flat(x.reshape(N, Mkv, M // Mkv, Lk, D).sum(2))  # noqa: E731
    gq = dS @ K * scale
    res["grad_q"] = (flat(gq), flat((d_q + (Lk + 4) * U * dS.abs()) @ K.abs() * scale + h * gq.abs() * 1.02 + tiny))
    R = Lq * (M // Mkv)
    gk = groups(dS.transpose(2, 3) @ Q * scale)
    b_k = groups((d_dS + (R + 4) * U * dS.abs()).transpose(2, 3) @ Q.abs() * scale)
    res["grad_k"] = (gk, b_k + h * gk.abs() * 1.02 + tiny)
    gv = groups(P.transpose(2, 3) @ G)
    d_P = torch.where(seen, P * (rho2 + hp + (R + 4) * U) * 1.02 + tp * 2.0 ** (-11 if carried else -8), zero)  # fp16: scaled by 2^8 at least
    res["grad_v"] = (gv, groups(d_P.transpose(2, 3) @ G.abs()) + h * gv.abs() * 1.02 + tiny)
    return res
