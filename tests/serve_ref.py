"""64-bit references of the serving operators (CPU) with elementwise error bounds, derived as those of layer_ref: fp32
arithmetic (u = 2^-24 per operation, sums counted by their longest chain of additions) plus the roundings to the element
type. Codes are compared bit by bit where they come from fp32 operations whose order is fixed."""
import math

import torch

from layer_ref import TINY, U, half_step, up

HALF16 = 2.0 ** -11  # half a step of fp16, relative
LEAST = 2.0 ** -100


# ---------------------------------------------------------------- rows in 8 bits


def codes_of(t):
    """(codes, u) of fp32 rows t: each operation in fp32, in the order that the header states."""
    assert t.dtype == torch.float32
    most = t.abs().amax(-1, keepdim=True)  # NaN where a row holds one
    u = most * torch.tensor(1 / 127, dtype=torch.float32)
    odd = ~torch.isfinite(most)
    u = torch.where(most < LEAST, torch.zeros_like(u), u)
    inverse = torch.where(u > 0, torch.ones_like(u) / u, torch.zeros_like(u))
    codes = torch.round(torch.where(odd, torch.zeros_like(t), t) * torch.where(odd, torch.zeros_like(u), inverse))
    return codes.clamp(-127, 127).to(torch.int8), torch.where(odd, torch.full_like(u, math.nan), u)[..., 0]


def quantized_rows(x, weight=None, residual=None):
    """codes and u of x (+ residual) (* weight), rows [rows, C]."""
    t = x.detach().cpu().float()
    if residual is not None:
        t = t + residual.cpu().float()
    if weight is not None:
        t = t * weight.cpu()
    return codes_of(t)


def rmsnorm(x, weight=None, residual=None, eps=1e-6, grad_out=None, grad_sum=None):
    """{name: (value, bound)} of every result for x [rows, C]; "scale_by" is rstd as a factor of the codes' scale."""
    h, tiny = half_step(x.dtype), TINY[x.dtype]
    C = x.shape[1]
    w = up(weight) if weight is not None else torch.ones(C, dtype=torch.float64)
    s = up(x) if residual is None else up(x) + up(residual)
    rstd = ((s * s).mean(1, keepdim=True) + eps).rsqrt()
    # the addition, the square, a sum over a row (16 elements a lane, 6 steps within a wave, 16 waves), the division,
    # the root and its inverse: half of the sum's relative error, as its root
    d_rstd = 0.5 * (40 + 6) * U + 4 * U
    # what a residual's addition rounds is relative to the sum, not to its parts
    xh = s * rstd
    d_xh = xh.abs() * (d_rstd + 3 * U)
    out = xh * w
    res = {"out": (out, w.abs() * d_xh + 2 * U * out.abs() + h * out.abs() * 1.01 + tiny),
           "rstd": (rstd[:, 0], (rstd * (d_rstd + U))[:, 0]), "sum": (s, (h + U) * s.abs() * 1.01 + tiny)}
    if grad_out is not None:
        go = up(grad_out)
        g = go * w
        m1 = (g * xh).mean(1, keepdim=True)
        gx = rstd * (g - xh * m1)
        d_m1 = (40 + 4) * U * (g * xh).abs().mean(1, keepdim=True) + (g.abs() * d_xh).mean(1, keepdim=True)
        d = rstd * (4 * U * (g.abs() + (xh * m1).abs()) + xh.abs() * d_m1 + d_xh * m1.abs()) + gx.abs() * (d_rstd + U)
        total = gx if grad_sum is None else gx + up(grad_sum)
        res["grad_x"] = (total, d + 2 * U * (gx.abs() + total.abs()) + h * total.abs() * 1.01 + tiny)
        adds = (math.ceil(x.shape[0] / 1024) + 80) * U  # rows of a lane, of a workgroup, and of the workgroups
        res["grad_weight"] = ((go * xh).sum(0), adds * (go * xh).abs().sum(0) + (go.abs() * d_xh).sum(0))
    return res


# ---------------------------------------------------------------- products


def product(a, b, a_scale, b_scale, bias, dtype):
    """(value, bound) of the scaled product; the sum itself is exact in 64 bits."""
    total = a.cpu().double() @ b.cpu().double().t()
    y = total * (up(a_scale)[:, None] * up(b_scale))
    bound = 3 * U * y.abs()  # the sum's conversion, and two products
    if bias is not None:
        y = y + up(bias)
        bound = bound + U * y.abs() * 1.01
    return y, bound * 1.01 + half_step(dtype) * y.abs() * 1.01 + TINY[dtype]


# ---------------------------------------------------------------- paged cache


def places(T, length, start, width, page_size):
    """Per sequence: (first new token of the call, how many, the first one's place)."""
    got = []
    for n, total in enumerate(length):
        a, b = (n, n + 1) if start is None else (min(max(start[n], 0), T), min(max(start[n + 1], 0), T))
        got.append((a, max(b - a, 0), max(total, 0) - max(b - a, 0)))
    return got


def turned(k, pos, freqs, interleaved):
    """(value, bound) of k [T, M, D] turned by pos . freqs, before any rounding."""
    x = up(k)
    if freqs is None or freqs.shape[1] == 0:
        return x, torch.zeros_like(x)
    p, f, R = up(pos), up(freqs), freqs.shape[1]
    angle = (p[:, :, None] * f).sum(1)[:, None]
    c, s = torch.cos(angle), torch.sin(angle)
    a, b = (slice(0, 2 * R, 2), slice(1, 2 * R, 2)) if interleaved else (slice(0, R), slice(R, 2 * R))
    y, bound = x.clone(), torch.zeros_like(x)
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., a] * s + x[..., b] * c
    # cosine and sine to 6 u, two products and a sum; the angle in fp64
    d = (9 * U + 2.0 ** -51 * (p.abs()[:, :, None] * f.abs()).sum(1)[:, None]) * (x[..., a].abs() + x[..., b].abs())
    bound[..., a] = bound[..., b] = d
    return y, bound


def check_append(before, after, values, bound, table, length, start):
    """Checks one of the caches (codes [pages, Mkv, P, D], scale [pages, Mkv]) against the values [T, Mkv, D] appended to it,
    which are known within `bound`. Returns how many codes were rounded anew."""
    codes0, scale0 = before
    codes1, scale1 = (x.cpu() for x in after)
    pages, Mkv, P, D = codes0.shape
    want_codes, want_scale = codes0.clone(), scale0.clone()
    T, width, anew = values.shape[0], table.shape[1], 0
    for n, (at, count, first) in enumerate(places(T, length, start, table.shape[1], P)):
        place, last = max(first, 0), min(max(length[n], 0), width * P)
        while place < last:
            stop, slot = min(last, (place // P + 1) * P), place % P
            page = int(table[n, place // P])
            t0 = at + place - first
            mine, off = values[t0:t0 + stop - place], bound[t0:t0 + stop - place]
            place = stop
            if not 0 <= page < pages:
                continue
            for h in range(Mkv):
                x, d = mine[:, h], off[:, h]
                got = float(scale1[page, h])
                old = float(scale0[page, h]) if slot else 0.0
                most = float(x.abs().max())
                if not math.isfinite(most) or not math.isfinite(old):
                    assert math.isnan(got), f"page {page}, head {h}: scale {got} of a block that is not finite"
                    assert not codes1[page, h, slot:slot + len(x)].any()
                    want_codes[page, h, slot:slot + len(x)] = 0
                    want_scale[page, h] = math.nan
                    continue
                want = max(old, 0.0 if most < LEAST else most / 127)
                # the values' own error, and the product with 1 / 127, which is rounded too
                assert abs(got - want) <= float(d.max()) / 127 + 2.1 * U * want, f"page {page}, head {h}: scale {got}, expected {want}"
                u = scale1[page, h]
                if old > 0 and got > old:  # rounded anew to the scale that the kernel found: the same fp32 operations
                    ratio = scale0[page, h] / u
                    want_codes[page, h, :slot] = torch.round(codes0[page, h, :slot].float() * ratio).to(torch.int8)
                    anew += slot * D
                new = codes1[page, h, slot:slot + len(x)].double()
                assert float(new.abs().max()) <= 127
                if got == 0.0:  # a block whose largest is below 2^-100 is held as zeros, by definition
                    assert most < LEAST and not new.any()
                # half a step; 1 / u and the product with it are each off by 2^-24 of up to 127 steps
                else:
                    near = (new * got - x).abs() <= got * (0.5 + 127 * 3 * U) + d
                    assert bool(near.all()), f"page {page}, head {h}: codes"
                want_codes[page, h, slot:slot + len(x)] = codes1[page, h, slot:slot + len(x)]
                want_scale[page, h] = u
    assert torch.equal(codes1, want_codes), "slots that no new token reaches have changed"
    assert torch.equal(torch.nan_to_num(scale1, -7.0), torch.nan_to_num(want_scale, -7.0)), "scales of other pages have changed"
    return anew


def attention(q, k_cache, v_cache, k_scale, v_scale, table, length, start=None, scale=None, softcap=0.0, causal=True):
    """{name: (value, bound)} of out [T, M, D] and lse [T, M]; rows of tokens of no sequence are NaN."""
    dt = q.dtype
    T, M, D = q.shape
    pages, Mkv, P, _ = k_cache.shape
    G, h, tiny = M // Mkv, half_step(dt), TINY[dt]
    two = dt == torch.float32
    hp = HALF16 ** 2 * 2 if two else HALF16  # probabilities: in fp16, or the sum of two of them
    scale = D ** -0.5 if scale is None else scale
    nan = math.nan
    out, d_out = torch.full((T, M, D), nan, dtype=torch.float64), torch.zeros((T, M, D), dtype=torch.float64)
    lse, d_lse = torch.full((T, M), nan, dtype=torch.float64), torch.zeros((T, M), dtype=torch.float64)
    table, lengths = table.cpu(), [int(x) for x in length]
    starts = None if start is None else [int(x) for x in start]
    kc, vc, ks, vs, qs = k_cache.cpu(), v_cache.cpu(), k_scale.cpu(), v_scale.cpu(), up(q)
    vs = torch.where(vs < 2.0 ** -126, torch.zeros_like(vs), vs)  # counted as 0, by definition
    for n, (at, count, first) in enumerate(places(T, lengths, starts, table.shape[1], P)):
        end = min(max(lengths[n], 0), table.shape[1] * P)
        place = torch.arange(end)
        page = table[n][place // P].long() if end else torch.zeros(0, dtype=torch.long)
        there = (page >= 0) & (page < pages)
        page = page.clamp(0, max(pages - 1, 0))
        if end:
            k = kc[page, :, place % P].double() * ks[page].double()[..., None]  # [end, Mkv, D]
            v = vc[page, :, place % P].double() * vs[page].double()[..., None]
            base = torch.where(there[:, None] & torch.isfinite(vs[page]), vs[page], torch.zeros_like(vs[page])).double().amax(0)
        for i in range(count):
            seen = there & (place <= first + i) if causal else there
            for m in range(M):
                t, hd = at + i, m // G
                if not bool(seen.any()):
                    out[t, m], lse[t, m] = 0.0, -math.inf
                    continue
                x, K, V = qs[t, m], k[seen, hd], v[seen, hd]
                raw = K @ x * scale
                # queries in fp16 (the sum of two in fp32), their largest at 2^14 or more; products summed in fp32
                dq = (HALF16 ** 2 * 2 * x.abs() if two else 0.0) + 2.0 ** -39 * x.abs().max()
                dz = ((D + 6) * U * (K.abs() @ x.abs()) + K.abs() @ (dq + torch.zeros_like(x))) * scale
                z = raw
                if softcap:
                    z = softcap * torch.tanh(raw / softcap)
                    # the series, or in 16 bits the short form up to a cap of 256: an fp32 rounding or two of 1, times the cap
                    dz = dz + 8 * U * softcap
                total = torch.logsumexp(z, 0)
                p = torch.exp(z - total)
                keys = len(z)
                rho = float(dz.max()) + 8 * U * (float(z.abs().max()) + 1)
                y = p @ V
                # a page's value scale is a factor in the exponent, known there to 2^-24 of a logarithm up to 128
                share = 2 * rho + hp + (2 * keys + 8) * U + 2 * 128 * U
                # half of fp16's smallest number, 2^-25, at 2^14 times a probability in units of the largest scale
                floor = 2.0 ** -39 * float(base[hd]) * 127 * keys
                out[t, m] = y
                d_out[t, m] = (share * (p @ V.abs()) + floor) * 1.02 + h * y.abs() * 1.01 + tiny
                lse[t, m] = total
                d_lse[t, m] = rho + (keys + 8) * U + 2 * 128 * U + 6 * U * abs(float(total))
    return {"out": (out, d_out), "lse": (lse, d_lse)}
