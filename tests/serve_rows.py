"""64-bit reference of single rows of the attention over the paged cache (CPU), with elementwise error bounds: for calls whose
rows are too many to check all, and for value scales that differ widely. As serve_ref.attention, but for what a probability is
rounded to: relative to the largest product of probability and value scale that the row itself sees."""
import math

import torch

from layer_ref import TINY, U, half_step, up
from serve_ref import HALF16


def attention_rows(c, tokens, scale=None, softcap=0.0, causal=True):
    """{name: (value, bound)} of the tokens' rows, out [n, M, D] and lse [n, M]. c: the call, as test_gpu_cache.Case."""
    dt, P = c.dt, c.P
    h, tiny, two = half_step(dt), TINY[dt], dt == torch.float32
    hp = HALF16 ** 2 * 2 if two else HALF16  # probabilities: in fp16, or the sum of two of them
    D, Mkv, M = c.D, c.Mkv, c.M
    scale = D ** -0.5 if scale is None else scale
    lengths, starts, table = c.length.tolist(), c.start.tolist(), c.table.cpu()
    pages, width = c.k_cache.shape[0], table.shape[1]
    got = {name: ([], []) for name in ("out", "lse")}
    held = {}  # by sequence
    for t in tokens:
        n = max(i for i in range(len(lengths)) if starts[i] <= t)
        assert t < starts[n + 1]
        if n not in held:
            end = min(max(lengths[n], 0), width * P)
            place = torch.arange(end)
            page = table[n][place // P].long()
            there = (page >= 0) & (page < pages)
            page = page.clamp(0, pages - 1)
            at = page.to(c.k_cache.device)
            slot = (place % P).to(at.device)
            vs = up(c.v_scale[at])
            vs = torch.where(vs < 2.0 ** -126, torch.zeros_like(vs), vs)  # counted as 0, by definition
            held[n] = (place, there, up(c.k_cache[at, :, slot]) * up(c.k_scale[at])[..., None], up(c.v_cache[at, :, slot]), vs)
        place, there, k, v, vs = held[n]
        seen = there & (place <= lengths[n] - starts[n + 1] + t) if causal else there
        keys = int(seen.sum())
        if keys == 0:
            for name, value in (("out", torch.zeros(M, D)), ("lse", torch.full((M,), -math.inf))):
                got[name][0].append(value.double())
                got[name][1].append(torch.zeros_like(value).double())
            continue
        x = up(c.q[t]).view(Mkv, M // Mkv, D)
        K, V, S = (y[seen].transpose(0, 1).contiguous() for y in (k, v, vs))  # [Mkv, keys, D] and [Mkv, keys]
        raw = x @ K.transpose(1, 2).contiguous() * scale
        # queries in fp16 (the sum of two in fp32), their largest at 2^14 or more; products summed in fp32
        dq = (HALF16 ** 2 * 2 * x.abs() if two else torch.zeros_like(x)) + 2.0 ** -39 * x.abs().amax(-1, keepdim=True)
        dz = ((D + 6) * U * x.abs() + dq) @ K.abs().transpose(1, 2).contiguous() * scale
        z = raw
        if softcap:
            z = softcap * torch.tanh(raw / softcap)
            dz = dz + 8 * U * softcap  # an fp32 rounding or two of 1, times the cap
        total = torch.logsumexp(z, -1, keepdim=True)
        p = torch.exp(z - total)
        rho = dz.amax(-1, keepdim=True) + 8 * U * (z.abs().amax(-1, keepdim=True) + 1)
        # A value scale is a factor in the exponent: its logarithm, its unit's, their difference, the exponent that they are part
        # of, and the two that turn the row's unit into the maximum's, each of up to 256 and rounded in fp32.
        share = 2 * rho + hp + (2 * keys + 8) * U + 6 * 256 * U
        weight = p * S[:, None]
        y = weight @ V
        # half of fp16's smallest number, 2^-25, where the largest product of probability and scale is 2^6 or more
        floor = 2.0 ** -31 * weight.amax(-1, keepdim=True) * V.abs().sum(1)[:, None]
        d = (share * (weight @ V.abs()) + floor) * 1.02 + h * y.abs() * 1.01 + tiny
        got["out"][0].append(y.reshape(M, D))
        got["out"][1].append(d.reshape(M, D))
        got["lse"][0].append(total.reshape(M))
        got["lse"][1].append((rho + (keys + 8) * U + 6 * 256 * U + 6 * U * total.abs()).reshape(M))
    return {name: tuple(torch.stack(y) for y in x) for name, x in got.items()}
