"""Timing cases of the operators that serve a transformer layer in 8 bits, and of its norm in training.

A decoder layer at inference, token by token or a chunk of a prompt at a time: the residual's addition with
a root-mean-square norm whose result leaves in 8 bits, products of 8-bit integers with scales for each token and
channel, new keys and values rotated on their way into a paged cache of 8 bits with a scale for each page and head, and the
attention that reads that cache. With ``own`` false a pass computes an operator in its plain form (elementary
torch operations in fp32), with ``own`` true through the library's entry points. Sizes are generic, with odd and ragged
ones among them; inputs are drawn on the GPU from the seed alone, lengths follow from the case.

  op            what a pass calls
  rms_quantize  msda.rmsnorm_quantize (inference)
  rms_step      msda.rmsnorm_forward and msda.rmsnorm_backward (training)
  mm            msda.quantize_rows on the activations, where they are not in 8 bits yet, and msda.quantized_matmul
  append        msda.cache_append
  attn          msda.cache_attention

What is held in 8 bits is returned as the values it stands for, in bf16, which holds a code's seven bits: a value
next to the border of two codes may get either.
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-6
THETA = 10000.0


def _rms(name, op, rows, C, dtype, residual):
    return {"name": name, "op": op, "rows": rows, "C": C, "dtype": dtype, "residual": residual}


def _mm(name, T, K, O, dtype, bias, codes):
    """codes: the activations are in 8 bits already, as a norm leaves them. (All those with results in fp32: one code that
    falls the other way at a border would outweigh fp32's roundings.)"""
    return {"name": name, "op": "mm", "T": T, "K": K, "O": O, "dtype": dtype, "bias": bias, "codes": codes}


def _cache(name, op, N, new, longest, M, Mkv, D, page, dtype, softcap=0.0, interleaved=False):
    """N sequences of up to `longest` tokens, of which up to `new`, the last ones, are new."""
    return {"name": name, "op": op, "N": N, "new": new, "longest": longest, "M": M, "Mkv": Mkv, "D": D, "page": page,
            "dtype": dtype, "softcap": softcap, "interleaved": interleaved}


def listed():
    return [
        # the norm before a projection, one token of each of 16 sequences: the call is its latency
        _rms("rms_token_q8_bf16", "rms_quantize", 16, 4096, "bf16", True),
        # the same over the tokens of several prompts, an odd number of rows of an odd number of pieces
        _rms("rms_chunk_q8_f16", "rms_quantize", 9973, 2568, "f16", True),
        # training in fp32, odd sizes
        _rms("rms_ragged_step_f32", "rms_step", 8997, 1000, "f32", True),
        # training: the tokens of two DETR encoder images, wide rows
        _rms("rms_encoder_step_bf16", "rms_step", 39894, 1024, "bf16", True),
        # a projection after attention, one token of each of eight sequences: the weights are read once
        _mm("mm_token_bf16", 8, 4096, 6144, "bf16", False, False),
        # odd sizes after a norm, results in fp32, with a bias
        _mm("mm_ragged_f32", 1019, 1360, 2050, "f32", True, True),
        # a projection after a norm of the tokens of several prompts
        _mm("mm_chunk_bf16", 8192, 4096, 12288, "bf16", False, True),
        # one token of each of 64 sequences that began lately (the pool holds their pages alone: it is returned whole)
        _cache("append_token_bf16", "append", 64, 1, 64, 32, 8, 128, 16, "bf16"),
        # chunks of prompts, of ragged lengths, after what is there
        _cache("append_chunk_f16", "append", 16, 2048, 2560, 32, 8, 128, 64, "f16"),
        # one token of each of 32 sequences over long caches, shared heads
        _cache("attn_token_bf16", "attn", 32, 1, 16411, 32, 8, 128, 64, "bf16"),
        # chunks of two prompts over what is there and themselves
        _cache("attn_chunk_bf16", "attn", 2, 2048, 10240, 32, 8, 128, 64, "bf16"),
        # a few guessed tokens of each of 12 sequences looked over at once, odd heads, capped scores, fp32
        _cache("attn_verify_f32", "attn", 12, 5, 3001, 10, 5, 48, 16, "f32", 30.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Any operator: rows of 16 to 8192 channels, products of 1 to 8192 tokens, 1 to 64 sequences of up to 20000 tokens."""
    while True:
        kind = rng.choice(["rms", "mm", "append", "attn"])
        dtype = rng.choice(["f32", "f16", "bf16"])
        if kind == "rms":
            c = _rms("", rng.choice(["rms_quantize", "rms_step"]), _log(rng, 1, 100000), _log(rng, 16, 8192), dtype,
                     rng.random() < 0.7)
            if c["rows"] * c["C"] > 39894 * 1024:
                continue
        elif kind == "mm":
            K = _log(rng, 16, 8192)
            c = _mm("", _log(rng, 1, 8192), K if rng.random() < 0.2 else -(-K // 16) * 16, _log(rng, 16, 12288), dtype,
                    rng.random() < 0.3, dtype == "f32" or rng.random() < 0.5)
            if c["T"] * c["K"] * c["O"] > 8192 * 4096 * 12288:
                continue
        else:
            Mkv, g = rng.choice([1, 2, 3, 4, 8]), rng.choice([1, 2, 4, 5, 8])
            N = _log(rng, 1, 64)
            new = rng.choice([1, 1, _log(rng, 2, 8), _log(rng, 8, 4096)])
            longest = max(new, _log(rng, 1, 4096 if kind == "append" else 20000))
            c = _cache("", kind, N, new, longest, Mkv * g, Mkv, rng.choice([16, 32, 48, 64, 80, 96, 112, 128, 128]),
                       rng.choice([16, 32, 64, 128]), dtype, rng.choice([0.0, 0.0, 30.0]) if kind == "attn" else 0.0,
                       kind == "append" and rng.random() < 0.5)
            if N * longest * Mkv * c["D"] > 32 * 16411 * 8 * 128 or N * c["M"] * new * longest > 2 * 32 * 2048 * 10240:
                continue
            if kind == "append" and N * longest * Mkv * c["D"] > 16 * 2560 * 8 * 128:
                continue
        del c["name"]
        return c


# ---------------------------------------------------------------- inputs


def _lengths(case):
    """Per sequence: (tokens in all, new ones among them)."""
    r = random.Random("%d %d %d" % (case["N"], case["new"], case["longest"]))
    got = []
    for _ in range(case["N"]):
        new = r.randint(max(1, case["new"] // 2), case["new"])
        got.append((r.randint(max(new, 2 * case["longest"] // 3), case["longest"]), new))
    return got


def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


def _rotation(case):
    """[1, D / 2] frequencies of the channels' pairs."""
    n = case["D"] // 2
    return (THETA ** (-torch.arange(n, dtype=torch.float64) / n)).float()[None].cuda()


def _inputs(case, seed):
    """The tensors of one pass, from the seed alone."""
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    dt, op = DTYPES[case["dtype"]], case["op"]
    if op.startswith("rms"):
        rows, C = case["rows"], case["C"]
        t = {"x": (_normal(gen, rows, C) * 1.5).to(dt), "residual": None}
        if case["residual"]:
            t["residual"] = _normal(gen, rows, C).to(dt)
        t["weight"] = 1 + 0.1 * _normal(gen, C)
        if op == "rms_step":
            t["gout"] = _normal(gen, rows, C).to(dt)
        return t
    if op == "mm":
        T, K, O = case["T"], case["K"], case["O"]
        t = {"x": _normal(gen, T, K).to(dt)}
        if case["codes"]:
            t["x_scale"] = t["x"].float().abs().amax(1) / 127
            t["x"] = torch.round(t["x"].float() / t["x_scale"][:, None]).clamp(-127, 127).to(torch.int8)
        w = _normal(gen, O, K)
        t["w_scale"] = w.abs().amax(1) / 127 / math.sqrt(K)  # the weights, laid out once
        t["w"] = torch.round(w * (127 / w.abs().amax(1, keepdim=True))).to(torch.int8)
        t["bias"] = _normal(gen, O) if case["bias"] else None
        return t
    N, M, Mkv, D, P = (case[k] for k in ("N", "M", "Mkv", "D", "page"))
    lengths = _lengths(case)
    T, width = sum(new for _, new in lengths), -(-case["longest"] // P)
    t = {"length": torch.tensor([n for n, _ in lengths], dtype=torch.int32, device="cuda"), "start": None}
    if case["new"] > 1:
        ends = [0]
        for _, new in lengths:
            ends.append(ends[-1] + new)
        t["start"] = torch.tensor(ends, dtype=torch.int32, device="cuda")
    # every sequence's pages lie anywhere in the pool
    t["table"] = torch.randperm(N * width, generator=gen, device="cuda").to(torch.int32).reshape(N, width)
    for x in ("k", "v"):
        codes = torch.empty((N * width, Mkv, P, D), dtype=torch.int8, device="cuda")
        codes.copy_((_normal(gen, N * width, Mkv, P, D) * 32).round_().clamp_(-127, 127))
        t[x + "_cache"] = codes
        t[x + "_scale"] = torch.exp(0.25 * _normal(gen, N * width, Mkv)) / 32
    if op == "attn":
        t["q"] = _normal(gen, T, M, D).to(dt)
        return t
    # the new tokens, as a projection leaves them: queries, keys and values of a token side by side
    packed = _normal(gen, T, M + 2 * Mkv, D).to(dt)
    t["k"], t["v"] = packed[:, M:M + Mkv], packed[:, M + Mkv:]
    t["pos"] = torch.cat([torch.arange(n - new, n) for n, new in lengths]).float()[:, None].cuda()
    t["freqs"] = _rotation(case)
    return t


def prepare(case, seed):
    return {"case": dict(case), **_inputs(case, seed)}


# ---------------------------------------------------------------- plain forms (fp32)


def _values(codes, scale):
    """What 8-bit codes stand for, in bf16."""
    out = torch.empty(codes.shape, dtype=torch.bfloat16, device=codes.device)
    return torch.mul(codes, scale.reshape(scale.shape + (1,) * (codes.dim() - scale.dim())), out=out)


def _plain_codes(x, scale):
    """x in steps of `scale`, the nearest code, even ones where two are as near; zeros where the scale is 0."""
    inverse = torch.where(scale > 0, torch.ones_like(scale) / scale, torch.zeros_like(scale))
    return torch.round(x * inverse).clamp(-127, 127).to(torch.int8)


def _plain_rms(s, step):
    x = s["x"].float()
    if s["residual"] is not None:
        x = x + s["residual"].float()
    dt = s["x"].dtype
    rstd = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)
    if not step:
        y = x * s["weight"]
        scale = y.abs().amax(-1, keepdim=True) * (1 / 127)
        return _values(_plain_codes(y, scale), (scale * rstd)[:, 0]), (scale * rstd)[:, 0], x.to(dt)
    xhat = x * rstd
    out = (xhat * s["weight"]).to(dt)
    g = s["gout"].float()
    gw = g * s["weight"]
    gx = rstd * (gw - xhat * (gw * xhat).mean(-1, keepdim=True))
    return out, rstd[:, 0], gx.to(dt), (g * xhat).sum(0)


def _plain_mm(s, case):
    a, b = s["x"].float(), s["w"].float()
    if case["codes"]:
        scale = s["x_scale"][:, None]
    else:
        scale = a.abs().amax(-1, keepdim=True) * (1 / 127)
        a = _plain_codes(a, scale).float()
    # runs of 1024 products of two codes are whole numbers that fp32 holds; their sums are taken in 64 bits
    run = 1024
    more = -case["K"] % run
    a, b = (torch.nn.functional.pad(y, (0, more)).reshape(y.shape[0], -1, run).transpose(0, 1).contiguous() for y in (a, b))
    total = torch.matmul(a, b.transpose(1, 2).contiguous()).double().sum(0).float()
    out = total * (scale * s["w_scale"])
    if s["bias"] is not None:
        out = out + s["bias"]
    return out.to(DTYPES[case["dtype"]])


def _plain_places(s, case, T):
    """Of every new token: its sequence, its place in it; and the first new place of each sequence."""
    start = s["start"] if s["start"] is not None else torch.arange(case["N"] + 1, device="cuda")
    t = torch.arange(T, device="cuda")
    n = (t[:, None] >= start[None, 1:]).sum(1)
    first = s["length"] - (start[1:] - start[:-1])
    return n, first[n] + t - start[n], first


def _plain_rotate(x, pos, freqs, interleaved):
    angle = (pos.double()[:, :, None] * freqs.double()).sum(1)  # far positions: in 64 bits
    c, s = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    R = freqs.shape[1]
    a, b = (slice(0, 2 * R, 2), slice(1, 2 * R, 2)) if interleaved else (slice(0, R), slice(R, 2 * R))
    y = x.float().clone()
    xa, xb = x[..., a].float(), x[..., b].float()
    y[..., a] = xa * c - xb * s
    y[..., b] = xa * s + xb * c
    return y


def _plain_append(s, case):
    P, width = case["page"], s["table"].shape[1]
    T = s["k"].shape[0]
    n, place, first = _plain_places(s, case, T)
    page = s["table"][n, place // P].long()
    slots = torch.arange(P, device="cuda")
    # the pages that new tokens reach, and how many of their tokens were there
    column = torch.arange(width, device="cuda")[None] * P
    reached = (column + P > first[:, None]) & (column < s["length"][:, None])
    before = (first[:, None] - column).clamp(0, P)[reached]
    pages = s["table"][reached].long()
    got = []
    for x, values in (("k", _plain_rotate(s["k"], s["pos"], s["freqs"], case["interleaved"])), ("v", s["v"].float())):
        codes, scale = s[x + "_cache"], s[x + "_scale"]
        old = torch.where((before > 0)[:, None], scale[pages], torch.zeros_like(scale[pages]))
        most = torch.zeros_like(scale)
        most.index_reduce_(0, page, values.abs().amax(-1), "amax")
        new = torch.maximum(old, most[pages] * (1 / 127))
        ratio = torch.where(new > 0, old / new, torch.zeros_like(new))
        held = codes[pages]
        again = torch.round(held.float() * ratio[:, :, None, None]).to(torch.int8)
        codes[pages] = torch.where((slots[None] < before[:, None])[:, None, :, None], again, held)
        scale[pages] = new
        codes[page, :, place % P] = _plain_codes(values, scale[page][..., None])
        got += [_values(codes, scale), scale]
    return tuple(got)


def _plain_attn(s, case):
    N, M, Mkv, D, P = (case[k] for k in ("N", "M", "Mkv", "D", "page"))
    T, G, Lq = s["q"].shape[0], M // Mkv, case["new"]
    n, place, first = _plain_places(s, case, T)
    i = place - first[n]
    pages = s["table"].long()

    def held(codes, scale):  # [N, Mkv, keys, D]
        x = codes[pages].float() * scale[pages][..., None, None]
        return x.transpose(1, 2).reshape(N, Mkv, -1, D)

    k, v = held(s["k_cache"], s["k_scale"]), held(s["v_cache"], s["v_scale"])
    q = torch.zeros((N, Lq, Mkv, G, D), device="cuda")
    q[n, i] = s["q"].float().reshape(T, Mkv, G, D)
    q = q.permute(0, 2, 3, 1, 4).reshape(N, Mkv, G * Lq, D)
    z = torch.matmul(q, k.transpose(2, 3).contiguous()) * (1.0 / math.sqrt(D))
    if case["softcap"]:
        z = case["softcap"] * torch.tanh(z / case["softcap"])
    z = z.reshape(N, Mkv, G, Lq, -1)
    last = first[:, None] + torch.arange(Lq, device="cuda")
    seen = (torch.arange(z.shape[-1], device="cuda") <= last[..., None]) & (last < s["length"][:, None])[..., None]
    z = z.masked_fill(~seen[:, None, None], -math.inf)
    top = z.amax(-1, keepdim=True)
    p = torch.exp(z - torch.where(torch.isinf(top), torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    lse = (torch.log(total) + top)[..., 0]
    p = p / torch.where(total > 0, total, torch.ones_like(total))
    o = torch.matmul(p.reshape(N, Mkv, G * Lq, -1), v).reshape(N, Mkv, G, Lq, D)
    return o.permute(0, 3, 1, 2, 4)[n, i].reshape(T, M, D).to(s["q"].dtype), lse.permute(0, 3, 1, 2)[n, i].reshape(T, M)


# ---------------------------------------------------------------- one pass


def run(s):
    if own:
        return _own(s)
    case = s["case"]
    if case["op"].startswith("rms"):
        return _plain_rms(s, case["op"] == "rms_step")
    if case["op"] == "mm":
        return _plain_mm(s, case)
    return _plain_append(s, case) if case["op"] == "append" else _plain_attn(s, case)


def _own(s):
    from paper_2505_14022_amd import msda

    case, op = s["case"], s["case"]["op"]
    if op == "rms_quantize":
        codes, scale, total = msda.rmsnorm_quantize(s["x"], s["weight"], residual=s["residual"], eps=EPS, want_sum=True)
        return _values(codes, scale), scale, total
    if op == "rms_step":
        out, rstd = msda.rmsnorm_forward(s["x"], s["weight"], residual=s["residual"], eps=EPS)
        return (out, rstd) + tuple(msda.rmsnorm_backward(s["x"], s["gout"], rstd, s["weight"], residual=s["residual"]))
    if op == "mm":
        codes, scale = (s["x"], s["x_scale"]) if case["codes"] else msda.quantize_rows(s["x"])
        return msda.quantized_matmul(codes, s["w"], scale, s["w_scale"], bias=s["bias"], dtype=DTYPES[case["dtype"]])
    cache = [s[x] for x in ("k_cache", "v_cache", "k_scale", "v_scale", "table", "length")]
    if op == "append":
        msda.cache_append(s["k"], s["v"], *cache, start=s["start"], pos=s["pos"], freqs=s["freqs"],
                          interleaved=case["interleaved"])
        return (_values(s["k_cache"], s["k_scale"]), s["k_scale"], _values(s["v_cache"], s["v_scale"]), s["v_scale"])
    return msda.cache_attention(s["q"], *cache, start=s["start"], softcap=case["softcap"])


# ---------------------------------------------------------------- floors and 64-bit results


def work(case):
    """Each input read once and each output written once; pages that new tokens do not reach are not read."""
    es = 4 if case["dtype"] == "f32" else 2
    op = case["op"]
    if op.startswith("rms"):
        n = case["rows"] * case["C"]
        if op == "rms_step":
            return {"bytes": (4 + case["residual"]) * n * es + 4 * case["rows"] + 8 * case["C"], "flops": n * 15}
        return {"bytes": (2 + case["residual"]) * n * es + n + 4 * case["rows"] + 4 * case["C"], "flops": n * 7}
    if op == "mm":
        T, K, O = case["T"], case["K"], case["O"]
        return {"bytes": T * K * (1 if case["codes"] else es) + O * K + T * O * es + 4 * O * (1 + case["bias"]), "flops": 2 * T * K * O}
    N, M, Mkv, D, P = (case[k] for k in ("N", "M", "Mkv", "D", "page"))
    lengths = _lengths(case)
    T = sum(new for _, new in lengths)
    if op == "append":
        old = sum((total - new) % P for total, new in lengths)  # tokens that stood in pages that new ones reach
        pages = sum(-(-total // P) - (total - new) // P for total, new in lengths)
        return {"bytes": 2 * (T * Mkv * D * (es + 1) + 2 * old * Mkv * D + 8 * pages * Mkv) + 8 * T, "flops": T * Mkv * D * 10}
    keys = sum(total for total, _ in lengths)
    pairs = sum(new * total - new * (new - 1) // 2 for total, new in lengths)
    return {"bytes": 2 * T * M * D * es + 4 * T * M + 2 * keys * Mkv * D + 12 * (keys // P) * Mkv, "flops": 4 * pairs * M * D}


def exact(case, seed):
    """run()'s outputs in 64 bits, from the definitions; gradients by automatic differentiation."""
    t, op = _inputs(case, seed), case["op"]
    if op.startswith("rms"):
        step = op == "rms_step"
        x, w = t["x"].double().requires_grad_(step), t["weight"].double().requires_grad_(step)
        total = x if t["residual"] is None else x + t["residual"].double()
        rstd = (total.square().sum(1) / case["C"] + EPS).pow(-0.5)
        y = total * rstd[:, None] * w
        if step:
            return (y.detach(), rstd.detach()) + torch.autograd.grad(y, (x, w), t["gout"].double())
        scale = y.abs().max(1).values / 127
        return torch.round(y / scale[:, None]) * scale[:, None], scale, total
    if op == "mm":
        codes = t["x"].double()
        if case["codes"]:
            scale = t["x_scale"].double()
        else:
            scale = codes.abs().max(1).values / 127
            codes = torch.round(codes / scale[:, None])
        y = (codes * scale[:, None]) @ (t["w"].double() * t["w_scale"].double()[:, None]).t().contiguous()
        return y if t["bias"] is None else y + t["bias"].double()
    N, M, Mkv, D, P = (case[k] for k in ("N", "M", "Mkv", "D", "page"))
    lengths, table, at = _lengths(case), t["table"].long().cpu(), 0
    if op == "append":
        turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), t["pos"].double() * t["freqs"].double())[:, None]
        k = t["k"].double()
        if case["interleaved"]:
            k = torch.view_as_real(torch.view_as_complex(k.reshape(k.shape[:2] + (-1, 2)).contiguous()) * turn).flatten(2)
        else:
            z = torch.complex(k[..., :D // 2].contiguous(), k[..., D // 2:].contiguous()) * turn
            k = torch.cat([z.real, z.imag], -1)
        got = []
        for x, new_values in (("k", k), ("v", t["v"].double())):
            codes, scale, at = t[x + "_cache"].double(), t[x + "_scale"].double(), 0
            for n, (total, new) in enumerate(lengths):
                place = total - new
                while place < total:  # a page at a time
                    stop, slot = min(total, (place // P + 1) * P), place % P
                    page = int(table[n, place // P])
                    mine = new_values[at:at + stop - place]
                    was = scale[page] if slot else torch.zeros_like(scale[page])
                    now = torch.maximum(was, mine.abs().amax((0, 2)) / 127)
                    codes[page, :, :slot] = torch.round(codes[page, :, :slot] * (was / now)[:, None, None])
                    codes[page, :, slot:slot + stop - place] = torch.round(mine.transpose(0, 1) / now[:, None, None])
                    scale[page] = now
                    at, place = at + stop - place, stop
            got += [codes * scale[..., None, None], scale]
        return tuple(got)
    out, lse = [], []
    for n, (total, new) in enumerate(lengths):
        pages = table[n, :-(-total // P)].cuda()

        def held(codes, scale):  # [Mkv, total, D]
            return (codes[pages].double() * scale[pages].double()[..., None, None]).transpose(0, 1).reshape(Mkv, -1, D)[:, :total]

        k, v = held(t["k_cache"], t["k_scale"]), held(t["v_cache"], t["v_scale"])
        q = t["q"][at:at + new].double().transpose(0, 1)  # [M, new, D]
        at += new
        later = torch.arange(total, device="cuda")[None] > torch.arange(total - new, total, device="cuda")[:, None]
        for h in range(M):  # one head at a time: the scores of all would not fit
            z = q[h] @ k[h // (M // Mkv)].t().contiguous() / math.sqrt(D)
            if case["softcap"]:
                z = torch.tanh(z / case["softcap"]) * case["softcap"]
            z[later] = -math.inf
            lse.append(torch.logsumexp(z, -1))
            out.append(torch.softmax(z, -1) @ v[h // (M // Mkv)])
    new = [m for _, m in lengths]
    join = lambda xs: torch.cat([torch.stack(xs[M * n:M * (n + 1)], 1) for n in range(len(new))])  # noqa: E731
    return join(out), join(lse)
