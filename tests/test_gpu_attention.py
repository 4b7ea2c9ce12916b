"""GPU parity of msda_attention_forward / msda_attention_backward with 64-bit attention, within bounds derived from
the arithmetic (tests/layer_ref.py): sizes around the tiles, head layouts, masks, strides, padding that holds
anything, streams, graphs and gradients against differences."""
import pytest

import layer_ref
from layer_ref import DT, assert_within
from paper_2505_14022_amd import msda
from gpu_util import require_gpu, say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    require_gpu()


def make(N, Lq, Lk, M, Mkv, D, dtype, seed=0, spread=1.0):
    import torch

    g = torch.Generator().manual_seed(seed)

    def normal(*shape):
        return (torch.randn(*shape, generator=g) * spread).to(DT[dtype]).cuda()

    return normal(N, Lq, M, D), normal(N, Lk, Mkv, D), normal(N, Lk, Mkv, D), normal(N, Lq, M, D)


def masks_of(N, Lq, Lk, M, docs="none", prefix=None, causal=False, softcap=0.0, bias=False, seed=0):
    """Keyword arguments of a call. docs: "pad" (ends of different lengths), "runs" (documents one after another, the
    last run padding), "mixed" (documents in any order, padding among them), "one" (one document)."""
    import torch

    g = torch.Generator().manual_seed(1000 + seed)
    how = {"causal": causal, "softcap": softcap}
    if docs != "none":
        L = max(Lq, Lk)
        if docs == "pad":
            t = torch.zeros(N, L, dtype=torch.int32)
            for n in range(N):
                t[n, int(torch.randint(0, L + 1, (1,), generator=g)):] = -1
        elif docs == "runs":
            step = max(1, L // 4)
            t = (torch.arange(L, dtype=torch.int32) // step)[None].repeat(N, 1)
            t[t == int(t.max())] = -1 if L > 4 else 0
        elif docs == "mixed":
            t = torch.randint(-1, 4, (N, L), generator=g).int()
        else:
            t = torch.full((N, L), 5, dtype=torch.int32)
        how["q_doc"], how["k_doc"] = t[:, :Lq].contiguous().cuda(), t[:, :Lk].contiguous().cuda()
    if prefix is not None:
        how["prefix"] = torch.tensor([prefix + n for n in range(N)], dtype=torch.int32, device="cuda")
    if bias:
        how["slopes"] = (torch.rand(M, generator=g) * 2).cuda()
        how["q_pos"], how["k_pos"] = torch.rand(N, Lq, 2, generator=g).cuda() * 3, torch.rand(N, Lk, 2, generator=g).cuda() * 3
    return how


def check(q, k, v, go, how, scale=None, backward=True, stream=None, few_keys=False):
    ref = layer_ref.attention(q, k, v, scale=scale, grad_out=go if backward else None, few_keys=few_keys, **how)
    out, lse = msda.attention_forward(q, k, v, scale=scale, stream=stream, **how)
    got = {"out": out, "lse": lse}
    if backward:
        grads = msda.attention_backward(q, k, v, out, lse, go, scale=scale, stream=stream, **how)
        got.update(zip(("grad_q", "grad_k", "grad_v"), grads))
    if stream is not None:
        stream.synchronize()
    for name, (value, bound) in ref.items():
        assert_within(name, got[name], value, bound)
    return got


SIZES = [
    # N, Lq, Lk, M, Mkv, D
    (1, 1, 1, 1, 1, 1), (2, 1, 33, 4, 1, 8), (1, 2, 31, 2, 2, 20), (1, 31, 32, 3, 3, 32), (2, 32, 63, 2, 1, 33),
    (1, 33, 64, 6, 2, 48), (1, 64, 65, 1, 1, 64), (2, 65, 127, 2, 2, 100), (1, 127, 129, 2, 1, 128),
    (1, 300, 300, 2, 2, 32), (1, 129, 40, 8, 1, 64), (3, 17, 500, 4, 4, 96),
    (1, 1, 3001, 8, 2, 128),   # one token: the keys are split
    (1, 700, 9, 4, 1, 32),     # few keys: the rows are split in the backward
    (1, 40, 2050, 3, 1, 64), (2, 520, 520, 1, 1, 16),
]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "N%d_Lq%d_Lk%d_M%d_Mkv%d_D%d" % s)
def test_attention_sizes(size, dtype):
    say(f"attention {size} {dtype}")
    N, Lq, Lk, M, Mkv, D = size
    check(*make(*size, dtype, seed=Lq + Lk), masks_of(N, Lq, Lk, M))


MASKS = [
    dict(causal=True), dict(causal=True, prefix=5), dict(docs="pad"), dict(docs="runs"), dict(docs="runs", causal=True),
    dict(docs="mixed"), dict(docs="mixed", prefix=9), dict(docs="mixed", prefix=70, causal=True), dict(docs="one", prefix=3),
    dict(docs="pad", prefix=500), dict(docs="runs", prefix=-4, causal=True), dict(softcap=3.0), dict(bias=True),
    dict(softcap=2.0, bias=True, docs="runs", prefix=6, causal=True), dict(prefix=5),
]


@pytest.mark.parametrize("dtype,D", [("f32", 32), ("f32", 128), ("f16", 64), ("bf16", 32), ("bf16", 128)])
@pytest.mark.parametrize("mask", MASKS, ids=lambda m: "-".join(f"{k}{v}" for k, v in m.items()))
def test_attention_masks(mask, dtype, D):
    say(f"attention masks {mask} {dtype} D={D}")
    for N, Lq, Lk, M, Mkv in ((2, 150, 150, 2, 1), (2, 1, 200, 4, 2), (2, 70, 330, 2, 2)):
        check(*make(N, Lq, Lk, M, Mkv, D, dtype, seed=Lk), masks_of(N, Lq, Lk, M, **mask, seed=Lk))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_of_groups_with_a_common_prefix(dtype):
    # a decoder's self-attention: matching queries, and denoising groups that see them and themselves
    import torch

    say(f"attention of denoising groups {dtype}")
    doc = torch.cat([torch.zeros(100), 1 + torch.arange(200) // 40]).int()[None].repeat(2, 1)
    doc[1, 260:] = -1
    how = {"q_doc": doc.cuda(), "k_doc": doc.cuda(), "prefix": torch.full((2,), 100, dtype=torch.int32, device="cuda")}
    seen = layer_ref.seen_pairs(2, 300, 300, **how)
    assert not seen[:, :100, 100:].any() and seen[0, 100:, :100].all() and not seen[1, 260:].any()
    check(*make(2, 300, 300, 2, 2, 32, dtype, seed=1), how)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_attention_rows_that_see_nothing(dtype):
    import torch

    say(f"attention rows that see nothing, {dtype}")
    q, k, v, go = make(2, 70, 90, 2, 1, 32, dtype, seed=2)
    how = masks_of(2, 70, 90, 2)
    how["q_doc"] = torch.full((2, 70), 1, dtype=torch.int32, device="cuda")
    how["k_doc"] = torch.full((2, 90), 1, dtype=torch.int32, device="cuda")
    how["q_doc"][0, 5:50] = 2  # a document without keys
    how["k_doc"][1] = -1       # a batch item without keys
    got = check(q, k, v, go, how)
    assert float(got["out"][0, 5:50].abs().max()) == 0 and float(got["grad_q"][1].abs().max()) == 0
    assert bool(torch.isneginf(got["lse"][0, :, 5:50]).all()) and bool(torch.isneginf(got["lse"][1]).all())
    assert float(got["grad_k"][1].abs().max()) == 0 and float(got["grad_v"][1].abs().max()) == 0


BAD = [float("nan"), float("inf"), float("-inf")]


@pytest.mark.parametrize("D", [32, 128])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_attention_padding_may_hold_anything(dtype, D):
    say(f"attention with infinities and NaN in the padding, {dtype} D={D}")
    q, k, v, go = make(2, 140, 140, 4, 2, D, dtype, seed=3)
    how = masks_of(2, 140, 140, 4, docs="mixed", prefix=10, bias=True)
    pad = how["q_doc"] < 0
    for i, t in enumerate((q, k, v, go)):
        t[pad] = BAD[i % 3]
    how["q_pos"][pad] = float("nan")
    how["k_pos"][pad] = float("inf")
    check(q, k, v, go, how)


@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_attention_of_a_document_with_infinities_leaves_the_others(dtype, D):
    import torch

    say(f"attention with infinities and NaN in one document, {dtype} D={D}")
    q, k, v, go = make(1, 120, 120, 2, 1, D, dtype, seed=4)
    doc = (torch.arange(120) // 25 % 3).int()[None].cuda()
    how = {"q_doc": doc, "k_doc": doc}
    mine = (doc[0] == 1).cpu()
    for i, t in enumerate((q, k, v, go)):
        t[:, mine.cuda()] = BAD[i % 3]
    ref = layer_ref.attention(q, k, v, grad_out=go, **how)  # the document's own values mean nothing there
    out, lse = msda.attention_forward(q, k, v, **how)
    grads = msda.attention_backward(q, k, v, out, lse, go, **how)
    for name, t in zip(("out", "grad_q", "grad_k", "grad_v"), (out,) + grads):
        assert_within(name, t[:, ~mine.cuda()], ref[name][0][:, ~mine], ref[name][1][:, ~mine])
    # the order rule: a NaN in the future reaches nobody before it, and everybody from it on
    q, k, v, go = make(1, 120, 120, 2, 1, D, dtype, seed=5)
    v[:, 77, 0, D // 2] = float("nan")
    clean = torch.nan_to_num(v)
    out = msda.attention_forward(q, k, v, causal=True)[0]
    ref = layer_ref.attention(q, k, clean, causal=True)["out"]
    assert_within("out", out[:, :77], ref[0][:, :77], ref[1][:, :77])
    assert bool(torch.isnan(out[:, 77:, :, D // 2]).all())
    rest = [d for d in range(D) if d != D // 2]
    assert_within("out", out[..., rest], ref[0][..., rest], ref[1][..., rest])
    # an infinite query, key and gradient of a row whose keys the others see as well
    for which in range(3):
        q, k, v, go = make(1, 120, 120, 2, 1, D, dtype, seed=6)
        out, lse = msda.attention_forward(q, k, v, causal=True)
        t = (q, k, go)[which]
        t[:, 100] = BAD[which]
        gq, gk, gv = msda.attention_backward(q, k, v, out, lse, go, causal=True)
        ref = layer_ref.attention(q, k, v, causal=True, grad_out=go)
        if which == 1:  # key 100 is not seen by the rows before it
            assert_within("grad_q", gq[:, :100], ref["grad_q"][0][:, :100], ref["grad_q"][1][:, :100])
        else:           # row 100 does not see the keys after it
            for name, g in (("grad_k", gk), ("grad_v", gv)):
                assert_within(name, g[:, 101:], ref[name][0][:, 101:], ref[name][1][:, 101:])


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_attention_scores_of_any_size(dtype):
    # scores up to some hundreds: one key takes nearly all, the running maximum moves
    say(f"attention with large scores {dtype}")
    q, k, v, go = make(1, 96, 400, 2, 2, 64, dtype, seed=7, spread=5.0)
    check(q, k, v, go, {})
    check(q, k, v, go, {"softcap": 30.0}, scale=1.0)
    check(q * 0, k, v, go, {}, scale=1e-3)


@pytest.mark.parametrize("dtype,D", [("f32", 48), ("bf16", 64), ("f16", 20)])
def test_attention_of_views(dtype, D):
    import torch

    say(f"attention of strided and unaligned views {dtype}")
    g = torch.Generator().manual_seed(8)
    qkv = torch.randn(2, 90, 3, 4, D, generator=g).to(DT[dtype]).cuda()
    go = torch.randn(2, 90, 4, D, generator=g).to(DT[dtype]).cuda()
    check(qkv[:, :, 0], qkv[:, :, 1], qkv[:, :, 2], go, masks_of(2, 90, 90, 4, causal=True))
    # a cache longer than what is in it, heads before tokens, an odd offset; keys and values shared by the batch
    cache = torch.randn(2, 2, 200, D + 1, generator=g).to(DT[dtype]).cuda()
    k = cache[0, :, :, 1:].transpose(0, 1)[None, :150].expand(2, 150, 2, D)
    v = cache[1, :, :, :D].transpose(0, 1)[None, :150].expand(2, 150, 2, D)
    check(qkv[:, 10:50, 0], k, v, go[:, :40].contiguous(), masks_of(2, 40, 150, 4, docs="pad"))


def test_attention_of_a_cache_past_32_bits():
    # 300 tokens 16 MB apart: offsets of 2.5e9 elements
    import torch

    say("attention of keys whose offsets pass 32 bits")
    step = 1 << 23
    cache = torch.empty(300 * step + 256, dtype=torch.bfloat16, device="cuda")
    k, v = (cache[o:].as_strided((1, 300, 2, 64), (300 * step, step, 64, 1)) for o in (0, 128))
    q, kk, vv, go = make(1, 3, 300, 4, 2, 64, "bf16", seed=9)
    k.copy_(kk)
    v.copy_(vv)
    check(q, k, v, go, {"causal": True})


def test_attention_empty_extents():
    import torch

    say("attention of no queries or no keys")
    q, k, v, go = make(2, 5, 0, 4, 2, 32, "bf16")
    out, lse = msda.attention_forward(q, k, v)
    assert float(out.abs().max()) == 0 and bool(torch.isneginf(lse).all())
    gq, gk, gv = msda.attention_backward(q, k, v, out, lse, go, grad_q=torch.full_like(q, 7.0))
    assert float(gq.abs().max()) == 0 and gk.numel() == 0
    q, k, v, go = make(2, 0, 70, 4, 2, 32, "f32")
    out, lse = msda.attention_forward(q, k, v)
    gq, gk, gv = msda.attention_backward(q, k, v, out, lse, go, grad_k=torch.full_like(k, 7.0))
    assert out.numel() == 0 and float(gk.abs().max()) == 0 and float(gv.abs().max()) == 0


def test_attention_writes_its_outputs_and_nothing_else():
    import torch

    say("attention between guards")
    q, k, v, go = make(2, 37, 71, 3, 3, 20, "f16", seed=10)
    how = masks_of(2, 37, 71, 3, docs="mixed")
    ref = layer_ref.attention(q, k, v, grad_out=go, **how)

    def guarded(shape, dtype):
        n = 1
        for x in shape:
            n *= x
        pad = 64
        flat = torch.full((n + 2 * pad,), float("nan"), dtype=dtype, device="cuda")
        return flat, flat[pad:pad + n].view(shape)

    bufs = [guarded(s, d) for s, d in ((q.shape, q.dtype), ((2, 3, 37), torch.float32), (q.shape, q.dtype),
                                       (k.shape, q.dtype), (k.shape, q.dtype))]
    out, lse, gq, gk, gv = (b[1] for b in bufs)
    wf = torch.empty(msda.attention_workspace_size(q, k, v, **how), dtype=torch.uint8, device="cuda")
    wb = torch.empty(msda.attention_workspace_size(q, k, v, backward=True, **how), dtype=torch.uint8, device="cuda")
    msda.attention_forward(q, k, v, out=out, lse=lse, workspace=wf, **how)
    msda.attention_backward(q, k, v, out, lse, go, grad_q=gq, grad_k=gk, grad_v=gv, workspace=wb, **how)
    for name, t in zip(("out", "lse", "grad_q", "grad_k", "grad_v"), (out, lse, gq, gk, gv)):
        assert_within(name, t, *ref[name])
    for flat, view in bufs:
        assert bool(torch.isnan(flat[:64]).all()) and bool(torch.isnan(flat[-64:]).all())
    assert msda.attention_forward(q, k, v, want_lse=False, **how)[1] is None
    with pytest.raises(msda.MsdaError, match="workspace"):
        msda.attention_forward(q, k, v, workspace=wf[:-256], **how)


def test_attention_is_reproducible_and_takes_any_stream():
    import torch

    say("attention on two streams at once")
    q, k, v, go = make(1, 200, 1500, 4, 2, 64, "bf16", seed=11)
    how = masks_of(1, 200, 1500, 4, docs="runs", causal=True, bias=True)
    first = check(q, k, v, go, how)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = []
    for s in streams * 2:
        out, lse = msda.attention_forward(q, k, v, stream=s, **how)
        got.append((out, lse) + msda.attention_backward(q, k, v, out, lse, go, stream=s, **how))
    torch.cuda.synchronize()
    for res in got:
        for name, t in zip(("out", "lse", "grad_q", "grad_k", "grad_v"), res):
            assert torch.equal(t, first[name]), name


def test_attention_gradients_against_differences():
    import torch

    say("attention's gradients against differences")
    q, k, v, go = make(1, 20, 24, 2, 1, 16, "f32", seed=12)
    how = masks_of(1, 20, 24, 2, docs="runs", prefix=3, causal=True, softcap=2.0, bias=True)
    out, lse = msda.attention_forward(q, k, v, **how)
    grads = msda.attention_backward(q, k, v, out, lse, go, **how)
    noise = float((layer_ref.attention(q, k, v, **how)["out"][1] * go.cpu().double().abs()).sum())

    def loss(d, e):
        o = msda.attention_forward(*(t + e * x for t, x in zip((q, k, v), d)), **how)[0]
        return float((o.double() * go.double()).sum())

    for seed in range(3):
        g = torch.Generator().manual_seed(seed)
        d = [torch.randn(t.shape, generator=g).cuda() for t in (q, k, v)]
        slope = sum(float((x.double() * y.double()).sum()) for x, y in zip(grads, d))
        e = 2.0 ** -8
        d1, d2 = ((loss(d, h) - loss(d, -h)) / (2 * h) for h in (e, e / 2))
        # a halved step leaves a quarter of the truncation; the rest is the outputs' rounding
        assert abs(d2 - slope) <= abs(d1 - d2) + 8 * noise / e, (d1, d2, slope)


FEW = [
    # N, Lq, Lk, M, Mkv, D, masks
    (1, 2, 2, 8, 2, 48, {}),
    (2, 2, 2, 4, 4, 32, {"causal": True}),
    (1, 1, 2, 8, 2, 128, {"docs": "pad"}),
    (2, 3, 5, 4, 2, 64, {"causal": True, "softcap": 4.0}),
    (1, 9, 7, 2, 1, 16, {"bias": True, "softcap": 4.0}),
    (1, 64, 64, 2, 2, 96, {"causal": True}),
    (3, 260, 260, 2, 1, 64, {"step": 4}),
    (1, 260, 260, 3, 3, 128, {"step": 4, "causal": True, "softcap": 9.0}),
    (1, 512, 512, 2, 2, 32, {"step": 8, "causal": True}),
]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("case", FEW, ids=lambda c: "-".join(map(str, c[:6])))
def test_attention_gradients_of_rows_with_few_keys(case, dtype):
    """Short rows: their gradients are off by their own roundings and not by that of out."""
    import torch

    N, Lq, Lk, M, Mkv, D, masks = case
    masks = dict(masks)
    step = masks.pop("step", 0)
    how = masks_of(N, Lq, Lk, M, **masks)
    if step:  # documents of `step` rows
        how["q_doc"] = how["k_doc"] = (torch.arange(Lq, dtype=torch.int32) // step)[None].repeat(N, 1).contiguous().cuda()
    q, k, v, go = make(N, Lq, Lk, M, Mkv, D, dtype)
    check(q, k, v, go, how, few_keys=True)
