"""Calls of msda_attention_forward / msda_attention_backward at the edges of what the header allows, against 64-bit
attention (tests/layer_ref.py)."""
import pytest

import layer_ref
from layer_ref import assert_within
from paper_2505_14022_amd import msda
from gpu_util import require_gpu, say
from test_gpu_attention import check, make, masks_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    require_gpu()


@pytest.mark.parametrize("prefix", [None, 9])
@pytest.mark.parametrize("dtype,D", [("f32", 32), ("f16", 64), ("bf16", 32), ("bf16", 128)])
def test_attention_any_negative_document_is_padding(dtype, D, prefix):
    import torch

    say(f"attention with documents of -2, -3 and the lowest integer, {dtype} D={D} prefix {prefix}")
    for N, Lq, Lk, M, Mkv in ((2, 150, 150, 2, 1), (2, 1, 200, 4, 2), (2, 70, 330, 2, 2)):
        how = masks_of(N, Lq, Lk, M, docs="mixed", prefix=prefix, seed=Lk)
        g = torch.Generator().manual_seed(Lk)
        for name in ("q_doc", "k_doc"):
            t = how[name].cpu()
            low = torch.tensor([-1, -2, -3, -2 ** 31])[torch.randint(0, 4, t.shape, generator=g)].int()
            how[name] = torch.where(t < 0, low, t).cuda()
        if Lq == 1:
            how["q_doc"].fill_(1)
        check(*make(N, Lq, Lk, M, Mkv, D, dtype, seed=Lk), how)
    # one document and its padding
    how = masks_of(1, 90, 90, 2, docs="one", prefix=prefix)
    how["q_doc"][:, 70:] = how["k_doc"][:, 70:] = -2
    check(*make(1, 90, 90, 2, 2, D, dtype, seed=1), how)


@pytest.mark.parametrize("dtype,D", [("f32", 32), ("f16", 64), ("bf16", 64), ("bf16", 128), ("bf16", 32)])
def test_attention_padding_before_a_last_tile_in_part(dtype, D):
    # padded queries at places that are no numbers, in the tile before the one that ends behind the last row
    import torch

    say(f"attention of left-padded queries without places, {dtype} D={D}")
    for L in (70, 134, 200):
        how = masks_of(1, L, L, 1, docs="one", bias=True)
        how["q_doc"][:, :20] = -1
        for bad in (float("nan"), float("inf")):
            how["q_pos"][:, :20] = bad
            check(*make(1, L, L, 1, 1, D, dtype, seed=L), how)


def _without_key(L, M, key):
    import torch

    doc = torch.zeros(1, L, dtype=torch.int32, device="cuda")
    k_doc = doc.clone()
    k_doc[:, key] = -1
    return {"q_doc": doc, "k_doc": k_doc}


@pytest.mark.parametrize("dtype,D", [("f32", 32), ("f16", 64), ("bf16", 32), ("bf16", 128)])
def test_attention_of_a_key_that_all_score_minus_infinity(dtype, D):
    # such a key has no weight: grad_k and grad_v of all keys are as if it were padding
    say(f"attention of a key with a score of minus infinity, {dtype} D={D}")
    L, M, key, c = 70, 2, 37, 5
    q, k, v, go = make(1, L, L, M, M, D, dtype, seed=3)
    q[..., c] = q[..., c].abs() + 0.25
    k[:, key, :, c] = float("-inf")
    ref = layer_ref.attention(q, k, v, grad_out=go, **_without_key(L, M, key))
    out, lse = msda.attention_forward(q, k, v)
    _, gk, gv = msda.attention_backward(q, k, v, out, lse, go)
    for name, t in (("out", out), ("lse", lse), ("grad_k", gk), ("grad_v", gv)):
        assert_within(name, t, *ref[name])


@pytest.mark.parametrize("dtype,D", [("f32", 32), ("f16", 64), ("bf16", 32), ("bf16", 128)])
def test_attention_infinities_in_a_last_tile_in_part(dtype, D):
    # the last rows and some keys of one document hold infinities; the other document's results have none
    import torch

    say(f"attention with infinities in the last rows, {dtype} D={D}")
    L = 70
    q, k, v, go = make(1, L, L, 2, 1, D, dtype, seed=4)
    doc = (torch.arange(L) >= 60).int()[None].cuda()
    how = {"q_doc": doc, "k_doc": doc, "causal": True}
    for t in (q, k, v, go):
        t[:, 65:, :, 1] = float("inf")
        t[:, 66, :, 3] = float("nan")
    ref = layer_ref.attention(q, k, v, grad_out=go, **how)
    out, lse = msda.attention_forward(q, k, v, **how)
    grads = msda.attention_backward(q, k, v, out, lse, go, **how)
    for name, t in zip(("out", "grad_q", "grad_k", "grad_v"), (out,) + grads):
        assert_within(name, t[:, :60], ref[name][0][:, :60], ref[name][1][:, :60])
    assert not bool(torch.isfinite(out[:, 66:]).all())


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("D", [20, 32, 64, 128])
def test_attention_of_one_wave_over_many_tiles(D, dtype):
    # up to 32 rows a head are one wave's, which stages every tile in the same place
    import torch

    say(f"attention of few rows over many tiles, {dtype} D={D}")
    for rows, Lk in ((1, 333), (4, 1999), (8, 640)):
        q, k, v, go = make(1, rows, Lk, 8, 2, D, dtype, seed=Lk)
        v += torch.arange(Lk, device="cuda")[None, :, None, None].to(v.dtype) % 17 - 8  # a tile read late shows
        how = masks_of(1, rows, Lk, 8, causal=True)
        first = check(q, k, v, go, how, backward=False)
        v[:, 100, 1, 3] = float("inf")  # noted by one half wave, added by both
        out = msda.attention_forward(q, k, v, **how)[0]
        assert torch.equal(out[..., :3], first["out"][..., :3]) and torch.equal(out[..., 4:], first["out"][..., 4:])
        assert bool((out[:, :, 4:, 3] == float("inf")).all()) and torch.equal(out[:, :, :4], first["out"][:, :, :4])


@pytest.mark.parametrize("softcap", [0.0, 3.0])
@pytest.mark.parametrize("dtype,D", [("f32", 32), ("f16", 64), ("bf16", 32), ("bf16", 128), ("f32", 128)])
def test_attention_masked_with_a_seen_key_of_minus_infinity(dtype, D, softcap):
    # a masked call's key that all who see it give a score of minus infinity, or of minus the cap: grad_q as without it
    # or, capped, as with a key far out; and NaN where it is seen with a score that is none
    import torch

    say(f"attention, masked, with a seen key of minus infinity, {dtype} D={D} softcap {softcap}")
    L, M, key, c = 128, 2, 37, 5
    q, k, v, go = make(1, L, L, M, M, D, dtype, seed=3)
    q[..., c] = q[..., c].abs() + 0.25
    how = {"causal": True, "softcap": softcap}
    k[:, key, :, c] = -30000.0
    ref = layer_ref.attention(q, k, v, grad_out=go, **how)
    k[:, key, :, c] = float("-inf")
    out, lse = msda.attention_forward(q, k, v, **how)
    gq, gk, gv = msda.attention_backward(q, k, v, out, lse, go, **how)
    rest = [d for d in range(D) if d != c]
    for name, t in (("out", out), ("grad_q", gq[..., rest]), ("grad_k", gk), ("grad_v", gv)):
        value, bound = ref[name]
        if name == "grad_q":
            value, bound = value[..., rest], bound[..., rest]
        if softcap == 0.0:  # from layer_ref of the call without the key: the rounding of a score of 30000 is not there
            plain = layer_ref.attention(q, k, v, grad_out=go, q_doc=torch.zeros(1, L).int(), softcap=softcap, causal=True,
                                        k_doc=-(torch.arange(L) == key).int()[None])
            value, bound = plain[name]
            if name == "grad_q":
                value, bound = value[..., rest], bound[..., rest]
        assert_within(name, t, value, bound)
    q[:, 100:, :, c] = -q[:, 100:, :, c]  # a score of plus infinity from query 100 on
    out, lse = msda.attention_forward(q, k, v, **how)
    gq = msda.attention_backward(q, k, v, out, lse, go, **how)[0]
    if softcap == 0.0:
        assert bool(torch.isnan(gq[:, 100:]).all()) and bool(torch.isfinite(gq[:, :100][..., rest]).all())
    else:
        assert bool(torch.isfinite(gq[..., rest]).all())


@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("dtype,D", [("f32", 32), ("f16", 64), ("bf16", 32), ("bf16", 128), ("f32", 48)])
def test_attention_masked_and_capped_with_an_infinite_query(dtype, D, bias):
    # its scores are plus and minus the cap, its weights numbers: as with a query far out
    say(f"attention, masked and capped, with an infinite query, {dtype} D={D} bias {bias}")
    L, M, row, c = 128, 2, 90, 5
    q, k, v, go = make(1, L, L, M, M, D, dtype, seed=5)
    k[..., c] += k[..., c].sign() * 0.25
    how = masks_of(1, L, L, M, docs="runs", causal=True, softcap=2.0, bias=bias)
    q[:, row, :, c] = 30000.0
    ref = layer_ref.attention(q, k, v, grad_out=go, **how)
    q[:, row, :, c] = float("inf")
    out, lse = msda.attention_forward(q, k, v, **how)
    gq, gk, gv = msda.attention_backward(q, k, v, out, lse, go, **how)
    rest = [d for d in range(D) if d != c]
    for name, t in (("out", out), ("lse", lse), ("grad_q", gq), ("grad_v", gv)):
        assert_within(name, t, *ref[name])
    assert_within("grad_k", gk[..., rest], *(x[..., rest] for x in ref["grad_k"]))


SHORT = [
    # rows, documents' lengths from the first row on (the last is repeated), masks
    (300, [1, 2], dict(causal=True)),                 # pairs that lie across blocks and tiles
    (300, [1, 3], dict()),
    (400, [150, 3], dict()),                          # short documents behind a long one, in one block with its end
    (400, [150, 5], dict(causal=True)),
    (700, [520, 2], dict(causal=True, softcap=5.0)),
    (460, [200, 1, 180, 4], dict(bias=True)),
    (330, [7], dict(prefix=40, causal=True)),         # short documents far behind common keys
]


@pytest.mark.parametrize("dtype,D,G", [("f16", 64, 1), ("bf16", 32, 1), ("bf16", 128, 4), ("bf16", 32, 3), ("f16", 20, 1)])
@pytest.mark.parametrize("case", SHORT, ids=lambda c: f"{c[0]}-{c[1]}-{'-'.join(c[2])}")
def test_attention_short_documents_wherever_they_lie(case, dtype, D, G):
    # rows that see at most 64 keys are off by their own roundings and not by that of out, whatever is beside them
    import torch

    L, sizes, masks = case
    say(f"attention of short documents {sizes} of {L}, {masks} {dtype} D={D} G={G}")
    how = masks_of(1, L, L, G, **masks)
    doc, n = [], 0
    while len(doc) < L:
        doc += [n] * sizes[min(n, len(sizes) - 1)]
        n += 1
    doc = torch.tensor(doc[:L]).int()[None].cuda()
    how["q_doc"] = how["k_doc"] = doc
    q, k, v, go = make(1, L, L, G, 1, D, dtype, seed=L)
    v += 3  # an offset that all keys share: dP - delta is without it, the rounding of out with it
    rows = layer_ref.seen_pairs(1, L, L, **{x: how.get(x) for x in ("q_doc", "k_doc", "prefix")},
                                causal=how["causal"])[0].sum(1) <= 64
    keys = torch.tensor([bool(rows[(doc[0] == d).cpu()].all()) for d in doc[0]])
    if "prefix" in how:
        keys[:40] = False
    assert rows.any() and keys.any()
    ref = layer_ref.attention(q, k, v, grad_out=go, few_keys=True, **how)
    out, lse = msda.attention_forward(q, k, v, **how)
    gq, gk, gv = msda.attention_backward(q, k, v, out, lse, go, **how)
    assert_within("grad_q", gq[:, rows.cuda()], *(x[:, rows] for x in ref["grad_q"]))
    for name, t in (("grad_k", gk), ("grad_v", gv)):
        assert_within(name, t[:, keys.cuda()], *(x[:, keys] for x in ref[name]))


@pytest.mark.parametrize("dtype,D", [("f16", 64), ("bf16", 32), ("bf16", 128)])
def test_attention_gradients_of_a_small_probability_with_a_large_value(dtype, D):
    # nearly all of a row's probability is on an early key, the rest on a late one, whose value outweighs that
    say(f"attention with a large value of small probability, {dtype} D={D}")
    L = 400
    q, k, v, go = make(1, L, L, 1, 1, D, dtype, seed=8)
    q[..., 1:] = 0
    q[..., 0] = 8
    k[..., 0] = -25     # scores of -200, of 0 and of -9
    k[:, 3, :, 0] = 0
    k[:, 300, :, 0] = -1.125
    v[:, 300] *= 1000
    how = masks_of(1, L, L, 1, docs="one")
    check(q, k, v, go, how, scale=1.0)


@pytest.mark.parametrize("size", [1.0, 1e-2, 1e-3, 1e-4])
@pytest.mark.parametrize("case", [(1, 8, 16384, 4, 2, 32, {}), (1, 40, 4099, 2, 1, 128, dict(causal=True)),
                                  (1, 1030, 1030, 2, 1, 64, dict(docs="pad", softcap=5.0)), (1, 2048, 70, 3, 1, 32, dict(bias=True))],
                         ids=lambda c: "-".join(map(str, c[:6])))
def test_attention_small_gradients_in_fp16(case, size):
    # gradients of scores are about grad_out / keys: below what fp16 holds with all its bits
    N, Lq, Lk, M, Mkv, D, masks = case
    say(f"attention's gradients of a grad_out of {size} in fp16, {case}")
    how = masks_of(N, Lq, Lk, M, **masks)
    q, k, v, go = make(N, Lq, Lk, M, Mkv, D, "f16", seed=Lk)
    go = (go.float() * size).half()
    out, lse = msda.attention_forward(q, k, v, **how)
    got = msda.attention_backward(q, k, v, out, lse, go, **how)
    ref = layer_ref.attention(q, k, v, grad_out=go, carried=True, **how)
    for name, t in zip(("grad_q", "grad_k", "grad_v"), got):
        assert_within(name, t, *ref[name])
        # and normwise: the rounding of the result, and as much again for the roundings within
        value = ref[name][0]
        off = float((t.cpu().double() - value).norm() / value.norm())
        own = float((value.half().double() - value).norm() / value.norm())
        say(f"  {name}: {off:.2e}, rounded {own:.2e}")
        assert off <= 2 * own + 2.0 ** -11, name


@pytest.mark.parametrize("D", [32, 64, 128])
def test_attention_large_gradients_of_scores_in_fp16(D):
    # P (dP - delta) beyond fp16's largest number, with results within it; the largest come late
    say(f"attention's gradients of scores beyond 65504 in fp16, D={D}")
    q, k, v, go = make(1, 150, 200, 2, 1, D, "f16", seed=D)
    k, v, go = k * 2.0 ** -10, v * 300, go * 300
    v[:, 150:] *= 30
    how = masks_of(1, 150, 200, 2, docs="mixed", prefix=9)
    ref = layer_ref.attention(q, k, v, grad_out=go, carried=True, **how)
    out, lse = msda.attention_forward(q, k, v, **how)
    gq, gk, gv = msda.attention_backward(q, k, v, out, lse, go, **how)
    assert float(ref["grad_q"][0].abs().max()) < 60000
    assert_within("grad_q", gq, *ref["grad_q"])
    k, q = k * 2.0 ** 10, q * 2.0 ** -10
    ref = layer_ref.attention(q, k, v, grad_out=go, carried=True, **how)
    out, lse = msda.attention_forward(q, k, v, **how)
    gq, gk, gv = msda.attention_backward(q, k, v, out, lse, go, **how)
    assert float(ref["grad_k"][0].abs().max()) < 60000
    assert_within("grad_k", gk, *ref["grad_k"])


@pytest.mark.parametrize("Lq,Lk", [(1, 1024), (40, 1500), (300, 4096)])
def test_attention_of_small_probabilities_in_fp16(Lq, Lk):
    # one key of weight 1 and no value, and many whose weights are less than two of fp16's smallest numbers
    say(f"attention of {Lk} small probabilities in fp16, {Lq} queries")
    q, k, v, go = make(1, Lq, Lk, 1, 1, 32, "f16", seed=3)
    q[..., 1:] = 0
    q[..., 0] = 8
    k[..., 0] = -2.0332  # scores of -16.27, weights of 1.45 times 2^-24
    k[:, 17, :, 0] = 0
    v += 1
    v *= 100
    v[:, 17] = 0
    ref = layer_ref.attention(q, k, v, scale=1.0, carried=True)
    out, lse = msda.attention_forward(q, k, v, scale=1.0)
    for name, t in (("out", out), ("lse", lse)):
        assert_within(name, t, *ref[name])


def test_attention_grad_v_of_small_probabilities_in_fp16():
    say("attention's grad_v of small probabilities in fp16")
    q, k, v, go = make(1, 64, 500, 1, 1, 32, "f16", seed=4)
    q[..., 1:] = 0
    q[..., 0] = 8
    k[..., 0] = -2.2932  # 1.45 times 2^-27
    k[:, 17, :, 0] = 0
    go = go.abs() * 1000
    ref = layer_ref.attention(q, k, v, grad_out=go, scale=1.0, carried=True)
    out, lse = msda.attention_forward(q, k, v, scale=1.0)
    gv = msda.attention_backward(q, k, v, out, lse, go, scale=1.0)[2]
    assert_within("grad_v", gv, *ref["grad_v"])


@pytest.mark.parametrize("softcap", [1e4, 1e6, 1e8])
@pytest.mark.parametrize("dtype,D", [("f32", 32), ("f16", 64), ("bf16", 32), ("bf16", 128)])
def test_attention_with_a_large_cap(dtype, D, softcap):
    # cap tanh(s / cap) is s to (s / cap)^2 / 3 of it, 1e-6 or less here (scores up to 20): as without a cap
    say(f"attention with a cap of {softcap}, {dtype} D={D}")
    q, k, v, go = make(2, 150, 170, 4, 2, D, dtype, seed=9)
    for bias in (False, True):
        how = masks_of(2, 150, 170, 4, docs="mixed", prefix=9, bias=bias)
        ref = layer_ref.attention(q, k, v, grad_out=go, **how)
        how["softcap"] = softcap
        out, lse = msda.attention_forward(q, k, v, **how)
        got = (out, lse) + tuple(msda.attention_backward(q, k, v, out, lse, go, **how))
        for name, t in zip(("out", "lse", "grad_q", "grad_k", "grad_v"), got):
            assert_within(name, t, *ref[name])


def test_attention_capped_scores_at_a_quarter_of_the_cap():
    # where the two forms of tanh meet in fp32: lse of one key is its score, to the roundings of it
    import torch

    say("attention's capped scores around a quarter of the cap, fp32")
    D = 8
    q = torch.zeros(1, 4096, 1, D, device="cuda")
    q[0, :, 0, 0] = torch.linspace(0.15, 0.3, 4096)
    k = torch.zeros(1, 1, 1, D, device="cuda")
    k[..., 0] = 1
    lse = msda.attention_forward(q, k, k, scale=1.0, softcap=1.0)[1]
    z = torch.tanh(q[0, :, 0, 0].double().cpu())
    # within the series (first half and more): the polynomial's four operations, s * a, the log 2 units and back; 10 u of z
    inside = q[0, :, 0, 0].cpu() < 0.25
    off = (lse[0, 0].double().cpu() - z).abs() / z
    assert float(off[inside].max()) <= 10 * layer_ref.U, float(off[inside].max()) / layer_ref.U
    assert float(off[~inside].max()) <= 6 * layer_ref.U / 0.24 + 4 * layer_ref.U


@pytest.mark.parametrize("Lq", [1, 90])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_attention_of_scores_of_ten_millions(dtype, Lq):
    # one key takes all: out is its value, to the rounding of a probability and of the result, and grad_v of the others is 0
    import torch

    say(f"attention with scores of ten millions, {dtype}")
    q, k, v, go = make(1, Lq, 400, 2, 2, 64, dtype, seed=Lq)
    q, k = q * 2500, k * 2500
    z = (q.cpu().double().transpose(1, 2) @ k.cpu().double().permute(0, 2, 3, 1)) / 8
    top2 = z.topk(2, -1)
    clear = top2.values[..., 0] - top2.values[..., 1] > 2000  # [N, M, Lq]; far beyond the rounding of a score
    assert float(top2.values.max()) > 1.2e7 and clear.float().mean() > 0.9
    out, lse = msda.attention_forward(q, k, v)
    want = torch.gather(v.cpu().double().transpose(1, 2), 2, top2.indices[..., :1].expand(-1, -1, -1, 64))
    off = (out.cpu().double().transpose(1, 2) - want).abs()[clear]
    assert bool(torch.isfinite(out).all()) and bool((off <= 3 * layer_ref.half_step(out.dtype) * want[clear].abs()).all())
    assert float(((lse.cpu().double() - top2.values[..., 0]).abs() / top2.values[..., 0]).max()) <= 70 * layer_ref.U * 64
    grads = msda.attention_backward(q, k, v, out, lse, go)
    assert all(bool(torch.isfinite(g).all()) for g in grads)


@pytest.mark.parametrize("dtype,D", [("f16", 64), ("bf16", 32), ("bf16", 128)])
def test_attention_of_16_bits_captured_and_replayed(dtype, D):
    # short and long documents (tables, delta, runs of tiles and their sums in the graph), new inputs for each replay
    import torch

    say(f"attention captured into a graph, {dtype} D={D}")
    L = 900
    doc = torch.cat([torch.arange(200) // 3, torch.full((650,), 100), torch.full((50,), -2)]).int()[None].cuda()
    how = {"q_doc": doc, "k_doc": doc.clone(), "causal": True, "softcap": 20.0}
    t = make(1, L, L, 4, 2, D, dtype, seed=0)

    def step(q, k, v, go):
        out, lse = msda.attention_forward(q, k, v, **how)
        return (out, lse) + tuple(msda.attention_backward(q, k, v, out, lse, go, **how))

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step(*t)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step(*t)
    for seed in (1, 2, 3):
        new = make(1, L, L, 4, 2, D, dtype, seed=seed)
        for a, b in zip(t, new):
            a.copy_(b)
        doc.copy_(torch.roll(doc, 7 * seed, 1))
        how["k_doc"].copy_(doc)
        graph.replay()
        torch.cuda.synchronize()
        eager = step(*new)  # between the replays, on the same allocator
        torch.cuda.synchronize()
        for name, a, b in zip(("out", "lse", "grad_q", "grad_k", "grad_v"), captured, eager):
            assert torch.equal(a, b), (seed, name)
