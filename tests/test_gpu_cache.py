"""GPU parity of the paged cache of 8-bit keys and values: appending and attention, against 64-bit references within derived
bounds (tests/serve_ref.py)."""
import math

import pytest

import serve_ref
from layer_ref import DT, assert_within
from paper_2505_14022_amd import msda
from gpu_util import require_gpu, say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    require_gpu()


class Case:
    """A pool with N sequences' pages anywhere in it, and the tokens of a call. lengths: tokens of each sequence in all; new:
    how many of them are new."""

    def __init__(self, lengths, new, Mkv=2, G=2, D=64, P=16, dtype="bf16", seed=0, width=None, spare=3, packed=True, axes=1):
        import torch

        g = torch.Generator().manual_seed(seed)
        self.g, self.dt = g, DT[dtype]
        self.lengths, self.new, self.Mkv, self.M, self.D, self.P = list(lengths), list(new), Mkv, Mkv * G, D, P
        N, T = len(lengths), sum(new)
        self.T, self.N = T, N
        width = width or max(1, -(-max(lengths) // P))
        pages = N * width + spare
        self.table = torch.randperm(pages, generator=g)[:N * width].to(torch.int32).view(N, width).cuda()
        self.length = torch.tensor(lengths, dtype=torch.int32).cuda()
        ends = [0]
        for x in new:
            ends.append(ends[-1] + x)
        self.ends = ends
        self.start = torch.tensor(ends, dtype=torch.int32).cuda()
        self.k_cache, self.v_cache = (torch.randint(-127, 128, (pages, Mkv, P, D), generator=g, dtype=torch.int8).cuda() for _ in range(2))
        self.k_scale, self.v_scale = ((torch.rand(pages, Mkv, generator=g) * 0.04 + 0.002).cuda() for _ in range(2))
        x = torch.randn(T, self.M + 2 * Mkv, D, generator=g).to(self.dt).cuda()
        self.q, self.k, self.v = x[:, :self.M], x[:, self.M:self.M + Mkv], x[:, self.M + Mkv:]
        if not packed:
            self.q, self.k, self.v = self.q.contiguous(), self.k.contiguous(), self.v.contiguous()
        self.pos = torch.rand(T, axes, generator=g).cuda() * 3000
        if axes == 1:
            self.pos = torch.tensor([float(p) for n, c in zip(lengths, new) for p in range(n - c, n)], device="cuda").view(T, 1)
        R = D // 2
        self.freqs = (10000.0 ** (-torch.arange(R, dtype=torch.float64) / R)).float().repeat(axes, 1).cuda()

    def cache(self):
        return self.k_cache, self.v_cache, self.k_scale, self.v_scale, self.table, self.length

    def append(self, start="own", stream=None, pos="own", freqs="own", **how):
        start, pos, freqs = (mine if x == "own" else x for x, mine in ((start, self.start), (pos, self.pos), (freqs, self.freqs)))
        msda.cache_append(self.k, self.v, *self.cache(), start=start, pos=pos, freqs=freqs, stream=stream, **how)

    def check_append(self, start="own", interleaved=False, pos="own", freqs="own"):
        before = [x.cpu() for x in (self.k_cache, self.k_scale, self.v_cache, self.v_scale)]
        self.append(start, interleaved=interleaved, pos=pos, freqs=freqs)
        starts = self.start if isinstance(start, str) else start
        starts = None if starts is None else starts.tolist()
        p = self.pos if isinstance(pos, str) or pos is None else pos
        f = self.freqs if isinstance(freqs, str) else freqs
        k, bound = serve_ref.turned(self.k, p, f, interleaved)
        v, none = serve_ref.turned(self.v, None, None, False)
        length, table = self.length.tolist(), self.table.cpu()
        a = serve_ref.check_append(before[:2], (self.k_cache, self.k_scale), k, bound, table, length, starts)
        return a + serve_ref.check_append(before[2:], (self.v_cache, self.v_scale), v, none, table, length, starts)

    def attend(self, start="own", **how):
        start = self.start if isinstance(start, str) else start
        return msda.cache_attention(self.q, *self.cache(), start=start, **how)

    def check_attention(self, start="own", scale=None, softcap=0.0, causal=True, **how):
        start = self.start if isinstance(start, str) else start
        out, lse = self.attend(start, scale=scale, softcap=softcap, causal=causal, **how)
        ref = serve_ref.attention(self.q, *self.cache(), start=start, scale=scale, softcap=softcap, causal=causal)
        assert_within("out", out, *ref["out"])
        assert_within("lse", lse, *ref["lse"])
        return out, lse


# ---------------------------------------------------------------- appending


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("D,P", [(16, 16), (32, 64), (48, 16), (64, 32), (80, 128), (96, 16), (112, 32), (128, 64), (128, 256)])
def test_append_sizes(dtype, D, P):
    say(f"append {dtype}, {D} channels, pages of {P}")
    # from nothing, into a page, over a page's end, over several pages, one token each at either side of an end, none
    lengths = [5, P, P + 1, 3 * P + 7, 2 * P + 1, 2 * P, 40, 1]
    new = [5, 1, 3, 2 * P + 9, 1, 1, 0, 1]
    for interleaved in (False, True):
        c = Case(lengths, new, D=D, P=P, dtype=dtype, seed=D + P + interleaved)
        c.check_append(interleaved=interleaved)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_append_one_token_each(dtype):
    say(f"append one token each, {dtype}")
    lengths = [1, 16, 17, 33, 64, 50, 2]
    a, b = (Case(lengths, [1] * 7, Mkv=3, dtype=dtype, seed=3) for _ in range(2))
    a.check_append()
    b.check_append(start=None)  # the same without the table of starts
    assert a.k_cache.equal(b.k_cache) and a.v_scale.equal(b.v_scale)


def test_append_rounds_what_stands_in_a_page_anew():
    say("append of larger values into pages")
    c = Case([12, 30, 64], [3, 4, 1], D=32, P=32, dtype="f32", seed=5)
    c.k_scale *= 0.05  # what stands there is small
    c.v_scale *= 0.01
    assert c.check_append() >= 2 * 2 * 32 * (9 + 26 + 31)
    # again: the scales are those of the new tokens by now, and nothing changes
    before = [x.clone() for x in (c.k_cache, c.v_cache, c.k_scale, c.v_scale)]
    assert c.check_append() == 0
    for x, y in zip(before, (c.k_cache, c.v_cache, c.k_scale, c.v_scale)):
        assert x.equal(y)


@pytest.mark.parametrize("how", ["place", "axes", "part", "none"])
def test_append_positions(how):
    say(f"append with positions: {how}")
    c = Case([21, 40, 300], [3, 20, 9], D=64, P=16, dtype="f32", seed=7, axes=3 if how == "axes" else 1)
    if how == "place":  # the place in the sequence is the position
        c.check_append(pos=None)
    elif how == "part":  # ten pairs are turned, which are no whole pieces
        c.freqs = c.freqs[:, :10].contiguous()
        c.check_append()
        c.check_append(interleaved=True)
    elif how == "none":
        c.check_append(pos=None, freqs=None)
    else:
        c.check_append()


def test_append_of_far_positions():
    say("append at far positions")
    c = Case([9, 20], [9, 4], D=32, P=16, dtype="f32", seed=8)
    c.pos += 10_000_000
    c.check_append()


@pytest.mark.parametrize("packed", [True, False])
@pytest.mark.parametrize("at", [0, 1])
def test_append_strides_and_alignment(packed, at):
    import torch

    say(f"append of strided keys, packed {packed}, {at} elements off alignment")
    c = Case([21, 40], [5, 20], D=64, dtype="f16", seed=9, packed=packed)
    if at:
        for name in ("k", "v"):
            x = getattr(c, name)
            flat = torch.empty(x.numel() + at, dtype=x.dtype, device="cuda")
            flat[at:] = x.reshape(-1)
            setattr(c, name, flat[at:].view(x.shape))
    c.check_append()
    # every head the same, and every token the same
    c.k = c.k[:, :1].expand(c.T, c.Mkv, c.D)
    c.v = c.v[:1].expand(c.T, c.Mkv, c.D)
    c.check_append()


def test_append_where_there_is_no_page():
    import torch

    say("append to pages that do not exist")
    c = Case([40, 33, 64, 20], [30, 5, 64, 20], seed=10)
    c.table[0, 1] = -1
    c.table[1, 2] = c.k_cache.shape[0]
    c.table[2, 0] = 2 ** 31 - 1
    c.length[3] = 12  # fewer than the new ones: the first 8 are outside
    c.check_append()
    c.length[0] = 10_000  # beyond the table
    c.length[1] = -5
    c.check_append()
    # starts that go backwards or beyond the tokens
    c.length[:] = torch.tensor([40, 33, 64, 20], dtype=torch.int32)
    c.start = torch.tensor([0, 30, 20, 84, 5000], dtype=torch.int32, device="cuda")
    before = [x.clone() for x in (c.k_cache, c.k_scale)]
    c.append()
    torch.cuda.synchronize()
    held = torch.zeros(c.k_cache.shape[0], dtype=torch.bool, device="cuda")
    t = c.table[(c.table >= 0) & (c.table < c.k_cache.shape[0])].long()
    held[t] = True
    assert c.k_cache[~held].equal(before[0][~held]) and c.k_scale[~held].equal(before[1][~held])


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_append_of_values_that_are_not_finite(dtype):
    import torch

    say("append of a NaN and of infinities")
    c = Case([20, 40, 18], [6, 20, 2], D=32, dtype=dtype, seed=11)
    k, v = c.k.clone(), c.v.clone()
    k[2, 0, 5] = float("nan")
    v[10, 1, 31] = float("inf")
    v[26, 0, 0] = -float("inf")
    c.k, c.v = k, v
    c.check_append()
    assert bool(torch.isnan(c.v_scale).any()) and bool(torch.isnan(c.k_scale).any())


def test_append_zeros_and_small_values():
    import torch

    say("append of zeros")
    c = Case([20, 40], [20, 3], D=32, dtype="f32", seed=12)
    c.k, c.v = torch.zeros_like(c.k), torch.full_like(c.v, 2.0 ** -110)
    c.check_append()
    fresh = c.table[0, 0].long()
    assert float(c.k_scale[fresh].abs().max()) == 0 and not bool(c.k_cache[fresh].any())


def test_append_of_nothing():
    import torch

    say("append of no tokens")
    c = Case([20, 40], [0, 0], seed=13)
    c.check_append()
    empty = Case([5], [5], seed=14)
    empty.table = empty.table[:0]
    empty.length, empty.start = empty.length[:0], empty.start[:1]
    empty.k, empty.v, empty.pos = empty.k[:0], empty.v[:0], empty.pos[:0]
    empty.append()


def test_append_many_sequences():
    import random

    say("append for 300 sequences")  # more than a wave looks over at once
    r = random.Random(1)
    new = [r.choice([0, 0, 1, 1, 2, 17]) for _ in range(300)]
    Case([max(1, x) + r.randint(0, 30) for x in new], new, Mkv=1, G=1, D=16, dtype="f32", seed=15).check_append()


def test_append_with_a_table_of_more_columns():
    import torch

    say("append through the first columns of a wider table")
    c = Case([33, 47], [4, 30], seed=16)
    wide = torch.full((2, 9), -7, dtype=torch.int32, device="cuda")
    wide[:, :c.table.shape[1]] = c.table
    c.table = wide[:, :c.table.shape[1]]
    c.check_append()
    c.check_attention()


# ---------------------------------------------------------------- attention


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("D,P,G", [(16, 16, 1), (32, 64, 4), (48, 16, 5), (64, 32, 8), (80, 128, 2), (96, 16, 3), (128, 64, 4),
                                   (128, 256, 1), (112, 32, 20), (32, 16, 40)])
def test_attention_of_one_token_each(dtype, D, P, G):
    say(f"attention of one token each: {dtype}, {D} channels, pages of {P}, {G} heads to a key head")
    lengths = [1, 2, P - 1, P, P + 1, 31, 32, 33, 129, 700]
    c = Case(lengths, [1] * len(lengths), G=G, D=D, P=P, dtype=dtype, seed=D + P + G)
    c.check_attention()
    a = c.attend()
    b = c.attend(start=None)
    assert a[0].equal(b[0]) and a[1].equal(b[1])
    # the same rows in any batch: a result does not depend on its neighbours' lengths
    again = c.attend()
    assert a[0].equal(again[0]) and a[1].equal(again[1])


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("D,P,G,new", [(32, 16, 2, 3), (64, 64, 4, 5), (128, 32, 3, 9), (48, 16, 1, 40), (128, 64, 2, 70),
                                       (80, 16, 5, 33), (16, 128, 8, 150)])
def test_attention_of_several_tokens(dtype, D, P, G, new):
    say(f"attention of up to {new} tokens each: {dtype}, {D} channels, pages of {P}, {G} heads to a key head")
    counts = [new, 1, max(1, new // 2), new, 0, new - 1]
    lengths = [new, 1, new // 2 + 200, new + 3 * P + 1, 7, 600]
    c = Case(lengths, counts, G=G, D=D, P=P, dtype=dtype, seed=D + P + G)
    c.check_attention()
    c.check_attention(causal=False, softcap=20.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("softcap", [0.5, 30.0, 1000.0])
def test_attention_with_capped_scores(dtype, softcap):
    say(f"attention with scores capped at {softcap}")
    Case([300, 41], [1, 6], D=64, dtype=dtype, seed=21).check_attention(softcap=softcap, scale=0.7)


@pytest.mark.parametrize("scale", [1e-30, 1e-3, 3.0])
def test_attention_scales(scale):
    say(f"attention with scale {scale}")
    Case([300, 41], [1, 6], D=32, dtype="f32", seed=22).check_attention(scale=scale)


def test_attention_over_long_sequences():
    import torch

    say("attention over long sequences, split")
    c = Case([5000, 1, 9001, 4097], [1, 1, 1, 1], Mkv=1, G=4, D=128, P=64, dtype="bf16", seed=23)
    assert msda.cache_attention_workspace_size(c.q, *c.cache(), start=c.start) > 0
    c.check_attention()
    c = Case([5000, 3, 4100], [60, 3, 2], Mkv=2, G=1, D=32, P=16, dtype="f32", seed=24)
    out, lse = c.check_attention()
    # into the caller's workspace and tensors
    ws = torch.empty(msda.cache_attention_workspace_size(c.q, *c.cache(), start=c.start), dtype=torch.uint8, device="cuda")
    o, x = torch.empty_like(out), torch.empty_like(lse)
    got = c.attend(workspace=ws, out=o, lse=x)
    assert got[0] is o and got[1] is x and o.equal(out) and x.equal(lse)
    assert c.attend(want_lse=False)[1] is None


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_of_rows_that_see_nothing(dtype):
    import torch

    say("attention of rows that see nothing")
    c = Case([40, 20, 9, 64], [5, 20, 1, 3], D=32, dtype=dtype, seed=25)
    c.length[1] = 12  # the first 8 of the new tokens are outside
    c.length[2] = 0
    c.table[3] = -1   # no pages at all
    out, lse = c.check_attention()
    for rows in (slice(5, 13), slice(25, 26), slice(26, 29)):
        assert float(out[rows].abs().max()) == 0.0 and bool((lse[rows] == -math.inf).all())


def test_attention_past_pages_that_do_not_exist():
    say("attention past pages that do not exist")
    c = Case([100, 70, 300], [1, 4, 1], D=64, P=16, dtype="f32", seed=26)
    c.table[0, 2] = -1
    c.table[1, 0] = c.k_cache.shape[0]
    c.table[2, 5:9] = 2 ** 30
    c.length[2] = 5000  # beyond the table
    c.check_attention()
    c.check_attention(causal=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_what_is_not_seen_has_no_effect(dtype):
    import torch

    say("attention beside pages and slots that are not seen")
    a, b = (Case([37, 100, 16], [3, 2, 1], D=64, P=16, dtype=dtype, seed=27, spare=5) for _ in range(2))
    used = torch.zeros(b.k_cache.shape[0], dtype=torch.bool, device="cuda")
    for n, total in enumerate(b.lengths):
        used[b.table[n, :-(-total // 16)].long()] = True
    for scale in (b.k_scale, b.v_scale):
        scale[~used] = float("nan")
    # the last pages' slots past the end, and columns of the table past it
    for n, total in enumerate(b.lengths):
        page = int(b.table[n, (total - 1) // 16])
        if total % 16:
            b.k_cache[page, :, total % 16:] = -128
            b.v_cache[page, :, total % 16:] = -128
        b.table[n, -(-total // 16):] = 2 ** 31 - 1
    x, y = a.attend(), b.attend()
    assert x[0].equal(y[0]) and x[1].equal(y[1])
    # a page that later tokens see, and earlier ones of the same block do not
    # (its value scale may be the unit of their probabilities, whose roundings change with it)
    c = Case([34], [6], D=64, P=16, dtype=dtype, seed=28)
    page = c.table[0, 2].long()
    ref = serve_ref.attention(c.q, *c.cache(), start=c.start)
    for name in ("k_scale", "v_scale"):
        for bad in (float("nan"), float("inf"), -1.0):
            keep = getattr(c, name)[page].clone()
            getattr(c, name)[page] = bad
            out, lse = c.attend()
            getattr(c, name)[page] = keep
            assert_within("out", out[:4], ref["out"][0][:4], ref["out"][1][:4])
            assert_within("lse", lse[:4], ref["lse"][0][:4], ref["lse"][1][:4])
            assert not bool(torch.isfinite(out[4:]).any())


def test_attention_with_scales_of_all_sizes():
    say("attention over pages whose scales differ by 2^20")
    c = Case([200, 90], [1, 5], D=32, P=16, dtype="f32", seed=29)
    c.v_scale *= 2.0 ** (-2.0 * (c.table.new_tensor(range(c.v_scale.shape[0])).float()[:, None] % 11))
    c.k_scale *= 2.0 ** -((c.table.new_tensor(range(c.k_scale.shape[0])).float()[:, None] + 3) % 7)
    c.check_attention()
    c.v_scale[::2] = 0  # and pages of zeros
    c.check_attention()
    c.v_scale[:] = 0
    out, lse = c.check_attention()
    assert float(out.abs().max()) == 0


@pytest.mark.parametrize("new", [1, 90])
@pytest.mark.parametrize("least", [2.0 ** -140, 2.0 ** -100])
def test_value_scales_at_the_ends_of_fp32(new, least):
    """Small scales first and large ones past the 64 pages that are looked up at once, small ones throughout, and zeros."""
    import torch

    say(f"attention over value scales of {least} and of 2^100, {new} tokens each")
    c = Case([1500, 1100], [new, new], G=2, D=64, P=16, dtype="bf16", seed=36)
    row = c.table.long()
    c.v_scale[row[0, :66]] = least
    c.v_scale[row[0, 66:]] = 2.0 ** 100
    c.v_scale[row[1]] = 0
    out, lse = c.check_attention()
    assert bool(torch.isfinite(out).all()) and bool(torch.isfinite(lse).all())
    assert float(out[new:].abs().max()) == 0
    c.v_scale[row[0]] = 2.0 ** 100
    c.v_scale[row[0, 66:]] = least
    c.check_attention()
    c.v_scale[row[0]] = least
    out, lse = c.check_attention()
    assert bool(torch.isfinite(lse).all())


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_queries_of_all_sizes(dtype):
    import torch

    say("attention of large, small and zero queries")
    c = Case([90, 50], [4, 3], D=64, dtype=dtype, seed=30)
    q = c.q.clone()
    q[0] *= 0
    q[1] *= 2.0 ** -20
    q[2] *= 2.0 ** 9
    q[3, :, ::2] *= 2.0 ** -10  # within a row
    if dtype != "f16":
        q[4] *= 2.0 ** -120
    c.q = q
    c.check_attention()


def test_queries_that_are_not_finite_stay_in_their_rows():
    import torch

    say("attention of queries that are not finite")
    c = Case([90, 50], [4, 3], D=64, dtype="bf16", seed=31)
    want = c.attend()
    c.q = c.q.clone()
    c.q[1, 0, 3] = float("nan")
    c.q[5, 2, 60] = float("inf")
    out, lse = c.attend()
    bad = torch.zeros(c.T, c.M, dtype=torch.bool, device="cuda")
    bad[1, 0] = bad[5, 2] = True
    assert out[~bad].equal(want[0][~bad]) and lse[~bad].equal(want[1][~bad])
    assert not bool(torch.isfinite(out[bad]).all())


@pytest.mark.parametrize("at", [0, 1])
def test_attention_strides_and_alignment(at):
    import torch

    say(f"attention of strided queries {at} elements off alignment")
    c = Case([90, 50], [4, 3], D=48, dtype="f16", seed=32, packed=False)
    want = c.attend()
    wide = torch.zeros(c.T * (c.M + 2) * c.D + at, dtype=c.dt, device="cuda")[at:].view(c.T, c.M + 2, c.D)
    wide[:, 1:-1] = c.q
    c.q = wide[:, 1:-1]
    got = c.attend()
    assert got[0].equal(want[0]) and got[1].equal(want[1])


def test_rows_of_no_sequence_are_left_as_they_were():
    import torch

    say("attention with a padded batch")
    c = Case([40, 30, 20], [4, 2, 3], D=64, seed=33)
    want = c.attend()
    pad = torch.randn(5, c.M, c.D, device="cuda").to(c.dt)
    c.q = torch.cat([pad[:2], c.q, pad[2:]])
    c.start = c.start + 2
    out = torch.full(c.q.shape, 7.0, dtype=c.dt, device="cuda")
    lse = torch.full(c.q.shape[:2], 7.0, device="cuda")
    c.attend(out=out, lse=lse)
    assert out[2:-3].equal(want[0]) and lse[2:-3].equal(want[1])
    for rows in (slice(0, 2), slice(-3, None)):
        assert bool((out[rows] == 7).all()) and bool((lse[rows] == 7).all())


def test_attention_of_many_sequences():
    import random

    say("attention of 300 sequences")
    r = random.Random(2)
    new = [r.choice([0, 0, 1, 1, 2, 17]) for _ in range(300)]
    Case([max(1, x) + r.randint(0, 30) for x in new], new, Mkv=1, G=2, D=16, dtype="f32", seed=34).check_attention()


def test_attention_over_a_cache_past_32_bits():
    import torch

    free, _ = torch.cuda.mem_get_info()
    if free < 12 << 30:
        pytest.skip("needs 12 GiB")
    say("a pool of more than 4 GiB of codes")
    pages, Mkv, P, D = 34000, 8, 128, 128  # 4.4e9 codes each of keys and values
    k = torch.zeros((pages, Mkv, P, D), dtype=torch.int8, device="cuda")
    v = torch.zeros_like(k)
    scale = torch.full((pages, Mkv), 0.01, device="cuda")
    table = torch.tensor([[pages - 1, pages - 2, 16400], [0, 33999 - 700, 1]], dtype=torch.int32, device="cuda")
    length = torch.tensor([300, 260], dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    start = torch.tensor([0, 300, 560], dtype=torch.int32, device="cuda")
    x = torch.randn(560, 2 * Mkv, D, generator=g, device="cuda")
    msda.cache_append(x[:, :Mkv], x[:, Mkv:], k, v, scale, scale.clone(), table, length, start=start)
    small = [torch.zeros((6, Mkv, P, D), dtype=torch.int8, device="cuda") for _ in range(2)]
    small_scale = [torch.full((6, Mkv), 0.01, device="cuda") for _ in range(2)]
    small_table = torch.arange(6, dtype=torch.int32, device="cuda").view(2, 3)
    msda.cache_append(x[:, :Mkv], x[:, Mkv:], *small, *small_scale, small_table, length, start=start)
    at = table.flatten().long()
    assert k[at].equal(small[0]) and v[at].equal(small[1])
    q = torch.randn(2, 2 * Mkv, D, generator=g, device="cuda").bfloat16()
    v_scale = scale.clone()
    scale[at], v_scale[at] = small_scale
    got = msda.cache_attention(q, k, v, scale, v_scale, table, length)
    want = msda.cache_attention(q, *small, *small_scale, small_table, length)
    assert got[0].equal(want[0]) and got[1].equal(want[1])


def test_cache_on_two_streams():
    import torch

    say("two caches on two streams at once")
    pair = [Case([700, 65], [1, 1], D=128, G=4, seed=40), Case([40, 800], [20, 30], D=64, P=32, seed=41)]
    want = []
    for c in pair:
        keep = [x.clone() for x in (c.k_cache, c.v_cache, c.k_scale, c.v_scale)]
        c.append()
        want.append(c.attend())
        torch.cuda.synchronize()
        for x, y in zip((c.k_cache, c.v_cache, c.k_scale, c.v_scale), keep):
            x.copy_(y)
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], []
    for _ in range(3):
        for s, c in zip(streams, pair):
            c.append(stream=s)
            got.append(c.attend(stream=s))
    torch.cuda.synchronize()
    for i, res in enumerate(got):
        assert res[0].equal(want[i % 2][0]) and res[1].equal(want[i % 2][1])
