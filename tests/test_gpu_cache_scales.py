"""Scales of the paged cache that differ widely: blocks of scale 0 whose codes are not, and value scales of pages that
a row does not see, sees with small probabilities, or comes to late."""
import pytest

import serve_ref
from gpu_util import require_gpu, say
from layer_ref import assert_within
from paper_2505_14022_amd import msda
from serve_rows import attention_rows
from test_gpu_cache import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    require_gpu()


# ---------------------------------------------------------------- appending


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("D,P", [(16, 16), (48, 32), (128, 64), (64, 256)])
def test_append_over_codes_of_scale_zero(dtype, D, P):
    """A code times its scale is the value it stands for: what stood for 0 does so afterwards, in the scale of the new tokens."""
    import torch

    say(f"append into blocks of scale 0 over codes that are not 0: {dtype}, {D} channels, pages of {P}")
    # one token, several, and over the page's end; the page begun anew; one token each is the same call without starts
    lengths, new = [P - 3, P // 2 + 5, P + 2, P + 1], [1, 5, 7, 1]
    for start in ("own", None):
        c = Case(lengths, new if start else [1] * 4, Mkv=3, D=D, P=P, dtype=dtype, seed=D + P)
        row = c.table.long()
        c.k_scale[row[:, 0], 0] = 0.0  # some heads' keys and others' values
        c.k_scale[row[1, 0], 2] = 0.0
        c.v_scale[row[:, 0], 1] = 0.0
        before = [x.clone() for x in (c.k_cache, c.v_cache)]
        scales = [x.clone() for x in (c.k_scale, c.v_scale)]
        c.append(None if start is None else "own", freqs=None, pos=None)
        for codes, scale, was, was_scale, x in zip((c.k_cache, c.v_cache), (c.k_scale, c.v_scale), before, scales, (c.k, c.v)):
            for n, (total, count) in enumerate(zip(lengths, c.new)):
                slot = max(total - count, 0)
                if slot >= P:
                    continue  # the first page is not reached
                page, stop = int(row[n, 0]), min(total, P)
                for h in range(c.Mkv):
                    u, old = float(scale[page, h]), float(was_scale[page, h])
                    mine = x[c.ends[n]:c.ends[n] + stop - slot, h].double()
                    assert u > 0
                    held = codes[page, h, :slot].double() * u
                    if old == 0:
                        assert float(held.abs().max()) == 0, f"page {page}, head {h}: zeros became {float(held.abs().max())}"
                    else:  # half a step of the new scale, if it is another, and the roundings of ratio, product and scale
                        want = was[page, h, :slot].double() * old
                        assert float((held - want).abs().max()) <= (0.5 * u if u > old else 0.0) + 127 * u * 2.0 ** -22
                    got = codes[page, h, slot:stop].double() * u
                    assert float((got - mine).abs().max()) <= u * (0.5 + 127 * 3 * serve_ref.U)
                    assert torch.equal(codes[page, h, stop:], was[page, h, stop:])


def test_append_of_zeros_over_codes_of_scale_zero():
    import torch

    say("append of zeros into blocks of scale 0")
    c = Case([9, 20], [2, 3], D=32, dtype="f32", seed=51)
    c.k_scale[:] = 0.0
    c.v_scale[:] = 0.0
    c.k, c.v = torch.zeros_like(c.k), torch.zeros_like(c.v)
    c.append()
    assert not bool(c.k_scale.any()) and not bool(c.v_scale.any())  # whatever the codes are, the values are 0


# ---------------------------------------------------------------- attention


def check_rows(c, tokens, **how):
    """The call's rows of some tokens against their reference; all of the results."""
    out, lse = c.attend(**how)
    ref = attention_rows(c, tokens, **how)
    assert_within("out", out[tokens], *ref["out"])
    assert_within("lse", lse[tokens], *ref["lse"])
    return out, lse


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("power", [-60, 7, 12, 20, 40, 100])
@pytest.mark.parametrize("softcap", [0.0, 20.0])
def test_scales_of_pages_that_earlier_tokens_do_not_see(dtype, power, softcap):
    """Blocks of new tokens of which the later ones open a page whose value scale is another by far."""
    say(f"attention beside pages that are 2^{power} larger and seen by later tokens alone: {dtype}, cap {softcap}")
    c = Case([34, 300, 100, 21], [6, 40, 90, 7], G=3, D=64, P=16, dtype=dtype, seed=60)
    row = c.table.long()
    if dtype == "f16":  # the results of the large pages stay within its range
        c.v_scale *= 2.0 ** (6 - power) if power > 0 else 1.0
    for n, column in ((0, 2), (1, 17), (1, 18), (2, 3), (3, 1)):
        c.v_scale[row[n, column]] *= 2.0 ** power
    check_rows(c, list(range(c.T)), softcap=softcap)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("power", [10, 30, 70])
def test_small_probabilities_of_large_scales(dtype, power):
    """Pages whose probabilities are as small as their value scales are large, more and less so."""
    import torch

    say(f"attention over pages 2^{power} larger whose probabilities are small: {dtype}")
    c = Case([200, 65], [1, 20], G=2, D=32, P=16, dtype=dtype, seed=61)
    row = c.table.long()
    c.q = (c.q.abs() + 0.5).to(c.dt)
    codes = c.k_cache.abs().clamp_min(1)
    c.k_cache.copy_(torch.where(codes < 60, codes, 60))
    for n, column in ((0, 1), (0, 4), (0, 12), (1, 0), (1, 2)):
        page = row[n, column]
        c.v_scale[page] *= 2.0 ** power
        # scores of -a half to -twice as much below the others', in units of log 2
        c.k_cache[page] *= -1
        c.k_scale[page] *= torch.rand(c.Mkv, generator=c.g).cuda() * power / 8
    check_rows(c, list(range(c.T)))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_pages_of_zeros_that_take_nearly_all(dtype):
    """Pages of value scale 0 (or below the smallest normal number) have the large scores: what is left is small, and no less exact."""
    import torch

    say(f"attention over pages of zeros with large scores: {dtype}")
    for zero in (0.0, 2.0 ** -130):
        c = Case([200, 65, 30], [1, 20, 4], G=2, D=32, P=16, dtype=dtype, seed=62)
        row = c.table.long()
        c.q = (c.q.abs() + 0.5).to(c.dt)
        c.k_cache.copy_(c.k_cache.abs().clamp(1, 60) * -1)
        for n, column in ((0, 1), (0, 12), (1, 0), (2, 0), (2, 1)):
            page = row[n, column]
            c.v_scale[page] = zero
            c.k_cache[page] *= -1
        out, _ = check_rows(c, list(range(c.T)))
        assert not bool(out[21:].any())  # the last sequence has no other pages


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("least", [2.0 ** -9, 2.0 ** -30, 2.0 ** -90, 0.0])
def test_scales_that_change_along_the_way(dtype, least):
    """So many rows that a workgroup goes through a sequence alone, in which it looks 64 pages up at a time: large scales first
    and small ones after, and the other way round."""
    import torch

    say(f"attention over long sequences whose scales change: {dtype}, {least}")
    N = 64
    c = Case([2300] * N, [1] * N, Mkv=16, G=2, D=32, P=16, dtype=dtype, seed=63)
    assert msda.cache_attention_workspace_size(c.q, *c.cache(), start=c.start) == 0  # one run to a sequence
    row = c.table.long()
    for n in range(0, N, 4):
        c.v_scale[row[n, 66:]] *= least
        c.v_scale[row[n + 1, :66]] *= least
        c.v_scale[row[n + 2, 130]] *= least
        c.v_scale[row[n + 3, 70:80]] *= least
        c.v_scale[row[n + 3, 135]] *= 2.0 ** 9
        # those with large scales are the less likely ones
        large = row[n + 1, 66:]
        c.q[n + 1] = (c.q[n + 1].abs() + 0.5).to(c.dt)
        c.k_cache[large] = -c.k_cache[large].abs().clamp_min(1)
    check_rows(c, [0, 1, 2, 3, 25, 38, 62, 63])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_scales_that_are_apart_in_some_runs_of_a_long_sequence(dtype):
    """Sequences that are split over workgroups, of which some meet scales that are apart and others do not."""
    import torch

    say(f"attention over long split sequences, scales apart in some runs: {dtype}")
    c = Case([5000, 3, 9001, 4100], [1, 3, 40, 2], Mkv=2, G=2, D=64, P=16, dtype=dtype, seed=64)
    assert msda.cache_attention_workspace_size(c.q, *c.cache(), start=c.start) > 0
    row = c.table.long()
    c.v_scale[row[0, 40]] *= 2.0 ** 30
    c.v_scale[row[0, 200:260]] *= 2.0 ** -40
    c.v_scale[row[2, 562]] *= 2.0 ** 50  # the last page, which the last tokens see alone
    c.v_scale[row[2, 100]] = 0
    c.v_scale[row[3, 256]] *= 2.0 ** 20
    c.k_scale[row[3, 255]] = float("nan")  # a page that makes NaN
    tokens = [0, 1, 2, 3, 4, 20, 30, 33, 34, 35, 36, 42, 43]
    out, lse = check_rows(c, tokens)
    assert not bool(torch.isfinite(out[44:]).any()) and not bool(torch.isfinite(lse[44:]).any())
    again = c.attend()
    assert out.nan_to_num(7).equal(again[0].nan_to_num(7)) and lse.nan_to_num(7).equal(again[1].nan_to_num(7))


def test_scales_apart_beside_pages_that_do_not_exist():
    say("attention past pages that do not exist, scales apart")
    for new in (1, 30):
        c = Case([200, 170, 100], [new] * 3, G=4, D=48, P=16, dtype="f16", seed=65)
        c.table[0, 2] = -1
        c.table[1, 0] = c.k_cache.shape[0]
        c.table[2] = -1
        row = c.table.long()
        for page in (row[0, 5], row[1, 10]):
            c.v_scale[page] *= 2.0 ** -25
        check_rows(c, list(range(c.T)))
        check_rows(c, list(range(c.T)), causal=False, softcap=400.0)
