"""Scales of the paged cache that differ widely: blocks of scale 0 whose codes are not."""
import pytest

import serve_ref
from gpu_util import require_gpu, say
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
