"""Attention over the paged cache for chunks of prompts so large that a workgroup takes 48 rows: a sample of the rows against
their 64-bit references (tests/serve_rows.py)."""
import math
import random

import pytest

from gpu_util import require_gpu, say
from layer_ref import assert_within
from paper_2505_14022_amd import msda
from serve_rows import attention_rows
from test_gpu_cache import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    require_gpu()


def tokens_of_a_block(c):
    """Of the call's 48 rows, which are taken for 16-bit queries where sequences bring 1024 rows and more to a key head on
    average, and their blocks, key heads and parts of the heads make 1024 workgroups."""
    G = c.M // c.Mkv
    group = min(G, 48)
    tokens, groups = 48 // group, -(-G // group)
    blocks = c.T // tokens + c.N
    assert -(-c.T // c.N) * G >= 1024 and blocks * c.Mkv * groups >= 1024
    assert msda.cache_attention_workspace_size(c.q, *c.cache(), start=c.start) == 0  # no splits
    return tokens


def sample(c, tokens, seed=0):
    """Tokens at the ends of sequences and of blocks, and any."""
    r, got = random.Random(seed), set()
    for a, b in zip(c.ends, c.ends[1:]):
        last = a + (b - a - 1) // tokens * tokens  # the first of the sequence's last block, which is not full
        got.update(t for t in (a, a + 1, a + tokens - 1, a + tokens, last - 1, last, b - 2, b - 1) if a <= t < b)
        got.update(r.randrange(a, b) for _ in range(6 if b > a else 0))
    return sorted(got)


def check(c, tokens, **how):
    out, lse = c.attend(**how)
    ref = attention_rows(c, tokens, **how)
    assert_within("out", out[tokens], *ref["out"])
    assert_within("lse", lse[tokens], *ref["lse"])
    return out, lse


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("Mkv,G,D,P,new", [(8, 4, 128, 64, [600, 421, 0, 530]),   # the sizes of the 48 rows: 12 tokens of 4 heads
                                           (8, 4, 64, 16, [601, 1, 700, 270]),
                                           (8, 5, 128, 32, [523, 300, 401]),       # 9 tokens of 5 heads, 3 rows idle
                                           (8, 5, 80, 128, [523, 300, 401]),
                                           (2, 64, 128, 16, [150, 31, 90]),        # a token's 64 heads in two parts of 48 and 16
                                           (2, 64, 48, 64, [150, 31, 90]),
                                           (24, 1, 32, 16, [1030, 1100]),          # 48 tokens of one head
                                           (16, 3, 16, 256, [700, 388]),
                                           (3, 20, 112, 16, [333, 340, 200])])     # two tokens of 20 heads, 8 rows idle
def test_chunks_of_48_rows(dtype, Mkv, G, D, P, new):
    say(f"attention of chunks in 48 rows: {dtype}, {Mkv} key heads, {G} heads to each, {D} channels, pages of {P}")
    past = [0, 333, 40, 211][:len(new)]
    c = Case([n + p for n, p in zip(new, past)], new, Mkv=Mkv, G=G, D=D, P=P, dtype=dtype, seed=D + G + P)
    tokens = sample(c, tokens_of_a_block(c))
    check(c, tokens)
    check(c, tokens, causal=False, softcap=20.0)
    check(c, tokens, softcap=400.0, scale=0.5)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_chunks_of_48_rows_where_some_see_nothing(dtype):
    say(f"attention of chunks in 48 rows, of which some see nothing: {dtype}")
    c = Case([600, 450, 530, 300], [600, 400, 530, 300], Mkv=8, G=4, D=64, P=16, dtype=dtype, seed=70)
    per_block = tokens_of_a_block(c)
    c.length[1] = 123    # the first 277 of the new tokens are outside
    c.table[2, 3:9] = -1  # pages 3 to 8 are missing
    c.table[3] = c.k_cache.shape[0]
    c.length[0] = 10_000  # beyond the table: the new tokens' places as well
    tokens = sorted(set(sample(c, per_block) + [600 + t for t in (275, 276, 277, 278)] + [1000 + t for t in (47, 48, 49, 143, 144)]))
    out, lse = check(c, tokens)
    for rows in (slice(600, 877), slice(1530, 1830)):
        assert float(out[rows].abs().max()) == 0.0 and bool((lse[rows] == -math.inf).all())


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_chunks_of_48_rows_whose_scales_are_apart(dtype):
    say(f"attention of chunks in 48 rows, value scales apart: {dtype}")
    c = Case([1500, 450, 530, 40], [600, 400, 530, 40], Mkv=8, G=4, D=128, P=16, dtype=dtype, seed=71)
    per_block = tokens_of_a_block(c)
    row = c.table.long()
    if dtype == "f16":
        c.v_scale *= 2.0 ** -6
    c.v_scale[row[0, 90]] *= 2.0 ** 14          # past the first 64 pages that are looked up
    c.v_scale[row[1, 20:25]] *= 2.0 ** -18
    c.v_scale[row[2, 33]] = 0                   # the last page
    c.v_scale[row[3, 1], 3] *= 2.0 ** 12        # of one head
    check(c, sample(c, per_block, 1))
    check(c, sample(c, per_block, 2), softcap=30.0)


def test_rows_of_a_large_batch_do_not_depend_on_their_neighbours():
    import torch

    say("a chunk alone, and among others that leave its blocks as they are")
    c = Case([1200, 700, 900], [1200, 500, 900], Mkv=8, G=4, D=128, P=64, dtype="bf16", seed=72)
    tokens_of_a_block(c)
    want = c.attend()
    order = [2, 0, 1]
    rows = torch.cat([torch.arange(c.ends[n], c.ends[n + 1]) for n in order]).cuda()
    c.q, c.table, c.length = c.q[rows], c.table[order].contiguous(), c.length[order].contiguous()
    c.start = torch.tensor([0, 900, 2100, 2600], dtype=torch.int32, device="cuda")
    got = c.attend()
    assert got[0].equal(want[0][rows]) and got[1].equal(want[1][rows])
    again = c.attend()
    assert got[0].equal(again[0]) and got[1].equal(again[1])
