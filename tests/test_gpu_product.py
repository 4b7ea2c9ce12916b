"""GPU parity of the product of 8-bit integers with exact sums (tests/serve_ref.py)."""
import pytest

import serve_ref
from layer_ref import DT, assert_within
from paper_2505_14022_amd import msda
from gpu_util import require_gpu, say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    require_gpu()


def make(T, K, O, seed=0, lo=-127, hi=127, at=0):
    import torch

    g = torch.Generator().manual_seed(seed)

    def codes(rows):
        flat = torch.zeros(rows * K + at, dtype=torch.int8, device="cuda")
        flat[at:] = torch.randint(lo, hi + 1, (rows * K,), generator=g, dtype=torch.int8).cuda()
        return flat[at:].view(rows, K)

    return (codes(T), codes(O), torch.rand(T, generator=g).cuda() + 0.01, torch.rand(O, generator=g).cuda() * 0.1 + 0.001,
            torch.randn(O, generator=g).cuda())


def check(a, b, a_scale, b_scale, bias, dtype, **how):
    got = msda.quantized_matmul(a, b, a_scale, b_scale, bias=bias, dtype=DT[dtype], **how)
    value, bound = serve_ref.product(a, b, a_scale, b_scale, bias, DT[dtype])
    assert got.dtype == DT[dtype]
    assert_within("out", got, value, bound)
    return got


# few tokens of 16, 32 and 64 to a workgroup, tiles of 64, 128 and 256; rows that are not whole pieces; tails of every kind
SIZES = [(1, 16, 16), (1, 1, 1), (3, 5, 2), (1, 4096, 48), (2, 130, 17), (16, 64, 33), (17, 48, 100), (32, 2064, 50), (33, 1000, 250),
         (64, 512, 129), (65, 128, 64), (70, 16, 5), (100, 144, 4), (130, 272, 257), (300, 1024, 512), (1019, 1360, 1030),
         (2100, 400, 2050), (4099, 144, 4101), (130, 77, 65), (3, 131071, 5), (70, 65552, 20)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("T,K,O", SIZES, ids=lambda v: str(v))
def test_product_sizes(T, K, O, dtype):
    say(f"product of {T} x {K} and {O} x {K} to {dtype}")
    a, b, a_scale, b_scale, bias = make(T, K, O, seed=T + K + O)
    if dtype == "f16":  # within its range
        a_scale, b_scale = a_scale / K ** 0.5 / 127, b_scale / 127
    check(a, b, a_scale, b_scale, bias, dtype)
    check(a, b, a_scale, b_scale, None, dtype)


@pytest.mark.parametrize("T,K,O", [(7, 131071, 9), (80, 131056, 12)])
def test_sums_of_the_largest_codes(T, K, O):
    # -128 times -128, as often as 32 bits hold, and the smallest of the other sign
    say(f"products of the largest codes, K = {K}")
    a, b, a_scale, b_scale, bias = make(T, K, O, lo=-128, hi=-128)
    check(a, b, a_scale, b_scale, None, "f32")
    b.fill_(127)
    check(a, b, a_scale, b_scale, None, "f32")


@pytest.mark.parametrize("at", [1, 4, 8])
@pytest.mark.parametrize("T", [5, 90])
def test_product_of_unaligned_codes(T, at):
    say(f"product of codes {at} bytes off alignment, {T} tokens")
    check(*make(T, 320, 70, seed=at, at=at), "bf16")


# rows that are not whole 16-byte pieces, in tiles of each size: one short step, whole steps and a rest, a rest of one
@pytest.mark.parametrize("T,K,O", [(65, 7, 40), (300, 777, 301), (2050, 129, 2049), (4100, 145, 4101), (4097, 383, 4098)],
                         ids=lambda v: str(v))
def test_product_of_odd_rows(T, K, O):
    say(f"product of {T} x {K} and {O} x {K}")
    check(*make(T, K, O, seed=T + K), "bf16")
    check(*make(T, K + 1, O, seed=T + K), "f32")


@pytest.mark.parametrize("T,O", [(5, 64), (90, 128), (5, 66)])
def test_product_into_a_given_tensor(T, O):
    import torch

    say("product into rows of a larger buffer")
    a, b, a_scale, b_scale, bias = make(T, 96, O, seed=9)
    flat = torch.full((T * O + 3,), 5.0, device="cuda", dtype=torch.float16)
    a_scale = a_scale / 1000
    out = flat[1:1 + T * O].view(T, O)  # not aligned
    assert check(a, b, a_scale, b_scale, bias, "f16", out=out) is out
    assert float(flat[0]) == 5.0 and bool((flat[-2:] == 5).all())


def test_product_of_tokens_in_batches_and_none():
    import torch

    a, b, a_scale, b_scale, bias = make(6, 64, 24, seed=2)
    say("product of tokens in batches, and of none")
    want = msda.quantized_matmul(a, b, a_scale, b_scale)
    got = msda.quantized_matmul(a.view(2, 3, 64), b, a_scale.view(2, 3), b_scale)
    assert got.shape == (2, 3, 24) and torch.equal(got.view(6, 24), want)
    assert msda.quantized_matmul(a[:0], b, a_scale[:0], b_scale).shape == (0, 24)
    assert msda.quantized_matmul(a, b[:0], a_scale, b_scale[:0]).shape == (6, 0)


def test_scales_that_are_not_finite_stay_in_their_row_and_channel():
    import torch

    a, b, a_scale, b_scale, bias = make(40, 64, 50, seed=5)
    a[3] = 0
    a_scale[3] = float("nan")
    b_scale[7] = float("inf")
    say("product with scales that are not finite")
    got = msda.quantized_matmul(a, b, a_scale, b_scale, dtype=torch.float32)
    assert bool(torch.isnan(got[3]).all())
    rows, cols = [i for i in range(40) if i != 3], [i for i in range(50) if i != 7]
    value, bound = serve_ref.product(a[rows], b[cols], a_scale[rows], b_scale[cols], None, torch.float32)
    assert_within("out", got[rows][:, cols], value, bound)
    assert not bool(torch.isfinite(got[rows][:, 7]).any())


def test_products_on_two_streams():
    import torch

    sets = [make(T, K, O, seed=T) for T, K, O in ((8, 2048, 512), (200, 512, 300))]
    want = [msda.quantized_matmul(a, b, s, t, bias=c) for a, b, s, t, c in sets]
    say("products on two streams at once")
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[msda.quantized_matmul(a, b, s, t, bias=c, stream=st) for st, (a, b, s, t, c) in zip(streams, sets)] for _ in range(4)]
    torch.cuda.synchronize()
    for pair in got:
        for x, y in zip(pair, want):
            assert torch.equal(x, y)
