"""GPU parity of msda_rotary_forward / msda_rotary_backward with 64-bit rotations (bounds of tests/layer_ref.py)."""
import pytest

import layer_ref
from layer_ref import DT, assert_within
from paper_2505_14022_amd import msda
from gpu_util import require_gpu, say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    require_gpu()


def freqs_of(A, R):
    import torch

    f = torch.zeros(A, R)
    for a in range(A):
        lo, hi = a * R // A, (a + 1) * R // A
        f[a, lo:hi] = 10000.0 ** (-torch.arange(hi - lo, dtype=torch.float32) / max(1, hi - lo))
    return f.cuda()


def make(N, T, M, D, A, dtype, seed=0, far=100.0, shared=False):
    import torch

    g = torch.Generator().manual_seed(seed)
    x = torch.randn(N, T, M, D, generator=g).to(DT[dtype]).cuda()
    pos = (torch.rand((T, A) if shared else (N, T, A), generator=g) * far).cuda()
    return x, pos


CASES = [
    # N, T, M, D, A, R, shared positions
    (1, 1, 1, 2, 1, 1, False), (2, 5, 3, 8, 2, 4, False), (1, 7, 2, 32, 2, 16, False), (3, 33, 5, 48, 3, 24, True),
    (2, 65, 8, 64, 2, 32, False), (1, 130, 3, 128, 3, 48, False), (2, 3, 1, 20, 1, 6, False), (1, 4, 2, 33, 4, 16, True),
    (1, 19, 64, 1024, 2, 512, False), (2, 9, 2, 40, 2, 0, False), (1, 3001, 8, 32, 3, 16, True),
]


@pytest.mark.parametrize("interleaved", [False, True], ids=["halves", "pairs"])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "N%d_T%d_M%d_D%d_A%d_R%d_%s" % c)
def test_rotary_sizes(case, dtype, interleaved):
    N, T, M, D, A, R, shared = case
    x, pos = make(N, T, M, D, A, dtype, seed=T + D, shared=shared)
    f = freqs_of(A, R)
    say(f"rotary {case} {dtype} interleaved={interleaved}")
    assert_within("out", msda.rotary_forward(x, pos, f, interleaved), *layer_ref.rotary(x, pos, f, interleaved))
    assert_within("grad_x", msda.rotary_backward(x, pos, f, interleaved), *layer_ref.rotary(x, pos, f, interleaved, -1.0))


@pytest.mark.parametrize("far", [1e4, 1e7, -3e6])
def test_rotary_of_far_positions(far):
    x, pos = make(1, 200, 2, 64, 1, "f32", seed=2, far=far)
    f = freqs_of(1, 32)
    say(f"rotary of positions up to {far}")
    assert_within("out", msda.rotary_forward(x, pos, f), *layer_ref.rotary(x, pos, f, False))


def test_rotary_with_mixed_axes():
    # every axis turns every pair, with frequencies of its own (and of either sign)
    import torch

    x, pos = make(2, 50, 4, 32, 3, "f32", seed=3)
    f = torch.randn(3, 16, generator=torch.Generator().manual_seed(1)).cuda()
    say("rotary with mixed axes")
    assert_within("out", msda.rotary_forward(x, pos, f, True), *layer_ref.rotary(x, pos, f, True))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rotary_of_views_and_in_place(dtype):
    # the queries and keys of a packed projection [N, T, 3, M, D], turned where they are
    import torch

    g = torch.Generator().manual_seed(4)
    qkv = torch.randn(2, 37, 3, 4, 32, generator=g).to(DT[dtype]).cuda()
    pos = (torch.rand(2, 37, 2, generator=g) * 50).cuda()
    f = freqs_of(2, 12)  # 24 of 32 channels
    before = qkv.clone()
    say(f"rotary of a packed projection in place, {dtype}")
    for which in (0, 1):
        view = qkv[:, :, which]
        assert msda.rotary_forward(view, pos, f, out=view) is view
        assert_within("out", view, *layer_ref.rotary(before[:, :, which], pos, f, False))
    assert torch.equal(qkv[:, :, 2], before[:, :, 2])
    # heads last but one in memory, channels at an odd offset, a batch that is one tensor seen twice
    base = torch.randn(4, 37, 33, generator=g).to(DT[dtype]).cuda()
    heads_first = base[:, :, 1:].permute(1, 0, 2)[None].expand(2, 37, 4, 32)
    assert_within("out", msda.rotary_forward(heads_first, pos, f, True), *layer_ref.rotary(heads_first, pos, f, True))
    out = torch.full((2, 37, 5, 40), 7.0, dtype=DT[dtype], device="cuda")
    msda.rotary_forward(heads_first, pos, f, True, out=out[:, :, :4, 3:35])
    assert_within("out", out[:, :, :4, 3:35], *layer_ref.rotary(heads_first, pos, f, True))
    assert float((out[:, :, 4] - 7).abs().max()) == 0 and float((out[..., 35:] - 7).abs().max()) == 0


def test_rotary_backward_undoes_forward_and_streams():
    import torch

    x, pos = make(3, 100, 8, 32, 2, "f32", seed=5)
    f = freqs_of(2, 16)
    say("rotary there and back on another stream")
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    y = msda.rotary_forward(x, pos, f, stream=s)
    z = msda.rotary_backward(y, pos, f, stream=s)
    s.synchronize()
    # both ways: 18 u of a pair's two values, which are at most sqrt(2) of its length each
    assert float((z - x).abs().max()) <= 40 * layer_ref.U * float(x.abs().max()) * 1.5
    assert torch.equal(y, msda.rotary_forward(x, pos, f))


def test_rotary_empty():
    import torch

    say("rotary of no tokens")
    x = torch.empty(2, 0, 3, 16, device="cuda")
    assert msda.rotary_forward(x, torch.empty(2, 0, 1, device="cuda"), freqs_of(1, 8)).shape == x.shape


@pytest.mark.parametrize("interleaved", [False, True], ids=["halves", "pairs"])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("T,M,D,R", [(37, 4, 32, 16), (5, 64, 128, 64), (9, 3, 96, 32), (3, 7, 1024, 512)])
def test_rotary_in_place_of_whole_pieces(T, M, D, R, dtype, interleaved):
    # heads of whole 16-byte pieces, each read by two threads, several turns of a workgroup to a token among them
    import torch

    g = torch.Generator().manual_seed(T)
    qkv = torch.randn(2, T, 3, M, D, generator=g).to(DT[dtype]).cuda()
    pos = (torch.rand(2, T, 2, generator=g) * 50).cuda()
    f = freqs_of(2, R)
    before = qkv.clone()
    say(f"rotary in place of {T} x {M} x {D}, {R} pairs, {dtype} interleaved={interleaved}")
    view = qkv[:, :, 1]
    msda.rotary_forward(view, pos, f, interleaved, out=view)
    assert_within("out", view, *layer_ref.rotary(before[:, :, 1], pos, f, interleaved))
    assert torch.equal(view, msda.rotary_forward(before[:, :, 1], pos, f, interleaved))
    msda.rotary_backward(view, pos, f, interleaved, grad_x=view)
    again = msda.rotary_backward(msda.rotary_forward(before[:, :, 1], pos, f, interleaved), pos, f, interleaved)
    assert torch.equal(view, again)
    assert torch.equal(qkv[:, :, 0], before[:, :, 0]) and torch.equal(qkv[:, :, 2], before[:, :, 2])
