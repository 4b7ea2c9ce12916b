"""GPU parity of the root-mean-square norm (forward, backward, in 8 bits) and of rows in 8 bits with 64-bit references
within derived bounds; codes bit by bit (tests/serve_ref.py)."""
import math

import pytest

import layer_ref
import serve_ref
from layer_ref import DT, assert_within
from paper_2505_14022_amd import msda
from gpu_util import require_gpu, say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    require_gpu()


def make(rows, C, dtype, seed=0, at=0):
    """x, residual, grad_out, grad_sum, weight on the GPU; `at` elements into their allocations."""
    import torch

    g = torch.Generator().manual_seed(seed)

    def put(t, dt):
        flat = torch.empty(t.numel() + at, dtype=dt, device="cuda")
        flat[at:] = t.to(dt).reshape(-1).cuda()
        return flat[at:].view(t.shape)

    dt = DT[dtype]
    return [put(torch.randn(rows, C, generator=g) * by, dt) for by in (2, 1, 1, 1)] + \
        [put(1 + 0.3 * torch.randn(C, generator=g), torch.float32)]


def check(x, r, go, gs, w, eps=1e-6, stream=None, workspace="auto"):
    ref = serve_ref.rmsnorm(x, w, r, eps, go, gs)
    got = dict(zip(("out", "rstd", "sum"), msda.rmsnorm_forward(x, w, residual=r, eps=eps, want_sum=True, stream=stream)))
    grads = msda.rmsnorm_backward(x, go, got["rstd"], w, residual=r, grad_sum=gs, stream=stream, workspace=workspace)
    got.update(zip(("grad_x", "grad_weight"), grads))
    if stream is not None:
        stream.synchronize()
    for name, (value, bound) in ref.items():
        assert_within(name, got[name], value, bound)
    return got


def check_codes(x, r, w, eps=1e-6, codes=None, scale=None):
    """rmsnorm_quantize against the fp32 operations that the header states, and its scales in 64 bits."""
    import torch

    ref = serve_ref.rmsnorm(x, w, r, eps)
    want, u = serve_ref.quantized_rows(x, w, r)
    codes, scale, total = msda.rmsnorm_quantize(x, w, residual=r, eps=eps, want_sum=True, codes=codes, scale=scale)
    assert torch.equal(codes.cpu(), want)
    rstd, bound = ref["rstd"]
    assert_within("scale", scale, u.double() * rstd, u.double() * (bound + 2 * serve_ref.U * rstd))
    assert_within("sum", total, *ref["sum"])
    return codes, scale


# every layout of a row: 8 .. 64 lanes, a workgroup of 256 or 1024 threads, one to sixteen pieces per lane
SIZES = [(1, 1), (5, 7), (3, 8), (33, 19), (70, 64), (9, 240), (300, 256), (41, 257), (7, 512), (6, 1000), (19, 1024),
         (4, 1030), (3, 2048), (2, 4100), (5, 8192), (2, 16383), (2, 16384), (1031, 2056), (5003, 32)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,C", SIZES, ids=lambda v: str(v))
def test_rmsnorm_sizes(rows, C, dtype):
    import torch

    say(f"root-mean-square norm of {rows} x {C} {dtype}")
    x, r, go, gs, w = make(rows, C, dtype, seed=rows + C)
    check(x, r, go, gs, w)
    check_codes(x, r, w)
    codes, scale = msda.quantize_rows(x)
    want, u = serve_ref.quantized_rows(x)
    assert torch.equal(codes.cpu(), want) and torch.equal(scale.cpu(), u)


@pytest.mark.parametrize("at", [1, 3])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rmsnorm_of_unaligned_tensors(dtype, at):
    import torch

    say(f"root-mean-square norm of tensors {at} elements off alignment, {dtype}")
    x, r, go, gs, w = make(37, 256, dtype, seed=3, at=at)
    check(x, r, go, gs, w)
    check_codes(x, r, w)
    # whole pieces into codes that are not aligned
    x, r, go, gs, w = make(37, 256, dtype, seed=4)
    flat = torch.full((37 * 256 + 5,), 99, dtype=torch.int8, device="cuda")
    check_codes(x, r, w, codes=flat[at:at + 37 * 256].view(37, 256))
    assert bool((flat[:at] == 99).all()) and bool((flat[at + 37 * 256:] == 99).all())


def test_rmsnorm_without_its_options():
    import torch

    x, r, go, gs, w = make(50, 96, "bf16", seed=4)
    say("root-mean-square norm without weight, residual and sums")
    ref = serve_ref.rmsnorm(x, None, None, 1e-3, go)
    out, rstd = msda.rmsnorm_forward(x, eps=1e-3)
    gx, gw = msda.rmsnorm_backward(x, go, rstd, want_weight_grad=False)
    assert gw is None
    for name, t in (("out", out), ("rstd", rstd), ("grad_x", gx)):
        assert_within(name, t, *ref[name])
    assert len(msda.rmsnorm_quantize(x)) == 2
    check_codes(x, None, None)
    # the caller's workspace
    ws = torch.empty(msda.rmsnorm_workspace_size(50, 96, msda.MSDA_BF16), dtype=torch.uint8, device="cuda")
    assert_within("grad_weight", msda.rmsnorm_backward(x, go, rstd, workspace=ws)[1], *ref["grad_weight"])


def test_rmsnorm_in_place():
    import torch

    # the residual stream's sum may take x's place, and the norm's result the residual's
    x, r, go, gs, w = make(200, 768, "bf16", seed=11)
    say("root-mean-square norm with its sum in place of the residual")
    out, rstd, total = msda.rmsnorm_forward(x, w, residual=r, want_sum=True)
    want, scale, _ = msda.rmsnorm_quantize(x, w, residual=r, want_sum=True)
    r2 = r.clone()
    codes, scale2, same = msda.rmsnorm_quantize(x, w, residual=r2, sum=r2)
    assert same is r2 and torch.equal(r2, total) and torch.equal(codes, want) and torch.equal(scale, scale2)
    r2 = r.clone()
    out2, _, _ = msda.rmsnorm_forward(x, w, residual=r2, sum=r2)
    assert torch.equal(out2, out) and torch.equal(r2, total)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_rows_that_are_not_finite(dtype):
    import torch

    x, r, go, gs, w = make(9, 100, dtype, seed=6)
    x[4, 17] = float("nan")
    x[7, 3] = float("inf")
    r[8, 99] = -float("inf")
    say("rows with a NaN and infinities")
    out, rstd = msda.rmsnorm_forward(x, w, residual=r)
    codes, scale = msda.rmsnorm_quantize(x, w, residual=r)
    keep = [i for i in range(9) if i not in (4, 7, 8)]
    assert_within("out", out[keep], *serve_ref.rmsnorm(x[keep], w, r[keep])["out"])
    want, u = serve_ref.quantized_rows(x, w, r)
    assert torch.equal(codes.cpu(), want) and not bool(codes[[4, 7, 8]].any())
    assert bool(torch.isnan(scale[[4, 7, 8]]).all()) and bool(torch.isfinite(scale[keep]).all())
    codes, scale = msda.quantize_rows(x)
    assert bool(torch.isnan(scale[[4, 7]]).all()) and not bool(codes[[4, 7]].any()) and bool(torch.isfinite(scale[8]))


def test_rows_of_zeros_and_of_small_values():
    import torch

    say("rows of zeros and of small values in 8 bits")
    x = torch.zeros(6, 72, device="cuda")
    x[1] = 2.0 ** -101
    x[2, 5] = -(2.0 ** -100)
    x[3] = 1e-42
    x[4] = 3e38
    codes, scale = msda.quantize_rows(x)
    want, u = serve_ref.quantized_rows(x)
    assert torch.equal(codes.cpu(), want) and torch.equal(scale.cpu(), u)
    assert scale[0] == 0 and scale[1] == 0 and scale[3] == 0 and scale[2] > 0 and int(codes[2, 5]) == -127 and int(codes[4, 0]) == 127
    out, rstd = msda.rmsnorm_forward(x[:1], eps=0.0)
    assert bool(torch.isnan(out).all()) and bool(torch.isinf(rstd).all())  # 0 / 0, as in the formula
    codes, scale = msda.rmsnorm_quantize(x[:1], eps=1e-6)
    assert not bool(codes.any()) and float(scale[0]) == 0.0


def test_codes_round_ties_to_even():
    import torch

    say("codes halfway between two")
    x = torch.tensor([[127.0, 0.5, 1.5, 2.5, -0.5, -1.5, -2.5, 126.5]], device="cuda")
    codes, scale = msda.quantize_rows(x)
    want, u = serve_ref.quantized_rows(x)
    assert torch.equal(codes.cpu(), want)
    if float(u[0]) == 1.0:
        assert codes[0].tolist() == [127, 0, 2, 2, 0, -2, -2, 126]


def test_rmsnorm_is_reproducible_on_other_streams():
    import torch

    args = make(2999, 240, "f32", seed=7)
    a = check(*args)
    x, r, go, gs, w = args
    codes, scale = check_codes(x, r, w)
    say("root-mean-square norm on two streams at once")
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    got = []
    for s in (s1, s2, s1):
        out, rstd = msda.rmsnorm_forward(x, w, residual=r, stream=s)
        got.append((out,) + msda.rmsnorm_backward(x, go, rstd, w, residual=r, grad_sum=gs, stream=s) +
                   msda.rmsnorm_quantize(x, w, residual=r, stream=s))
    torch.cuda.synchronize()
    for res in got:
        for name, t in zip(("out", "grad_x", "grad_weight"), res):
            assert torch.equal(t, a[name]), name
        assert torch.equal(res[3], codes) and torch.equal(res[4], scale)


def test_rmsnorm_empty():
    import torch

    say("root-mean-square norm of no rows")
    x = torch.empty((0, 48), device="cuda", dtype=torch.bfloat16)
    out, rstd = msda.rmsnorm_forward(x)
    gw = torch.full((48,), 7.0, device="cuda")
    gx, gw = msda.rmsnorm_backward(x, x, rstd, grad_weight=gw)
    assert out.shape == (0, 48) and gx.shape == (0, 48) and float(gw.abs().max()) == 0.0
    codes, scale = msda.quantize_rows(x)
    assert codes.shape == (0, 48) and scale.shape == (0,)


def test_rmsnorm_gradient_against_differences():
    import torch

    x, r, go, gs, w = make(6, 40, "f32", seed=8)
    out, rstd = msda.rmsnorm_forward(x, w)
    gx, gw = msda.rmsnorm_backward(x, go, rstd, w)
    say("root-mean-square norm's gradient against differences")

    def loss(dx, dw):
        return float((msda.rmsnorm_forward(x + dx, w + dw)[0].double() * go.double()).sum())

    noise = float((serve_ref.rmsnorm(x, w)["out"][1] * go.cpu().double().abs()).sum())
    for seed in range(3):
        g = torch.Generator().manual_seed(seed)
        dx, dw = torch.randn(6, 40, generator=g).cuda(), torch.randn(40, generator=g).cuda()
        slope = float((gx.double() * dx.double()).sum() + (gw.double() * dw.double()).sum())
        e = 2.0 ** -7
        d1 = (loss(e * dx, e * dw) - loss(-e * dx, -e * dw)) / (2 * e)
        d2 = (loss(e / 2 * dx, e / 2 * dw) - loss(-e / 2 * dx, -e / 2 * dw)) / e
        # a halved step leaves a quarter of the truncation; the inputs' steps are rounded too (6e-8 of 8)
        assert abs(d2 - slope) <= abs(d1 - d2) + 8 * noise / e, (d1, d2, slope)
