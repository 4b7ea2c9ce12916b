"""GPU parity of msda_layernorm_forward / msda_layernorm_backward with a 64-bit layer norm, within bounds derived
from the arithmetic (tests/layer_ref.py)."""
import pytest

import layer_ref
from layer_ref import DT, assert_within
from paper_2505_14022_amd import msda
from gpu_util import require_gpu, say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    require_gpu()


def make(rows, C, dtype, seed=0, shift=0.0, at=0):
    """x, residual, grad_out, grad_sum, weight, bias on the GPU; `at` elements into their allocations."""
    import torch

    g = torch.Generator().manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g)

    def put(t, dt):
        flat = torch.empty(t.numel() + at, dtype=dt, device="cuda")
        flat[at:] = t.to(dt).reshape(-1).cuda()
        return flat[at:].view(t.shape)

    dt = DT[dtype]
    return [put(normal(rows, C) * 2 + shift, dt), put(normal(rows, C), dt), put(normal(rows, C), dt),
            put(normal(rows, C), dt), put(1 + 0.3 * normal(C), torch.float32), put(0.3 * normal(C), torch.float32)]


def check(x, r, go, gs, w, b, eps=1e-5, stream=None, workspace="auto"):
    ref = layer_ref.layernorm(x, w, b, r, eps, go, gs)
    got = msda.layernorm_forward(x, w, b, residual=r, eps=eps, want_sum=True, stream=stream)
    got = dict(zip(("out", "mean", "rstd", "sum"), got))
    grads = msda.layernorm_backward(x, go, got["mean"], got["rstd"], w, residual=r, grad_sum=gs, stream=stream,
                                    workspace=workspace)
    got.update(zip(("grad_x", "grad_weight", "grad_bias"), grads))
    if stream is not None:
        stream.synchronize()
    for name, (value, bound) in ref.items():
        assert_within(name, got[name], value, bound)
    return got


# every layout of a row: 8 .. 64 lanes, a workgroup of 256 or 1024 threads, one to sixteen pieces per lane
SIZES = [(1, 1), (5, 7), (3, 8), (33, 19), (70, 64), (9, 240), (300, 256), (41, 257), (7, 512), (6, 1000), (19, 1024),
         (4, 1030), (3, 2048), (2, 4100), (5, 8192), (2, 16383), (2, 16384), (1031, 2056), (5003, 32)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,C", SIZES, ids=lambda v: str(v))
def test_layernorm_sizes(rows, C, dtype):
    say(f"layer norm of {rows} x {C} {dtype}")
    check(*make(rows, C, dtype, seed=rows + C))


@pytest.mark.parametrize("at", [1, 3])
@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_layernorm_of_unaligned_tensors(dtype, at):
    say(f"layer norm of tensors {at} elements off alignment, {dtype}")
    check(*make(37, 256, dtype, seed=3, at=at))


def test_layernorm_without_its_options():
    import torch

    x, r, go, gs, w, b = make(50, 96, "bf16", seed=4)
    say("layer norm without weight, bias, residual and sums")
    ref = layer_ref.layernorm(x, None, None, None, 1e-3, go)
    res = msda.layernorm_forward(x, eps=1e-3)
    assert len(res) == 3
    gx, gw, gb = msda.layernorm_backward(x, go, res[1], res[2], want_weight_grads=False)
    assert gw is None and gb is None
    for name, t in (("out", res[0]), ("mean", res[1]), ("rstd", res[2]), ("grad_x", gx)):
        assert_within(name, t, *ref[name])
    # one of the two sums alone, and the caller's workspace
    only = torch.full((96,), float("nan"), device="cuda")
    ws = torch.empty(msda.layernorm_workspace_size(50, 96, msda.MSDA_BF16), dtype=torch.uint8, device="cuda")
    _, gw, gb = msda.layernorm_backward(x, go, res[1], res[2], want_weight_grads=False, grad_bias=only, workspace=ws)
    assert gw is None and gb is only
    assert_within("grad_bias", gb, *ref["grad_bias"])


def test_layernorm_of_rows_far_from_zero():
    # the variance is not a difference of large sums: rows at 1000 with a spread of 2 keep their digits
    x, r, go, gs, w, b = make(40, 384, "f32", seed=5, shift=1000.0)
    say("layer norm of rows far from zero")
    check(x, None, go, None, w, b)


def test_layernorm_of_constant_rows():
    import torch

    x = torch.full((6, 80), 3.5, device="cuda", dtype=torch.float16)
    go = torch.randn(6, 80, device="cuda").half()
    say("layer norm of constant rows")
    out, mean, rstd = msda.layernorm_forward(x, eps=1e-5)
    assert float(out.abs().max()) == 0.0 and float((mean - 3.5).abs().max()) == 0.0
    assert_within("grad_x", msda.layernorm_backward(x, go, mean, rstd)[0], *layer_ref.layernorm(x, grad_out=go)["grad_x"])


def test_layernorm_keeps_nan_in_its_row():
    import torch

    x, r, go, gs, w, b = make(9, 100, "f16", seed=6)
    x[4, 17] = float("nan")
    x[7, 3] = float("inf")
    say("layer norm with a NaN and an infinity in two rows")
    out, mean, rstd = msda.layernorm_forward(x, w, b, residual=r)
    keep = [i for i in range(9) if i not in (4, 7)]
    ref = layer_ref.layernorm(x[keep], w, b, r[keep])
    assert_within("out", out[keep], *ref["out"])
    assert bool(torch.isnan(out[4]).all()) and bool(torch.isnan(out[7]).all())


def test_layernorm_is_reproducible_on_other_streams():
    import torch

    args = make(2999, 240, "f32", seed=7)
    a = check(*args)
    say("layer norm on two streams at once")
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    x, r, go, gs, w, b = args
    got = []
    for s in (s1, s2, s1):
        out, mean, rstd = msda.layernorm_forward(x, w, b, residual=r, stream=s)
        got.append((out,) + msda.layernorm_backward(x, go, mean, rstd, w, residual=r, grad_sum=gs, stream=s))
    torch.cuda.synchronize()
    for res in got:
        for name, t in zip(("out", "grad_x", "grad_weight", "grad_bias"), res):
            assert torch.equal(t, a[name]), name


def test_layernorm_empty():
    import torch

    say("layer norm of no rows")
    x = torch.empty((0, 48), device="cuda", dtype=torch.bfloat16)
    out, mean, rstd = msda.layernorm_forward(x)
    gw = torch.full((48,), 7.0, device="cuda")
    gx, gw, gb = msda.layernorm_backward(x, x, mean, rstd, grad_weight=gw)
    assert out.shape == (0, 48) and gx.shape == (0, 48)
    assert float(gw.abs().max()) == 0.0 and float(gb.abs().max()) == 0.0


def test_layernorm_gradient_against_differences():
    import torch

    x, r, go, gs, w, b = make(6, 40, "f32", seed=8)
    out, mean, rstd = msda.layernorm_forward(x, w, b)
    gx, gw, gb = msda.layernorm_backward(x, go, mean, rstd, w)
    say("layer norm's gradient against differences")

    def loss(dx, dw):
        return float((msda.layernorm_forward(x + dx, w + dw, b)[0].double() * go.double()).sum())

    noise = float((layer_ref.layernorm(x, w, b)["out"][1] * go.cpu().double().abs()).sum())
    for seed in range(3):
        g = torch.Generator().manual_seed(seed)
        dx, dw = torch.randn(6, 40, generator=g).cuda(), torch.randn(40, generator=g).cuda()
        slope = float((gx.double() * dx.double()).sum() + (gw.double() * dw.double()).sum())
        e = 2.0 ** -7
        d1 = (loss(e * dx, e * dw) - loss(-e * dx, -e * dw)) / (2 * e)
        d2 = (loss(e / 2 * dx, e / 2 * dw) - loss(-e / 2 * dx, -e / 2 * dw)) / e
        # a halved step leaves a quarter of the truncation; the inputs' steps are rounded too (6e-8 of 8)
        assert abs(d2 - slope) <= abs(d1 - d2) + 8 * noise / e, (d1, d2, slope)
