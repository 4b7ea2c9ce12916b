"""The layer operators run together, as a decoder layer runs them: rotary positions on the queries and keys, masked
self-attention, residual and norm, then deformable attention over the feature maps and another norm, forward and
backward; and the same captured into a graph and replayed between eager work."""
import numpy as np
import pytest

import layer_ref
from paper_2505_14022_amd import msda
from gpu_util import require_gpu, say

pytestmark = pytest.mark.gpu

N, L, M, D = 2, 90, 4, 32
C = M * D
SHAPES = np.asarray([[9, 12], [5, 6]], dtype=np.int64)
STARTS = np.asarray([0, 108], dtype=np.int64)
S, LEVELS, P = 138, 2, 3


@pytest.fixture(scope="module", autouse=True)
def gpu():
    require_gpu()


def inputs(seed):
    import torch

    g = torch.Generator().manual_seed(seed)

    def normal(*shape, by=1.0):
        return (torch.randn(*shape, generator=g) * by).cuda()

    t = {"x": normal(N, L, C), "wq": normal(C, C, by=C ** -0.5), "wk": normal(C, C, by=C ** -0.5),
         "wv": normal(C, C, by=C ** -0.5), "w1": 1 + normal(C, by=0.1), "b1": normal(C, by=0.1),
         "w2": 1 + normal(C, by=0.1), "b2": normal(C, by=0.1), "value": normal(N, S, M, D),
         "loc": torch.rand(N, L, M, LEVELS, P, 2, generator=g).cuda(),
         "attn": torch.softmax(torch.randn(N, L, M, LEVELS * P, generator=g), -1).reshape(N, L, M, LEVELS, P).cuda(),
         "grad": normal(N, L, C), "pos": torch.rand(N, L, 2, generator=g).cuda()}
    t["freqs"] = torch.zeros(2, D // 2, device="cuda")
    t["freqs"][0, :8] = t["freqs"][1, 8:] = 6.28 * 4.0 ** -torch.arange(8, dtype=torch.float32, device="cuda")
    doc = torch.cat([torch.zeros(40), 1 + torch.arange(50) // 10]).int()[None].repeat(N, 1)
    doc[1, 80:] = -1
    t["doc"] = doc.cuda()
    t["prefix"] = torch.full((N,), 40, dtype=torch.int32, device="cuda")
    return t


def layer(t):
    """The library's calls, with the projections as plain products between them; outputs and gradients."""
    import torch

    how = {"q_doc": t["doc"], "k_doc": t["doc"], "prefix": t["prefix"], "softcap": 20.0}
    x = t["x"]
    q, k, v = (torch.matmul(x, t[w]).view(N, L, M, D) for w in ("wq", "wk", "wv"))
    qr, kr = (msda.rotary_forward(y, t["pos"], t["freqs"]) for y in (q, k))
    o, lse = msda.attention_forward(qr, kr, v, **how)
    y, mean1, rstd1 = msda.layernorm_forward(x, t["w1"], t["b1"], residual=o.view(N, L, C))
    s = msda.forward(t["value"], SHAPES, STARTS, t["loc"], t["attn"])
    out, mean2, rstd2 = msda.layernorm_forward(y, t["w2"], t["b2"], residual=s)
    gy, gw2, gb2 = msda.layernorm_backward(y, t["grad"], mean2, rstd2, t["w2"], residual=s)
    gvalue, gloc, gattn = msda.backward(t["value"], SHAPES, STARTS, t["loc"], t["attn"], gy)
    gx, gw1, gb1 = msda.layernorm_backward(x, gy, mean1, rstd1, t["w1"], residual=o.view(N, L, C))
    gqr, gkr, gv = msda.attention_backward(qr, kr, v, o, lse, gx.view(N, L, M, D), **how)
    gq, gk = (msda.rotary_backward(g, t["pos"], t["freqs"]) for g in (gqr, gkr))
    for g, w in ((gq, "wq"), (gk, "wk"), (gv, "wv")):
        gx = gx + torch.matmul(g.view(N, L, C), t[w].t())
    return {"out": out, "gx": gx, "gq": gq, "gk": gk, "gv": gv, "gw1": gw1, "gb1": gb1, "gw2": gw2, "gb2": gb2,
            "gvalue": gvalue}


def layer64(t):
    """The same in 64 bits on the CPU by automatic differentiation; the sampling of the maps enters as its own result."""
    import torch

    u = {k: v.cpu().double() if v.is_floating_point() else v.cpu() for k, v in t.items()}
    x = u["x"].requires_grad_()
    q, k, v = (torch.matmul(x, u[w]).view(N, L, M, D) for w in ("wq", "wk", "wv"))
    leaves = [y for y in (q, k, v)]
    angle = (u["pos"][..., None] * u["freqs"]).sum(-2)[:, :, None]
    turn = torch.polar(torch.ones_like(angle), angle)

    def rotated(y):
        z = torch.complex(y[..., :D // 2], y[..., D // 2:]) * turn
        return torch.cat([z.real, z.imag], -1)

    z = torch.einsum("nimd,njmd->nmij", rotated(q), rotated(k)) * D ** -0.5
    z = 20.0 * torch.tanh(z / 20.0)
    seen = layer_ref.seen_pairs(N, L, L, u["doc"], u["doc"], u["prefix"])[:, None]
    e = torch.where(seen, torch.exp(z), torch.zeros_like(z))
    total = e.sum(-1, keepdim=True)
    o = torch.einsum("nmij,njmd->nimd", e / torch.where(total > 0, total, torch.ones_like(total)), v)
    params = [u[w].requires_grad_() for w in ("w1", "b1", "w2", "b2")]
    y = torch.nn.functional.layer_norm(x + o.reshape(N, L, C), (C,), params[0], params[1])
    s = msda.forward(t["value"], SHAPES, STARTS, t["loc"], t["attn"]).cpu().double()
    out = torch.nn.functional.layer_norm(y + s, (C,), params[2], params[3])
    g = torch.autograd.grad(out, [x] + leaves + params, u["grad"])
    return dict(zip(("out", "gx", "gq", "gk", "gv", "gw1", "gb1", "gw2", "gb2"), (out.detach(),) + g))


def test_decoder_layer_in_fp32():
    t = inputs(1)
    say("a decoder layer of the operators together")
    got, want = layer(t), layer64(t)
    for name, w in want.items():
        # a chain of at most ten fp32 operators, each within 3e-6 of its result's norm (products of 128 terms, sums
        # of 90 keys or 180 rows), with condition numbers of some units
        err = float((got[name].cpu().double() - w).norm() / w.norm())
        say(f"  {name}: {err:.2e}")
        assert err <= 3e-5, name


def test_decoder_layer_captured_and_replayed():
    import torch

    t = inputs(2)
    say("a decoder layer captured into a graph")
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        layer(t)  # warm: libraries and the allocator
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = layer(t)
    for seed in (3, 4, 5):
        new = inputs(seed)
        for name in t:
            t[name].copy_(new[name])
        graph.replay()
        torch.cuda.synchronize()
        eager = layer(new)  # between the replays, on the same allocator
        torch.cuda.synchronize()
        for name, w in eager.items():
            if name == "gvalue":  # its sums' order is not fixed
                assert float((captured[name] - w).abs().max()) <= 1e-5 * float(w.abs().max())
            else:
                assert torch.equal(captured[name], w), name


def test_two_captured_graphs_with_workspaces_of_their_own():
    import torch

    say("two captured graphs replayed at once")
    pair = []
    for seed in (6, 7):
        t = inputs(seed)
        layer(t)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            res = layer(t)
        pair.append((graph, res, layer(t), t))  # a graph reads its inputs where they were
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        for s, (graph, _, _, _) in zip(streams, pair):
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        for _, res, want, _ in pair:
            for name in ("out", "gq", "gk", "gv", "gw1", "gb1"):
                assert torch.equal(res[name], want[name]), name
