"""Calls of msda_attention_forward / msda_attention_backward at the edges of what the header allows, against 64-bit
attention (tests/layer_ref.py)."""
import pytest

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
