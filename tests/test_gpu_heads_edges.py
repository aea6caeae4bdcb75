"""Query and key heads at the edges of what the entry points take, on the GPU:
kinds without heads.  Bounds as in test_gpu_qk_norm_rope."""
import pytest
import torch

from paper_2603_13180_amd import mxnorm
from test_gpu_qk_norm_rope import DEV, Case

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        raise RuntimeError("these tests need a GPU (run them with -m gpu on an MI355X)")
    mxnorm.load()


@pytest.mark.parametrize("R", [0, 16, 64])
@pytest.mark.parametrize("T", [1, 9, 1500])
@pytest.mark.parametrize("Hq,Hk", [(3, 0), (0, 2), (16, 0), (0, 0)])
def test_kinds_without_heads(T, Hq, Hk, R):
    c = Case(T, Hq, Hk, 64, R, False)
    hq, hk = c.qkv[:, :Hq * 64].view(T, Hq, 64), c.qkv[:, Hq * 64:(Hq + Hk) * 64].view(T, Hk, 64)
    q, k = hq.to(DEV), hk.to(DEV)
    yq, yk = mxnorm.qk_norm_rope_fwd(q, k, *c.on_gpu(), **c.kw())
    gq, gk, gqg, gkg = mxnorm.qk_norm_rope_bwd(c.gq.to(DEV), c.gk.to(DEV), q, k, *c.on_gpu(), **c.kw())
    for i, (y, g, gg, heads, gy) in enumerate([(yq, gq, gqg, hq, c.gq), (yk, gk, gkg, hk, c.gk)]):
        assert y.shape == g.shape == heads.shape
        if heads.shape[1]:
            c.check_forward(y, heads, i)
            c.check_backward(g, gg, heads, gy, i)
        else:
            assert (gg == 0).all()
