"""Query and key heads at the edges of what the entry points take, on the GPU:
kinds without heads,
heads beside others that have no norm or are missing, heads of subnormals
and of the largest values, gain gradients over many tokens.  Bounds as in test_gpu_qk_norm_rope."""
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


@pytest.mark.parametrize("D,R,inter", [(128, 128, False), (64, 32, True), (256, 0, False), (512, 512, False)])
def test_a_head_does_not_depend_on_its_neighbours(D, R, inter):
    # the same heads by themselves, beside others, and beside heads of zeros, of
    # tiny and of huge values (whose squares leave the float range), NaN among them
    T, H = 3000, 3
    c = Case(T, 16, 16, D, R, inter)
    q, gq = c.qkv[:, :16 * D].view(T, 16, D).to(DEV), c.gq.to(DEV)
    beside = q.clone()
    beside[:, H] = 0
    beside[:, H + 1] *= 1e-30
    beside[:, H + 2] *= 1e30
    beside[1::2, H + 3] = float("nan")
    # and, of every other token, one of the heads itself
    beside[::2, 1] = 0
    keep = torch.ones(T, H, dtype=torch.bool, device=DEV)
    keep[::2, 1] = False
    args = (c.on_gpu()[0], None, *c.on_gpu()[2:])

    def both(x, gy):
        y, _ = mxnorm.qk_norm_rope_fwd(x, x[:, :0], *args, **c.kw())
        g = mxnorm.qk_norm_rope_bwd(gy, gy[:, :0], x, x[:, :0], *args, **c.kw())
        return y[:, :H], g[0][:, :H]
    for got in (both(q[:, :H], gq[:, :H]), both(q[:, :H + 1], gq[:, :H + 1]), both(beside, gq)):
        for a, b in zip(got, both(q, gq)):
            assert torch.equal(a[keep], b[keep])


@pytest.mark.parametrize("D,R,inter,Hq,Hk", [(128, 128, False, 8, 8), (64, 32, True, 3, 1), (512, 0, False, 2, 1),
                                             (512, 512, False, 2, 2), (8, 0, False, 5, 1)])
def test_heads_of_subnormals_without_eps(D, R, inter, Hq, Hk):
    # multiples of 2^-133, the least value: an inverse RMS of up to 2^133 sqrt(D)
    T = 12
    c = Case(T, Hq, Hk, D, R, inter, eps=0.0)
    g = torch.Generator().manual_seed(D + R)
    k = torch.randint(-127, 128, (T, Hq + 2 * Hk, D), generator=g)
    k[1] %= 2
    k[2] = 0
    k[1:3, :, 3] = -1                    # one element alone
    k = k.reshape(T, -1)
    bits = k.abs() | (k < 0).long() << 15
    some = torch.arange(T) % 4 != 3      # and tokens of ordinary heads beside them
    c.qkv = torch.where(some[:, None], bits.to(torch.int16).view(torch.bfloat16), c.qkv)
    q, kk = c.views(c.qkv.to(DEV))
    hq, hk = c.views(c.qkv)
    y = mxnorm.qk_norm_rope_fwd(q, kk, *c.on_gpu(), **c.kw())
    c.check_forward(y[0], hq, 0)
    c.check_forward(y[1], hk, 1)
    # output gradients under which those of x stay below the largest bf16: 2^-30 2^138
    c.gq, c.gk = c.gq * 2.0 ** -30, c.gk * 2.0 ** -30
    gx = mxnorm.qk_norm_rope_bwd(c.gq.to(DEV), c.gk.to(DEV), q, kk, *c.on_gpu(), **c.kw())
    c.check_backward(gx[0], gx[2], hq, c.gq, 0)
    c.check_backward(gx[1], gx[3], hk, c.gk, 1)


def test_gain_gradients_do_not_lose_bits_with_the_tokens():
    # 2^27 equal heads, 4096 of them to a lane: a float sum of so many is 2.5e-5
    # off in the median.  Bound: r 2^-20, x r and its product 2^-24 each, 64 terms in
    # float 64 2^-24, then double, rounded to float twice: below 2^-17.6
    T, H, D = 1 << 21, 64, 8
    g = torch.Generator().manual_seed(1)
    x, gy = [torch.randn(1, 1, D, generator=g).bfloat16() for _ in range(2)]
    gain = torch.ones(D, dtype=torch.bfloat16, device=DEV)
    q, dq = [t.to(DEV).expand(T, H, D) for t in (x, gy)]
    got = mxnorm.qk_norm_rope_bwd(dq, dq[:, :1], q, q[:, :1], gain, gain, None, None, rotary=0)
    xd = x.double().flatten()
    term = xd * (xd.square().mean() + 1e-6).rsqrt() * gy.double().flatten()
    for gg, n in ((got[2], T * H), (got[3], T)):
        err = (gg.cpu().double() / (term * n) - 1).abs()
        assert (err <= 2.0 ** -17.6).all(), err.max()


@pytest.mark.parametrize("D,R,inter,Hq,Hk", [(128, 128, False, 8, 8), (64, 32, True, 3, 1), (512, 512, False, 2, 1)])
def test_heads_of_the_largest_values(D, R, inter, Hq, Hk):
    # from 2^126 up to the largest bf16 number: an inverse RMS below 2^-126, a
    # subnormal with 21 bits or more, 2^-22 of it (the bounds count 2^-20 for it)
    c = Case(11, Hq, Hk, D, R, inter, eps=0.0)
    g = torch.Generator().manual_seed(D)
    bits = torch.randint(0x7E80, 0x7F80, c.qkv.shape, generator=g) | torch.randint(0, 2, c.qkv.shape, generator=g) << 15
    some = torch.arange(11) % 4 != 3     # and tokens of ordinary heads beside them
    c.qkv = torch.where(some[:, None], bits.to(torch.int16).view(torch.bfloat16), c.qkv)
    assert c.qkv.isfinite().all()
    q, k = c.views(c.qkv.to(DEV))
    hq, hk = c.views(c.qkv)
    y = mxnorm.qk_norm_rope_fwd(q, k, *c.on_gpu(), **c.kw())
    c.check_forward(y[0], hq, 0)
    c.check_forward(y[1], hk, 1)
    # gradients of x well above the subnormals: 2^60 2^-128
    c.gq, c.gk = c.gq * 2.0 ** 60, c.gk * 2.0 ** 60
    gx = mxnorm.qk_norm_rope_bwd(c.gq.to(DEV), c.gk.to(DEV), q, k, *c.on_gpu(), **c.kw())
    c.check_backward(gx[0], gx[2], hq, c.gq, 0)
    c.check_backward(gx[1], gx[3], hk, c.gk, 1)
