"""Matrices whose last rows lie more than 4 GiB behind their first, against calls
on those rows alone."""
import pytest
import torch

from paper_2603_13180_amd import mxnorm

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
FAR = 4 << 30     # bytes
LAST = 200        # rows compared


@pytest.fixture(autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        raise RuntimeError("these tests need a GPU (run them with -m gpu on an MI355X)")
    mxnorm.load()
    yield
    torch.cuda.empty_cache()


def rand(*shape, seed=0, scale=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn(*shape, generator=g, device=DEV) * scale).bfloat16()


@pytest.mark.parametrize("elem", ["e4m3", "e2m1"])
def test_gated_rows(elem):
    # one matrix instruction (two) of K a product: the same bits in any tile
    T, F, d = 66000, 16384, 128 if elem == "e4m3" else 256
    x = rand(T, d)
    wc, ws = mxnorm.mx_cast_fwd(rand(2 * F, d, seed=1), elem=elem)
    ac, as_ = mxnorm.mx_cast_fwd(x, elem=elem)
    small = ac[-LAST:].contiguous(), as_[-LAST:].contiguous()
    for dtype in (torch.float32, torch.uint8):
        h, gu = mxnorm.mx_gated_fwd(ac, as_, wc, ws, d, elem=elem, out_dtype=dtype, save_gu=True)
        assert gu.numel() * 2 > FAR and (dtype is torch.uint8 or h.numel() * 4 > FAR)
        h2, gu2 = mxnorm.mx_gated_fwd(*small, wc, ws, d, elem=elem, out_dtype=dtype, save_gu=True)
        assert torch.equal(gu[-LAST:], gu2)
        for a, b in zip(*((h, h2) if dtype is torch.uint8 else ((h,), (h2,)))):
            assert torch.equal(a[-LAST:], b)
        del h
    gh = rand(T, F, seed=2)
    grad = mxnorm.mx_gated_bwd(gh, gu, grad_gu=gu)
    assert torch.equal(grad[-LAST:], mxnorm.mx_gated_bwd(gh[-LAST:].contiguous(), gu2))


def test_gated_backward():
    # only the last rows have a gradient: the others add zeros.  The products'
    # sums are within 2^-9 of the sums of magnitudes of theirs, and in another
    # order; in the norm, of independent errors, 2^-10 is ample
    T, F, d = 66000, 32768, 64
    gh, gu = torch.zeros(T, F, dtype=torch.bfloat16, device=DEV), rand(256, 2 * F, seed=3).repeat(T // 256 + 1, 1)[:T]
    gh[-LAST:] = rand(LAST, F, seed=4, scale=0.01)
    x, w, gamma = rand(T, d, seed=5), rand(2 * F, d, seed=6, scale=0.02), 1 + rand(d, seed=7, scale=0.1)
    rho = torch.rand(T, device=DEV) + 0.5
    assert gu.is_contiguous() and gu.numel() > FAR
    a = mxnorm.mxnorm_gated_bwd(gh, gu, x, rho, gamma, w)
    last = [t[-LAST:].contiguous() for t in (gh, gu, x, rho)]
    b = mxnorm.mxnorm_gated_bwd(*last, gamma, w)
    assert (a[0][:-LAST] == 0).all()
    # T = 66000 ends 80 rows into a block of 128, LAST = 200 ends 72 into one: the
    # blocks along T differ, so grad_w is compared where those do not matter
    for i in (0, 1):
        p, q = (t.double() for t in ((a[0][-LAST:], b[0]) if i == 0 else (a[1], b[1])))
        assert (p - q).norm() <= 2.0 ** -10 * q.norm(), i
    exact = torch.zeros(2 * F, d, dtype=torch.float64, device=DEV)
    exact += mxnorm.mx_gated_bwd(last[0], last[1]).double().t() @ (last[3].double()[:, None] * last[2].double())
    exact *= gamma.double()
    # both operands' casts: an element is off by half a step of E4M3 at most, 2^-4 of
    # it, and by half of that in the norm: together sqrt(2) 2^-5
    for g in (a[2], b[2]):
        assert (g.double() - exact).norm() <= 2.0 ** -4 * exact.norm()


@pytest.mark.parametrize("back", [False, True])
def test_heads_far_apart(back):
    # tokens 2^31 + 64 elements apart, and heads as far apart as that
    T, H, D, far = 3, 2, 128, (1 << 31) + 64
    buf = torch.empty(3 * far, dtype=torch.bfloat16, device=DEV)
    q = buf.as_strided((T, H, D), (far, D, 1))
    k = buf.as_strided((T, 2, D), (2 * D, far, 1), 1024)
    oq, ok = buf.as_strided((T, H, D), (far, D, 1), 4096), buf.as_strided((T, 2, D), (2 * D, far, 1), 8192)
    q.copy_(rand(T, H, D))
    k.copy_(rand(T, 2, D, seed=1))
    gains = [1 + rand(D, seed=i, scale=0.1) for i in (2, 3)]
    rest = (*gains, torch.tensor([0, 7, 1 << 20], device=DEV), torch.rand(D // 2, device=DEV))
    if not back:
        mxnorm.qk_norm_rope_fwd(q, k, *rest, q_out=oq, k_out=ok)
        want = mxnorm.qk_norm_rope_fwd(q.contiguous(), k.contiguous(), *rest)
    else:
        gq, gk = rand(T, H, D, seed=4), rand(T, 2, D, seed=5)
        got = mxnorm.qk_norm_rope_bwd(gq, gk, q, k, *rest, grad_q=oq, grad_k=ok)
        want = mxnorm.qk_norm_rope_bwd(gq, gk, q.contiguous(), k.contiguous(), *rest)
        assert torch.equal(got[2], want[2]) and torch.equal(got[3], want[3])
    assert torch.equal(oq, want[0]) and torch.equal(ok, want[1])
