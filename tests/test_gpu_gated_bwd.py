"""The gradients of the gated feed-forward on the GPU: the gate's own against
64 bits, the whole backward against its definition in 64 bits from casts that
other tests hold to the oracle."""
import math

import numpy as np
import pytest
import torch

from paper_2603_13180_amd import mxnorm

DEV = "cuda:0"
ACTS = ["silu", "gelu_tanh"]
ELEMS = ["e4m3", "e2m1"]
HALF = 2.0 ** -8   # half a bf16 step


@pytest.fixture(autouse=True)
def _need_gpu(request):
    if request.node.get_closest_marker("gpu"):
        if not torch.cuda.is_available():
            raise RuntimeError("these tests need a GPU (run them with -m gpu on an MI355X)")
        mxnorm.load()


def gate64(g, act):
    """(sigma(z(g)), z'(g)) in 64 bits."""
    if act == "silu":
        return torch.sigmoid(g), torch.ones_like(g)
    c = 2 * math.sqrt(2 / math.pi)
    return torch.sigmoid(c * (g + 0.044715 * g ** 3)), c * (1 + 3 * 0.044715 * g * g)


def gradients64(gh, gu, act):
    """(dg, du) in float64, and how far float arithmetic may be from each: sigma
    is within 2^-14 s (1 - s) relatively to its exponential and 2^-22 in all
    (gate.h's arithmetic); the 2^-22 of 1 - sigma meets g z' <= 40 where sigma is
    not 1 in float (z < 17): 2^-16 sigma.  Doubled.  A sigma below 2^-126 is 0 in
    float (the reciprocal's subnormal results are), where dg's terms are below
    2^-126 |h u| (1 + |g| z') and du below 2^-126 |h g|, with |g| held at 128."""
    g, u = gu.double().chunk(2, 1)
    h = gh.double()
    s, dz = gate64(g, act)
    t = torch.where(s * (1 - s) == 0, torch.zeros_like(s), g * s * (1 - s) * dz)
    none = 2.0 ** -126 * h.abs()
    most = 1 + 128 * gate64(torch.full_like(g, 128.0), act)[1]
    return (h * u * (s + t), h * g * s,
            (h * u).abs() * (2.0 ** -13 * (s + t.abs()) + 2.0 ** -15 * s) + none * u.abs() * most,
            2.0 ** -13 * (h * g * s).abs() + none * g.abs())


@pytest.mark.parametrize("act", ACTS)
def test_reference_gradients_by_differences(act):
    gen = torch.Generator().manual_seed(1)
    gu = (torch.randn(4, 12, generator=gen, dtype=torch.float64) * 3).requires_grad_()
    gh = torch.randn(4, 6, generator=gen, dtype=torch.float64)

    def h(p):
        g, u = p.chunk(2, 1)
        return g * gate64(g, act)[0] * u
    assert torch.autograd.gradcheck(h, (gu,))
    want, = torch.autograd.grad(h(gu), gu, gh)
    dg, du, _, _ = gradients64(gh, gu.detach(), act)
    assert torch.allclose(torch.cat((dg, du), 1), want, rtol=1e-12, atol=1e-14)


def check_gate(got, gh, gu, act, only=None):
    dg, du, eg, eu = gradients64(gh, gu, act)
    for a, want, tol, name in zip(got.double().chunk(2, 1), (dg, du), (eg, eu), ("gate", "up")):
        # (below 2^-126 bf16 values lie 2^-133 apart: half that, absolutely)
        bad = (a - want).abs() > HALF * want.abs() + tol + 2.0 ** -134
        if only is not None:
            bad &= only
        at = bad.nonzero()[:4].tolist()
        assert not at, [(name, i, j, a[i, j].item(), want[i, j].item(), tol[i, j].item(), gu[i, j].item()) for i, j in at]


@pytest.mark.gpu
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("T,F", [(1, 8), (3, 24), (37, 96), (1000, 2048), (129, 4104)])
def test_gate_gradient(T, F, act):
    gen = torch.Generator(device=DEV).manual_seed(T + F)
    gu = (torch.randn(T, 2 * F, generator=gen, device=DEV) * 4).bfloat16()
    gh = torch.randn(T, F, generator=gen, device=DEV).bfloat16()
    buf = torch.full((T * 2 * F + 64,), 7.0, dtype=torch.bfloat16, device=DEV)
    got = mxnorm.mx_gated_bwd(gh, gu, act, grad_gu=buf[:T * 2 * F].view(T, 2 * F))
    assert (buf[T * 2 * F:] == 7.0).all()
    check_gate(got, gh, gu, act)
    assert torch.equal(mxnorm.mx_gated_bwd(gh, gu, act, grad_gu=gu), got)     # in place


@pytest.mark.gpu
@pytest.mark.parametrize("act", ACTS)
def test_gate_gradient_over_the_whole_range(act):
    # every bf16 gate value; the derivative of an infinite or huge one is 0 or 1
    g = torch.arange(65536, device=DEV, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    g = g.view(64, 1024)
    one = torch.ones(64, 1024, dtype=torch.bfloat16, device=DEV)
    got = mxnorm.mx_gated_bwd(one, torch.cat((g, one), 1), act)
    a, b = got.double().chunk(2, 1)
    assert a[g.isnan()].isnan().all() and b[g.isnan()].isnan().all()
    fin = g.isfinite()
    inf = g.isinf()
    assert (a[inf & (g > 0)] == 1).all() and (a[inf & (g < 0)] == 0).all()
    assert (b[inf & (g > 0)] == math.inf).all() and b[inf & (g < 0)].isnan().all()
    check_gate(got, one, torch.cat((g, one), 1), act, only=fin)


# ------------------------------------------------------- the whole backward --

def decode(codes, scales, elem):
    """Float64 values of MX codes."""
    if elem == "e4m3":
        v = codes.view(torch.float8_e4m3fn).double()
    else:
        n = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).long()
        v = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, 0, -.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64,
                         device=codes.device)[n]
    return v * torch.exp2(scales.double() - 127).repeat_interleave(32, 1)


def padded(t, elem):
    step = 128 if elem == "e4m3" else 256
    return torch.cat((t, t.new_zeros((-t.shape[0] % step,) + t.shape[1:])))


class Case:
    def __init__(self, T, F, d, seed=0, gain=True):
        gen = torch.Generator(device=DEV).manual_seed(seed + T + F + d)
        n = lambda *s: torch.randn(*s, generator=gen, device=DEV)  # noqa: E731
        self.T, self.F, self.d = T, F, d
        self.gh, self.gu = (0.1 * n(T, F)).bfloat16(), (2 * n(T, 2 * F)).bfloat16()
        self.x, self.w = n(T, d).bfloat16(), (0.1 * n(2 * F, d)).bfloat16()
        self.gamma = (1 + 0.2 * n(d)).bfloat16() if gain else None
        self.rho = 0.5 + torch.rand(T, generator=gen, device=DEV)

    def args(self):
        return self.gh, self.gu, self.x, self.rho, self.gamma, self.w

    def parts(self, elem, act):
        """The casts of the definition: grad_P by rows and by columns, W and
        rho X by columns, as (codes, scales)."""
        gp = mxnorm.mx_gated_bwd(self.gh, self.gu, act)
        return dict(gh=mxnorm.mx_cast_fwd(gp, elem=elem), ght=mxnorm.mx_cast_t_fwd(padded(gp, elem), elem=elem),
                    wt=mxnorm.mx_cast_t_fwd(self.w, elem=elem),
                    xt=mxnorm.mx_cast_t_fwd(padded(self.x, elem), padded(self.rho, elem), elem=elem))

    def check(self, got, elem, act):
        gx, gg, gw = (t.double() for t in got)
        step = [0.0 if t.dtype == torch.float32 else HALF for t in got]
        p = {k: decode(*v, elem) for k, v in self.parts(elem, act).items()}
        gz, mag = p["gh"] @ p["wt"].t().contiguous(), p["gh"].abs() @ p["wt"].abs().t().contiguous()
        # the product within 2^-9 of its magnitudes (mx_matmul_fwd), then bf16
        ez = 2.0 ** -9 * mag * (1 + HALF) + HALF * gz.abs()
        x, r = self.x.double(), self.rho.double()[:, None]
        w = torch.ones(self.d, dtype=torch.float64, device=DEV) if self.gamma is None else self.gamma.double()
        u = (gz * w * x).sum(1, keepdim=True)
        want = r * w * gz - r ** 3 / self.d * u * x
        back = r ** 3 / self.d * x.abs()
        tol = r * w.abs() * ez + back * (w.abs() * x.abs() * ez).sum(1, keepdim=True)
        tol += 2.0 ** -21 * (r * w.abs() * (gz.abs() + ez) + back * u.abs())
        err = (gx - want).abs()
        assert (err <= (1 + step[0]) * tol + step[0] * want.abs() + 1e-30).all(), ("grad_x", (err / tol).max())
        want, terms = (r * x * gz).sum(0), (r * x * gz).abs().sum(0)
        tol = (r * x.abs() * ez).sum(0) + 2.0 ** -17 * terms
        err = (gg - want).abs()
        assert (err <= (1 + step[1]) * tol + step[1] * want.abs() + 1e-30).all(), ("grad_gamma", (err / tol).max())
        want, mag = p["ght"] @ p["xt"].t().contiguous() * w, p["ght"].abs() @ p["xt"].abs().t().contiguous() * w.abs()
        tol = 2.0 ** -9 * mag + 2.0 ** -22 * want.abs()
        err = (gw - want).abs()
        assert (err <= (1 + step[2]) * tol + step[2] * want.abs() + 1e-30).all(), ("grad_w", (err / tol).max())


@pytest.mark.gpu
@pytest.mark.parametrize("grad_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("elem", ELEMS)
@pytest.mark.parametrize("T,F,d", [(1, 128, 16), (37, 128, 48), (128, 256, 272), (300, 384, 512), (1024, 512, 768),
                                   (1999, 896, 256)])
def test_whole_backward(elem, T, F, d, grad_dtype):
    act = ACTS[T % 2]
    c = Case(T, F, d)
    got = mxnorm.mxnorm_gated_bwd(*c.args(), elem=elem, act=act, grad_dtype=grad_dtype,
                                  grad_x_dtype=torch.bfloat16 if T % 3 else torch.float32)
    assert got[1].dtype == got[2].dtype == grad_dtype
    c.check(got, elem, act)
    again = mxnorm.mxnorm_gated_bwd(*c.args(), elem=elem, act=act, grad_dtype=grad_dtype,
                                    grad_x_dtype=torch.bfloat16 if T % 3 else torch.float32)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


@pytest.mark.gpu
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("elem", ELEMS)
@pytest.mark.parametrize("T,F,d", [(1, 128, 16), (37, 384, 48), (128, 128, 272), (300, 640, 512), (1025, 1152, 256),
                                   (160, 6272, 64), (150, 64, 32), (70, 192, 16), (200, 6208, 32),
                                   (4130, 8256, 48), (2100, 14400, 32)])
def test_casts_byte_for_byte(elem, act, T, F, d):
    if elem == "e2m1" and F % 128:
        F += 64
    # what the products take, in a workspace of the test's own: the casts of the
    # gradient that mx_gated_bwd gives, padded with rows of zeros.  6272: from 48
    # column tiles on they are visited in another order; the last two have over 2048
    # tiles, which are then of 128 columns, not 64.  Infinities and NaN too
    c = Case(T, F, d, seed=9)
    c.gh[T // 2, 5] = float("inf")
    c.gh[0, F - 1] = float("nan")
    c.gu[T - 1, 7] = -float("inf")
    c.gu[T - 1, F + 40] = 0.0
    lib, e = mxnorm.load(), mxnorm.ELEMS[elem]
    size = lib.mxnorm_gated_bwd_workspace_bytes(T, F, d, e)
    ws = torch.full((size + 256,), 7, dtype=torch.uint8, device=DEV)
    gx, gg, gw = [torch.empty(s, dtype=torch.bfloat16, device=DEV) for s in ((T, d), (d,), (2 * F, d))]
    mxnorm._check(lib.mxnorm_gated_bwd(
        c.gh.data_ptr(), c.gu.data_ptr(), c.x.data_ptr(), c.rho.data_ptr(), c.gamma.data_ptr(), c.w.data_ptr(),
        T, F, d, 32, e, mxnorm.ACTS[act], 1, 1, gx.data_ptr(), gg.data_ptr(), gw.data_ptr(), ws.data_ptr(), size,
        mxnorm._stream(c.x.device)))
    assert (ws[size:] == 7).all()
    at = 0
    parts = c.parts(elem, act)
    for name in ("gh", "wt", "ght", "xt"):
        for want, what in zip(parts[name], ("codes", "scales")):
            got = ws[at:at + want.numel()].view(want.shape)
            bad = (got != want).nonzero()
            assert not len(bad), (name, what, len(bad), bad[0].tolist(), got[tuple(bad[0])], want[tuple(bad[0])])
            at += (want.numel() + 255) // 256 * 256


@pytest.mark.gpu
def test_without_a_gain_and_narrow_feed_forward():
    for F in (64, 192):                       # a single partial tile of columns
        c = Case(200, F, 128, gain=False)
        c.check(mxnorm.mxnorm_gated_bwd(*c.args()), "e4m3", "silu")


@pytest.mark.gpu
def test_large_products():
    # 256 x 256 tiles shared out by load, gradients in both types
    for dt in (torch.float32, torch.bfloat16):
        c = Case(2304, 2048, 1024)
        c.check(mxnorm.mxnorm_gated_bwd(*c.args(), grad_dtype=dt), "e4m3", "silu")


@pytest.mark.gpu
def test_captured_graph_and_another_stream():
    c = Case(130, 256, 256)

    def run():
        return mxnorm.mxnorm_gated_bwd(*c.args(), grad_dtype=torch.bfloat16)
    want = run()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = run()
    torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run()
    for seed in range(3):
        c.gh.copy_(torch.randn(c.gh.shape, device=DEV, generator=torch.Generator(device=DEV).manual_seed(seed)))
        graph.replay()
        want = run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


@pytest.mark.gpu
def test_a_layer_forward_and_back():
    """The operators chained as a layer chains them, QKV projection, heads,
    feed-forward, and back; the gradient of the feed-forward against differences
    of its loss in 64 bits along the gradient itself."""
    T, d, F, Hq, Hk, D = 96, 256, 512, 4, 2, 64
    gen = torch.Generator(device=DEV).manual_seed(3)
    n = lambda *s: torch.randn(*s, generator=gen, device=DEV)  # noqa: E731
    x, gamma = n(T, d).bfloat16(), (1 + 0.1 * n(d)).bfloat16()
    w_qkv, w_gu = (0.06 * n((Hq + 2 * Hk) * D, d)).bfloat16(), (0.06 * n(2 * F, d)).bfloat16()
    w_down = (0.06 * n(d, F)).bfloat16()
    qg, kg = (1 + 0.1 * n(D)).bfloat16(), (1 + 0.1 * n(D)).bfloat16()
    freq = (10000.0 ** (-torch.arange(0, D, 2, device=DEV).double() / D)).float()
    # attention's inputs: normed and turned heads, in place in the projection
    qkv, _ = mxnorm.mxnorm_linear_fwd(x, *mxnorm.mx_cast_fwd(w_qkv, gamma))
    q, k = qkv[:, :Hq * D].view(T, Hq, D), qkv[:, Hq * D:(Hq + Hk) * D].view(T, Hk, D)
    yq, yk = mxnorm.qk_norm_rope_fwd(q, k, qg, kg, None, freq)
    assert torch.isfinite(yq.float()).all() and abs(yq.float().square().mean().item() - 1) < 0.2
    # the feed-forward, with the down projection's operand as codes and as bf16
    wc, ws = mxnorm.mx_cast_fwd(w_gu, gamma)
    dc, ds = mxnorm.mx_cast_fwd(w_down)
    (hc, hs), gu, rho = mxnorm.mxnorm_gated_fwd(x, wc, ws, out_dtype=torch.uint8, save_gu=True)
    y = mxnorm.mx_matmul_fwd(hc, hs, dc, ds, F)
    h, _, _ = mxnorm.mxnorm_gated_fwd(x, wc, ws)
    y2 = mxnorm.mx_matmul_fwd(*mxnorm.mx_cast_fwd(h), dc, ds, F)
    # H rounded to bf16 first: an element v moves by at most 2^-8 v, 2^-9 v on
    # average, and so crosses a code's border with probability 2^-9 v / step;
    # then it changes by the step, at most 2^-3 v: a mean square of 2^-9 2^-3 v^2,
    # 2^-6 in the norm.  Doubled
    assert (y - y2).norm() <= 2.0 ** -5 * y.norm()
    # back: a loss <y, v>
    v = n(T, d).bfloat16()
    gh = (v.double() @ w_down.double()).bfloat16()
    gx, gg, gw = mxnorm.mxnorm_gated_bwd(gh, gu, x, rho, gamma, w_gu)

    def loss(w):
        """The same function without casts, in 64 bits."""
        z = x.double() * rho.double()[:, None] * gamma.double()
        g, u = (z @ w.t().contiguous()).chunk(2, 1)
        return ((g * torch.sigmoid(g) * u) * (v.double() @ w_down.double())).sum()
    w = w_gu.double()
    # grad_w is that of the weight the gain is folded into, times the gain
    step = 1e-4 / gw.double().abs().max()
    slope = (loss(w + step * gw.double()) - loss(w - step * gw.double())) / (2 * step)
    # each cast moves a value by at most 2^-4, on average nothing: the slope
    # along grad_W is its norm squared to a few per cent
    assert abs(slope / gw.double().square().sum() - 1) < 2.0 ** -4
    # and the heads' gradient goes into the projection's
    gqkv = torch.zeros_like(qkv)
    oq, ok = gqkv[:, :Hq * D].view(T, Hq, D), gqkv[:, Hq * D:(Hq + Hk) * D].view(T, Hk, D)
    mxnorm.qk_norm_rope_bwd(yq, yk, q, k, qg, kg, None, freq, grad_q=oq, grad_k=ok)
    # T is no multiple of 128: the projection's backward takes whole blocks
    pad = lambda t: torch.cat((t, t.new_zeros((32,) + t.shape[1:])))  # noqa: E731
    _, rho1 = mxnorm.mxnorm_linear_fwd(x, *mxnorm.mx_cast_fwd(w_qkv, gamma))
    g = mxnorm.mxnorm_linear_bwd(pad(gqkv), pad(x), pad(rho1), gamma, w_qkv)
    assert all(torch.isfinite(t.float()).all() for t in g) and (g[0][T:] == 0).all()


# -------------------------------------------------------------- refusals (CPU) --

A16, A8, A4, W256 = 0x10000, 0x10008, 0x10004, 0x100000


@pytest.mark.parametrize("kw,status", [
    (dict(T=0), 1), (dict(F=0), 1), (dict(d=0), 1), (dict(T=-1), 1), (dict(F=96), 2), (dict(F=64, elem=1), 2),
    (dict(F=1 << 22), 2), (dict(T=(1 << 22) + 1), 2), (dict(d=24), 2), (dict(d=65536), 2), (dict(block=16), 2),
    (dict(elem=2), 1), (dict(act=2), 1), (dict(out_dtype=2), 1), (dict(grad_dtype=2), 1), (dict(gh=None), 1),
    (dict(gu=None), 1), (dict(x=None), 1), (dict(rho=None), 1), (dict(w=None), 1), (dict(grad_x=None), 1),
    (dict(grad_w=None), 1), (dict(gh=A8), 1), (dict(gu=A8), 1), (dict(x=A8), 1), (dict(w=A8), 1),
    (dict(rho=A16 + 2), 1), (dict(gamma=A8), 1), (dict(grad_x=A8), 1), (dict(grad_w=A8), 1),
    (dict(grad_gamma=A16 + 2), 1), (dict(ws=None), 1), (dict(ws=0x100010), 1), (dict(wb=4096), 1),
])
def test_whole_backward_refusals(kw, status):
    a = dict(gh=A16, gu=A16, x=A16, rho=A4, gamma=A16, w=A16, T=37, F=256, d=256, block=32, elem=0, act=0,
             out_dtype=1, grad_dtype=0, grad_x=A16, grad_gamma=A4, grad_w=A16, ws=W256, wb=1 << 60)
    a.update(kw)
    got = mxnorm.load().mxnorm_gated_bwd(a["gh"], a["gu"], a["x"], a["rho"], a["gamma"], a["w"], a["T"], a["F"],
                                         a["d"], a["block"], a["elem"], a["act"], a["out_dtype"], a["grad_dtype"],
                                         a["grad_x"], a["grad_gamma"], a["grad_w"], a["ws"], a["wb"], None)
    assert got == status
    assert mxnorm.mx_last_error() != ""


@pytest.mark.parametrize("args,status", [
    ((A16, A16, -1, 8, 0, A16), 1), ((A16, A16, 4, -8, 0, A16), 1), ((A16, A16, 4, 12, 0, A16), 1),
    ((A16, A16, 4, 8, 2, A16), 1), ((None, A16, 4, 8, 0, A16), 1), ((A16, None, 4, 8, 0, A16), 1),
    ((A16, A16, 4, 8, 0, None), 1), ((A8, A16, 4, 8, 0, A16), 1), ((A16, A8, 4, 8, 0, A16), 1),
    ((A16, A16, 4, 8, 0, A8), 1), ((A16, A16, 1 << 31, 8, 0, A16), 2), ((A16, A16, 4, (1 << 23) + 8, 0, A16), 2),
    ((None, None, 0, 8, 0, None), 0), ((None, None, 4, 0, 1, None), 0),
])
def test_gate_gradient_refusals(args, status):
    assert mxnorm.load().mx_gated_bwd(*args, None) == status
    assert (mxnorm.mx_last_error() != "") == (status != 0)


def test_binding_refuses():
    gh, gu = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(4, 128, dtype=torch.bfloat16)
    with pytest.raises(RuntimeError, match="GPU"):
        mxnorm.mx_gated_bwd(gh, gu)
    with pytest.raises(TypeError):
        mxnorm.mx_gated_bwd(gh.float(), gu)
    with pytest.raises(RuntimeError, match="GPU"):
        mxnorm.mxnorm_gated_bwd(gh, gu, gh, torch.zeros(4), None, gh)
    assert np.isfinite(mxnorm.load().mxnorm_gated_bwd_workspace_bytes(1, 64, 64, 0))
    for bad in ((0, 64, 64, 0), (1, 0, 64, 0), (1, 64, 0, 0), (1, 64, 64, 2)):
        assert mxnorm.load().mxnorm_gated_bwd_workspace_bytes(*bad) == 0
