"""The norm and rotation of query and key heads, and its gradients, on the GPU
against a plain implementation in 64 bits.

Bounds, from the arithmetic that include/mxnorm.h states: with (a, b) a pair
before (or, backward, its gradient after) the turn, the angle's fraction is
rounded to float (2^-26 turns = 2^-23.3 radians), sine and cosine are within two
units (2^-22), two products by r and gamma and the turn's two operations 2^-24
each: 2^-21 (|a| + |b|).  A head's sum takes 16 additions in a lane and up to 5
between lanes, of positive terms: 21 2^-24 of the sum, half of that in r, its
square root a unit more: 2^-20.5.  Together below 2^-19.6 before the rounding to
bf16, half a step or 2^-8 |y|.  k adds the same number of terms: 2^-19.6 of the
sum of their magnitudes.  Bounds below take 2^-19."""
import numpy as np
import pytest
import torch

from paper_2603_13180_amd import mxnorm

DEV = "cuda:0"
HALF = 2.0 ** -8   # half a bf16 step
E = 2.0 ** -19


@pytest.fixture(autouse=True)
def _need_gpu(request):
    if request.node.get_closest_marker("gpu"):
        if not torch.cuda.is_available():
            raise RuntimeError("these tests need a GPU (run them with -m gpu on an MI355X)")
        mxnorm.load()


def turned(y, pos, freq, R, inter, back=False):
    """y with the first R elements turned, and per element |a| + |b| of its pair."""
    i = torch.arange(R)
    first, second = (i[0::2], i[1::2]) if inter else (i[:R // 2], i[R // 2:])
    t = (pos.double()[:, None, None] * freq.double()) * (-1 if back else 1)
    a, b = y[..., first], y[..., second]
    out, mag = y.clone(), y.detach().abs().clone()
    out[..., first] = a * torch.cos(t) - b * torch.sin(t)
    out[..., second] = b * torch.cos(t) + a * torch.sin(t)
    mag[..., first] = mag[..., second] = (a.abs() + b.abs()).detach()
    return out, mag


def forward(x, gamma, pos, freq, R, inter, eps):
    """(y, |a| + |b|) of float64 heads x [T, H, D]."""
    n = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + eps) * gamma
    return turned(n, pos, freq, R, inter)


def test_reference_gradients_by_differences():
    g = torch.Generator().manual_seed(0)
    x = torch.randn(3, 2, 24, generator=g, dtype=torch.float64, requires_grad=True)
    gamma = torch.randn(24, generator=g, dtype=torch.float64, requires_grad=True)
    freq, pos = torch.rand(8, generator=g), torch.tensor([0, 5, -3])
    for inter in (False, True):
        assert torch.autograd.gradcheck(lambda x, w: forward(x, w, pos, freq, 16, inter, 1e-3)[0], (x, gamma))


class Case:
    def __init__(self, T, Hq, Hk, D, R, inter, seed=0, far=4096, gains=True, eps=1e-6, pos=True):
        g = torch.Generator().manual_seed(seed + T + 7 * Hq + D)
        self.T, self.Hq, self.Hk, self.D, self.R, self.inter, self.eps = T, Hq, Hk, D, R, inter, eps
        self.qkv = (torch.randn(T, (Hq + 2 * Hk) * D, generator=g) * 2).bfloat16()
        self.gq, self.gk = [torch.randn(T, h, D, generator=g).bfloat16() for h in (Hq, Hk)]
        self.gammas = [(1 + 0.2 * torch.randn(D, generator=g)).bfloat16() if gains else None for _ in range(2)]
        self.pos = torch.randint(-far, far, (T,), generator=g) if pos else None
        self.freq = (10000.0 ** (-torch.arange(0, R, 2).double() / max(R, 1))).float()

    def views(self, buf):
        Hq, Hk, D = self.Hq, self.Hk, self.D
        return buf[:, :Hq * D].view(-1, Hq, D), buf[:, Hq * D:(Hq + Hk) * D].view(-1, Hk, D)

    def on_gpu(self):
        put = lambda t: None if t is None else t.to(DEV)  # noqa: E731
        return [put(t) for t in self.gammas] + [put(self.pos), put(self.freq)]

    def kw(self):
        return dict(rotary=self.R, interleaved=self.inter, eps=self.eps)

    def position(self):
        return torch.arange(self.T) if self.pos is None else self.pos

    def gamma64(self, i):
        return torch.ones(self.D, dtype=torch.float64) if self.gammas[i] is None else self.gammas[i].double()

    def check_forward(self, got, heads, i, ctx=""):
        want, mag = forward(heads.double(), self.gamma64(i), self.position(), self.freq, self.R, self.inter, self.eps)
        err = (got.cpu().double() - want).abs()
        assert (err <= HALF * want.abs() + E * mag).all(), (ctx, err.max())

    def check_backward(self, got, got_gain, heads, gy, i, ctx=""):
        x = heads.double().requires_grad_()
        w = self.gamma64(i).requires_grad_()
        forward(x, w, self.position(), self.freq, self.R, self.inter, self.eps)[0].backward(gy.double())
        _, mag = turned(gy.double(), self.position(), self.freq, self.R, self.inter, back=True)
        xd, wd = heads.double(), w.detach().abs()
        r = torch.rsqrt((xd * xd).mean(-1, keepdim=True) + self.eps)
        scale = r * wd * mag + r ** 3 / self.D * xd.abs() * (wd * mag * xd.abs()).sum(-1, keepdim=True)
        err = (got.cpu().double() - x.grad).abs()
        assert (err <= HALF * x.grad.abs() + E * scale).all(), (ctx, err.max())
        if got_gain is not None:
            # at most 64 heads in a row and 64 lanes are added in float
            terms = (r * xd.abs() * mag).sum((0, 1))
            err = (got_gain.cpu().double() - w.grad).abs()
            assert (err <= 2.0 ** -17 * terms).all(), (ctx, (err / terms).max())


SHAPES = [
    (1, 1, 1, 64, 64, False), (1, 32, 8, 128, 128, False), (3, 5, 1, 128, 128, True), (16, 32, 8, 128, 128, False),
    (37, 12, 4, 64, 32, True), (65, 7, 7, 80, 80, False), (50, 3, 1, 96, 48, False), (29, 4, 2, 256, 256, True),
    (11, 3, 2, 256, 64, False), (7, 2, 1, 512, 512, False), (9, 3, 1, 512, 128, True), (33, 9, 3, 24, 16, False),
    (20, 2, 2, 8, 0, False), (13, 2, 1, 40, 0, True), (21, 17, 2, 72, 64, False), (5000, 2, 1, 64, 64, False),
    (4099, 3, 1, 32, 16, True),
]


@pytest.mark.gpu
@pytest.mark.parametrize("shape", SHAPES)
def test_forward(shape):
    c = Case(*shape)
    q, k = c.views(c.qkv.to(DEV))
    yq, yk = mxnorm.qk_norm_rope_fwd(q, k, *c.on_gpu(), **c.kw())
    hq, hk = c.views(c.qkv)
    c.check_forward(yq, hq, 0, "q")
    c.check_forward(yk, hk, 1, "k")


@pytest.mark.gpu
@pytest.mark.parametrize("shape", SHAPES)
def test_backward(shape):
    c = Case(*shape)
    q, k = c.views(c.qkv.to(DEV))
    args = (c.gq.to(DEV), c.gk.to(DEV), q, k, *c.on_gpu())
    gqkv = torch.full(c.qkv.shape, 7.0, dtype=torch.bfloat16, device=DEV)
    oq, ok = c.views(gqkv)
    got = mxnorm.qk_norm_rope_bwd(*args, grad_q=oq, grad_k=ok, **c.kw())
    hq, hk = c.views(c.qkv)
    c.check_backward(oq, got[2], hq, c.gq, 0, "q")
    c.check_backward(ok, got[3], hk, c.gk, 1, "k")
    assert (gqkv[:, (c.Hq + c.Hk) * c.D:] == 7.0).all()   # the values' part is the caller's
    again = mxnorm.qk_norm_rope_bwd(*args, **c.kw())
    for a, b in zip(got, again):
        assert torch.equal(a, b)


@pytest.mark.gpu
@pytest.mark.parametrize("far", [1 << 20, 1 << 27])
@pytest.mark.parametrize("inter", [False, True])
def test_far_positions(far, inter):
    c = Case(64, 4, 2, 128, 128, inter, far=far)
    q, k = c.views(c.qkv.to(DEV))
    yq, yk = mxnorm.qk_norm_rope_fwd(q, k, *c.on_gpu(), **c.kw())
    hq, hk = c.views(c.qkv)
    c.check_forward(yq, hq, 0)
    c.check_forward(yk, hk, 1)


@pytest.mark.gpu
def test_no_gains_and_counted_positions():
    c = Case(45, 6, 2, 128, 64, False, gains=False, pos=False)
    q, k = c.views(c.qkv.to(DEV))
    yq, yk = mxnorm.qk_norm_rope_fwd(q, k, *c.on_gpu(), **c.kw())
    hq, hk = c.views(c.qkv)
    c.check_forward(yq, hq, 0)
    c.check_forward(yk, hk, 1)
    gx = mxnorm.qk_norm_rope_bwd(c.gq.to(DEV), c.gk.to(DEV), q, k, *c.on_gpu(), **c.kw())
    assert gx[2] is None and gx[3] is None
    c.check_backward(gx[0], None, hq, c.gq, 0)
    c.check_backward(gx[1], None, hk, c.gk, 1)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [19, 4100])
def test_layouts_and_in_place(T):
    # heads before tokens, views with gaps, the input as the output
    c = Case(T, 5, 3, 64, 64, False)
    q, k = c.views(c.qkv.to(DEV))
    want = mxnorm.qk_norm_rope_fwd(q, k, *c.on_gpu(), **c.kw())
    buf = torch.full((2, 5, T + 1, 2, 64), 7.0, dtype=torch.bfloat16, device=DEV)
    oq, ok = buf[0, :, :T, 0].transpose(0, 1), buf[1, 1:4, :T, 1].transpose(0, 1)
    mxnorm.qk_norm_rope_fwd(q, k, *c.on_gpu(), q_out=oq, k_out=ok, **c.kw())
    assert torch.equal(oq, want[0]) and torch.equal(ok, want[1])
    oq.fill_(7.0)
    ok.fill_(7.0)
    assert (buf == 7.0).all()
    wide = torch.zeros(3, T, 8, 128, dtype=torch.bfloat16, device=DEV)[1, :, 2:7, 64:]
    wide.copy_(q)
    got = mxnorm.qk_norm_rope_fwd(wide, k, *c.on_gpu(), q_out=wide, k_out=ok, **c.kw())
    assert got[0] is wide and torch.equal(wide, want[0]) and torch.equal(ok, want[1])
    args = (q, k, *c.on_gpu())
    gq, gk = c.gq.to(DEV), c.gk.to(DEV)
    wantg = mxnorm.qk_norm_rope_bwd(gq, gk, *args, **c.kw())
    got = mxnorm.qk_norm_rope_bwd(gq, gk, *args, grad_q=gq, grad_k=gk, **c.kw())
    assert all(torch.equal(a, b) for a, b in zip(got, wantg))
    # one head's gradient for all heads, one token's input for all tokens
    shared = c.gk[:, :1].to(DEV).expand(-1, 3, -1)
    a = mxnorm.qk_norm_rope_bwd(c.gq.to(DEV), shared, *args, **c.kw())
    b = mxnorm.qk_norm_rope_bwd(c.gq.to(DEV), shared.contiguous(), *args, **c.kw())
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    one = q[:1].expand(T, -1, -1)
    a = mxnorm.qk_norm_rope_fwd(one, k, *c.on_gpu(), **c.kw())
    b = mxnorm.qk_norm_rope_fwd(one.contiguous(), k, *c.on_gpu(), **c.kw())
    assert torch.equal(a[0], b[0])


@pytest.mark.gpu
def test_heads_without_norm_and_not_finite():
    # an all-zero head without epsilon gives zeros; what is not finite stays in
    # its own head; infinite values have no inverse RMS but 0
    c = Case(6, 4, 2, 128, 64, False, eps=0.0)
    c.qkv[1, :128] = 0
    c.qkv[2, 128:256] = float("nan")
    c.qkv[3, 300] = float("inf")
    c.qkv[4, 4 * 128] = float("nan")
    q, k = c.views(c.qkv.to(DEV))
    yq, yk = mxnorm.qk_norm_rope_fwd(q, k, *c.on_gpu(), **c.kw())
    assert (yq[1, 0] == 0).all() and yq[2, 1].isnan().all() and yk[4, 0].isnan().all()
    head = yq[3, 2].cpu()                       # element 44 = 300 - 256, paired with 12
    bad = torch.zeros(128, dtype=torch.bool)
    bad[[44, 12]] = True
    assert (head[~bad] == 0).all() and head[bad].isnan().all()
    gx = mxnorm.qk_norm_rope_bwd(c.gq.to(DEV), c.gk.to(DEV), q, k, *c.on_gpu(), **c.kw())
    assert (gx[0][1, 0] == 0).all() and gx[0][2, 1].isnan().all()
    hq, hk = c.views(c.qkv)
    ok = torch.tensor([True, False, False, False, True, True])
    for name in ("pos", "gq", "gk", "qkv"):
        setattr(c, name, getattr(c, name)[ok])
    c.T = 3
    hq, _ = c.views(c.qkv)
    c.check_forward(yq[ok.to(DEV)], hq, 0)
    c.check_backward(gx[0][ok.to(DEV)], None, hq, c.gq, 0)


@pytest.mark.gpu
def test_large_and_tiny_values():
    # squares beyond the float range, and below it
    for scale in (1e30, 1e-30):
        c = Case(8, 2, 1, 128, 128, True, eps=0.0)
        c.qkv = (c.qkv.float() * scale).bfloat16()
        q, k = c.views(c.qkv.to(DEV))
        y = mxnorm.qk_norm_rope_fwd(q, k, *c.on_gpu(), **c.kw())
        hq, hk = c.views(c.qkv)
        c.check_forward(y[0], hq, 0)
        c.check_forward(y[1], hk, 1)
        gx = mxnorm.qk_norm_rope_bwd(c.gq.to(DEV), c.gk.to(DEV), q, k, *c.on_gpu(), **c.kw())
        c.check_backward(gx[0], gx[2], hq, c.gq, 0)
        c.check_backward(gx[1], gx[3], hk, c.gk, 1)


@pytest.mark.gpu
def test_no_tokens_or_heads():
    c = Case(4, 2, 1, 64, 64, False)
    q, k = c.views(c.qkv.to(DEV))
    y = mxnorm.qk_norm_rope_fwd(q[:0], k[:0], c.on_gpu()[0], None, c.on_gpu()[2][:0], c.on_gpu()[3], **c.kw())
    assert y[0].shape == (0, 2, 64)
    g = mxnorm.qk_norm_rope_bwd(q[:0], k[:0], q[:0], k[:0], *c.on_gpu()[:2], c.on_gpu()[2][:0], c.on_gpu()[3], **c.kw())
    assert (g[2] == 0).all() and (g[3] == 0).all()
    y = mxnorm.qk_norm_rope_fwd(q, k[:, :0], *c.on_gpu(), **c.kw())
    hq, _ = c.views(c.qkv)
    c.check_forward(y[0], hq, 0)
    g = mxnorm.qk_norm_rope_bwd(c.gq.to(DEV), k[:, :0], q, k[:, :0], *c.on_gpu(), **c.kw())
    c.check_backward(g[0], g[2], hq, c.gq, 0)
    assert (g[3] == 0).all()


@pytest.mark.gpu
def test_another_stream_and_a_captured_graph():
    c = Case(130, 4, 2, 128, 128, False)
    q, k = c.views(c.qkv.to(DEV))
    args = (q, k, *c.on_gpu())
    gq, gk = c.gq.to(DEV), c.gk.to(DEV)

    def both():
        return (*mxnorm.qk_norm_rope_fwd(*args, **c.kw()), *mxnorm.qk_norm_rope_bwd(gq, gk, *args, **c.kw()))
    want = both()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = both()
    torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both()
    for seed in range(3):
        q.copy_(torch.randn(q.shape, device=DEV, generator=torch.Generator(device=DEV).manual_seed(seed)))
        graph.replay()
        want = both()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


# -------------------------------------------------------------- refusals (CPU) --

A16, A8, A4 = 0x10000, 0x10008, 0x10004


def heads(data=A16, n=4, st=512, sh=64):
    return mxnorm._Heads(data, n, st, sh)


FWD = [
    (dict(T=-1), 1), (dict(D=0), 1), (dict(D=60), 1), (dict(D=1024, R=64), 2), (dict(R=8), 1), (dict(R=128), 1),
    (dict(R=-16), 1), (dict(eps=-1.0), 1), (dict(eps=float("nan")), 1), (dict(eps=float("inf")), 1),
    (dict(freq=None), 1), (dict(freq=A16 + 2), 1), (dict(pos=A4), 1), (dict(qg=A8), 1), (dict(kg=A8), 1),
    (dict(q=None), 1), (dict(k=None), 1), (dict(qo=None), 1), (dict(q=heads(data=None)), 1),
    (dict(q=heads(data=A8)), 1), (dict(q=heads(st=516)), 1), (dict(q=heads(sh=60)), 1), (dict(q=heads(st=-512)), 1),
    (dict(q=heads(st=1 << 62)), 1), (dict(q=heads(n=-1), qo=heads(n=-1)), 1), (dict(q=heads(n=5)), 1),
    (dict(q=heads(n=1 << 17), qo=heads(n=1 << 17)), 2), (dict(T=1 << 41), 2),
    (dict(qo=heads(st=0)), 1), (dict(qo=heads(sh=0)), 1), (dict(qo=heads(sh=32)), 1), (dict(qo=heads(st=128)), 1),
    (dict(qo=heads(st=64, sh=64)), 1), (dict(ko=heads(st=64, sh=448)), 1),
    (dict(T=0, q=heads(data=None), qo=heads(data=None), freq=None), 0),
]


def call(kw, bwd=False):
    a = dict(q=heads(), k=heads(), qg=A16, kg=A16, T=8, D=64, R=64, pos=A16, freq=A4, eps=1e-6, qo=heads(), ko=heads(),
             gq=heads(), gk=heads(), gqg=A4, gkg=A4, ws=A16, wb=1 << 30)
    a.update(kw)
    import ctypes
    ref = lambda h: None if h is None else ctypes.byref(h)  # noqa: E731
    tail = (a["qg"], a["kg"], a["T"], a["D"], a["R"], a["pos"], a["freq"], 0, a["eps"], ref(a["qo"]), ref(a["ko"]))
    lib = mxnorm.load()
    if not bwd:
        return lib.qk_norm_rope_fwd(ref(a["q"]), ref(a["k"]), *tail, None)
    return lib.qk_norm_rope_bwd(ref(a["gq"]), ref(a["gk"]), ref(a["q"]), ref(a["k"]), *tail, a["gqg"], a["gkg"],
                                a["ws"], a["wb"], None)


@pytest.mark.parametrize("kw,status", FWD)
def test_refusals(kw, status):
    assert call(kw) == status
    assert (mxnorm.mx_last_error() != "") == (status != 0)
    if status:
        assert call(kw, bwd=True) == status


@pytest.mark.parametrize("kw", [
    dict(gq=None), dict(gk=heads(data=None)), dict(gq=heads(n=3)), dict(gq=heads(st=4)), dict(gqg=A16 + 2),
    dict(gkg=A16 + 2), dict(ws=None), dict(ws=A8), dict(wb=64),
])
def test_backward_refusals(kw):
    assert call(kw, bwd=True) == 1 and mxnorm.mx_last_error() != ""


def test_backward_workspace():
    f = mxnorm.load().qk_norm_rope_bwd_workspace_bytes
    assert f(1, 128) == 2 * 2 * 128 * 4 and f(1 << 20, 128) == 512 * 2 * 128 * 4
    assert f(0, 128) == 0 and f(8, 1024) == 0 and f(-1, 64) == 0


def test_binding_refuses():
    q, k = torch.zeros(4, 2, 64, dtype=torch.bfloat16), torch.zeros(4, 1, 64, dtype=torch.bfloat16)
    with pytest.raises(RuntimeError, match="GPU"):
        mxnorm.qk_norm_rope_fwd(q, k, None, None, None, None)
    with pytest.raises(TypeError):
        mxnorm.qk_norm_rope_fwd(q.float(), k, None, None, None, None)
    with pytest.raises(TypeError):
        mxnorm.qk_norm_rope_fwd(q.view(4, 128), k, None, None, None, None)
