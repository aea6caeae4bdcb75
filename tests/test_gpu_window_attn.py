"""Attention with a window and sinks, and its gradients, on the GPU against a
plain implementation in 64 bits (attn_reference.py, which derives the bounds)."""
import ctypes
import math

import pytest
import torch

from attn_reference import Attention, off, packed, visible
from paper_2603_13180_amd import mxnorm

DEV = "cuda:0"
gpu = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _need_gpu(request):
    if request.node.get_closest_marker("gpu"):
        if not torch.cuda.is_available():
            raise RuntimeError("these tests need a GPU (run them with -m gpu on an MI355X)")
        mxnorm.load()


def test_reference_gradients_by_differences():
    g = torch.Generator().manual_seed(0)
    q, k, v, go = (torch.randn(n, 8, generator=g, dtype=torch.float64) for n in (5, 7, 7, 5))
    see = visible(torch.arange(5) + 1, torch.arange(7), 3, 1)
    see[0] = False  # a query that sees nothing
    want = Attention(q, k, v, see, 0.3).gradients(go, 8)[0]
    for i, t in enumerate((q, k, v)):
        for e in range(0, t.numel(), 3):
            step = torch.zeros_like(t).view(-1)
            step[e] = 1e-6
            ends = [t + s * step.view_as(t) for s in (1, -1)]
            f = [(Attention(*(x if j == i else y for j, y in enumerate((q, k, v))), see, 0.3).o * go).sum() for x in ends]
            assert abs((f[0] - f[1]) / 2e-6 - want[i].view(-1)[e]) < 1e-8


class Case:
    """Packed sequences of the given numbers of queries and keys."""

    def __init__(self, queries, keys, Hq, Hk, D, seed=0, tail=0):
        g = torch.Generator(device=DEV).manual_seed(seed + 31 * sum(queries) + D)
        def rand(*s):
            return torch.randn(*s, generator=g, device=DEV).bfloat16()
        self.qs, self.ks = ([sum(n[:i]) for i in range(len(n) + 1)] for n in (queries, keys))
        self.T, self.S = self.qs[-1] + tail, self.ks[-1] + tail
        self.q, self.k, self.v = rand(self.T, Hq, D), rand(self.S, Hk, D), rand(self.S, Hk, D)
        self.go = rand(self.T, Hq, D)

    def starts(self):
        return dict(q_start=torch.tensor(self.qs, dtype=torch.int32, device=DEV),
                    k_start=torch.tensor(self.ks, dtype=torch.int32, device=DEV))

    def want(self, window, sinks, scale=None, back=True):
        return packed(self.q, self.k, self.v, self.qs, self.ks, window, sinks,
                      self.q.shape[2] ** -0.5 if scale is None else scale, self.go if back else None)

    def forward(self, window, sinks, **kw):
        return mxnorm.window_attn_fwd(self.q, self.k, self.v, window, sinks, **kw)

    def backward(self, o, lse, window, sinks, **kw):
        return mxnorm.window_attn_bwd(self.go, self.q, self.k, self.v, o, lse, window, sinks, **kw)


def check(c, window, sinks, scale=None, starts=True):
    kw = dict(scale=scale, **(c.starts() if starts else {}))
    want, bound = c.want(window, sinks, scale)
    o, lse = c.forward(window, sinks, **kw)
    n = c.qs[-1], c.ks[-1]
    worst = {"o": off(o[:n[0]], want["o"][:n[0]], bound["o"][:n[0]]),
             "lse": off(lse[:, :n[0]], want["lse"][:, :n[0]], bound["lse"][:, :n[0]])}
    assert max(worst.values()) <= 1, worst
    grads = c.backward(o, lse, window, sinks, **kw)
    worst = {name: off(t[:m], want[name][:m], bound[name][:m]) for name, t, m in zip(("gq", "gk", "gv"), grads, (n[0], n[1], n[1]))}
    assert max(worst.values()) <= 1, worst
    again = c.backward(o, lse, window, sinks, **kw)
    assert all(torch.equal(x[:m], y[:m]) for x, y, m in zip(grads, again, (n[0], n[1], n[1])))


SHAPES = [  # heads, head size
    (4, 2, 128), (3, 1, 64), (2, 2, 96), (8, 1, 80), (16, 8, 72), (6, 3, 8), (5, 5, 40), (4, 4, 120)]


@gpu
@pytest.mark.parametrize("Hq,Hk,D", SHAPES)
@pytest.mark.parametrize("n", [1, 2, 31, 65, 300])
def test_one_sequence(n, Hq, Hk, D):
    c = Case([n], [n], Hq, Hk, D)
    check(c, 0, 0, starts=False)
    check(c, 33, 3, starts=False)


@gpu
@pytest.mark.parametrize("window,sinks", [(0, 0), (0, 5), (1, 0), (1, 1), (64, 0), (100, 4), (63, 65), (200, 256), (5, 130), (2000, 7)])
def test_windows_and_sinks(window, sinks):
    check(Case([700], [700], 4, 2, 64), window, sinks)


@gpu
@pytest.mark.parametrize("window,sinks", [(0, 0), (50, 4)])
@pytest.mark.parametrize("queries,keys", [
    ([5, 0, 257, 1, 64, 128], [5, 0, 257, 1, 64, 128]),      # packed, an empty one
    ([3, 100, 1], [400, 100, 129]),                          # behind kept keys
    ([70, 3, 5], [20, 0, 9]),                                # more queries than keys: rows that see none
    ([0, 0, 9], [30, 0, 9]),                                 # keys without queries
    ([1] * 40, list(range(1, 41)))])
def test_packed(queries, keys, window, sinks):
    check(Case(queries, keys, 4, 2, 64), window, sinks)


@gpu
def test_many_far_chunks():
    # sinks' sums over several chunks of queries behind the window
    check(Case([2500, 777], [2500, 777], 2, 1, 64), 100, 40)


@gpu
@pytest.mark.parametrize("scale", [2.0 ** -20, 1.0, 30.0])
def test_scales(scale):
    # 30: rows where one key has all the weight
    check(Case([200], [200], 2, 1, 64), 0, 0, scale=scale)


@gpu
def test_views_of_a_projection_and_rows_behind_the_last_sequence():
    c = Case([40, 25], [40, 25], 6, 2, 80, tail=11)
    qkv = torch.cat((c.q, c.k, c.v), 1)
    parts = qkv.split([6, 2, 2], 1)
    grad = torch.full_like(qkv, 7.0)
    o, lse = torch.full_like(c.q, 5.0), torch.full((6, c.T), 3.0, device=DEV)
    st = torch.tensor(c.qs, dtype=torch.int32, device=DEV)
    mxnorm.window_attn_fwd(*parts, 16, 2, q_start=st, out=o, lse=lse)
    o2, lse2 = c.forward(16, 2, q_start=st)
    n = c.qs[-1]
    assert torch.equal(o[:n], o2[:n]) and torch.equal(lse[:, :n], lse2[:, :n])
    assert (o[n:] == 5).all() and (lse[:, n:] == 3).all()
    gq, gk, gv = grad.split([6, 2, 2], 1)
    mxnorm.window_attn_bwd(c.go, *parts, o, lse, 16, 2, q_start=st, grad_q=gq, grad_k=gk, grad_v=gv)
    want = c.backward(o2, lse2, 16, 2, q_start=st)
    for x, y in zip((gq, gk, gv), want):
        assert torch.equal(x[:n], y[:n])
    assert (grad[n:] == 7).all()


@gpu
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("D", [64, 128])
def test_masked_places_may_hold_anything(bad, D):
    # token 70 is visible to tokens 70 .. 79 alone, token 1 as a sink to all from 1 on
    T, W, S = 150, 10, 1
    c = Case([T], [T], 2, 1, D)
    c.k[70], c.v[70] = bad, bad
    o, lse = c.forward(W, S)
    clean = Case([T], [T], 2, 1, D)
    want, bound = clean.want(W, S)
    rows = torch.tensor([i for i in range(T) if not 70 <= i < 80], device=DEV)
    assert off(o[rows], want["o"][rows], bound["o"][rows]) <= 1
    assert off(lse[:, rows], want["lse"][:, rows], bound["lse"][:, rows]) <= 1
    assert o[70:80].isnan().any()
    # backward: a query and its gradient, and a key that one query alone sees
    clean = Case([T], [T], 2, 1, D)
    o, lse = clean.forward(W, S)
    clean.q[100], clean.go[100], o[100], lse[:, 100] = bad, bad, bad, bad
    gq, gk, gv = clean.backward(o, lse, W, S)
    keep = Case([T], [T], 2, 1, D)
    keep.go[100] = 0
    want, bound = keep.want(W, S)
    mine = torch.tensor([j for j in range(T) if not (90 < j <= 100 or j < S)], device=DEV)
    rows = torch.tensor([i for i in range(T) if i != 100], device=DEV)
    assert off(gq[rows], want["gq"][rows], bound["gq"][rows]) <= 1
    for n, t in (("gk", gk), ("gv", gv)):
        assert off(t[mine], want[n][mine], bound[n][mine]) <= 1
    c = Case([T], [T], 2, 1, D)
    o, lse = c.forward(W, S)
    c.k[70], c.v[70] = bad, bad
    gq, gk, gv = c.backward(o, lse, W, S)
    clean = Case([T], [T], 2, 1, D)
    clean.go[70:80] = 0
    rows = torch.tensor([i for i in range(T) if not 70 <= i < 80], device=DEV)
    full, bound = Case([T], [T], 2, 1, D).want(W, S)
    assert off(gq[rows], full["gq"][rows], bound["gq"][rows]) <= 1
    far = torch.tensor([j for j in range(S, T) if not 60 < j < 80], device=DEV)
    for n, t in (("gk", gk), ("gv", gv)):
        assert off(t[far], full[n][far], bound[n][far]) <= 1


@gpu
def test_rows_of_large_scores():
    # scores beyond float: a row whose visible ones are all -inf gives NaN
    c = Case([3], [3], 1, 1, 64)
    c.q[:] = 3e38
    c.k[:] = -3e38
    o, lse = c.forward(0, 0)
    assert o.isnan().all() and (lse == -torch.inf).all()


@gpu
def test_captured_and_replayed():
    c = Case([300, 77], [300, 77], 4, 2, 64)
    kw = c.starts()
    o, lse = c.forward(64, 4, **kw)
    want = [o, lse, *c.backward(o, lse, 64, 4, **kw)]
    got = [torch.empty_like(t) for t in want]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.forward(64, 4, out=got[0], lse=got[1], **kw)
        c.backward(got[0], got[1], 64, 4, grad_q=got[2], grad_k=got[3], grad_v=got[4], **kw)
    for i in range(3):
        for t in got:
            t.fill_(float(i))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want)), i


@gpu
def test_another_stream():
    c = Case([500], [500], 4, 2, 64)
    want = c.forward(0, 0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        o, lse = c.forward(0, 0)
    side.synchronize()
    assert torch.equal(o, want[0]) and torch.equal(lse, want[1])


@gpu
def test_tokens_far_apart():
    # tokens, and heads, 2^31 + 64 elements apart
    T, far = 3, (1 << 31) + 64
    buf = torch.empty(3 * far, dtype=torch.bfloat16, device=DEV)
    c = Case([T], [T], 2, 2, 64)
    q, k = buf.as_strided((T, 2, 64), (far, 64, 1)), buf.as_strided((T, 2, 64), (128, far, 1), 1024)
    v = buf.as_strided((T, 2, 64), (far, 64, 1), 2048)
    out = [buf.as_strided((T, 2, 64), (far, 64, 1), 4096 + 1024 * i) for i in range(4)]
    q.copy_(c.q), k.copy_(c.k), v.copy_(c.v)
    o, lse = mxnorm.window_attn_fwd(q, k, v, out=out[0])
    want = c.forward(0, 0)
    assert torch.equal(o, want[0]) and torch.equal(lse, want[1])
    got = mxnorm.window_attn_bwd(c.go, q, k, v, o, lse, grad_q=out[1], grad_k=out[2], grad_v=out[3])
    assert all(torch.equal(x, y) for x, y in zip(got, c.backward(*want, 0, 0)))
    del buf, q, k, v, out, o, got
    torch.cuda.empty_cache()


@gpu
@pytest.mark.parametrize("Hq,Hk", [(8, 2), (3, 3), (2, 1), (16, 8)])
@pytest.mark.parametrize("D", [64, 96, 128, 120])
def test_larger(Hq, Hk, D):
    # several tiles of queries a head, workgroups of both sizes, shares of a key block's queries
    check(Case([1500, 700], [1500, 700], Hq, Hk, D), 0, 0)
    check(Case([1500, 700], [1600, 700], Hq, Hk, D), 300, 20)


@gpu
def test_many_heads():
    # enough workgroups that none shares a key block's queries
    check(Case([1100], [1100], 64, 32, 64), 500, 4)


@gpu
def test_two_streams_at_once():
    c, d = Case([900], [900], 4, 2, 64), Case([800], [800], 4, 2, 64, seed=5)
    want = []
    for x in (c, d):
        o, lse = x.forward(100, 2)
        want.append([o, lse, *x.backward(o, lse, 100, 2)])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = [None, None]
    for _ in range(3):
        with torch.cuda.stream(side):
            o, lse = d.forward(100, 2)
            got[1] = [o, lse, *d.backward(o, lse, 100, 2)]
        o, lse = c.forward(100, 2)
        got[0] = [o, lse, *c.backward(o, lse, 100, 2)]
    side.synchronize()
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


@gpu
def test_a_row_that_is_used_twice():
    # queries that share their memory (a stride of 0), keys and values the same heads
    c = Case([130], [130], 4, 2, 64)
    q = c.q[:, :1].expand(-1, 4, -1)
    o, lse = mxnorm.window_attn_fwd(q, c.k, c.k, 50, 2)
    want = mxnorm.window_attn_fwd(q.contiguous(), c.k, c.k.clone(), 50, 2)
    assert torch.equal(o, want[0]) and torch.equal(lse, want[1])
    got = mxnorm.window_attn_bwd(c.go, q, c.k, c.k, o, lse, 50, 2)
    want = mxnorm.window_attn_bwd(c.go, q.contiguous(), c.k, c.k.clone(), o, lse, 50, 2)
    assert all(torch.equal(x, y) for x, y in zip(got, want))


@gpu
def test_starts_that_do_not_fit():
    # past the end, descending, negative: no row outside the tensors is touched
    c = Case([100, 60], [100, 60], 2, 1, 64)
    for st in ([0, 1 << 30, 160], [0, 200, 50], [-5, 100, 1 << 20], [160, 0, 160]):
        starts = torch.tensor(st, dtype=torch.int32, device=DEV)
        o, lse = c.forward(0, 3, q_start=starts)
        c.backward(o, lse, 20, 3, q_start=starts)
    torch.cuda.synchronize()
    check(c, 20, 3)


@gpu
def test_small_heads_and_wide_strides():
    # tokens 2^24 elements apart take the loads of whole addresses
    T, far = 70, 1 << 24
    buf = torch.empty(T * far + 4096, dtype=torch.bfloat16, device=DEV)
    c = Case([T], [T], 2, 2, 64)
    k, v = (buf.as_strided((T, 2, 64), (far, 64, 1), 128 * i) for i in range(2))
    k.copy_(c.k), v.copy_(c.v)
    o, lse = mxnorm.window_attn_fwd(c.q, k, v)
    want = c.forward(0, 0)
    assert torch.equal(o, want[0]) and torch.equal(lse, want[1])
    got = mxnorm.window_attn_bwd(c.go, c.q, k, v, o, lse)
    assert all(torch.equal(x, y) for x, y in zip(got, c.backward(*want, 0, 0)))
    del buf, k, v
    torch.cuda.empty_cache()


@gpu
def test_the_largest_window():
    c = Case([1100], [1100], 4, 2, 64)
    o, lse = c.forward(0, 0)
    want = [o, lse, *c.backward(o, lse, 0, 0)]
    for sinks in (0, 9):
        o, lse = c.forward((1 << 63) - 1, sinks)
        got = [o, lse, *c.backward(o, lse, (1 << 63) - 1, sinks)]
        assert all(torch.equal(x, y) for x, y in zip(got, want))


def backward_with_guards(c, window, sinks, **kw):
    """The gradients by a call whose workspace lies between guards, which have to hold."""
    lib, ref = mxnorm.load(), ctypes.byref
    o, lse = c.forward(window, sinks, **kw)
    dq, dk, dv, T, S, D, B, scale = mxnorm._attn_arguments(c.q, c.k, c.v, kw["q_start"], kw.get("k_start"), None)
    need = lib.window_attn_bwd_workspace_bytes(T, S, dq.heads, dk.heads, D, B, window, sinks)
    buf = torch.full((need + (2 << 20),), 0xA5, dtype=torch.uint8, device=DEV)
    ws = buf[1 << 20:][:need]
    grads = [torch.empty_like(t) for t in (c.q, c.k, c.v)]
    mxnorm._call(lib.window_attn_bwd, c.q.device, ref(mxnorm._heads(c.go, "grad_out")), ref(dq), ref(dk), ref(dv),
                 ref(mxnorm._heads(o, "out")), lse.data_ptr(), T, S, D, kw["q_start"].data_ptr(),
                 kw["k_start"].data_ptr() if "k_start" in kw else None, B, window, sinks, scale,
                 *[ref(mxnorm._heads(g, "grad")) for g in grads], ws.data_ptr(), need)
    assert (buf[:1 << 20] == 0xA5).all() and (buf[(1 << 20) + need:] == 0xA5).all()
    return grads


@gpu
@pytest.mark.parametrize("Hq,Hk,D", [(4, 2, 64), (2, 1, 96), (3, 3, 128)])
@pytest.mark.parametrize("window,sinks", [(10, 4), (40, 70), (1, 1), (300, 256)])
def test_far_sums_of_many_sequences(window, sinks, Hq, Hk, D):
    # short and long sequences in turn, empty ones, keys without queries and kept ones;
    # those longer than the window alone have room for far sums
    queries = [(7 * b * b + 3 * b) % 53 if b % 9 else 400 * (b % 2) for b in range(70)]
    keys = [n + (0 if b % 4 else 11 * b % 60) for b, n in enumerate(queries)]
    for q, k in ((queries, queries), (queries, keys)):
        c = Case(q, k, Hq, Hk, D)
        check(c, window, sinks)
        want, bound = c.want(window, sinks)
        for name, got in zip(("gq", "gk", "gv"), backward_with_guards(c, window, sinks, **c.starts())):
            assert off(got, want[name], bound[name]) <= 1


@gpu
def test_far_sums_of_starts_that_do_not_fit():
    c = Case([300, 60, 200], [300, 60, 200], 2, 1, 64)
    for st in ([0, 1 << 30, 160, 560], [0, 200, 50, 560], [-5, 100, 1 << 20, 3], [560, 0, 560, 0]):
        starts = torch.tensor(st, dtype=torch.int32, device=DEV)
        for window, sinks in ((20, 40), (1, 1), (500, 256)):
            backward_with_guards(c, window, sinks, q_start=starts)


@gpu
@pytest.mark.parametrize("D", [64, 80, 128])
def test_starts_that_do_not_fit_write_their_own_rows(D):
    # the memory around the output, the lse and the gradients holds
    c = Case([100, 60, 200], [100, 60, 200], 4, 2, D)
    far = (1 << 31) - 1

    def guarded(*shape, dtype=torch.bfloat16):
        n, edge = math.prod(shape), 4096
        big = torch.full((n + 2 * edge,), 7.0, dtype=dtype, device=DEV)
        return big, big[edge:-edge].view(shape)

    bufs = [guarded(*c.q.shape), guarded(4, c.T, dtype=torch.float32)] + [guarded(*t.shape) for t in (c.q, c.k, c.v)]
    (_, o), (_, lse), (_, gq), (_, gk), (_, gv) = bufs
    for st in ([0, 1 << 30, 160, 360], [0, 200, 50, far], [-far - 1, 100, 1 << 20, -1], [360, 0, 360, 0], [300, 310, 311, 312]):
        for kst in (st, [0, 360, 360, 360], [far, 0, -5, 200]):
            kw = {n: torch.tensor(x, dtype=torch.int32, device=DEV) for n, x in (("q_start", st), ("k_start", kst))}
            for window, sinks in ((0, 0), (20, 40), (1, 1)):
                c.forward(window, sinks, out=o, lse=lse, **kw)
                c.backward(o, lse, window, sinks, grad_q=gq, grad_k=gk, grad_v=gv, **kw)
    torch.cuda.synchronize()
    for big, _ in bufs:
        assert (big[:4096] == 7).all() and (big[-4096:] == 7).all()
    check(c, 20, 3)


@gpu
@pytest.mark.parametrize("Hq,Hk", [(512, 1), (200, 200)])
def test_very_many_heads(Hq, Hk):
    check(Case([70, 9], [70, 9], Hq, Hk, 64), 20, 2)


@gpu
def test_no_keys_at_all():
    c = Case([5], [0], 4, 2, 64)
    for kw in (dict(), dict(q_start=torch.tensor([0, 2, 5], dtype=torch.int32, device=DEV),
                            k_start=torch.zeros(3, dtype=torch.int32, device=DEV))):
        o, lse = c.forward(0, 0, **kw)
        assert (o == 0).all() and (lse == -torch.inf).all()
        gq, gk, gv = c.backward(o, lse, 0, 0, **kw)
        assert (gq == 0).all() and gk.numel() == gv.numel() == 0
    # and no queries: the keys' gradients are 0
    c = Case([0], [7], 4, 2, 64)
    for kw in (dict(), dict(window=3, sinks=2)):
        o, lse = mxnorm.window_attn_fwd(c.q, c.k, c.v, **kw)
        _, gk, gv = mxnorm.window_attn_bwd(c.go, c.q, c.k, c.v, o, lse, **kw)
        assert (gk == 0).all() and (gv == 0).all()


@gpu
def test_a_hundred_thousand_sequences():
    # each of one token: its value
    n = 100000
    c = Case([n], [n], 2, 1, 8)
    starts = torch.arange(n + 1, dtype=torch.int32, device=DEV)
    o, lse = c.forward(9, 3, q_start=starts)
    assert torch.equal(o, c.v.expand(-1, 2, -1))
    gq, gk, gv = c.backward(o, lse, 9, 3, q_start=starts)
    # P is 1, so grad_v is the sum of two heads' gradients, rounded once
    assert torch.equal(gv, c.go.float().sum(1, keepdim=True).bfloat16())


@gpu
@pytest.mark.parametrize("bad", [float("nan"), -float("inf")])
@pytest.mark.parametrize("Hq,Hk,D", [(64, 32, 96), (64, 32, 80), (6, 2, 96), (64, 32, 64)])
def test_masked_places_of_many_heads(bad, Hq, Hk, D):
    # token 300 is visible to tokens 300 .. 339 alone; more workgroups than share tiles or queries, and fewer
    T, W, S = 700, 40, 2
    near = torch.zeros(T, dtype=torch.bool, device=DEV)
    near[300:340] = True
    clean, c = Case([T], [T], Hq, Hk, D), Case([T], [T], Hq, Hk, D)
    want, bound = clean.want(W, S)
    c.k[300], c.v[300] = bad, bad
    o, lse = c.forward(W, S)
    assert off(o[~near], want["o"][~near], bound["o"][~near]) <= 1
    assert off(lse[:, ~near], want["lse"][:, ~near], bound["lse"][:, ~near]) <= 1
    o, lse = clean.forward(W, S)
    gq, _, _ = c.backward(o, lse, W, S)
    assert off(gq[~near], want["gq"][~near], bound["gq"][~near]) <= 1
    # a query, its gradient, output and lse: the keys that it does not see, as sinks or in its window
    c = Case([T], [T], Hq, Hk, D)
    c.q[500], c.go[500], o[500], lse[:, 500] = bad, bad, bad, bad
    _, gk, gv = c.backward(o, lse, W, S)
    unseen = torch.tensor([j for j in range(S, T) if not 460 < j <= 500], device=DEV)
    for n, t in (("gk", gk), ("gv", gv)):
        assert off(t[unseen], want[n][unseen], bound[n][unseen]) <= 1
