"""The paged cache of keys and values, and attention of new tokens over it, on the
GPU against a plain implementation in 64 bits (attn_reference.py)."""
import pytest
import torch

from attn_reference import HALF, Attention, off
from paper_2603_13180_amd import mxnorm

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        raise RuntimeError("these tests need a GPU (run them with -m gpu on an MI355X)")
    mxnorm.load()


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def decode(codes, scales):
    """float64 values of E4M3 codes and E8M0 scales."""
    x = codes.view(torch.float8_e4m3fn).double().unflatten(-1, (-1, 32))
    s = torch.where(scales == 255, torch.nan, torch.ldexp(torch.ones((), dtype=torch.float64, device=DEV), scales.int() - 127))
    return (x * s[..., None]).flatten(-2)


class Case:
    """Sequences with `cached` and `new` tokens; a cache with every new token in it,
    NaN in all slots that no token has."""

    def __init__(self, cached, new, Hq, Hk, D, page=16, mx=False, seed=0, tree=False, tail=0, slack=1):
        g = torch.Generator().manual_seed(seed + 31 * sum(cached) + 7 * sum(new) + D)
        self.cached, self.new, self.page, self.mx = cached, new, page, mx
        self.Hq, self.Hk, self.D = Hq, Hk, D
        self.st = [sum(new[:i]) for i in range(len(new) + 1)]
        self.T = self.st[-1] + tail
        need = [-(-(a + b) // page) for a, b in zip(cached, new)]
        self.pages = sum(need) + 2
        order = torch.randperm(self.pages, generator=g).tolist()
        table = torch.full((len(new), max(need + [0]) + slack), -1, dtype=torch.int32)
        for b, n in enumerate(need):
            for i in range(n):
                table[b, i] = order.pop()
        self.table = table.to(DEV)
        shape = (self.pages, Hk, page, D)
        # halves of one buffer
        self.buf = torch.full((self.pages, 2, Hk, page, D), torch.nan, dtype=torch.bfloat16, device=DEV)
        self.scales = [None, None]
        self.kc, self.vc = self.buf[:, 0], self.buf[:, 1]
        if mx:
            self.buf = torch.full((self.pages, 2, Hk, page, D), 0x7F, dtype=torch.uint8, device=DEV)
            self.kc, self.vc = self.buf[:, 0], self.buf[:, 1]
            self.scales = [torch.full((self.pages, Hk, page, D // 32), 255, dtype=torch.uint8, device=DEV) for _ in range(2)]
        assert self.kc.shape == shape
        self.length, self.start = i32(cached), i32(self.st)
        self.q = torch.randn(self.T, Hq, D, generator=g).bfloat16().to(DEV)
        # all tokens of a sequence, by the append under test from nothing
        whole = [a + b for a, b in zip(cached, new)]
        self.k, self.v = [(torch.randn(sum(whole), Hk, D, generator=g) * 1.5).bfloat16().to(DEV) for _ in range(2)]
        self.append(self.k, self.v, torch.zeros_like(self.length), i32([sum(whole[:i]) for i in range(len(whole) + 1)]))
        self.bits = None
        if tree:
            bits = []
            for n in new:
                mine = []
                for i in range(n):
                    parent = int(torch.randint(-1, i, (1,), generator=g)) if i else -1
                    mine.append((1 << i) | (mine[parent] if parent >= 0 else 0))
                bits += mine
            bits = [b - (1 << 64) if b >> 63 else b for b in bits] + [0] * tail
            self.bits = torch.tensor(bits, dtype=torch.int64, device=DEV)

    def kw(self):
        return dict(k_scales=self.scales[0], v_scales=self.scales[1])

    def append(self, k, v, length, start, rows=None):
        return mxnorm.kv_cache_append(k, v, self.kc, self.vc, self.table, length, start=start, rows=rows, **self.kw())

    def run(self, window=0, sinks=0, **kw):
        args = dict(start=self.start, max_new=max(self.new + [1]), ancestors=self.bits, window=window, sinks=sinks)
        return mxnorm.kv_cache_attn_fwd(self.q, self.kc, self.vc, self.table, self.length, **self.kw(), **{**args, **kw})

    def keys(self, b, codes, scales):
        """float64 [keys, heads, D] of sequence b, and whether its page is there."""
        j = torch.arange(self.cached[b] + self.new[b], device=DEV)
        i = j // self.page
        page = torch.where(i < self.table.shape[1], self.table[b].long()[i.clamp(max=self.table.shape[1] - 1)], -1)
        there = (page >= 0) & (page < self.pages)
        at = page.clamp(0, self.pages - 1)
        x = codes[at, :, j % self.page]
        return (x.double() if scales is None else decode(x, scales[at, :, j % self.page])), there

    def want(self, window=0, sinks=0, scale=None):
        o = torch.zeros(self.T, self.Hq, self.D, dtype=torch.float64, device=DEV)
        bound = torch.ones_like(o)
        scale = self.D ** -0.5 if scale is None else scale
        for b, (c, n) in enumerate(zip(self.cached, self.new)):
            (k, there), (v, _) = self.keys(b, self.kc, self.scales[0]), self.keys(b, self.vc, self.scales[1])
            drafted = torch.ones(n, n, dtype=torch.bool, device=DEV).tril()
            if self.bits is not None:
                drafted = self.bits[self.st[b]:self.st[b + 1], None] >> torch.arange(n, device=DEV) & 1 == 1
            place = c - 1 + drafted.sum(1)
            at = torch.cat((torch.arange(c, device=DEV), place))
            see = torch.cat((torch.ones(n, c, dtype=torch.bool, device=DEV), drafted), 1) & there
            if window:
                see = see & ((place[:, None] - at < window) | (at < sinks))
            unseen = ~see.any(0)
            k, v = [t.masked_fill(unseen[:, None, None], 0) for t in (k, v)]
            for h in range(self.Hq):
                x = Attention(self.q[self.st[b]:self.st[b + 1], h].double(), k[:, h * self.Hk // self.Hq],
                              v[:, h * self.Hk // self.Hq], see, scale)
                o[self.st[b]:self.st[b + 1], h], bound[self.st[b]:self.st[b + 1], h] = x.o, x.o_bound
        return o, bound


def check(c, window=0, sinks=0, **kw):
    want, bound = c.want(window, sinks, kw.get("scale"))
    o = c.run(window, sinks, **kw)
    n = c.st[-1]
    worst = off(o[:n], want[:n], bound[:n])
    assert worst <= 1, worst
    return o


@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("Hk,D,page", [(2, 64, 16), (8, 128, 64), (1, 96, 32), (3, 32, 16)])
def test_append(mx, Hk, D, page):
    c = Case([0, 5, 40, 100], [3, 0, 70, 1], 4 * Hk, Hk, D, page, mx)
    kept = c.kc.clone(), c.vc.clone()
    S = 200
    qkv = torch.randn(S, 3 * Hk, D, device=DEV).bfloat16()
    qkv[7, Hk, 3] = torch.inf
    qkv[9, 2 * Hk, 1] = torch.nan
    k, v = qkv[:, Hk:2 * Hk], qkv[:, 2 * Hk:]
    rows = torch.randperm(S, device=DEV)[:c.T].to(torch.int32)
    rows[0], rows[1], rows[2] = 7, 9, S  # the last is none
    got = c.append(k, v, c.length, c.start, rows)
    assert got[0] is c.kc
    want = [kept[0], kept[1]]
    scales = [None, None] if not mx else [s.clone() for s in c.scales]
    for which, x in ((0, k), (1, v)):
        for t in range(c.T):
            b = next(b for b in range(4) if c.st[b] <= t < c.st[b + 1])
            place = c.cached[b] + t - c.st[b]
            at, slot = int(c.table[b, place // page]), place % page
            if t == 2:
                continue
            row = x[rows[t].long()]
            if mx:
                codes, sc = mxnorm.mx_cast_fwd(row.contiguous())
                want[which][at, :, slot], scales[which][at, :, slot] = codes, sc
            else:
                want[which][at, :, slot] = row
    for a, b in zip((c.kc, c.vc), want):
        assert torch.equal(a.view(torch.uint8), b.contiguous().view(torch.uint8))
    if mx:
        assert all(torch.equal(a, b) for a, b in zip(c.scales, scales))


def test_append_skips_pages_that_are_not_there():
    c = Case([0, 0], [40, 20], 2, 1, 64)
    before = c.buf.clone()
    c.table[0, 1], c.table[1, 0] = c.pages, -1
    k = torch.full((60, 1, 64), 2.0, dtype=torch.bfloat16, device=DEV)
    c.append(k, k, c.length, c.start)
    pages = [int(c.table[0, 0]), int(c.table[0, 2]), int(c.table[1, 1])]
    rest = [p for p in range(c.pages) if p not in pages]
    assert torch.equal(c.buf[rest].view(torch.int16), before[rest].view(torch.int16))
    assert (c.kc[pages[0]] == 2).all() and (c.vc[pages[1], :, :8] == 2).all() and (c.kc[pages[2], :, :4] == 2).all()
    # past the table, and a negative length past its start
    c.append(k, k, i32([1 << 20, 0]), c.start)
    assert torch.equal(c.buf[rest].view(torch.int16), before[rest].view(torch.int16))


def test_append_many_sequences():
    # more starts than the kernel keeps near
    n = 1500
    c = Case([17] * n, [1] * n, 1, 1, 64)
    k = torch.randn(n, 1, 64, device=DEV).bfloat16()
    c.append(k, k, c.length, c.start)
    page = c.table[:, 1].long()
    assert torch.equal(c.kc[page, 0, 1], k[:, 0]) and torch.equal(c.vc[page, 0, 1], k[:, 0])
    c.append(-k, k, c.length + 1, None)
    assert torch.equal(c.kc[page, 0, 2], -k[:, 0]) and torch.equal(c.kc[page, 0, 1], k[:, 0])


SHAPES = [(4, 2, 128), (3, 1, 64), (2, 2, 96), (8, 1, 80), (12, 3, 32), (32, 1, 128), (5, 5, 40)]


@pytest.mark.parametrize("Hq,Hk,D", SHAPES)
@pytest.mark.parametrize("mx", [False, True])
def test_one_token(Hq, Hk, D, mx):
    if mx and D % 32:
        pytest.skip("codes come in blocks of 32")
    c = Case([0, 1, 15, 16, 33, 500, 2000], [1] * 7, Hq, Hk, D, mx=mx)
    check(c)
    check(c, window=20, sinks=3)
    check(c, start=None)


@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("new", [[64, 1, 0, 17], [3, 2, 3, 1], [33, 31, 5, 9]])
@pytest.mark.parametrize("Hq,Hk", [(4, 4), (4, 2), (8, 1)])
def test_chains_and_trees(new, mx, Hq, Hk):
    for tree in (False, True):
        c = Case([0, 700, 30, 129], new, Hq, Hk, 64, mx=mx, tree=tree)
        check(c)
        check(c, window=40, sinks=5)
        check(c, window=2, sinks=700)


@pytest.mark.parametrize("page", [16, 32, 256, 4096])
@pytest.mark.parametrize("splits", [False, True])
def test_pages(page, splits):
    # with max_length 1 the keys are not shared out
    c = Case([5000, 4097, 31], [1, 2, 3], 8, 2, 128, page=page)
    check(c, max_length=0 if splits else 1)


def test_any_mask_bits():
    # masks that name later tokens, none, and tokens that the sequence does not have
    c = Case([0, 20, 0], [5, 6, 2], 4, 2, 64, tree=True)
    c.bits[:5] = torch.tensor([0, 1 << 4, -1, 0b10110, 1 << 40], device=DEV)
    c.bits[5:11] = torch.tensor([0, 1 << 5, -1, 0b111000, -(1 << 63), 32], device=DEV)
    o = check(c)
    assert (o[0] == 0).all() and (o[4] == 0).all()
    check(c, window=3, sinks=1)


@pytest.mark.parametrize("mx", [False, True])
def test_pages_that_are_not_there_are_not_seen(mx):
    c = Case([300, 100], [4, 2], 4, 2, 64, mx=mx, tree=True)
    c.table[0, 3], c.table[0, 7], c.table[1, 0] = -1, c.pages, 1 << 30
    check(c)
    c.table = c.table[:, :10].contiguous()  # the last keys have no pages
    check(c, window=64, sinks=70)
    c.table[:] = -1
    assert (c.run() == 0).all()
    c.table = c.table[:, :0].contiguous()
    assert (c.run() == 0).all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("new", [1, 40])
def test_masked_keys_may_hold_anything(bad, new):
    c = Case([200], [new], 4, 2, 64, tree=new > 1)
    want, bound = c.want(50, 2)
    place = 200 + (new > 1)
    # keys behind the window but above the sinks, in its first tile and the sinks'
    for j in list(range(2, 20)) + list(range(140, 150)):
        c.kc[int(c.table[0, j // 16]), :, j % 16] = bad
        c.vc[int(c.table[0, j // 16]), :, j % 16] = bad
    assert place - 149 > 50
    assert off(c.run(50, 2), want, bound) <= 1


@pytest.mark.parametrize("new", [1, 40])
def test_drafted_tokens_do_not_see_each_other(new):
    # siblings: whatever one holds, the others' rows stay; it itself is NaN
    c = Case([37], [new], 2, 1, 64, tree=True)
    c.bits[:] = 1 << torch.arange(new, device=DEV)
    want, bound = c.want()
    at = 37 + new - 1
    c.vc[int(c.table[0, at // 16]), :, at % 16] = torch.nan
    o = c.run()
    if new > 1:
        assert off(o[:-1], want[:-1], bound[:-1]) <= 1
    assert o[-1].isnan().all()


def test_scale_of_255_is_nan_and_of_0_the_smallest():
    c = Case([20], [1], 1, 1, 64, mx=True)
    page = int(c.table[0, 0])
    c.scales[1][page, 0, 5, 1], c.scales[1][page, 0, 6, 0] = 255, 0
    c.vc[page, 0, 5, 32:] = 0x38
    o = c.run()
    assert o[0, 0, 32:].isnan().all() and not o[0, 0, :32].isnan().any()
    c.scales[1][page, 0, 5, 1] = 127
    check(c)


def test_rows_behind_the_last_sequence():
    c = Case([50, 2000], [2, 1], 4, 2, 64, tail=3)
    for kw in ({}, {"max_length": 1}):
        out = torch.full_like(c.q, 7.0)
        c.run(out=out, **kw)
        assert (out[3:] == 7).all() and torch.equal(out[:3], c.run(**kw)[:3])


def test_strided_queries_and_output():
    c = Case([300, 3000], [2, 5], 6, 2, 96)
    buf = torch.randn(7, 10, 96, device=DEV).bfloat16()
    buf[:, :6] = c.q
    out = torch.zeros(7, 8, 96, dtype=torch.bfloat16, device=DEV)
    want = c.run()
    c.q = buf[:, :6]
    assert torch.equal(c.run(out=out[:, 1:7]), want) and (out[:, 0] == 0).all() and (out[:, 7] == 0).all()


def test_far_pages():
    # a page more than 4 GiB behind the first
    Hk, D, far = 1, 64, (4 << 30) // 2 + 4096
    buf = torch.zeros(2 * far, dtype=torch.bfloat16, device=DEV)
    kc, vc = buf.as_strided((2, Hk, 16, D), (far, 16 * D, D, 1)), buf.as_strided((2, Hk, 16, D), (far, 16 * D, D, 1), 1 << 20)
    c = Case([10], [1], 2, Hk, D)
    table = i32([[1]])
    mxnorm.kv_cache_append(c.k, c.v, kc, vc, table, i32([0]), start=i32([0, 11]))
    assert torch.equal(kc[1, 0, :11], c.k[:, 0]) and torch.equal(vc[1, 0, :11], c.v[:, 0]) and (kc[0] == 0).all()
    o = mxnorm.kv_cache_attn_fwd(c.q, kc, vc, table, i32([10]))
    want, bound = c.want()
    assert off(o, want, bound) <= 1
    del buf, kc, vc
    torch.cuda.empty_cache()


def test_captured_and_replayed():
    # append and attention of one step, lengths moved on between replays
    c = Case([100, 3000], [1, 1], 8, 2, 128)
    k, v = torch.randn(2, 2, 2, 128, device=DEV).bfloat16()
    length, out = c.length.clone(), torch.empty_like(c.q)
    c.append(k, v, length, None)
    want = c.run(start=None)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.append(k, v, length, None)
        mxnorm.kv_cache_attn_fwd(c.q, c.kc, c.vc, c.table, length, out=out)
    for i in range(3):
        out.fill_(float(i))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), i
    length += 1
    graph.replay()
    torch.cuda.synchronize()
    c.length, c.cached = length, [101, 3001]
    assert torch.equal(out, c.run(start=None))
    want, bound = c.want()
    assert off(out, want, bound) <= 1


def test_a_prompt_then_steps_then_a_draft():
    """Norm and rotation, packed attention, the cache and attention over it as a
    program runs them: token by token and drafted, the same as packed at once."""
    g = torch.Generator(device=DEV).manual_seed(3)
    Hq, Hk, D, prompt, steps = 8, 2, 64, [70, 33], 3
    n = [p + steps for p in prompt]
    qkv = torch.randn(sum(n), Hq + 2 * Hk, D, generator=g, device=DEV).bfloat16()
    q, k, v = qkv.split([Hq, Hk, Hk], 1)
    gain = [(1 + 0.1 * torch.randn(D, generator=g, device=DEV)).bfloat16() for _ in range(2)]
    pos = torch.cat([torch.arange(m, device=DEV) for m in n])
    freq = 10000.0 ** (-torch.arange(0, D, 2, device=DEV).float() / D)
    mxnorm.qk_norm_rope_fwd(q, k, *gain, pos, freq, q_out=q, k_out=k)
    st = [0, n[0], sum(n)]
    kw = dict(window=24, sinks=2)
    whole, _ = mxnorm.window_attn_fwd(q, k, v, q_start=i32(st), want_lse=False, **kw)
    kc, vc = [torch.full((20, Hk, 16, D), torch.nan, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    table = torch.randperm(20, generator=g, device=DEV).to(torch.int32).view(2, 10)
    rows = torch.cat([torch.arange(a, a + p, device=DEV) for a, p in zip(st, prompt)])
    mxnorm.kv_cache_append(k, v, kc, vc, table, i32([0, 0]), start=i32([0, prompt[0], sum(prompt)]), rows=rows.to(torch.int32))

    def near(got, want):
        # two orders of the same sums of 24 to 26 terms with P and outputs rounded
        # to bf16: each within (HALF + 2^-10) of the terms' magnitudes and HALF of itself
        assert ((got.double() - want.double()).abs() <= 2 * (2 * HALF + 2.0 ** -10) * v.double().abs().max()).all()

    for i in range(steps):  # one token at a time
        t = torch.tensor([a + p + i for a, p in zip(st, prompt)], device=DEV)
        length = i32([p + i for p in prompt])
        mxnorm.kv_cache_append(k[t], v[t], kc, vc, table, length)
        near(mxnorm.kv_cache_attn_fwd(q[t], kc, vc, table, length, **kw), whole[t])
    # the same three as a draft of two branches: the tokens, and others before each
    length = i32(prompt)
    t = torch.cat([torch.tensor([a + p + i for i in range(steps)], device=DEV) for a, p in zip(st, prompt)])
    dq, dk, dv = [torch.randn(2 * t.numel(), x.shape[1], D, generator=g, device=DEV).bfloat16() for x in (q, k, v)]
    for x, y in ((dq, q), (dk, k), (dv, v)):
        x[1::2] = y[t]
    bits = torch.tensor([1, 2, 5, 10, 21, 42] * 2, device=DEV)
    start = i32([0, 2 * steps, 4 * steps])
    mxnorm.kv_cache_append(dk, dv, kc, vc, table, length, start=start)
    near(mxnorm.kv_cache_attn_fwd(dq, kc, vc, table, length, start=start, max_new=2 * steps, ancestors=bits, **kw)[1::2], whole[t])
    # those kept, one behind the other
    mxnorm.kv_cache_append(dk, dv, kc, vc, table, length, start=i32([0, steps, 2 * steps]),
                           rows=torch.arange(1, 4 * steps, 2, dtype=torch.int32, device=DEV))
    last = torch.tensor([s - 1 for s in st[1:]], device=DEV)
    near(mxnorm.kv_cache_attn_fwd(q[last], kc, vc, table, i32([m - 1 for m in n]), **kw), whole[last])


def test_many_sequences_by_length():
    # long and short ones, taken in the order of their lengths; more than that order covers
    for n in (40, 300):
        cached = [(37 * i * i) % 2500 for i in range(n)]
        c = Case(cached, [1] * n, 4, 2, 64)
        check(c)
        check(c, window=300, sinks=2)


@pytest.mark.parametrize("mx", [False, True])
def test_slots_past_the_end_may_hold_anything(mx):
    # the slots behind the last token, their scales too, are NaN (the case's filling)
    for n in (1, 17, 33):
        c = Case([n], [1], 4, 2, 128, page=64, mx=mx)
        check(c)


def test_lengths_that_do_not_fit():
    # negative, and past the table: no slot outside the cache is read
    c = Case([40, 50], [1, 1], 4, 2, 64)
    c.length = i32([-7, 1 << 30])
    c.run()
    torch.cuda.synchronize()
    c.length, want = i32([-7, 50]), i32([0, 50])
    o = c.run()
    c.length = want
    assert torch.equal(o, c.run())
    # sinks and a window far past what the table has room for
    c.length = i32([1 << 28, 50])
    c.run(window=5, sinks=1 << 27)
    c.length = i32([40, 50])
    check(c, window=5, sinks=1 << 27)


def test_starts_that_do_not_fit():
    c = Case([40, 50], [3, 2], 4, 2, 64, tree=True)
    for st in ([0, 1 << 30, 5], [3, 0, 5], [-4, 3, 99]):
        c.start = i32(st)
        c.run()
        c.append(c.k[:5], c.v[:5], c.length, c.start)
    torch.cuda.synchronize()


def test_max_new_bounds_what_is_read():
    # a sequence has more new tokens than max_new says: the rows of the others hold
    c = Case([20, 30, 40], [2, 9, 2], 4, 2, 64)
    want = c.run()
    got = c.run(max_new=2)
    assert torch.equal(got[:2], want[:2]) and torch.equal(got[11:], want[11:])


def uneven(B, longest, new=1, **kw):
    """A long sequence, one of half its length, empty ones and short ones; some without new tokens."""
    cached = [longest if b == B // 3 else longest // 2 if b == B - 1 else 0 if b % 7 == 1 else 5 + 37 * b % 200 for b in range(B)]
    return Case(cached, [0 if b % 5 == 4 and b < B - 1 else max(1, new - b % 3) for b in range(B)], D=64, **kw)


@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("B,longest,new,Hq,Hk", [
    (24, 6000, 1, 4, 2), (60, 5001, 1, 8, 2), (256, 2500, 1, 2, 1), (9, 4100, 5, 16, 4), (24, 3001, 40, 8, 2), (40, 2200, 20, 8, 2)])
def test_uneven_lengths(B, longest, new, Hq, Hk, mx):
    c = uneven(B, longest, new, Hq=Hq, Hk=Hk, mx=mx, tree=new > 1)
    a = check(c)
    assert torch.equal(a, c.run())
    check(c, window=300, sinks=20)
    # a bound of the lengths changes the shares
    near = c.run(max_length=longest + 900)
    o, bound = c.want()
    assert off(near, o, bound) <= 1


def test_uneven_lengths_captured():
    # lengths that change between a graph's replays
    c = uneven(30, 4000, Hq=8, Hk=2)
    out = torch.empty_like(c.q)
    c.run(out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run(out=out)
    for turn in range(4):
        now = [n if turn != 1 else n // 3 for n in c.cached]
        if turn == 2:
            now[0], now[10] = 150, 17
        c.length.copy_(i32(now))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        # (bits: the slots that a grown length brings in hold NaN)
        assert torch.equal(out.view(torch.int16), c.run().view(torch.int16))


def test_uneven_starts_and_lengths_that_do_not_fit():
    c = uneven(24, 6000, 3, Hq=4, Hk=2)
    st, length = c.start.clone(), c.length.clone()
    for i, x in ((3, 1 << 30), (5, -9), (24, 10), (0, 40)):
        c.start = st.clone()
        c.start[i] = x
        c.run()
    c.start = st
    c.length[2], c.length[9] = 1 << 30, -5
    c.run()
    c.length = length
    check(c)


def test_two_streams_at_once():
    c, d = Case([3000, 100], [1, 1], 8, 2, 128), Case([2500, 4000], [1, 1], 8, 2, 128, mx=True)
    want = c.run(), d.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        with torch.cuda.stream(side):
            b = d.run()
        a = c.run()
        torch.cuda.synchronize()
        assert torch.equal(a, want[0]) and torch.equal(b, want[1])


@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("length", [-1, -5, -(1 << 31)])
def test_append_takes_a_negative_length_as_0(length, mx):
    # below 0 by less than the new tokens, by as many, and by far more
    c, d = [Case([0, 0, 0], [20, 3, 5], 2, 2, 64, mx=mx) for _ in range(2)]
    k, v = torch.randn(2, 28, 2, 64, device=DEV).bfloat16()
    c.append(k, v, i32([length, 0, length]), c.start)
    d.append(k, v, i32([0, 0, 0]), d.start)
    assert torch.equal(c.buf.view(torch.uint8), d.buf.view(torch.uint8))
    assert not mx or all(torch.equal(x, y) for x, y in zip(c.scales, d.scales))
    # and attention finds them
    c.length = i32([length, 0, length])
    check(c)


@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("length", [-1, -5, -(1 << 31)])
def test_append_takes_a_negative_length_as_0(length, mx):
    # below 0 by less than the new tokens, by as many, and by far more
    c, d = [Case([0, 0, 0], [20, 3, 5], 2, 2, 64, mx=mx) for _ in range(2)]
    k, v = torch.randn(2, 28, 2, 64, device=DEV).bfloat16()
    c.append(k, v, i32([length, 0, length]), c.start)
    d.append(k, v, i32([0, 0, 0]), d.start)
    assert torch.equal(c.buf.view(torch.uint8), d.buf.view(torch.uint8))
    assert not mx or all(torch.equal(x, y) for x, y in zip(c.scales, d.scales))
    # and attention finds them
    c.length = i32([length, 0, length])
    check(c)


@pytest.mark.parametrize("Hq,Hk", [(2, 2), (4, 2), (8, 1)])
@pytest.mark.parametrize("window", [62, 63, 64, 65])
def test_windows_as_long_as_a_draft(window, Hq, Hk):
    # a token whose mask is empty has a place 64 before that of one that names all 64
    c = Case([30], [64], Hq, Hk, 64, tree=True)
    c.bits[0], c.bits[40], c.bits[63], c.bits[62] = 0, 0, -1, (1 << 63) - 1
    for i in (0, 40):
        at = 30 + i
        c.vc[int(c.table[0, at // 16]), :, at % 16] *= 30
    check(c, window=window)
    check(c, window=window, sinks=29)
    check(c, window=window, sinks=30)  # their place, 29, is a sink


def test_the_largest_window_and_sinks():
    most = (1 << 63) - 1
    c = Case([5000, 70], [1, 1], 4, 2, 64)
    want = c.run()
    for window, sinks in ((most, 0), (most, most), (9, most)):
        assert torch.equal(c.run(window, sinks), want)


@pytest.mark.parametrize("mx", [False, True])
def test_a_cache_of_one_page(mx):
    # its stride is not used: k and v need not agree in it
    c = Case([5], [3], 4, 2, 64, page=16, mx=mx)
    want = c.run()
    at = int(c.table[0, 0])
    c.kc, c.vc = c.buf[at:at + 1, 0], c.buf[at, 1].clone()[None]
    if mx:
        wide = torch.stack((c.scales[0], c.scales[1]), 1)
        c.scales = [wide[at:at + 1, 0], c.scales[1][at:at + 1].clone()]
    c.table[0, 0] = 0
    assert c.kc.stride() != c.vc.stride()
    assert torch.equal(c.run(), want)
    c.append(-c.k, c.v, torch.zeros_like(c.length), i32([0, 8]))
    c.pages = 1
    check(c)


@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("new", [[3, 2, 4], [40, 2, 30]])
def test_calls_that_do_not_fit_write_their_own_rows(new, mx):
    """Starts, lengths, rows and pages that do not fit: the memory around the cache, the
    scales and the output holds, and so do the pages that no table row names."""
    c = Case([400, 0, 3], new, 4, 2, 64, mx=mx, tree=True)
    P, T = c.pages, c.T

    def guarded(t, fill):
        big = torch.full((t.shape[0] + 8,) + t.shape[1:], fill, dtype=t.dtype, device=DEV)
        big[4:-4] = t
        return big, big[4:-4]

    buf, inner = guarded(c.buf, 7)
    c.kc, c.vc = inner[:, 0], inner[:, 1]
    scales = [guarded(s, 7) for s in c.scales] if mx else []
    c.scales = [s for _, s in scales] if mx else [None, None]
    outs, out = guarded(c.q, 7)
    named = torch.tensor(sorted(set(c.table.flatten().tolist()) - {-1}), device=DEV)
    spare = torch.tensor([p for p in range(P) if p not in named.tolist()], device=DEV)
    assert len(spare) == 2
    before = [t[4 + spare].clone() for t in [buf] + [s for s, _ in scales]]
    far = (1 << 31) - 1
    st, length, table, bits = c.start.clone(), c.length.clone(), c.table.clone(), c.bits.clone()
    rows = torch.arange(T, dtype=torch.int32, device=DEV)
    wild = rows.clone()
    wild[::3], wild[1::3] = far, -far - 1
    for starts in (st, i32([0, 1 << 30, 5, T]), i32([3, 0, 5, far]), i32([-far - 1, 3, 99, -1]), i32([T, T, 0, 0])):
        for lengths in (length, i32([-5, far, -far - 1]), i32([1 << 28, 401, 390])):
            for pages in (table, torch.where(table % 2 == 0, table, far), torch.where(table % 3 == 0, table, -far - 1)):
                c.start, c.length, c.table = starts, lengths, pages
                for kw in (dict(), dict(window=9, sinks=5), dict(window=300, sinks=far, max_length=1)):
                    c.run(out=out, **kw)
                c.append(c.k[:T], c.v[:T], lengths, starts)
                c.append(c.k[:T], c.v[:T], lengths, starts, wild)
    torch.cuda.synchronize()
    for t in [buf, outs] + [s for s, _ in scales]:
        assert (t[:4] == 7).all() and (t[-4:] == 7).all()
    for t, b in zip([buf] + [s for s, _ in scales], before):
        assert torch.equal(t[4 + spare].view(torch.uint8), b.view(torch.uint8))
    # and calls that fit are right after them
    c.start, c.length, c.table = st, length, table
    c.append(c.k[:T], c.v[:T], length, st)
    whole = i32([sum(c.cached[:b]) + sum(c.new[:b]) for b in range(4)])
    c.append(c.k, c.v, torch.zeros_like(length), whole)
    check(c)


@pytest.mark.parametrize("byte", [0, 1, 5, 100])
def test_values_of_small_scales(byte):
    # codes of 2 .. 448 times 2^(byte - 127), none below bf16's normal numbers
    c = Case([40], [1], 2, 1, 64, mx=True)
    g = torch.Generator().manual_seed(byte)
    c.vc[:] = torch.randint(0x40, 0x7F, c.vc.shape, generator=g, dtype=torch.uint8).to(DEV)
    c.scales[1].fill_(byte)
    want, _ = c.want()
    big = 448 * 2.0 ** (byte - 127)
    # P's rounding is at most HALF of the largest value, the output's too; P itself and
    # the sums of 41 terms are off by less than 2^-12 of it
    assert ((c.run().double() - want).abs() <= (2 * HALF + 2.0 ** -12) * big).all()
    assert (want > 2 * 2.0 ** (byte - 127)).all()


@pytest.mark.parametrize("mx", [False, True])
def test_sequences_that_write_the_same_token_at_one_place(mx):
    # a page that two sequences share, and the same rows named twice
    c = Case([0, 0], [12, 12], 4, 2, 64, mx=mx)
    c.table[1] = c.table[0]
    k, v = torch.randn(2, 12, 2, 64, device=DEV).bfloat16()
    rows = torch.arange(12, dtype=torch.int32, device=DEV).repeat(2)
    c.append(k, v, c.length, c.start, rows)
    at = int(c.table[0, 0])
    for which, x in ((0, k), (1, v)):
        got = (c.kc, c.vc)[which][at, :, :12].transpose(0, 1)
        if mx:
            codes, scales = mxnorm.mx_cast_fwd(x.flatten(0, 1))
            assert torch.equal(got, codes.view_as(got))
            assert torch.equal(c.scales[which][at, :, :12].transpose(0, 1), scales.view(12, 2, 2))
        else:
            assert torch.equal(got, x)
    c.q[12:] = c.q[:12]
    o = check(c)
    assert torch.equal(o[:12], o[12:])


@pytest.mark.parametrize("Hq,Hk,new", [(4096, 1, 1), (512, 2, 64)])
def test_many_heads(Hq, Hk, new):
    check(Case([40, 3], [new, 1], Hq, Hk, 64), window=30, sinks=2)


def test_an_empty_cache():
    # no pages: no token sees a key
    q = torch.randn(2, 4, 64, device=DEV).bfloat16()
    kc = torch.empty(0, 2, 16, 64, dtype=torch.bfloat16, device=DEV)
    k = torch.randn(2, 2, 64, device=DEV).bfloat16()
    table = i32([[0, 1], [2, 3]])
    mxnorm.kv_cache_append(k, k, kc, kc, table, i32([5, 0]))
    assert (mxnorm.kv_cache_attn_fwd(q, kc, kc, table, i32([5, 0])) == 0).all()


@pytest.mark.parametrize("new,Hq", [(1, 4), (1, 64), (30, 4), (30, 8), (60, 16)])
def test_masked_codes_may_hold_anything(new, Hq):
    # codes and scales that are NaN, behind the window but above the sinks; rows of every kind of workgroup
    for long in (200, 6000):
        c = Case([long], [new], Hq, 2, 64, mx=True, tree=new > 1)
        want, bound = c.want(50, 2)
        for j in list(range(2, 20)) + list(range(long - 60, long - 50)):
            at = int(c.table[0, j // 16]), slice(None), j % 16
            if j % 2:
                c.kc[at] = c.vc[at] = 0x7F
            else:
                c.scales[0][at] = c.scales[1][at] = 255
        assert off(c.run(50, 2), want, bound) <= 1
        # and with as many shares as a cache without a window has
        c = Case([long], [new], Hq, 2, 64, mx=True, tree=new > 1)
        at = int(c.table[0, 5])
        c.vc[at], c.kc[at], c.scales[0][at] = 0xFF, 0x7F, 255
        c.table[0, 5] = -1
        check(c)
