"""Host-side checks of the attention and cache entry points (no GPU needed): what
they refuse before a launch, calls that launch nothing, workspace sizes."""
import ctypes
import os

import pytest
import torch

import launch_rules
from paper_2603_13180_amd import mxnorm

pytestmark = pytest.mark.skipif(not os.path.exists(mxnorm.LIB_PATH), reason="libmxnorm.so not built")

P = 0x10000          # an aligned address that no call reads
BIG = 1 << 28


def heads(n, D=64, data=P, token=None, head=None):
    return mxnorm._Heads(data, n, n * D if token is None else token, D if head is None else head)


def call(fn, *args):
    status = getattr(mxnorm.load(), fn)(*(ctypes.byref(a) if isinstance(a, ctypes.Structure) else a for a in args))
    return status, mxnorm.load().mx_last_error().decode()


def forward(**kw):
    a = dict(q=heads(4), k=heads(2), v=heads(2), Tq=10, Tk=10, D=64, qs=None, ks=None, B=1, window=0, sinks=0, scale=0.125,
             out=heads(4), lse=P)
    a.update(kw)
    return call("window_attn_fwd", *[a[n] for n in ("q", "k", "v", "Tq", "Tk", "D", "qs", "ks", "B", "window", "sinks", "scale",
                                                   "out", "lse")], None)


def backward(**kw):
    a = dict(go=heads(4), q=heads(4), k=heads(2), v=heads(2), out=heads(4), lse=P, Tq=10, Tk=10, D=64, qs=None, ks=None, B=1,
             window=0, sinks=0, scale=0.125, gq=heads(4), gk=heads(2), gv=heads(2), ws=P, n=1 << 40)
    a.update(kw)
    return call("window_attn_bwd", *[a[n] for n in ("go", "q", "k", "v", "out", "lse", "Tq", "Tk", "D", "qs", "ks", "B", "window",
                                                   "sinks", "scale", "gq", "gk", "gv", "ws", "n")], None)


def cache(**kw):
    a = dict(k=P, v=P, k_scales=None, v_scales=None, pages=8, page_size=16, heads=2, page_stride=2 * 16 * 64,
             scale_page_stride=0, type=0)
    a.update(kw)
    return mxnorm._Cache(*[a[n] for n in ("k", "v", "k_scales", "v_scales", "pages", "page_size", "heads", "page_stride",
                                          "scale_page_stride", "type")])


def append(**kw):
    a = dict(c=cache(), k=heads(2), v=heads(2), T=5, S=5, D=64, table=P, width=4, length=P, start=P, B=3, rows=None)
    a.update(kw)
    return call("kv_cache_append", *[a[n] for n in ("c", "k", "v", "T", "S", "D", "table", "width", "length", "start", "B",
                                                   "rows")], None)


def cached(**kw):
    a = dict(c=cache(), q=heads(4), T=5, D=64, table=P, width=4, length=P, start=P, B=3, max_new=4, max_length=0, bits=None,
             window=0, sinks=0, scale=0.125, out=heads(4), ws=P, n=1 << 40)
    a.update(kw)
    return call("kv_cache_attn_fwd", *[a[n] for n in ("c", "q", "T", "D", "table", "width", "length", "start", "B", "max_new",
                                                     "max_length", "bits", "window", "sinks", "scale", "out", "ws", "n")], None)


EINVAL, UNSUPPORTED = mxnorm.MX_EINVAL, mxnorm.MX_EUNSUPPORTED
COMMON = [
    (dict(Tq=-1), EINVAL), (dict(Tk=-1), EINVAL), (dict(D=0), EINVAL), (dict(D=12), EINVAL), (dict(D=136), UNSUPPORTED),
    (dict(q=heads(0)), EINVAL), (dict(q=heads(5)), EINVAL), (dict(k=heads(3)), EINVAL), (dict(v=heads(1)), EINVAL),
    (dict(q=None), EINVAL), (dict(k=None), EINVAL), (dict(v=None), EINVAL), (dict(out=None), EINVAL),
    (dict(q=heads(4, data=P + 8)), EINVAL), (dict(k=heads(2, data=None)), EINVAL), (dict(v=heads(2, token=132)), EINVAL),
    (dict(window=-1), EINVAL), (dict(sinks=-1), EINVAL), (dict(sinks=257), UNSUPPORTED),
    (dict(scale=0.0), EINVAL), (dict(scale=-1.0), EINVAL), (dict(scale=float("nan")), EINVAL), (dict(scale=float("inf")), EINVAL),
    (dict(B=2), EINVAL), (dict(ks=P), EINVAL), (dict(qs=P, B=0), EINVAL), (dict(qs=P + 2, B=1), EINVAL),
    (dict(qs=P, ks=P + 1, B=1), EINVAL), (dict(qs=P, Tk=11), EINVAL), (dict(qs=P, B=(1 << 20) + 1), UNSUPPORTED),
    (dict(Tq=BIG + 1), UNSUPPORTED), (dict(Tk=BIG + 1), UNSUPPORTED), (dict(q=heads(8192), k=heads(8192), v=heads(8192)), UNSUPPORTED),
    (dict(Tq=BIG, Tk=BIG, q=heads(4096, 64), k=heads(4096), v=heads(4096)), UNSUPPORTED),
    (dict(Tk=BIG, q=heads(4096, 64), k=heads(4096), v=heads(4096)), UNSUPPORTED)]


@pytest.mark.parametrize("kw,status", COMMON + [
    (dict(out=heads(4, token=200)), EINVAL), (dict(out=heads(2)), EINVAL), (dict(lse=P + 2), EINVAL)])
def test_forward_refuses(kw, status):
    got, text = forward(**kw)
    assert got == status and text


@pytest.mark.parametrize("kw,status", COMMON + [
    (dict(go=None), EINVAL), (dict(go=heads(2)), EINVAL), (dict(gq=heads(4, token=64)), EINVAL), (dict(gk=heads(4)), EINVAL),
    (dict(gv=heads(2, head=32)), EINVAL), (dict(lse=None), EINVAL), (dict(lse=P + 1), EINVAL), (dict(ws=None), EINVAL),
    (dict(ws=P + 16), EINVAL), (dict(n=100), EINVAL)])
def test_backward_refuses(kw, status):
    got, text = backward(**kw)
    assert got == status and text


MX = dict(type=1, k_scales=P, v_scales=P, page_stride=2 * 16 * 64, scale_page_stride=2 * 16 * 2)
PAGED = [
    (dict(c=None), EINVAL), (dict(c=cache(heads=0)), EINVAL), (dict(c=cache(pages=-1)), EINVAL), (dict(c=cache(type=2)), EINVAL),
    (dict(c=cache(page_size=8)), EINVAL), (dict(c=cache(page_size=48)), EINVAL), (dict(c=cache(page_size=0)), EINVAL),
    (dict(c=cache(page_stride=2 * 16 * 64 - 8)), EINVAL), (dict(c=cache(page_stride=2 * 16 * 64 + 4)), EINVAL),
    (dict(c=cache(k=P + 8)), EINVAL), (dict(c=cache(v=None)), EINVAL), (dict(c=cache(pages=1 << 31)), UNSUPPORTED),
    (dict(c=cache(**{**MX, "k_scales": None})), EINVAL), (dict(c=cache(**{**MX, "v_scales": P + 4})), EINVAL),
    (dict(c=cache(**{**MX, "scale_page_stride": 2 * 16 * 2 + 8})), EINVAL), (dict(c=cache(**{**MX, "scale_page_stride": 48})), EINVAL),
    (dict(c=cache(**{**MX, "page_stride": 2 * 16 * 64 + 8})), EINVAL),
    (dict(D=0), EINVAL), (dict(D=60), EINVAL), (dict(D=136, c=cache(page_stride=1 << 20)), UNSUPPORTED),
    (dict(D=40, c=cache(**MX)), EINVAL), (dict(T=-1), EINVAL), (dict(B=-1), EINVAL), (dict(width=-1), EINVAL),
    (dict(width=BIG // 16 + 1), UNSUPPORTED), (dict(table=None), EINVAL), (dict(table=P + 2), EINVAL), (dict(length=None), EINVAL),
    (dict(length=P + 1), EINVAL), (dict(start=P + 2), EINVAL), (dict(start=None), EINVAL), (dict(B=(1 << 20) + 1), UNSUPPORTED),
    (dict(T=BIG + 1), UNSUPPORTED)]


@pytest.mark.parametrize("kw,status", PAGED + [
    (dict(S=4), EINVAL), (dict(S=-1), EINVAL), (dict(rows=P + 2), EINVAL), (dict(k=heads(3)), EINVAL), (dict(v=None), EINVAL),
    (dict(k=heads(2, data=P + 4)), EINVAL)])
def test_append_refuses(kw, status):
    got, text = append(**kw)
    assert got == status and text


@pytest.mark.parametrize("kw,status", PAGED + [
    (dict(q=None), EINVAL), (dict(q=heads(3)), EINVAL), (dict(q=heads(0)), EINVAL), (dict(q=heads(4098)), UNSUPPORTED),
    (dict(out=heads(2)), EINVAL), (dict(out=None), EINVAL), (dict(out=heads(4, token=0)), EINVAL), (dict(max_new=0), EINVAL),
    (dict(max_new=65), UNSUPPORTED), (dict(max_length=-1), EINVAL), (dict(max_length=BIG + 1), UNSUPPORTED),
    (dict(window=-1), EINVAL), (dict(sinks=-1), EINVAL), (dict(scale=0.0), EINVAL), (dict(scale=float("nan")), EINVAL),
    (dict(bits=P + 4), EINVAL), (dict(width=4096, ws=None), EINVAL), (dict(width=4096, n=100), EINVAL),
    (dict(width=4096, ws=P + 128), EINVAL)])
def test_cached_refuses(kw, status):
    got, text = cached(**kw)
    assert got == status and text


@pytest.mark.parametrize("fn,kw", [
    # 2^24 workgroups of 256 threads, 2^23 of 512: a launch's threads no longer fit 32 bits
    (forward, dict(Tq=BIG, Tk=BIG, q=heads(8), out=heads(8))),
    (forward, dict(Tq=BIG, Tk=BIG, q=heads(8), out=heads(8), k=heads(8), v=heads(8))),
    (backward, dict(Tq=BIG, Tk=BIG, go=heads(8), q=heads(8), out=heads(8), gq=heads(8))),
    (backward, dict(Tk=BIG, k=heads(4), v=heads(4), gk=heads(4), gv=heads(4))),
    (append, dict(T=BIG, S=BIG, c=cache(heads=64, page_stride=64 * 16 * 64), k=heads(64), v=heads(64))),
    (cached, dict(T=BIG, q=heads(4), B=1, width=1024)),
    (cached, dict(T=1 << 20, B=1 << 20, start=None, c=cache(heads=16, page_stride=16 * 16 * 64), q=heads(16), out=heads(16)))])
def test_more_workgroups_than_a_launch_counts(fn, kw):
    got, text = fn(**kw)
    assert got == UNSUPPORTED and text


def test_calls_that_launch_nothing():
    none = heads(4, data=None), heads(2, data=None)
    assert forward(Tq=0, q=none[0], out=none[0])[0] == 0
    assert forward(Tq=0, Tk=0, q=none[0], k=none[1], v=none[1], out=none[0], lse=None)[0] == 0
    assert backward(Tq=0, Tk=0, go=none[0], q=none[0], k=none[1], v=none[1], out=none[0], gq=none[0], gk=none[1], gv=none[1],
                    lse=None, ws=None, n=0)[0] == 0
    assert append(T=0, S=0, k=none[1], v=none[1], table=None, length=None)[0] == 0
    assert append(T=0, B=0, table=None, length=None)[0] == 0
    assert append(c=cache(pages=0, k=None, v=None))[0] == 0
    assert cached(T=0, q=none[0], out=none[0], table=None, length=None)[0] == 0


def test_workspace_sizes():
    lib = mxnorm.load()
    bwd = lib.window_attn_bwd_workspace_bytes
    assert bwd(8192, 8192, 32, 8, 128, 1, 0, 0) >= 2 * 4 * 8192 * 32
    assert bwd(8192, 8192, 32, 8, 128, 1, 512, 4) > bwd(8192, 8192, 32, 8, 128, 1, 512, 0)
    assert bwd(0, 100, 4, 2, 64, 1, 0, 0) == 0 and bwd(10, 10, 4, 2, 64, 1, 0, 257) == 0 and bwd(10, 10, 2, 4, 64, 1, 0, 0) == 0
    att = lib.kv_cache_attn_fwd_workspace_bytes
    assert att(1, 32, 8, 128, 1, 64, 2048, 1, 0, 0, 0) >= 32 * 130 * 4
    # a bound of the lengths, or a window, leaves no keys to share out
    assert att(1, 32, 8, 128, 1, 64, 2048, 1, 100, 0, 0) == 0 and att(1, 32, 8, 128, 1, 64, 2048, 1, 0, 100, 4) == 0
    assert att(1, 32, 8, 128, 1, 64, 2048, 65, 0, 0, 0) == 0 and att(0, 32, 8, 128, 1, 64, 2048, 1, 0, 0, 0) == 0


def test_binding_refuses():
    t = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(RuntimeError, match="GPU"):
        mxnorm.window_attn_fwd(t, t, t)
    with pytest.raises(TypeError):
        mxnorm.window_attn_fwd(t.float(), t, t)
    with pytest.raises(TypeError):
        mxnorm.kv_cache_append(t[0], t, t, t, t, t)
    with pytest.raises(RuntimeError, match="GPU"):
        mxnorm.kv_cache_attn_fwd(t, t, t, t, t)


@pytest.mark.parametrize("waves", [2, 4, 8])
@pytest.mark.parametrize("D", range(8, 129, 8))
def test_a_tile_loads_its_heads_alone(D, waves):
    # every lane's loads: each 16 bytes of a head once, nothing behind it
    want = (torch.arange(16) * 8 < D).to(torch.uint8).expand(64, 16)
    assert torch.equal(launch_rules.attn_tile_loads(D, waves), want)


def test_windows_and_sinks_of_any_size_plan_as_no_window():
    # as far as 64 bits go, without overflow in the choice of shares
    lib, most = mxnorm.load(), (1 << 63) - 1
    att, bwd = lib.kv_cache_attn_fwd_workspace_bytes, lib.window_attn_bwd_workspace_bytes
    want = att(1, 32, 8, 128, 1, 64, 2048, 1, 0, 0, 0)
    assert want > 0
    for window, sinks in ((most, 0), (most, most), (most - 1, 4), (100, most), (BIG, BIG)):
        assert att(1, 32, 8, 128, 1, 64, 2048, 1, 0, window, sinks) == want
    want = bwd(1024, 1024, 12, 12, 64, 1, 0, 0)
    assert want > 2 * 4 * 1024 * 12
    for window in (BIG, most - 200, most - 100, most):
        assert bwd(1024, 1024, 12, 12, 64, 1, window, 0) == want


def test_far_sums_take_room_for_sequences_longer_than_the_window():
    bwd = mxnorm.load().window_attn_bwd_workspace_bytes
    args = (8192, 8192, 32, 8, 128, 512)
    # no query lies a window of all keys behind a sink
    for window in (8192, 8191 + 2, 0, (1 << 63) - 1):
        assert bwd(*args, window, 256) == bwd(*args, window, 0)
    # 32 chunks of 256 queries, and at most 8192 // 1001 sequences of more than 1000 keys
    block = 8 * 4 * 2 * 16 * 64 * 4
    assert 0 < bwd(*args, 1000, 4) - bwd(*args, 1000, 0) <= block * (32 + 8192 // 1001 + 1)
    # of 256 sinks 8192 - 8160 have such queries
    assert bwd(*args, 8160, 256) - bwd(*args, 8160, 0) <= block * (32 + 1 + 1)
