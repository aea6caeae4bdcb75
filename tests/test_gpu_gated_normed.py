"""MXNorm of a few rows within the gated product's launch, against the norm and
the product in two launches: the same bits.

The inputs' block absmaxes are powers of two times 1 to 2, within 2^12 of each
other in a row: their squares are multiples of a 2^-14 part of the smallest
(16-bit products), 512 of them below 2^(24 + 9) of it, so a row's sum has at
most 14 + 33 = 47 bits and is exact in double in any order."""
import ctypes

import numpy as np
import pytest
import torch

from launch_rules import ELEM, UNITS
from paper_2603_13180_amd import mxnorm

DEV = "cuda:0"
gpu = pytest.mark.gpu
_I, _L, _P = ctypes.c_int, ctypes.c_int64, ctypes.c_void_p


def normed(T, F, d, elem, units=UNITS):
    f = mxnorm.load().mxt_gated_normed
    f.restype, f.argtypes = _I, [_L] * 3 + [_I] * 2
    return f(T, F, d, ELEM[elem], units)


@pytest.mark.parametrize("T,d,elem,want", [
    (1, 128, "e4m3", 4), (4, 2048, "e4m3", 4), (4, 2176, "e4m3", 8), (4, 4096, "e4m3", 8), (5, 4096, "e4m3", 0),
    (4, 4224, "e4m3", 0), (1, 8192, "e4m3", 4), (1, 16384, "e4m3", 8), (1, 16512, "e4m3", 0),
    (2, 4096, "e2m1", 4), (2, 8192, "e2m1", 8), (4, 256, "e2m1", 4), (4, 4096, "e2m1", 8), (4, 4352, "e2m1", 0),
    (1, 16384, "e2m1", 8), (0, 256, "e4m3", 0), (16, 256, "e4m3", 0)])
def test_which_rows_are_normed_in_the_product(T, d, elem, want):
    assert normed(T, 4096, d, elem) == want


def rows(T, d, seed, special=False):
    rng = np.random.default_rng(seed)
    # a block's scale, then values below it and one at it
    s = np.exp2(rng.integers(-6, 6, (T, d // 32, 1)))
    v = s * rng.uniform(-1.0, 1.0, (T, d // 32, 32))
    v[:, :, 7] = s[:, :, 0] * rng.uniform(1.0, 1.99, (T, d // 32))
    x = torch.from_numpy(v.reshape(T, d)).to(torch.bfloat16)
    if special:
        x[T - 1] = 0
        x[0, d - 1] = float("inf")
        if T > 2:
            x[1, 33] = float("nan")
            x[1, 40] = float("-inf")
    return x


def weight(F, d, elem, seed=3):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    w = torch.randn(2 * F, d, generator=g, device=DEV).to(torch.bfloat16)
    return mxnorm.mx_cast_fwd(w, elem=elem)


def bits(t):
    return t.contiguous().view(torch.uint8)


def one_call(x, wc, ws, F, elem, p, mode, act, dtype, keep, want_rho):
    """The C entry point; nothing is written behind its outputs."""
    lib = mxnorm.load()
    T, d = x.shape
    codes = dtype is torch.uint8

    def guarded(shape, dt):
        n = int(np.prod(shape))
        buf = torch.full((n + 512,), 7, dtype=dt, device=DEV)
        return buf, buf[:n].view(shape)
    bufs = [guarded((T, F // 2 if codes and elem == "e2m1" else F), dtype), guarded((T, F // 32), torch.uint8),
            guarded((T, 2 * F), torch.bfloat16), guarded((T,), torch.float32)]
    out, sc, gu, rho = (b[1] for b in bufs)
    n = lib.mxnorm_gated_fwd_workspace_bytes(T, d, 32, ELEM[elem])
    wk = torch.empty(n, dtype=torch.uint8, device=DEV)
    mxnorm._check(lib.mxnorm_gated_fwd(
        x.data_ptr(), T, d, wc.data_ptr(), ws.data_ptr(), F, 32, ELEM[elem], p, 0.0, 1e-6,
        mxnorm.SCALE_MODES[mode], mxnorm.ACTS[act], mxnorm.GATED_DTYPES[dtype], out.data_ptr(),
        sc.data_ptr() if codes else None, gu.data_ptr() if keep else None,
        rho.data_ptr() if want_rho else None, wk.data_ptr(), n, mxnorm._stream(x.device)))
    used = [True, codes, keep, want_rho]
    for (buf, t), on in zip(bufs, used):
        assert (buf[t.numel() if on else 0:] == 7).all()
    return [t for (_, t), on in zip(bufs, used) if on]


def two_calls(x, wc, ws, elem, p, mode, act, dtype, keep, want_rho):
    ac, as_, rho = mxnorm.mxnorm_mx_fwd(x, elem=elem, p=p, scale_mode=mode)
    h, gu = mxnorm.mx_gated_fwd(ac, as_, wc, ws, x.shape[1], elem=elem, act=act, out_dtype=dtype,
                                scale_mode=mode, save_gu=keep)
    return list(h if dtype is torch.uint8 else (h,)) + [gu] * keep + [rho] * want_rho


# one K step (three waves without one), steps that no four waves share evenly,
# the longest rows that fit, for both numbers of chunks; F of half a tile, of a tile and a half, of many
SIZES = {"e4m3": [(1, 128, 32), (2, 384, 96), (3, 640, 32), (4, 1152, 1024), (2, 4096, 64), (1, 8192, 96),
                  (3, 2176, 32), (4, 4096, 64), (2, 8192, 32), (1, 16384, 64), (2, 4096, 12800), (3, 4096, 12800)],
         "e2m1": [(1, 256, 32), (2, 768, 96), (3, 1280, 32), (4, 1792, 1024), (2, 4096, 64), (1, 8192, 96),
                  (3, 2304, 32), (4, 4096, 64), (2, 8192, 32), (1, 16384, 64), (1, 8192, 12800), (2, 8192, 12800)]}


@gpu
@pytest.mark.parametrize("special", [False, True])
@pytest.mark.parametrize("elem", ["e4m3", "e2m1"])
def test_one_launch_has_the_bits_of_two(elem, special):
    ways = [(2, "rceil", "silu", torch.bfloat16, True, True), (1, "floor", "gelu_tanh", torch.float32, False, True),
            (2, "floor", "silu", torch.uint8, True, False), (1, "rceil", "gelu_tanh", torch.uint8, False, False)]
    for T, d, F in SIZES[elem]:
        assert normed(T, F, d, elem)
        x = rows(T, d, T + d, special).to(DEV)
        wc, ws = weight(F, d, elem)
        for way in ways:
            got, want = one_call(x, wc, ws, F, elem, *way), two_calls(x, wc, ws, elem, *way)
            for i, (a, b) in enumerate(zip(got, want)):
                assert torch.equal(bits(a), bits(b)), (T, d, F, way, i)


@gpu
@pytest.mark.parametrize("elem", ["e4m3", "e2m1"])
def test_columns_short_of_a_block_and_a_row_alone(elem):
    # F = 48: a tile whose last 16 columns lie outside; and every row of four
    # as it is by itself
    T, d, F = 4, 1024, 48
    x = rows(T, d, 9).to(DEV)
    wc, ws = weight(F, d, elem)
    whole = one_call(x, wc, ws, F, elem, 2, "rceil", "silu", torch.bfloat16, True, True)
    for t in range(T):
        alone = one_call(x[t:t + 1].contiguous(), wc, ws, F, elem, 2, "rceil", "silu", torch.bfloat16, True, True)
        for a, b in zip(whole, alone):
            assert torch.equal(bits(a[t:t + 1]), bits(b)), t


@gpu
def test_captured_and_replayed():
    T, d, F = 2, 2048, 512
    x = rows(T, d, 1).to(DEV)
    wc, ws = weight(F, d, "e4m3")
    mxnorm.mxnorm_gated_fwd(x, wc, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        h, gu, rho = mxnorm.mxnorm_gated_fwd(x, wc, ws, save_gu=True)
    for seed in (2, 3, 4):
        x.copy_(rows(T, d, seed))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((h, gu, rho), two_calls(x, wc, ws, "e4m3", 2, "rceil", "silu", torch.bfloat16, True, True)):
            assert torch.equal(bits(a), bits(b)), seed
