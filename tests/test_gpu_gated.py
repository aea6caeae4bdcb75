"""The gated feed-forward's first half on the GPU: every kernel that computes
it, its three kinds of output, and the entry points.

Operands are small multiples of a power of two, a row's blocks within a factor
of four of each other, so that every sum of products is exact in float in any
order (at most 512 products below 2^12 units).  Then:

* the kept products are the exact ones rounded to bf16, bit for bit;
* float H is act(G) U of those in 64 bits within the error of the activation and
  of two products.  With |z| <= 100, the exponential's argument -z log2(e) is
  rounded at most four times (GELU: g^2, the polynomial, its product with g, and
  the constants), 100 * 4 * 2^-24 < 2^-15; exp2 and the reciprocal are within a
  unit, 2^-23, the sum and both products within 2^-24 each.  Where the
  exponential overflows (z < -88) H is 0 against |H| < 2^-126 |G U|.  Together
  2^-14 |H| + 2^-120 |G U|;
* bf16 H is the float H rounded, MX codes are the oracle's cast of the float H,
  both bit for bit (one kernel, one order of sums).
"""
import ctypes

import numpy as np
import pytest
import torch

import oracle
from launch_rules import ELEM, SHAPES
from paper_2603_13180_amd import mxnorm, synth
from test_gpu_gemm import dev_u8

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ELEMS = ["e4m3", "e2m1"]
ACTS = ["silu", "gelu_tanh"]
NAMES = SHAPES + ["g16x64", "g32x64", "g64x64"]
GATED_SHAPES = NAMES[4:]
# (tile shape, 256 x 256 cells before it, compute units; 0: the device's)
WAYS = [(s, 0, 0) for s in GATED_SHAPES] + \
    [(s, 0, u) for s in ("r64x128", "r128x128", "t256x256") for u in (1, 2)] + \
    [(s, n, 1) for s in GATED_SHAPES if s != "t256x256" for n in (2, 5)]
_I, _L, _P = ctypes.c_int, ctypes.c_int64, ctypes.c_void_p


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        raise RuntimeError("GPU gated tests need a GPU (run them with -m gpu on an MI355X)")
    mxnorm.load()


def guarded(shape, dtype):
    """A tensor of `shape` at the start of a buffer of sevens."""
    n = int(np.prod(shape))
    buf = torch.full((n + 4096,), 7, dtype=dtype, device=DEV)
    return buf, buf[:n].view(shape)


def gated_as(ac, as_, wc, ws, K, elem, act, dtype, shape, whole=0, units=0, mode="rceil", keep=True):
    """mx_gated_fwd by the named kernel: (H or (codes, scales), gu), each with
    nothing written behind it."""
    M, F = ac.shape[0], wc.shape[0] // 2
    codes = dtype is torch.uint8
    bo, out = guarded((M, F // 2 if codes and elem == "e2m1" else F), dtype)
    bs, sc = guarded((M, F // 32), torch.uint8)
    bg, gu = guarded((M, 2 * F), torch.bfloat16)
    f = mxnorm.load().mxt_gated
    f.restype, f.argtypes = _I, [_P] * 4 + [_L] * 3 + [_I] * 4 + [_P] * 3 + [_I] * 3 + [_P]
    mxnorm._check(f(ac.data_ptr(), as_.data_ptr(), wc.data_ptr(), ws.data_ptr(), M, F, K, ELEM[elem],
                    mxnorm.ACTS[act], mxnorm.SCALE_MODES[mode], mxnorm.GATED_DTYPES[dtype],
                    out.data_ptr(), sc.data_ptr() if codes else None, gu.data_ptr() if keep else None,
                    NAMES.index(shape), whole, units, mxnorm._stream(ac.device)))
    assert (bo[out.numel():] == 7).all() and (bg[gu.numel():] == 7).all()
    assert (bs[sc.numel() if codes else 0:] == 7).all()
    if not keep:
        assert (gu == 7).all()
    return ((out, sc) if codes else out), gu


def operand(rows, K, elem, rng, base):
    """(codes, scales, their values in 64 bits): row r's scales are 2^base[r] to
    four times that."""
    if elem == "e4m3":
        codes = rng.choice(np.array([0, 0x38, 0x40, 0x44, 0x48, 0x4C, 0xB8, 0xC0, 0xC4, 0xC8, 0xCC], np.uint8),
                           (rows, K))
        v = oracle.e4m3_value(codes)
    else:
        n = rng.integers(0, 16, (rows, K), dtype=np.uint8)
        codes, v = n[:, 0::2] | n[:, 1::2] << 4, oracle.e2m1_value(n)
    e = np.asarray(base)[:, None] + rng.integers(0, 3, (rows, K // 32))
    return codes, (e + 127).astype(np.uint8), v.astype(np.float64) * np.repeat(np.exp2(e), 32, 1)


def operands(elem, M, F, K, seed=0, abase=None, wbase=None):
    """The four operands on the GPU and the exact products [M, 2F]."""
    rng = np.random.default_rng(seed + M + 3 * F + 5 * K + len(elem))
    ac, as_, a = operand(M, K, elem, rng, np.full(M, -4) if abase is None else abase(rng))
    wc, ws, w = operand(2 * F, K, elem, rng, np.full(2 * F, -3) if wbase is None else wbase(rng))
    return [dev_u8(v) for v in (ac, as_, wc, ws)], a @ w.T


def decode(codes, scales, elem):
    v = oracle.e4m3_value(codes) if elem == "e4m3" else \
        oracle.e2m1_value(np.stack((codes & 15, codes >> 4), -1).reshape(codes.shape[0], -1))
    return v.astype(np.float64) * np.repeat(np.exp2(scales.astype(np.float64) - 127), 32, 1)


def kept(products):
    return bits(torch.from_numpy(products).float().bfloat16().to(DEV))


def bits(t):
    return t.contiguous().view(torch.int16 if t.element_size() == 2 else torch.int32)


def act64(g, act):
    """act(g) in 64 bits, g >= -700 or so beyond which it is 0."""
    z = g if act == "silu" else 2 * np.sqrt(2 / np.pi) * (g + 0.044715 * g ** 3)
    with np.errstate(over="ignore"):
        return g / (1 + np.exp(-z))


def check_float(h, products, act):
    g, u = np.split(products, 2, axis=1)
    with np.errstate(invalid="ignore", over="ignore"):
        want = act64(g, act) * u
        err = np.abs(h.cpu().numpy().astype(np.float64) - want)
        bad = ~(err <= 2.0 ** -14 * np.abs(want) + 2.0 ** -120 * np.abs(g * u))
    assert not bad.any(), "%d outputs off, first %s: %r, want %r" % (
        bad.sum(), np.argwhere(bad)[0], h[tuple(np.argwhere(bad)[0])].item(), want[tuple(np.argwhere(bad)[0])])


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("elem", ELEMS)
@pytest.mark.parametrize("shape,whole,units", WAYS)
def test_every_kernel(elem, shape, whole, units, act):
    # 300 x 416: two row cells, four column cells of 128, the last of each
    # partial
    M, F, K = 300, 416, 512
    t, p = operands(elem, M, F, K)
    assert 5 < p[:, :F].std() < 40
    h, gu = gated_as(*t, K, elem, act, torch.float32, shape, whole, units)
    assert torch.equal(bits(gu), kept(p))
    check_float(h, p, act)
    hb, _ = gated_as(*t, K, elem, act, torch.bfloat16, shape, whole, units, keep=False)
    assert torch.equal(bits(hb), bits(h.to(torch.bfloat16)))
    for mode in ("rceil", "floor"):
        (c, s), gm = gated_as(*t, K, elem, act, torch.uint8, shape, whole, units, mode)
        wc, ws = oracle.mxcast(h.cpu().numpy(), elem=elem, mode=mode)
        assert np.array_equal(s.cpu().numpy(), ws) and np.array_equal(c.cpu().numpy(), wc)
        assert torch.equal(bits(gm), bits(gu))


@pytest.mark.parametrize("elem", ELEMS)
@pytest.mark.parametrize("M,F,K", [(1, 16, 256), (1, 32, 256), (17, 48, 512), (64, 32, 1024), (65, 80, 256),
                                   (257, 144, 256), (3, 4112, 256)])
@pytest.mark.parametrize("shape", GATED_SHAPES)
def test_edges_of_tiles(elem, shape, M, F, K):
    t, p = operands(elem, M, F, K, seed=7)
    h, gu = gated_as(*t, K, elem, "silu", torch.float32, shape)
    assert torch.equal(bits(gu), kept(p))
    check_float(h, p, "silu")
    hb, _ = gated_as(*t, K, elem, "silu", torch.bfloat16, shape)
    assert torch.equal(bits(hb), bits(h.to(torch.bfloat16)))
    if F % 32 == 0:
        (c, s), _ = gated_as(*t, K, elem, "silu", torch.uint8, shape)
        wc, ws = oracle.mxcast(h.cpu().numpy(), elem=elem)
        assert np.array_equal(s.cpu().numpy(), ws) and np.array_equal(c.cpu().numpy(), wc)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("elem", ELEMS)
@pytest.mark.parametrize("shape", ["g16x64", "r64x128", "t256x256"])
def test_wide_ranges_and_non_finite_values(elem, shape, act):
    # gate products from below the exponential's range to beyond it, rows of
    # NaN, sums that overflow to infinity
    M, F, K = 70, 64, 256
    t, p = operands(elem, M, F, K, seed=3, abase=lambda r: r.integers(-27, 20, M), wbase=lambda r: r.integers(-17, 6, 2 * F))
    t[1][5] = 0xFF
    p[5] = np.nan
    # one product of row 9, and one of up column 50, beyond or below float's
    # range (sums of several would depend on their order)
    big = 0x4C if elem == "e4m3" else 0x77
    for codes, scales, row in ((t[0], t[1], 9), (t[2], t[3], F + 50)):
        codes[row] = 0
        codes[row, 3] = big
        scales[row] = 254
    one = [decode(c.cpu().numpy(), s.cpu().numpy(), elem) for c, s in ((t[0], t[1]), (t[2], t[3]))]
    with np.errstate(all="ignore"):
        p[9], p[:, F + 50] = one[0][9] @ one[1].T, one[0] @ one[1][F + 50]
        p = np.where(np.abs(p) > 3.4028236e38, np.copysign(np.inf, p), p)
    p[5] = np.nan
    t[3][40, 3] = 0xFF                     # gate column 40
    p[:, 40] = np.nan
    assert np.isinf(p).sum() > 10
    g, u = np.split(p, 2, axis=1)
    h, _ = gated_as(*t, K, elem, act, torch.float32, shape)
    got = h.cpu().numpy().astype(np.float64)
    assert np.isnan(got[5]).all() and np.isnan(got[:, 40]).all()
    with np.errstate(all="ignore"):
        a = act64(g, act)
        a[np.isneginf(g)] = np.nan         # -inf times 0
        want = (a.astype(np.float32) * u.astype(np.float32)).astype(np.float64)
        # where act(G) U is 0 * inf only after the activation has underflowed
        # the formula's value is anything between: those are left out
        tiny = np.isinf(u) & (np.abs(a) < 2.0 ** -100)
        exact = a * u
        ok = (np.isnan(got) & np.isnan(want)) | (got == want) | \
            (np.abs(got - exact) <= 2.0 ** -14 * np.abs(exact) + 2.0 ** -100 * np.abs(g * u)) | \
            (np.isinf(got) & (np.abs(exact) > 3.4e38)) | tiny
        ok[9, 50] = True                   # 2^127 twice
    assert ok.all(), "%d off, first %s" % ((~ok).sum(), np.argwhere(~ok)[0])
    for mode in ("rceil", "floor"):
        (c, s), _ = gated_as(*t, K, elem, act, torch.uint8, shape, mode=mode)
        wc_, ws_ = oracle.mxcast(h.cpu().numpy(), elem=elem, mode=mode)
        s, c = s.cpu().numpy(), c.cpu().numpy()
        assert np.array_equal(s, ws_)
        nan = np.repeat(ws_ == 0xFF, 32 if elem == "e4m3" else 16, axis=1)
        # a NaN's sign is the hardware's: in NaN blocks the magnitudes count
        mag = 0x7F if elem == "e4m3" else 0x77
        assert np.array_equal(c[~nan], wc_[~nan]) and (c[nan] & mag == mag).all() and nan.any()


# ------------------------------------------------------------ entry points --

def planned(M, F, K, elem):
    whole, tail, us = _I(), _I(), ctypes.c_double()
    f = mxnorm.load().mxt_gated_plan
    f.restype, f.argtypes = _I, [_L] * 3 + [_I] * 2 + [_P] * 3
    s = f(M, F, K, ELEM[elem], torch.cuda.get_device_properties(0).multi_processor_count,
          ctypes.byref(whole), ctypes.byref(tail), ctypes.byref(us))
    return (NAMES[tail.value], whole.value) if whole.value else (NAMES[s], 0)


def same(a, b):
    if isinstance(a, tuple):
        return all(same(x, y) for x, y in zip(a, b))
    return torch.equal(bits(a) if a.is_floating_point() else a, bits(b) if b.is_floating_point() else b)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.uint8])
@pytest.mark.parametrize("elem", ELEMS)
@pytest.mark.parametrize("M,F,K", [(1, 512, 512), (61, 2048, 512), (1000, 2048, 768), (2304, 4224, 256)])
def test_entry_point_runs_its_plan(elem, dtype, M, F, K):
    t, _ = operands(elem, M, F, K, seed=1)
    shape, whole = planned(M, F, K, elem)
    for keep in (False, True):
        h, gu = mxnorm.mx_gated_fwd(*t, K, elem=elem, act="gelu_tanh", out_dtype=dtype, save_gu=keep)
        want, wgu = gated_as(*t, K, elem, "gelu_tanh", dtype, shape, whole)
        assert same(h, want) and (same(gu, wgu) if keep else gu is None)


@pytest.mark.parametrize("elem", ELEMS)
@pytest.mark.parametrize("T,d,F", [(1, 256, 32), (33, 512, 96), (1000, 1024, 1056)])
def test_norm_and_gate_as_one_call(elem, T, d, F):
    x = torch.from_numpy(synth.gaussian(T, d, seed=T, scale=2.0).view(np.int16)).to(DEV).view(torch.bfloat16)
    gen = torch.Generator(device=DEV).manual_seed(d)
    w = (0.05 * torch.randn(2 * F, d, generator=gen, device=DEV)).bfloat16()
    wc, ws = mxnorm.mx_cast_fwd(w, elem=elem)
    for p, mode in ((2, "rceil"), (1, "floor")):
        ac, as_, rho = mxnorm.mxnorm_mx_fwd(x, elem=elem, p=p, scale_mode=mode)
        for dtype in (torch.float32, torch.bfloat16, torch.uint8):
            h, gu, r = mxnorm.mxnorm_gated_fwd(x, wc, ws, elem=elem, p=p, scale_mode=mode, out_dtype=dtype,
                                               save_gu=True)
            want, wgu = mxnorm.mx_gated_fwd(ac, as_, wc, ws, d, elem=elem, scale_mode=mode, out_dtype=dtype,
                                            save_gu=True)
            assert same(h, want) and same(gu, wgu) and same(r, rho)
    h, gu, r = mxnorm.mxnorm_gated_fwd(x, wc, ws, elem=elem, want_rho=False)
    assert gu is None and r is None and h.dtype == torch.bfloat16


def test_no_rows_and_no_columns():
    wc, ws = torch.zeros(64, 256, dtype=torch.uint8, device=DEV), torch.zeros(64, 8, dtype=torch.uint8, device=DEV)
    h, gu = mxnorm.mx_gated_fwd(wc[:0], ws[:0], wc, ws, 256, save_gu=True)
    assert h.shape == (0, 32) and gu.shape == (0, 64)
    h, gu = mxnorm.mx_gated_fwd(wc, ws, wc[:0], ws[:0], 256)
    assert h.shape == (64, 0)
    x = torch.empty(0, 256, dtype=torch.bfloat16, device=DEV)
    (c, s), _, rho = mxnorm.mxnorm_gated_fwd(x, wc, ws, out_dtype=torch.uint8)
    assert c.shape == (0, 32) and s.shape == (0, 1) and rho.shape == (0,)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.uint8])
def test_another_stream_and_a_captured_graph(dtype):
    T, d, F = 130, 512, 256
    x = torch.randn(T, d, device=DEV).bfloat16()
    wc, ws = mxnorm.mx_cast_fwd((0.05 * torch.randn(2 * F, d, device=DEV)).bfloat16())
    want = mxnorm.mxnorm_gated_fwd(x, wc, ws, out_dtype=dtype, save_gu=True)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = mxnorm.mxnorm_gated_fwd(x, wc, ws, out_dtype=dtype, save_gu=True)
    torch.cuda.current_stream().wait_stream(s)
    assert same(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = mxnorm.mxnorm_gated_fwd(x, wc, ws, out_dtype=dtype, save_gu=True)
    for seed in range(3):
        x.copy_(torch.randn(T, d, device=DEV, generator=torch.Generator(device=DEV).manual_seed(seed)))
        graph.replay()
        want = mxnorm.mxnorm_gated_fwd(x, wc, ws, out_dtype=dtype, save_gu=True)
        torch.cuda.synchronize()
        assert same(out, want)


def test_feed_forward_forward():
    """Norm, gate, down projection as a user chains them, against the oracle's
    steps in 64 bits: the casts' half steps dominate (2^-4 of an element for x
    and H each, weights are given as codes), random over the sums."""
    T, d, F = 50, 512, 768
    xb = synth.gaussian(T, d, seed=11, scale=1.0)
    x = torch.from_numpy(xb.view(np.int16)).to(DEV).view(torch.bfloat16)
    gen = torch.Generator(device=DEV).manual_seed(5)
    w = (0.1 * torch.randn(2 * F, d, generator=gen, device=DEV)).bfloat16()
    wd = (0.1 * torch.randn(d, F, generator=gen, device=DEV)).bfloat16()
    wc, ws = mxnorm.mx_cast_fwd(w)
    dc, ds = mxnorm.mx_cast_fwd(wd)
    (hc, hs), _, _ = mxnorm.mxnorm_gated_fwd(x, wc, ws, out_dtype=torch.uint8)
    y = mxnorm.mx_matmul_fwd(hc, hs, dc, ds, F)
    a = oracle.mxnorm_mx(xb)
    gu = oracle.mx_matmul(a[0], a[1], wc.cpu().numpy(), ws.cpu().numpy(), d)
    h = act64(gu[:, :F], "silu") * gu[:, F:]
    oc, os_ = oracle.mxcast(h.astype(np.float32))
    want = oracle.mx_matmul(oc, os_, dc.cpu().numpy(), ds.cpu().numpy(), F)
    # H before its cast is within the products' 2^-9 of sum |a b|; a code then
    # differs by at most one step, 2^-3 of the element, in few places
    err = np.linalg.norm(y.cpu().numpy() - want) / np.linalg.norm(want)
    assert err <= 2.0 ** -8, err


@pytest.mark.parametrize("elem", ELEMS)
@pytest.mark.parametrize("M", [1, 5, 29, 61, 120])
def test_large_weights_read_once(elem, M):
    # over 96 MB: a tile's K steps in an order of its own.  Codes of 0, 1 and -1 and
    # scales of 1 and 2: sums below 2^16, exact in any order
    F, K = (12800, 4096) if elem == "e4m3" else (12800, 8192)
    gen = torch.Generator(device=DEV).manual_seed(M)
    val = torch.tensor([0.0, 1.0, -1.0, 0.0], device=DEV)
    code = torch.tensor([0x00, 0x38, 0xB8, 0x00] if elem == "e4m3" else [0, 2, 10, 0], dtype=torch.uint8, device=DEV)

    def operand(rows):
        i = torch.randint(0, 4, (rows, K), generator=gen, device=DEV)
        e = torch.randint(0, 2, (rows, K // 32), generator=gen, device=DEV)
        c = code[i]
        if elem == "e2m1":
            c = c[:, 0::2] | (c[:, 1::2] << 4)
        return c.contiguous(), (127 + e).to(torch.uint8), val[i] * torch.exp2(e.float()).repeat_interleave(32, 1)
    (ac, as_, a), (wc, ws, w) = operand(M), operand(2 * F)
    assert wc.numel() >= 96 << 20
    h, gu = mxnorm.mx_gated_fwd(ac, as_, wc, ws, K, elem=elem, out_dtype=torch.float32, save_gu=True)
    exact = torch.cat([a.double() @ p.double().t() for p in w.split(3200)], 1)
    assert exact.abs().max() < 1 << 16 and torch.equal(gu, exact.to(torch.bfloat16))
    want = act64(exact.cpu().numpy()[:, :F], "silu") * exact.cpu().numpy()[:, F:]
    assert (np.abs(h.cpu().numpy() - want) <= 2.0 ** -14 * np.abs(want) + 2.0 ** -120 * np.abs(exact.cpu().numpy()[:, :F] * exact.cpu().numpy()[:, F:])).all()
