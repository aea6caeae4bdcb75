"""The launch of a gated backward's two products in which the second has its K split
over four waves: every output against the oracle, and where it is chosen."""
import ctypes

import pytest
import torch

import launch_rules
from launch_rules import ELEM, PAIRS, UNITS
from paper_2603_13180_amd import mxnorm

DEV = "cuda:0"
SPLIT = len(PAIRS)     # mxt_gated_pair_plan's number
_I, _L = ctypes.c_int, ctypes.c_int64


def plan(T, F, d, elem):
    step = 128 if elem == "e4m3" else 256
    Tp = -(-T // step) * step
    f = launch_rules._fn("mxt_gated_pair_plan", [_L] * 6 + [_I] * 2)
    return f(2 * F, d, Tp, T, d, 2 * F, ELEM[elem], UNITS)


@pytest.mark.parametrize("T,F,d,elem,split", [
    (1024, 2048, 768, "e4m3", True), (1024, 2048, 768, "e2m1", True), (64, 1024, 512, "e4m3", True),
    (512, 2048, 1024, "e4m3", True), (50, 5120, 512, "e4m3", False), (8192, 14336, 4096, "e4m3", False),
    (3000, 3200, 2176, "e2m1", False)])
def test_where_it_is_chosen(T, F, d, elem, split):
    assert (plan(T, F, d, elem) == SPLIT) == split


def test_the_plain_backward_does_not_take_it():
    for T, F, d in ((1024, 2048, 768), (64, 1024, 512), (512, 2048, 1024)):
        for elem in ("e4m3", "e2m1"):
            assert launch_rules.pair_plan(-(-T // 256) * 256, 2 * F, d, elem)[0] in PAIRS


# products of partial tiles; the longer chain of steps first and second, fewer
# steps than waves, uneven shares
SIZES = [((531, 560, 256), (777, 304, 2304)), ((531, 560, 2560), (77, 304, 768)), ((257, 144, 512), (1, 16, 256)),
         ((64, 128, 256), (64, 64, 1280)), ((16, 16, 1024), (200, 528, 4096))]


@pytest.mark.gpu
@pytest.mark.parametrize("elem", ["e4m3", "e2m1"])
@pytest.mark.parametrize("sizes", SIZES)
def test_every_output(elem, sizes):
    if not torch.cuda.is_available():
        raise RuntimeError("pair tests need a GPU (run them with -m gpu on an MI355X)")
    from test_gpu_tile_shapes import check, guarded, random_case
    cases = [random_case(elem, *s, special=i == 1 and s[0] > 16 and s[1] > 17) for i, s in enumerate(sizes)]
    for gains in ((False, False), (True, False), (True, True)):
        outs = [guarded(s[0], s[1], dt) for s, dt in zip(sizes, (torch.float32, torch.bfloat16))]
        g = [c[3].to(DEV) if on else None for c, on in zip(cases, gains)]
        p = [launch_rules._Product(*(t.data_ptr() for t in c[0]), *s, None if gi is None else gi.data_ptr(),
                                   o[1].data_ptr()) for c, s, gi, o in zip(cases, sizes, g, outs)]
        f = launch_rules._fn("mxt_matmul_pair", [ctypes.c_void_p] * 2 + [_I] * 3 + [ctypes.c_void_p])
        mxnorm._check(f(ctypes.byref(p[0]), ctypes.byref(p[1]), ELEM[elem], SPLIT, 0,
                        mxnorm._stream(torch.device(DEV))))
        for i, ((buf, h), c) in enumerate(zip(outs, cases)):
            assert (buf[h.numel():] == 7.0).all()
            check(h, c[1], c[2], None if g[i] is None else c[3], "%s product %d" % (elem, i))
