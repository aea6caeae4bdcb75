"""Host-side checks of the gated feed-forward's entry points (no GPU needed):
what they refuse, before any launch."""
import ctypes
import os

import pytest
import torch

from paper_2603_13180_amd import mxnorm

pytestmark = pytest.mark.skipif(not os.path.exists(mxnorm.LIB_PATH), reason="libmxnorm.so not built")

A16, A8, A4, W256 = 0x10000, 0x10008, 0x10004, 0x100000

GATED = [
    (dict(M=-1), 1), (dict(F=-32), 1), (dict(K=0), 1), (dict(elem=2), 1), (dict(act=2), 1), (dict(act=-1), 1),
    (dict(out_dtype=3), 1), (dict(mode=2), 1), (dict(block=16), 2), (dict(block=64), 2), (dict(K=192), 2),
    (dict(K=128, elem=1), 2), (dict(F=24), 2), (dict(F=48), 2), (dict(F=8, out_dtype=0, scales=None), 2),
    (dict(K=1 << 23), 2), (dict(a=None), 1), (dict(as_=None), 1), (dict(w=None), 1), (dict(ws=None), 1),
    (dict(out=None), 1), (dict(scales=None), 1), (dict(out_dtype=1), 1), (dict(out_dtype=0), 1), (dict(a=A8), 1),
    (dict(w=A8), 1), (dict(as_=A16 + 2), 1), (dict(ws=A16 + 2), 1), (dict(out=A8), 1), (dict(gu=A8), 1),
    (dict(M=1 << 31), 2), (dict(F=(1 << 23) + 32), 2), (dict(M=1 << 24, F=1 << 22), 2),
    (dict(M=0, a=None, out=None), 0), (dict(F=0, w=None, out=None), 0), (dict(M=0, K=192), 2),
]


@pytest.mark.parametrize("kw,status", GATED)
def test_gated_forward_refusals(kw, status):
    a = dict(a=A16, as_=A4, w=A16, ws=A4, M=8, F=64, K=256, block=32, elem=0, act=0, mode=0, out_dtype=2,
             out=A16, scales=A4 + 1, gu=A16)
    a.update(kw)
    lib = mxnorm.load()
    assert lib.mx_gated_fwd(a["a"], a["as_"], a["w"], a["ws"], a["M"], a["F"], a["K"], a["block"], a["elem"],
                            a["act"], a["mode"], a["out_dtype"], a["out"], a["scales"], a["gu"], None) == status
    assert (mxnorm.mx_last_error() != "") == (status != 0)


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), 1), (dict(x=A8), 1), (dict(d=1000), 1), (dict(d=1056), 2), (dict(d=65536), 2), (dict(p=3), 1),
    (dict(eps=-1.0), 1), (dict(coef=float("nan")), 1), (dict(rho=A16 + 2), 1), (dict(F=24), 2), (dict(act=5), 1),
    (dict(block=16), 2), (dict(block=7), 1), (dict(elem=2), 1), (dict(mode=2), 1), (dict(out_dtype=3), 1),
    (dict(scales=A4), 1), (dict(w=None), 1), (dict(out=A8), 1), (dict(gu=A8), 1), (dict(ws=None), 1),
    (dict(wspace=0x100010), 1), (dict(wspace=None), 1), (dict(wbytes=1024), 1), (dict(T=-1), 1),
    (dict(T=0, x=None, out=None, wspace=None), 0),
])
def test_norm_and_gate_checks_both_parts_before_a_launch(kw, status):
    a = dict(x=A16, T=8, d=1024, w=A16, ws=A4, F=64, block=32, elem=0, p=2, coef=0.0, eps=1e-6, mode=0, act=0,
             out_dtype=1, out=A16, scales=None, gu=A16, rho=A4, wspace=W256, wbytes=1 << 40)
    a.update(kw)
    lib = mxnorm.load()
    got = lib.mxnorm_gated_fwd(a["x"], a["T"], a["d"], a["w"], a["ws"], a["F"], a["block"], a["elem"], a["p"],
                               a["coef"], a["eps"], a["mode"], a["act"], a["out_dtype"], a["out"], a["scales"],
                               a["gu"], a["rho"], a["wspace"], a["wbytes"], None)
    assert got == status
    assert (mxnorm.mx_last_error() != "") == (status != 0)


def test_workspace_sizes():
    lib = mxnorm.load()
    assert lib.mxnorm_gated_fwd_workspace_bytes(8, 1024, 32, 0) >= 8 * 1024 + 8 * 32
    for bad in ((0, 1024, 32, 0), (8, 0, 32, 0), (8, 1024, 0, 0), (8, 1024, 32, 2)):
        assert lib.mxnorm_gated_fwd_workspace_bytes(*bad) == 0


def test_binding_refuses_cpu_tensors_and_bad_names():
    x = torch.zeros(4, 256, dtype=torch.bfloat16)
    c, s = torch.zeros(64, 256, dtype=torch.uint8), torch.zeros(64, 8, dtype=torch.uint8)
    with pytest.raises(RuntimeError, match="GPU"):
        mxnorm.mxnorm_gated_fwd(x, c, s)
    with pytest.raises(ValueError):
        mxnorm.mx_gated_fwd(c, s, c, s, 256)
    with pytest.raises(ValueError):
        mxnorm.mx_gated_fwd(c, s, c, s, 256, elem="e5m2")


@pytest.mark.parametrize("M,F,K,want", [
    # decoding: the narrowest tiles that hold the rows, rings where 64 rows share
    # a weight; prefill: 256 x 256
    (1, 14336, 4096, 7), (16, 14336, 4096, 7), (32, 14336, 4096, 4), (61, 14336, 4096, 4), (61, 8192, 8192, 9),
    (32, 8192, 8192, 8), (61, 4096, 2048, 8), (128, 14336, 4096, 5), (1000, 4096, 2048, 5), (16384, 14336, 4096, 6),
])
def test_plan_names_a_gated_kernel(M, F, K, want):
    whole, tail, us = ctypes.c_int(), ctypes.c_int(), ctypes.c_double()
    f = mxnorm.load().mxt_gated_plan
    f.restype, f.argtypes = ctypes.c_int, [ctypes.c_int64] * 3 + [ctypes.c_int] * 2 + [ctypes.c_void_p] * 3
    for elem in (0, 1):
        shape = f(M, F, K, elem, 256, ctypes.byref(whole), ctypes.byref(tail), ctypes.byref(us))
        assert shape in (4, 5, 6, 7, 8, 9) and us.value > 0
        assert elem or shape == want
        assert not whole.value or (shape == 6 and tail.value in (4, 5, 7, 8, 9))
    assert f(M, F, 100, 0, 256, ctypes.byref(whole), ctypes.byref(tail), ctypes.byref(us)) == -1


@pytest.mark.parametrize("M,F,K,elem,want", [
    # one row of tiles, from 96 MB of weights on; a first launch of 256 x 256 tiles
    # has one up to 256 rows, the smaller tiles of its tail do not
    (1, 14336, 4096, 0, 1), (61, 14336, 4096, 0, 1), (61, 14336, 4096, 1, 0), (129, 14336, 4096, 0, 0),
    (200, 36096, 4096, 0, 1), (200, 37120, 4096, 0, 1), (200, 65792, 4096, 0, 1), (256, 37120, 8192, 1, 1),
    (257, 65792, 4096, 0, 0),
])
def test_weights_that_are_read_once(M, F, K, elem, want):
    f = mxnorm.load().mxt_gated_once
    f.restype, f.argtypes = ctypes.c_int, [ctypes.c_int64] * 3 + [ctypes.c_int] * 2
    assert f(M, F, K, elem, 256) == want
