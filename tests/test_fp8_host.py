"""Refusals of the eight-bit entry points, through the C ABI on the CPU (every check is made before a launch), and the binding's own."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2505_03803_b200 import binding as B

EINVAL, ESHAPE, EALIGN, EUNSUPPORTED = 1, 2, 3, 7




def _aligned():
    buf = np.zeros(8192, np.uint8)
    return buf, (buf.ctypes.data + 255) // 256 * 256


def quantize(x=0, dtype=0, rows=4, cols=128, x_row=None, block=1, codes=0, scale=0):
    buf, p = _aligned()
    x, codes, scale = (p if v == 0 else v for v in (x, codes, scale))
    return B.lib().rwkvq_fp8_quantize(x, dtype, rows, cols, cols if x_row is None else x_row, block, codes, scale, None)


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), EINVAL), (dict(codes=None), EINVAL), (dict(scale=None), EINVAL), (dict(dtype=3), EINVAL), (dict(dtype=-1), EINVAL),
    (dict(rows=0), EINVAL), (dict(rows=-1), EINVAL), (dict(cols=0), EINVAL), (dict(cols=-16), EINVAL), (dict(block=2), EINVAL), (dict(block=0), EINVAL),
    (dict(cols=24), ESHAPE), (dict(cols=1), ESHAPE), (dict(x_row=112), EINVAL), (dict(x_row=130), EALIGN), (dict(dtype=1, x_row=132), EALIGN),
    (dict(rows=2**31 - 1, cols=2**12), EUNSUPPORTED)], ids=str)
def test_quantize_refusals(kw, status):
    assert quantize(**kw) == status


@pytest.mark.parametrize("which", ["x", "codes", "scale"])
def test_quantize_refuses_unaligned(which):
    buf, p = _aligned()
    assert quantize(**{which: p + 8}) == EALIGN


def product(w=0, ws=0, oc=64, ic=128, x=0, xs=0, M=4, y=0, dtype=0, y_row=None):
    buf, p = _aligned()
    w, ws, x, xs, y = (p if v == 0 else v for v in (w, ws, x, xs, y))
    return B.lib().rwkvq_gemm_fp8(w, ws, oc, ic, x, xs, M, y, dtype, oc if y_row is None else y_row, None)


@pytest.mark.parametrize("kw,status", [
    (dict(w=None), EINVAL), (dict(ws=None), EINVAL), (dict(x=None), EINVAL), (dict(xs=None), EINVAL), (dict(y=None), EINVAL),
    (dict(oc=0), EINVAL), (dict(ic=0), EINVAL), (dict(M=0), EINVAL), (dict(M=-3), EINVAL), (dict(dtype=3), EINVAL), (dict(y_row=63), EINVAL),
    (dict(ic=120), ESHAPE), (dict(oc=2**31 - 1, M=2**31 - 1), EUNSUPPORTED)], ids=str)
def test_product_refusals(kw, status):
    assert product(**kw) == status


@pytest.mark.parametrize("which", ["w", "ws", "x", "xs", "y"])
def test_product_refuses_unaligned(which):
    buf, p = _aligned()
    assert product(**{which: p + 4}) == EALIGN


def test_scale_pitch():
    assert [B.rwkvq_fp8_scale_pitch(c) for c in (0, -5, 1, 128, 2048, 2049, 4096, 14336)] == [0, 0, 16, 16, 16, 32, 32, 112]


def test_binding_refuses_what_is_not_on_the_device_or_ill_shaped():
    x, codes, scale = torch.zeros((4, 128)), torch.zeros((4, 128), dtype=torch.uint8), torch.zeros((4, 16), dtype=torch.uint8)
    with pytest.raises(B.RwkvqError) as e:
        B.rwkvq_fp8_quantize(x, codes, scale, 1)
    assert e.value.status == EINVAL
    with pytest.raises(B.RwkvqError):
        B.rwkvq_fp8_quantize(x, codes, scale, 64)
    with pytest.raises(B.RwkvqError):
        B.rwkvq_fp8_quantize(x.T, codes, scale, 1)
    with pytest.raises(B.RwkvqError):
        B.rwkvq_gemm_fp8(codes, scale, codes, scale, x)
    with pytest.raises(B.RwkvqError):
        B.rwkvq_fp8_quantize(x, codes.view(torch.float8_e5m2), scale, 1)


def test_the_call_that_loses_scales_refuses():
    buf, p = _aligned()
    call = lambda announced, lost: B.lib().rwkvq_gemm_fp8_lost(p, p, 64, 128, p, p, 4, p, 0, 64, 0, announced, lost, None)
    assert call(0, None) == EINVAL and call(-1, p) == EINVAL


def test_plan():
    plan = (C.c_int32 * 6)()
    for args, status in [((0, 64, 128), EINVAL), ((1, 0, 128), EINVAL), ((1, 64, 0), EINVAL), ((1, 64, 120), ESHAPE), ((2**31 - 1, 2**31 - 1, 128), EUNSUPPORTED), ((1, 64, 128), 0)]:
        assert B.lib().rwkvq_gemm_fp8_plan(*args, plan) == status
    assert B.lib().rwkvq_gemm_fp8_plan(1, 64, 128, None) == EINVAL
    for M in (1, 16, 100, 241, 2048, 70000):
        for oc in (1, 128, 4100, 65536):
            for ic in (16, 2048, 4112, 14336):
                p = B.rwkvq_gemm_fp8_plan(M, oc, ic)
                tall, wide = -(-oc // p["w_rows"]), -(-M // p["x_rows"])
                assert p["w_rows"] in (128, 256) and p["x_rows"] % 16 == 0 and 16 <= p["x_rows"] <= 240 and p["tiles"] == tall * wide
                assert p["slices"] in (1, 2, 4, 8) and p["slices"] * 4 <= -(-ic // 128) + 3 and 3 <= p["stages"] <= 12
                assert p["blocks"] == (p["tiles"] * p["slices"] if p["slices"] > 1 else min(p["tiles"], p["blocks"])) and p["blocks"] <= 148
    with pytest.raises(B.RwkvqError):
        B.rwkvq_gemm_fp8_plan(1, 64, 8)
