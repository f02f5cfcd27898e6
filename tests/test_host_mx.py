"""What the calls on 4-bit operands refuse, and their size functions; nothing here reaches a GPU."""
import ctypes as C

import pytest
import torch

from paper_2202_09368_b200 import binding as B
from paper_2202_09368_b200 import build as BUILD

import _mx as M

BAD, NOT, WS = B.EC_ERR_INVALID_ARG, B.EC_ERR_UNSUPPORTED, B.EC_ERR_WORKSPACE


@pytest.fixture(scope="module", autouse=True)
def built():
    BUILD.build()


def test_pitches():
    for cols in (1, 31, 32, 33, 511, 512, 513, 4096, (1 << 22) - 64):
        assert (B.lib().ec_mx_code_pitch(cols), B.lib().ec_mx_scale_pitch(cols)) == M.pitches(cols) == B._mx_pitches(cols)
    for cols in (0, -1, -2 ** 63):
        assert B.lib().ec_mx_code_pitch(cols) == B.lib().ec_mx_scale_pitch(cols) == 0


@pytest.mark.parametrize("args,code", [
    ((2, 4096, 1, 8, 64, 0, 4096, 4096), BAD), ((-1, 4096, 1, 8, 64, 0, 4096, 4096), BAD), ((1, 4096, 1, 8, 64, 2, 4096, 4096), BAD),
    ((1, 4096, -1, 8, 64, 0, 4096, 4096), BAD), ((1, 4096, 1, -8, 64, 0, 4096, 4096), BAD), ((1, 4096, 1, 8, 0, 0, 4096, 4096), BAD),
    ((1, None, 1, 8, 64, 0, 4096, 4096), BAD), ((1, 4096, 1, 8, 64, 0, None, 4096), BAD), ((1, 4096, 1, 8, 64, 0, 4096, None), BAD),
    ((1, 4104, 1, 8, 64, 0, 4096, 4096), BAD), ((1, 4096, 1, 8, 64, 0, 4104, 4096), BAD), ((1, 4096, 1, 8, 64, 0, 4096, 4097), BAD),
    ((1, 4096, 1, 8, 62, 0, 4096, 4096), NOT), ((0, 4096, 1, 8, 62, 0, 4096, 4096), NOT), ((1, 4096, 1, 62, 64, 1, 4096, 4096), NOT),
    ((1, 4096, 1, 8, 1 << 22, 0, 4096, 4096), NOT), ((1, 4096, 1, 1 << 22, 64, 1, 4096, 4096), NOT), ((1, 4096, 1 << 16, 1 << 15, 64, 0, 4096, 4096), NOT),
    ((1, 4096, 1 << 62, 8, 64, 0, 4096, 4096), NOT), ((1, 4096, 1, 1 << 62, 64, 0, 4096, 4096), NOT),
    ((1, None, 0, 8, 64, 0, None, None), B.EC_OK), ((1, None, 8, 0, 64, 0, None, None), B.EC_OK), ((1, None, 8, 0, 64, 1, None, None), B.EC_OK),
])
def test_quantize_refuses(args, code):
    assert B.lib().ec_mx_quantize(*args, None) == code


@pytest.mark.parametrize("args,code", [
    ((2, 4096, 4096, 8, 64, 4096), BAD), ((1, 4096, 4096, -1, 64, 4096), BAD), ((1, 4096, 4096, 8, 0, 4096), BAD), ((1, None, 4096, 8, 64, 4096), BAD),
    ((1, 4096, 4097, 8, 64, 4096), BAD), ((1, 4096, 4096, 8, 64, 4104), BAD), ((1, 4096, 4096, 8, 60, 4096), NOT), ((1, 4096, 4096, 1 << 31, 64, 4096), NOT),
    ((1, 4096, 4096, 8, 1 << 22, 4096), NOT), ((1, None, None, 0, 64, None), B.EC_OK),
])
def test_dequantize_refuses(args, code):
    assert B.lib().ec_mx_dequantize(*args, None) == code


def test_dispatch_refuses():
    L, p = B.lib(), 4096
    cfg = B.make_sort_config(16, 64, 8, 2, torch.bfloat16)
    for args in ((None, p, p, p), (p, None, p, p), (p, p, 4104, p), (p, p, p, None)):
        assert L.ec_mx_dispatch(C.byref(cfg), *args, None) == BAD
    assert L.ec_mx_dispatch(C.byref(B.make_sort_config(16, 60, 8, 2, torch.bfloat16)), p, p, p, p, None) == NOT
    assert L.ec_mx_dispatch(C.byref(B.make_sort_config(0, 64, 8, 2)), None, None, None, None, None) == B.EC_OK


def _gemm(rows=16, N=64, K=64, E=2, out=B.EC_MX_OUT_BF16, act=0, bias_dtype=0, A=4096, As=4096, off=4096, Bc=4096, Bs=4096, bias=None, Cp=4096, Cs=None,
          ws=4096, ws_bytes=256):
    cfg = B.ec_mx_gemm_config(rows, N, K, E, out, act, bias_dtype)
    return B.lib().ec_mx_expert_gemm(C.byref(cfg), A, As, off, Bc, Bs, bias, Cp, Cs, ws, ws_bytes, None)


@pytest.mark.parametrize("change,code", [
    (dict(rows=-1), BAD), (dict(N=0), BAD), (dict(K=0), BAD), (dict(E=0), BAD), (dict(out=3), BAD), (dict(out=-1), BAD), (dict(act=3), BAD), (dict(act=-1), BAD),
    (dict(bias_dtype=2), BAD), (dict(A=None), BAD), (dict(As=None), BAD), (dict(off=None), BAD), (dict(Bc=None), BAD), (dict(Bs=None), BAD), (dict(Cp=None), BAD),
    (dict(A=4104), BAD), (dict(bias=4104), BAD), (dict(Cs=4096), BAD), (dict(out=B.EC_MX_OUT_MX), BAD), (dict(out=B.EC_MX_OUT_MX, Cs=4100), BAD), (dict(ws=None), BAD),
    (dict(ws=4096 + 128), BAD), (dict(ws_bytes=255), WS), (dict(E=257), NOT), (dict(N=1 << 22), NOT), (dict(K=1 << 22), NOT), (dict(rows=(1 << 31) - 256), NOT),
    (dict(N=60), NOT), (dict(N=62, out=B.EC_MX_OUT_F32), NOT), (dict(rows=1 << 30, N=1 << 20), NOT),
    (dict(rows=0), B.EC_OK), (dict(rows=0, A=None, As=None, Cp=None), B.EC_OK),
])
def test_product_refuses(change, code):
    assert _gemm(**change) == code


def test_product_without_a_configuration():
    assert B.lib().ec_mx_expert_gemm(None, 4096, 4096, 4096, 4096, 4096, None, 4096, None, 4096, 256, None) == BAD


def test_tensors_that_are_refused():
    """Host tensors, types, ranks and shapes, before an address leaves for the library."""
    x = torch.zeros(8, 64)
    q = B.alloc_mx((8, 64), "cpu")
    cfg = B.make_sort_config(8, 64, 4, 1)
    for call in (lambda: B.ec_mx_quantize(x), lambda: B.ec_mx_quantize(x.half()), lambda: B.ec_mx_dequantize(q), lambda: B.ec_mx_dispatch(cfg, x, torch.zeros(8, 1, dtype=torch.int32)),
                 lambda: B.ec_mx_expert_gemm(q, B.alloc_mx((2, 8, 64), "cpu"), torch.zeros(3, dtype=torch.int32))):
        with pytest.raises(B.EcError) as e:
            call()
        assert e.value.code == BAD
    W, off = B.alloc_mx((2, 8, 64), "cpu"), torch.zeros(3, dtype=torch.int32)
    for call in (lambda: B.ec_mx_expert_gemm(q, W, off, act="relu"), lambda: B.ec_mx_expert_gemm(q, q, off), lambda: B.ec_mx_expert_gemm(W, W, off)):
        with pytest.raises(B.EcError) as e:
            call()
        assert e.value.code == BAD
    dev = -1                                              # what torch says of a host tensor
    assert len(B._mx_operands("x", dev, q, (8, 64))) == 2
    for shape in ((8, 65), (8, 96), (4, 64), (1, 8, 64)):
        with pytest.raises(B.EcError):
            B._mx_operands("x", dev, q, shape)


def test_the_restated_format():
    """The oracle's own worked values: ties to the even code, 6 beyond, scales from the largest magnitude."""
    import numpy as np
    x = np.zeros((1, 32))
    x[0, :12] = [4.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -7.0, -0.2, 0.26, 6.5]
    codes, scales = M.encode(x)
    assert scales[0, 0] == 127 and list(M.decode(codes, scales, 32)[0, :12]) == [4, 0, 1, 1, 2, 2, 4, 4, -6, -0.0, 0.5, 6]
    assert M.encode(x * 2.0 ** -140)[1][0, 0] == 0 and M.encode(np.zeros((1, 32)))[1][0, 0] == 0
    assert M.encode(np.full((1, 32), 3.4028234663852886e38))[1][0, 0] == 252
