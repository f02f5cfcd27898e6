"""The 4-bit products in the debug build: the same bits as the normal one, and waits that run out are reported, not waited for."""
import ctypes

import pytest
import torch

from paper_2202_09368_b200 import binding as B

import _mx as M
from test_gpu_debug_build import D  # noqa: F401  (the fixture: a second binding, of the debug library)

pytestmark = pytest.mark.gpu


def _operands(M, rows, N, K, E):
    g = torch.Generator(device="cuda").manual_seed(rows)
    A = M.ec_mx_quantize(torch.empty(rows, K, device="cuda").normal_(generator=g))
    W = M.ec_mx_quantize(torch.empty(E, N, K, device="cuda").normal_(generator=g))
    return A, W, torch.arange(E + 1, dtype=torch.int32, device="cuda") * (rows // E)


@pytest.mark.parametrize("rows,N,K,E", [(1, 128, 8192, 1), (30, 264, 6144, 2), (64, 256, 512, 2), (300, 1000, 1000, 2), (900, 384, 512, 2)])
def test_a_product_whose_loads_never_come(D, rows, N, K, E):
    """One CTA loads nothing: the call ends, with the status of a wait that ran out, and the next one on the same workspace is as ever."""
    A, W, offsets = _operands(D, rows, N, K, E)
    ws = torch.empty(D.EC_MX_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
    want = D.ec_mx_expert_gemm(A, W, offsets, ws=ws)
    assert D.ec_read_status(ws) == D.EC_OK and torch.equal(want, B.ec_mx_expert_gemm(A, W, offsets))
    cfg = D.ec_mx_gemm_config(rows, N, K, E, D.EC_MX_OUT_BF16, 0, 0)
    call = D.lib().ec_debug_mx_wait
    call.argtypes = [ctypes.POINTER(D.ec_mx_gemm_config)] + [ctypes.c_void_p] * 9 + [ctypes.c_size_t, ctypes.c_void_p]
    out = torch.zeros_like(want)
    assert call(ctypes.byref(cfg), A.codes.data_ptr(), A.scales.data_ptr(), offsets.data_ptr(), W.codes.data_ptr(), W.scales.data_ptr(), None,
                out.data_ptr(), None, ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream) == D.EC_OK
    assert D.ec_read_status(ws) == D.EC_ERR_TIMEOUT
    assert torch.equal(D.ec_mx_expert_gemm(A, W, offsets, ws=ws), want) and D.ec_read_status(ws) == D.EC_OK


@pytest.mark.parametrize("rows,N,K,E,columns", [(2400, 4096, 520, 8, 128), (4000, 8192, 4104, 8, 256)])
def test_loads_that_never_come_where_a_cta_has_several_tiles(D, rows, N, K, E, columns):
    """The same with three tiles and more to a CTA, in tiles of 128 and of 256 columns: the roles leave in the middle of their tiles."""
    A, W, offsets = _operands(D, rows, N, K, E)
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    assert M.form(rows, N, K, E, sms) == (192, columns) and M.tiles(offsets.cpu(), N, 192, columns) > 2 * sms
    ws = torch.empty(D.EC_MX_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
    want = D.ec_mx_expert_gemm(A, W, offsets, ws=ws)
    assert D.ec_read_status(ws) == D.EC_OK and torch.equal(want, B.ec_mx_expert_gemm(A, W, offsets))
    cfg = D.ec_mx_gemm_config(rows, N, K, E, D.EC_MX_OUT_BF16, 0, 0)
    call = D.lib().ec_debug_mx_wait
    call.argtypes = [ctypes.POINTER(D.ec_mx_gemm_config)] + [ctypes.c_void_p] * 9 + [ctypes.c_size_t, ctypes.c_void_p]
    out = torch.zeros_like(want)
    assert call(ctypes.byref(cfg), A.codes.data_ptr(), A.scales.data_ptr(), offsets.data_ptr(), W.codes.data_ptr(), W.scales.data_ptr(), None,
                out.data_ptr(), None, ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream) == D.EC_OK
    assert D.ec_read_status(ws) == D.EC_ERR_TIMEOUT
    assert torch.equal(D.ec_mx_expert_gemm(A, W, offsets, ws=ws), want) and D.ec_read_status(ws) == D.EC_OK


def _silent(D, cfg, A, W, offsets, out, ws):
    """A product whose first CTA loads nothing."""
    call = D.lib().ec_debug_mx_wait
    call.argtypes = [ctypes.POINTER(D.ec_mx_gemm_config)] + [ctypes.c_void_p] * 9 + [ctypes.c_size_t, ctypes.c_void_p]
    assert call(ctypes.byref(cfg), A.codes.data_ptr(), A.scales.data_ptr(), offsets.data_ptr(), W.codes.data_ptr(), W.scales.data_ptr(), None,
                out.data_ptr(), None, ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream) == D.EC_OK


@pytest.mark.parametrize("rows,N,K,E", [(1, 128, 8192, 1), (64, 256, 512, 2), (900, 384, 512, 2)])
def test_a_wait_that_ran_out_is_not_lost_behind_a_later_product(D, rows, N, K, E):
    """A chain of products on one workspace is asked once, at its end; the answer is given once, and a call of another kind starts anew."""
    A, W, offsets = _operands(D, rows, N, K, E)
    for fill in (0, 0xA5, 5):                             # whatever the workspace holds before its first use
        ws = torch.full((D.EC_MX_WORKSPACE_BYTES,), fill, dtype=torch.uint8, device="cuda")
        want = D.ec_mx_expert_gemm(A, W, offsets, ws=ws)
        assert D.ec_read_status(ws) == D.EC_OK
    cfg = D.ec_mx_gemm_config(rows, N, K, E, D.EC_MX_OUT_BF16, 0, 0)
    _silent(D, cfg, A, W, offsets, torch.zeros_like(want), ws)
    for _ in range(3):
        assert torch.equal(D.ec_mx_expert_gemm(A, W, offsets, ws=ws), want)
    assert D.ec_read_status(ws) == D.EC_ERR_TIMEOUT
    assert D.ec_read_status(ws) == D.EC_OK
    assert torch.equal(D.ec_mx_expert_gemm(A, W, offsets, ws=ws), want) and D.ec_read_status(ws) == D.EC_OK
    layer = D.make_config(256, 64, 128, 4, 2.0, torch.bfloat16)
    ws = D.alloc_workspace(layer)
    _silent(D, cfg, A, W, offsets, torch.zeros_like(want), ws)
    g = torch.Generator(device="cuda").manual_seed(1)
    D.ec_route(layer, *(torch.empty(s, device="cuda").normal_(generator=g).to(torch.bfloat16) for s in ((256, 64), (64, 4))), ws=ws)
    assert D.ec_read_status(ws) == D.EC_OK


@pytest.mark.parametrize("n", [3, 3000, 20000])
def test_nor_behind_a_plan(D, n):
    """Nor do a plan's counts land in the word: in one CTA, in a cluster and in two launches."""
    A, W, offsets = _operands(D, 64, 256, 512, 2)
    sort = D.make_sort_config(n, 64, 200, 2)
    choice = torch.randint(0, 200, (n, 2), generator=torch.Generator().manual_seed(n), dtype=torch.int32).cuda()
    ws = torch.empty(D.ec_sort_workspace_bytes(sort), dtype=torch.uint8, device="cuda")
    _silent(D, D.ec_mx_gemm_config(64, 256, 512, 2, D.EC_MX_OUT_BF16, 0, 0), A, W, offsets, torch.zeros(64, 256, dtype=torch.bfloat16, device="cuda"), ws)
    D.ec_sort_tokens(sort, choice, ws=ws)
    assert D.ec_read_status(ws) == D.EC_ERR_TIMEOUT
