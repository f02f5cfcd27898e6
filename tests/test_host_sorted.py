"""What the calls on tokens sorted by expert refuse, and their size functions; nothing here reaches a GPU."""
import ctypes as C
import itertools

import pytest
import torch

from paper_2202_09368_b200 import binding as B
from paper_2202_09368_b200 import build as BUILD


@pytest.fixture(scope="module", autouse=True)
def built():
    BUILD.build()


def _codes(cfg, p=4096):
    """The status of every call with the pointer p in each place, a workspace of 256 KiB at 4096."""
    L, r = B.lib(), C.byref(cfg)
    return [L.ec_sort_tokens(r, p, p, p, p, 4096, 1 << 18, None), L.ec_dispatch(r, p, p, p, None), L.ec_combine(r, p, None, p, p, None),
            L.ec_combine_backward(r, p, p, p, p, p, p, None)]


@pytest.mark.parametrize("change,code", [
    (dict(n=-1), B.EC_ERR_INVALID_ARG), (dict(d=0), B.EC_ERR_INVALID_ARG), (dict(E=0), B.EC_ERR_INVALID_ARG), (dict(K=0), B.EC_ERR_INVALID_ARG),
    (dict(dtype=torch.float32, y_dtype=torch.bfloat16), B.EC_ERR_INVALID_ARG),
    (dict(E=257), B.EC_ERR_UNSUPPORTED), (dict(K=33), B.EC_ERR_UNSUPPORTED), (dict(d=62), B.EC_ERR_UNSUPPORTED), (dict(d=1 << 22), B.EC_ERR_UNSUPPORTED),
    (dict(d=60), B.EC_ERR_UNSUPPORTED), (dict(n=1 << 31, K=1), B.EC_ERR_UNSUPPORTED), (dict(n=1 << 30, K=2), B.EC_ERR_UNSUPPORTED), (dict(n=1 << 62, K=32), B.EC_ERR_UNSUPPORTED),
])
def test_configurations_that_are_refused(change, code):
    a = dict(n=16, d=64, E=8, K=2, dtype=torch.bfloat16, y_dtype=None) | change
    cfg = B.make_sort_config(a["n"], a["d"], a["E"], a["K"], a["dtype"], a["y_dtype"])
    assert _codes(cfg) == [code] * 4
    assert B.ec_sort_workspace_bytes(cfg) == 0


def test_types_outside_their_range():
    for field in ("dtype", "y_dtype"):
        for v in (-1, 2):
            cfg = B.make_sort_config(16, 64, 8, 2)
            setattr(cfg, field, v)
            assert _codes(cfg) == [B.EC_ERR_INVALID_ARG] * 4


def test_pointers():
    cfg = B.make_sort_config(16, 64, 8, 2)
    for p in (None, 4096 + 4):
        assert _codes(cfg, p) == [B.EC_ERR_INVALID_ARG] * 4
    L, r, p = B.lib(), C.byref(cfg), 4096
    assert L.ec_combine(r, p, 4100, p, p, None) == B.EC_ERR_INVALID_ARG
    assert L.ec_sort_tokens(r, p, p, p, p, None, 1 << 18, None) == B.EC_ERR_INVALID_ARG
    assert L.ec_sort_tokens(r, p, p, p, p, 4096 + 16, 1 << 18, None) == B.EC_ERR_INVALID_ARG
    need = B.ec_sort_workspace_bytes(cfg)
    assert 0 < need <= 1 << 18
    assert L.ec_sort_tokens(r, p, p, p, p, 4096, need - 1, None) == B.EC_ERR_WORKSPACE
    assert B.ec_sort_workspace_bytes(B.make_sort_config(1, 64, 256, 32)) <= 1 << 18
    for f in (L.ec_sort_workspace_bytes,):
        assert f(None) == 0


@pytest.mark.parametrize("at", [4097, 4098, 4102])
def test_indices_that_are_not_whole_words(at):
    """choice, offsets, order and place need 4 bytes' alignment, and that they need."""
    cfg, L, p = B.make_sort_config(16, 64, 8, 2), B.lib(), [i << 20 for i in range(1, 8)]
    r = C.byref(cfg)
    for i in range(4):
        args = p[:4]
        args[i] += at - 4096
        assert L.ec_sort_tokens(r, *args, 16 << 20, 1 << 18, None) == B.EC_ERR_INVALID_ARG
    assert L.ec_dispatch(r, p[0], at, p[1], None) == B.EC_ERR_INVALID_ARG
    assert L.ec_combine(r, p[0], None, at, p[1], None) == B.EC_ERR_INVALID_ARG
    assert L.ec_combine_backward(r, p[0], p[1], p[2], at, p[3], p[4], None) == B.EC_ERR_INVALID_ARG
    assert L.ec_mx_dispatch(r, p[0], at, p[1], p[2], None) == B.EC_ERR_INVALID_ARG
    gemm = B.ec_mx_gemm_config(16, 64, 64, 2, B.EC_MX_OUT_BF16, 0, 0)
    assert L.ec_mx_expert_gemm(C.byref(gemm), p[0], p[1], at, p[2], p[3], None, p[4], None, p[5], 256, None) == B.EC_ERR_INVALID_ARG


@pytest.mark.parametrize("one,other", list(itertools.combinations(range(5), 2)))
@pytest.mark.parametrize("shift", [0, 16])
def test_arrays_of_the_plan_that_overlap(one, other, shift):
    """Two of choice, offsets, order, place and the workspace on one another: the kernels index shared memory and `order` by what they
    read back of these, so the call is refused."""
    cfg, L = B.make_sort_config(1 << 16, 64, 8, 2), B.lib()
    args = [(i + 1) << 22 for i in range(5)]
    args[one] = args[other] + shift
    assert L.ec_sort_tokens(C.byref(cfg), *args, 1 << 18, None) == B.EC_ERR_INVALID_ARG


def test_no_tokens():
    """n = 0: arguments that would be empty may be NULL, and nothing but offsets is written (on a GPU)."""
    cfg, L = B.make_sort_config(0, 64, 8, 2), B.lib()
    r = C.byref(cfg)
    assert [L.ec_dispatch(r, None, None, None, None), L.ec_combine(r, None, None, None, None, None),
            L.ec_combine_backward(r, None, None, None, None, None, None, None)] == [B.EC_OK] * 3


def test_no_tokens_and_offsets_on_the_workspace():
    """The plan of no tokens writes its offsets and the status word: not on one another."""
    cfg, L = B.make_sort_config(0, 64, 8, 2), B.lib()
    for ws in (4096, 4096 - 256):
        assert L.ec_sort_tokens(C.byref(cfg), None, 4096 + 16, None, None, ws, 1 << 18, None) == B.EC_ERR_INVALID_ARG


def test_tensors_that_are_not_the_current_device_s():
    cfg = B.make_sort_config(16, 64, 8, 2)
    x, p = torch.zeros(16, 64), torch.zeros(16, 2, dtype=torch.int32)
    for call in (lambda: B.ec_sort_tokens(cfg, p), lambda: B.ec_dispatch(cfg, x, p), lambda: B.ec_combine(cfg, x, None, p),
                 lambda: B.ec_combine_backward(cfg, x, x, x, p)):
        with pytest.raises(B.EcError) as e:
            call()
        assert e.value.code == B.EC_ERR_INVALID_ARG


def test_operands_are_looked_at():
    """Types, shapes and layouts, before an address leaves for the library."""
    dev = -1                                              # what torch says of a host tensor
    i32, x = torch.int32, torch.zeros(16, 64)
    assert B._dense("x", dev, (x, torch.float32, (16, 64))) == [x.data_ptr()]
    for t, dtype, shape in ((x, torch.bfloat16, (16, 64)), (x, torch.float32, (64, 16)), (x.t(), torch.float32, (64, 16)), (x[:, ::2], torch.float32, (16, 32)),
                            (x, i32, (16, 64))):
        with pytest.raises(B.EcError):
            B._dense("x", dev, (t, dtype, shape))
    for t in (x, torch.zeros(16, 64, device="meta")):     # not on device 0
        with pytest.raises(B.EcError):
            B._dense("x", 0, (t, torch.float32, (16, 64)))
