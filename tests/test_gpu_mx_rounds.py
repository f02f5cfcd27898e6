"""Expert products in which every CTA takes several tiles, in each form of the kernel: the accumulators, the stages and the scales are used
again and again, over uneven and empty groups, and each sum is exact."""
import numpy as np
import pytest
import torch

from paper_2202_09368_b200 import binding as B

import _mx as M

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def _values(q, K):
    """What codes and scales stand for, in 64 bits on the device: scales here are those of normal numbers."""
    levels = torch.tensor(list(M.LEVELS) + [-v for v in M.LEVELS], dtype=torch.float64, device="cuda")
    v = levels[torch.stack((q.codes & 15, q.codes >> 4), -1).flatten(-2).int()].unflatten(-1, (-1, 32))
    return (v * torch.exp2(q.scales[..., : v.shape[-2]].double() - 127)[..., None]).flatten(-2)[..., :K]


def _random(shape, K, g):
    """Scales of 1/2 and 1: a product is a multiple of 2^-4 not above 36, a sum of 8200 below 2^19: 23 bits, so any order of exact additions
    gives the same value."""
    q = B.alloc_mx(shape + (K,))
    q.codes.random_(0, 256, generator=g)
    q.codes[..., K // 2:] = 0                             # what the format wants behind the last column
    q.scales.random_(126, 128, generator=g)
    return q


def _offsets(rows, E, seed):
    """Groups of very different lengths, some empty, between a first and a last row of no expert."""
    g = np.random.default_rng(seed)
    share = np.exp(1.5 * g.standard_normal(E)) * (g.random(E) < 0.85)
    share[0] += 1e-3
    cut = np.floor(np.cumsum(share) / share.sum() * (rows - 4)).astype(np.int64)
    return np.concatenate([[1], 1 + cut])


CASES = [                                                 # rows, N, K, E: by the rows of a tile
    (200, 640, 1096, 100, 32), (500, 1024, 264, 250, 32), (256, 4096, 776, 16, 64), (1200, 1096, 2056, 64, 64), (480, 8192, 2056, 8, 128),
    (2000, 4072, 1000, 30, 128), (2400, 4096, 520, 8, 192), (3000, 6008, 96, 5, 192), (4000, 8192, 4104, 8, 256), (6000, 4096, 8200, 3, 256),
]


@pytest.mark.parametrize("rows,N,K,E,kind", CASES)
def test_several_tiles_to_a_cta(rows, N, K, E, kind):
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    g = torch.Generator(device="cuda").manual_seed(rows)
    A, W = _random((rows,), K, g), _random((E, N), K, g)
    offsets = _offsets(rows, E, rows + E)
    row_tile, columns = M.form(rows, N, K, E, sms)
    assert (row_tile if columns == 128 else 256) == kind
    assert M.tiles(offsets, N, row_tile, columns) > 2 * sms           # so that some CTA takes three
    off = torch.from_numpy(offsets).int().cuda()
    ws = torch.empty(B.EC_MX_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
    want = torch.full((rows, N), 7.0, device="cuda")
    for e in range(E):
        r = slice(int(offsets[e]), int(offsets[e + 1]))
        want[r] = (_values(B.Mx(A.codes[r], A.scales[r], K), K) @ _values(B.Mx(W.codes[e], W.scales[e], K), K).T).float()
    for _ in range(3):
        out = torch.full((rows, N), 7.0, device="cuda")
        B.ec_mx_expert_gemm(A, W, off, out=out, ws=ws)
        assert B.ec_read_status(ws) == B.EC_OK and torch.equal(out, want)
    half = B.ec_mx_expert_gemm(A, W, off, out=torch.full((rows, N), 7.0, dtype=BF16, device="cuda"))
    assert torch.equal(half, want.to(BF16))
    inside = slice(int(offsets[0]), int(offsets[-1]))
    for act in ("none", "erf"):                           # the epilogues that take longest: the same sums, activated and quantised
        full = B.ec_mx_expert_gemm(A, W, off, act=act, dtype=F32)
        q = B.alloc_mx((rows, N))
        q.codes.fill_(0xAA); q.scales.fill_(0xAA)
        B.ec_mx_expert_gemm(A, W, off, act=act, out=q, ws=ws)
        assert B.ec_read_status(ws) == B.EC_OK
        same = B.ec_mx_quantize(full)
        blocks = -(-N // 32)
        assert torch.equal(q.codes[inside], same.codes[inside]) and torch.equal(q.scales[inside, :blocks], same.scales[inside, :blocks])
        for r in (slice(0, inside.start), slice(inside.stop, rows)):
            assert (q.codes[r] == 0xAA).all() and (q.scales[r] == 0xAA).all()


@pytest.mark.parametrize("rows,N,K,E", [(256, 4096, 4104, 16), (480, 8192, 2056, 8), (2400, 4096, 520, 8), (4000, 8192, 4104, 8)])
def test_the_same_bits_every_time(rows, N, K, E):
    """Back to back, where a barrier passes a phase every few hundred cycles: no lane of the issuing warps misses one (it would wait for two
    seconds and give up), and no result differs."""
    g = torch.Generator(device="cuda").manual_seed(N)
    A, W = _random((rows,), K, g), _random((E, N), K, g)
    off = torch.from_numpy(_offsets(rows, E, 5)).int().cuda()
    ws = torch.empty(B.EC_MX_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
    want = B.ec_mx_expert_gemm(A, W, off, out=torch.zeros(rows, N, device="cuda"), ws=ws)
    assert B.ec_read_status(ws) == B.EC_OK
    out = torch.zeros(rows, N, device="cuda")
    wrong = torch.zeros((), dtype=torch.bool, device="cuda")
    codes = torch.zeros((), dtype=torch.int32, device="cuda")
    for _ in range(100):
        B.ec_mx_expert_gemm(A, W, off, out=out, ws=ws)
        codes |= ws[:4].view(torch.int32)[0]              # the status word of each call
        wrong |= (out != want).any()
    assert not wrong and codes == 0
