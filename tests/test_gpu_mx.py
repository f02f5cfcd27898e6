"""The 4-bit microscaled format against its definition, bit for bit, and expert products on it against 64 bits."""
import math
import threading

import numpy as np
import pytest
import torch

from paper_2202_09368_b200 import binding as B

import _mx as M
import _sorted as R

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def _np(t):
    return t.detach().cpu().double().numpy() if t.is_floating_point() else t.detach().cpu().numpy()


def _special(rows, cols, dtype, seed):
    """Values of every size, ties, signed zeros, subnormals, the largest number; some rows all zero."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * torch.exp2(torch.randint(-140, 120, (rows, 1), generator=g).float())
    ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, 0.0, -0.0, 0.5, 3.0])
    pick = ties[torch.randint(0, len(ties), (rows, cols), generator=g)] * torch.where(torch.rand(rows, cols, generator=g) < 0.5, -1.0, 1.0)
    at = torch.exp2(torch.randint(-120, 120, (rows, 1), generator=g).float())
    x = torch.where(torch.rand(rows, 1, generator=g) < 0.5, x, pick * at)
    x[rows // 3] = 0
    x[rows // 2] = torch.finfo(dtype).max
    x[2 * rows // 3] = torch.randint(-3, 4, (cols,), generator=g).float() * torch.finfo(dtype).smallest_normal / 8      # subnormal in either type
    return x.to(dtype)


SHAPES = [(1, 8), (3, 32), (5, 40), (7, 64), (9, 72), (33, 128), (6, 136), (7, 256), (64, 264), (9, 512), (33, 520), (130, 1000), (17, 2056), (4, 16384)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_quantised_rows_and_back(rows, cols, dtype):
    x = _special(rows, cols, dtype, rows + cols)
    want = M.encode(_np(x))
    out = B.alloc_mx((rows, cols))
    out.codes.fill_(0xAA); out.scales.fill_(0xAA)
    q = B.ec_mx_quantize(x.cuda(), out=out)
    assert np.array_equal(_np(q.scales), want[1]) and np.array_equal(_np(q.codes), want[0])
    for dt in (F32, BF16):
        back = B.ec_mx_dequantize(q, dtype=dt)
        value = torch.from_numpy(M.decode(*want, cols))
        assert torch.equal(back.cpu(), value.to(dt)) and torch.equal(value.to(dt).double(), value)
        assert torch.equal(torch.signbit(back.cpu()), torch.signbit(value))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("batches,rows,cols", [(1, 8, 1), (1, 8, 33), (2, 64, 64), (3, 72, 1000), (2, 200, 256), (1, 136, 31), (1, 4104, 40), (2, 1000, 520), (5, 16, 2050)])
def test_quantised_from_transposed_storage(batches, rows, cols, dtype):
    x = torch.stack([_special(rows, cols, dtype, rows + cols + b) for b in range(batches)])
    want = [M.encode(_np(v)) for v in x]
    out = B.alloc_mx((batches, rows, cols))
    out.codes.fill_(0xAA); out.scales.fill_(0xAA)
    q = B.ec_mx_quantize(x.transpose(1, 2).contiguous().cuda(), transposed=True, out=out)
    for b in range(batches):
        assert np.array_equal(_np(q.scales[b]), want[b][1]) and np.array_equal(_np(q.codes[b]), want[b][0])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_infinities_and_nan_take_their_block(dtype):
    x = torch.randn(40, 520, generator=torch.Generator().manual_seed(3)).to(dtype)
    x[3, 7], x[5, 64], x[5, 519], x[39, 31] = float("nan"), float("inf"), -float("inf"), -float("nan")
    want = M.encode(_np(x))
    for q in (B.ec_mx_quantize(x.cuda()), B.ec_mx_quantize(x.t().contiguous().cuda(), transposed=True)):
        assert np.array_equal(_np(q.scales), want[1]) and np.array_equal(_np(q.codes), want[0])
        back = B.ec_mx_dequantize(q, dtype=dtype).cpu()
        nan = torch.zeros(40, 520, dtype=torch.bool)
        for r, c in ((3, 0), (5, 64), (5, 512), (39, 0)):
            nan[r, c:c + 32] = True
        assert torch.equal(torch.isnan(back), nan)


def test_no_rows():
    for shape in ((0, 64), (0, 8, 64), (3, 0, 64)):
        q = B.ec_mx_quantize(torch.zeros(shape, dtype=BF16, device="cuda"))
        assert q.codes.shape[:-1] == shape[:-1] and B.ec_mx_dequantize(q).shape == shape
    W = B.ec_mx_quantize(torch.zeros(2, 8, 64, dtype=BF16, device="cuda"))
    assert B.ec_mx_expert_gemm(B.ec_mx_quantize(torch.zeros(0, 64, device="cuda")), W, torch.zeros(3, dtype=torch.int32, device="cuda")).shape == (0, 8)


@pytest.mark.parametrize("dtype,n,K,E,d", [(BF16, 1, 1, 4, 8), (BF16, 37, 3, 10, 1000), (F32, 50, 2, 4, 200), (BF16, 21, 2, 4, 120), (F32, 64, 8, 16, 36), (F32, 5, 32, 256, 520), (BF16, 300, 2, 8, 4096)])
def test_dispatch_of_quantised_rows(dtype, n, K, E, d):
    """The bits of the quantised rows, at the places of a plan with holes; the other rows as they were."""
    g = torch.Generator().manual_seed(9)
    choice = torch.randint(-2, E + 1, (n, K), generator=g, dtype=torch.int32)
    cfg = B.make_sort_config(n, d, E, K, dtype)
    plan = B.ec_sort_tokens(cfg, choice.cuda())
    X = torch.randn(n, d, generator=g).to(dtype)
    out = B.alloc_mx((n * K, d))
    out.codes.fill_(0xAA); out.scales.fill_(0xAA)
    q = B.ec_mx_dispatch(cfg, X.cuda(), plan.place, out=out)
    codes, scales = M.encode(_np(X))
    offsets, order, _ = R.plan(choice.numpy(), E)
    m = int(offsets[-1])
    assert np.array_equal(_np(q.codes)[:m], codes[order // K]) and np.array_equal(_np(q.scales)[:m], scales[order // K])
    assert (_np(q.codes)[m:] == 0xAA).all() and (_np(q.scales)[m:] == 0xAA).all()


def _groups(rows, E, kind, seed):
    g = np.random.default_rng(seed)
    if kind == "even":
        return np.array([i * rows // E for i in range(E + 1)])
    if kind == "one":                                     # a single expert holds them all
        at = g.integers(0, E)
        return np.array([0] * (at + 1) + [rows] * (E - at))
    if kind == "tail":                                    # starts behind row 0 and ends before the last
        return np.sort(g.integers(min(rows, 1), max(rows - 1, 1) + 0, E + 1))
    if kind == "none":
        return np.full(E + 1, rows // 2)
    return np.concatenate([[0], np.sort(g.integers(0, rows + 1, E - 1)), [rows]])       # any lengths, some none


def _case(rows, N, K, E, seed, spread=3):
    g = torch.Generator().manual_seed(seed)
    a = torch.randn(rows, K, generator=g) * torch.exp2(torch.randint(-spread, spread + 1, (rows, 1), generator=g).float())
    w = torch.randn(E, N, K, generator=g) * K ** -0.5
    A, W = B.ec_mx_quantize(a.cuda()), B.ec_mx_quantize(w.cuda())
    av = M.decode(_np(A.codes), _np(A.scales), K)
    wv = np.stack([M.decode(_np(W.codes[e]), _np(W.scales[e]), K) for e in range(E)])
    return A, W, av, wv


PRODUCTS = [                                              # rows, N, K, E, groups
    (1, 8, 32, 1, "even"), (1, 128, 256, 4, "one"), (2, 136, 64, 8, "any"), (5, 128, 8, 2, "even"), (8, 1000, 512, 64, "any"),
    (31, 128, 544, 1, "even"), (32, 256, 1024, 1, "even"), (33, 128, 288, 1, "even"), (64, 264, 320, 1, "even"), (65, 128, 96, 1, "even"),
    (129, 128, 1000, 1, "even"), (193, 136, 776, 1, "even"), (192, 128, 4096, 1, "even"), (400, 40, 520, 3, "any"), (700, 384, 264, 5, "any"),
    (777, 520, 1032, 7, "tail"), (300, 72, 40, 256, "any"), (300, 128, 128, 4, "none"), (1500, 128, 64, 2, "one"), (1024, 1096, 512, 16, "even"),
    (2000, 256, 2056, 9, "any"), (4000, 1096, 4104, 2, "any"), (2900, 2000, 5000, 3, "tail"),
]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,N,K,E,kind", PRODUCTS)
def test_product(rows, N, K, E, kind, dtype):
    A, W, a, w = _case(rows, N, K, E, rows + N + K)
    offsets = _groups(rows, E, kind, rows)
    out = torch.full((rows, N), 7.0, dtype=dtype, device="cuda")
    ws = torch.empty(B.EC_MX_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
    B.ec_mx_expert_gemm(A, W, torch.from_numpy(offsets).int().cuda(), out=out, ws=ws)
    assert B.ec_read_status(ws) == B.EC_OK
    z, size = M.product(a, w, offsets)
    M.check_product(_np(out), z, size, K, dtype)
    assert (_np(out)[np.isnan(z)] == 7.0).all()           # rows of no expert: as they were


@pytest.mark.parametrize("rows,N,K,E", [(3, 128, 4096, 2), (40, 136, 4096, 1), (90, 256, 2048, 1), (600, 384, 4096, 2), (2, 264, 4096, 8), (17, 72, 3080, 4), (1, 1000, 1096, 1)])
def test_sums_that_fp32_holds_are_exact(rows, N, K, E):
    """Scales of 1/2 to 2: every product is a multiple of 2^-4 below 144, a sum of 4096 below 2^20 in steps of 2^-4: 24 bits, so any order of
    exact additions gives the same value."""
    g = torch.Generator().manual_seed(rows)
    A, W = B.alloc_mx((rows, K)), B.alloc_mx((E, N, K))
    for q in (A, W):
        q.codes.copy_(torch.randint(0, 256, q.codes.shape, generator=g, dtype=torch.uint8))
        q.codes[..., K // 2:] = 0                         # what the format wants behind the last column
        q.scales.copy_(torch.randint(126, 129, q.scales.shape, generator=g, dtype=torch.uint8))
    offsets = _groups(rows, E, "even", 0)
    out = B.ec_mx_expert_gemm(A, W, torch.from_numpy(offsets).int().cuda(), dtype=F32)
    a = M.decode(_np(A.codes), _np(A.scales), K)
    w = np.stack([M.decode(_np(W.codes[e]), _np(W.scales[e]), K) for e in range(E)])
    assert np.array_equal(_np(out), M.product(a, w, offsets)[0])


@pytest.mark.parametrize("rows,N,K,E", [(9, 136, 520, 4), (100, 256, 128, 1), (200, 1000, 96, 1), (500, 72, 1000, 2), (4000, 1096, 8200, 2)])
@pytest.mark.parametrize("act", ["none", "erf", "tanh"])
def test_bias_activation_and_each_result_type(rows, N, K, E, act):
    A, W, a, w = _case(rows, N, K, E, N, spread=1)
    offsets = _groups(rows, E, "any", 4)
    off = torch.from_numpy(offsets).int().cuda()
    g = torch.Generator().manual_seed(2)
    for bias_dtype in (F32, BF16, None):
        bias = None if bias_dtype is None else torch.randn(E, N, generator=g).to(bias_dtype)
        z, size = M.product(a, w, offsets, None if bias is None else _np(bias))
        on = None if bias is None else bias.cuda()
        full = B.ec_mx_expert_gemm(A, W, off, bias=on, act=act, dtype=F32)
        M.check_product(_np(full), z, size, K, F32, act)
        half = B.ec_mx_expert_gemm(A, W, off, bias=on, act=act, dtype=BF16)
        assert torch.equal(half, full.to(BF16))           # the same sums, rounded once
        out = B.alloc_mx((rows, N))
        out.codes.fill_(0xAA); out.scales.fill_(0xAA)
        B.ec_mx_expert_gemm(A, W, off, bias=on, act=act, out=out)
        codes, scales = M.encode(_np(full))               # the same sums, quantised
        blocks = -(-N // 32)
        assert np.array_equal(_np(out.scales)[:, :blocks], scales[:, :blocks]) and np.array_equal(_np(out.codes), codes)
        assert (_np(out.scales)[:, blocks:] == 0xAA).all()


@pytest.mark.parametrize("rows", [1, 100])
def test_gelu_over_its_range(rows):
    """Zero rows, so that z is the bias.  The erf form is within 2.6e-7 |z| of the definition and never of the other sign, tails among
    them; NaN stays NaN."""
    N, K = 40000, 32
    g = torch.Generator().manual_seed(3)
    z = torch.cat([torch.linspace(-8, 8, 20000), torch.linspace(-6, -4, 15000), torch.randn(4984, generator=g) * 20,
                   torch.tensor([0.0, -0.0, 1e-38, -1e-38, 1e-45, -5.374011538, -5.3740120, -5.3740110, 5.374, 1e30, -1e30, float("nan"), 0.5, -0.5, 4.0, -4.0])])
    A, W = B.ec_mx_quantize(torch.zeros(rows, K, device="cuda")), B.ec_mx_quantize(torch.zeros(1, N, K, device="cuda"))
    off = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    got = B.ec_mx_expert_gemm(A, W, off, bias=z[None].cuda(), act="erf", dtype=F32)
    assert torch.equal(got.nan_to_num(99.0), got[:1].nan_to_num(99.0).expand(rows, N))
    h, z = _np(got[0]), z.double().numpy()
    nan = np.isnan(z)
    assert np.array_equal(np.isnan(h), nan)
    h, z = h[~nan], z[~nan]
    want = 0.5 * z * np.vectorize(math.erfc, otypes=[float])(-z * math.sqrt(0.5))
    assert (h * np.sign(z) >= 0).all(), h[(h * np.sign(z) < 0)]
    assert (np.abs(h - want) <= 2.6e-7 * np.abs(z) + 2.0 ** -24 * np.abs(want) + 2.0 ** -149).all()
    assert (np.abs(h) <= np.abs(z)).all()


@pytest.mark.parametrize("rows", [20, 60, 100, 300])
def test_nan_and_what_lies_outside(rows):
    """A NaN block reaches its own row or column and no other; scale bytes behind the contraction's end and rows of no expert are not
    read, whatever they hold."""
    N, K, E = 200, 200, 1
    A, W, a, w = _case(rows, N, K, E, 1, spread=0)
    offsets = torch.tensor([2, rows - 3], dtype=torch.int32, device="cuda")
    want = B.ec_mx_expert_gemm(A, W, offsets, dtype=F32, out=torch.full((rows, N), 7.0, device="cuda"))
    A.scales[:, 7:] = 255; W.scales[:, :, 7:] = 255
    A.scales[:2] = 255; A.scales[rows - 3:] = 255
    got = B.ec_mx_expert_gemm(A, W, offsets, dtype=F32, out=torch.full((rows, N), 7.0, device="cuda"))
    assert torch.equal(got, want)
    A.scales[5, 3] = 255; W.scales[0, 131, 6] = 255
    got = B.ec_mx_expert_gemm(A, W, offsets, dtype=F32, out=torch.full((rows, N), 7.0, device="cuda"))
    nan = torch.zeros(rows, N, dtype=torch.bool, device="cuda")
    nan[5] = True
    nan[2:rows - 3, 131] = True
    assert torch.equal(torch.isnan(got), nan) and torch.equal(got[~nan], want[~nan])
    q = B.ec_mx_expert_gemm(A, W, offsets, out=B.alloc_mx((rows, N)))
    assert (q.scales[5, :7] == 255).all() and (q.scales[2:rows - 3, 4] == 255).all() and (q.codes[5] == 0).all()
    assert (q.scales[2:5, :4] != 255).all() and (q.scales[6:rows - 3, 5:7] != 255).all()


@pytest.mark.parametrize("rows", [3, 40, 100, 250])
def test_the_ends_of_the_range(rows):
    """Scales at both ends: sums beyond fp32 are infinities of their sign, those below its normal range are off by at most 2^-126 per
    product, and zeros times the largest scale stay zeros."""
    K, N = 96, 136
    g = torch.Generator().manual_seed(rows)
    A, W = B.alloc_mx((rows, K)), B.alloc_mx((1, N, K))
    for q in (A, W):
        q.codes.copy_(torch.randint(0, 256, q.codes.shape, generator=g, dtype=torch.uint8))
    W.codes &= 0x77                                       # no negative weights
    A.codes[0] = 0x11; A.codes[1] = 0x99; W.codes[0, 0] = 0x22
    off = torch.tensor([0, rows], dtype=torch.int32, device="cuda")

    def run(a, w):
        A.scales.fill_(a); W.scales.fill_(w)
        return _np(B.ec_mx_expert_gemm(A, W, off, dtype=F32))

    big = run(254, 254)
    assert big[0, 0] == np.inf and big[1, 0] == -np.inf
    plain = run(127, 127)
    assert plain[0, 0] == K / 2 and plain[1, 0] == -K / 2
    for a, w in ((60, 70), (1, 126), (0, 127), (0, 100), (0, 0), (1, 60)):
        assert (np.abs(run(a, w) - np.ldexp(plain, a + w - 254)) <= K * 2.0 ** -126).all(), (a, w)
    assert np.array_equal(run(150, 140), np.ldexp(plain, 36)) and np.array_equal(run(10, 244), plain)
    A.codes.fill_(0x08)                                   # zeros of either sign
    assert (run(254, 254) == 0).all()


def test_offsets_are_cut_to_the_rows():
    """Offsets are the caller's memory: below 0 counts as 0, beyond the rows as their number, a decrease as an empty group."""
    rows, N, K, E = 150, 136, 64, 6
    A, W, a, w = _case(rows, N, K, E, 8)
    bad = [-2 ** 31, 20, 10, 60, 2 ** 31 - 1, 40, 2 ** 31 - 1]
    out = B.ec_mx_expert_gemm(A, W, torch.tensor(bad, dtype=torch.int32, device="cuda"), dtype=F32, out=torch.full((rows, N), 7.0, device="cuda"))
    lo = np.clip(bad, 0, rows)
    whole = [(0, 0, 20), (2, 10, 60), (3, 60, 150), (5, 40, 150)]         # overlapping groups: rows 10-19 and 60-149 are written twice
    got = _np(out)
    for r in range(rows):
        fits = [e for e, x, y in whole if x <= r < y]
        ok = np.zeros(N, bool)                            # tiles of either group write such a row, each its columns
        for e in fits:
            z, size = a[r] @ w[e].T, np.abs(a[r]) @ np.abs(w[e]).T
            ok |= np.abs(got[r] - z) <= (K + 2) * 2.0 ** -23 * size + 2.0 ** -24 * np.abs(z) + 1e-30
        assert ok.all(), r
    assert lo[0] == 0 and lo[-1] == rows


@pytest.mark.parametrize("rows,N,K,E", [(150, 136, 64, 6), (3, 72, 2048, 40), (700, 264, 96, 33), (900, 384, 512, 256), (2000, 512, 72, 5)])
def test_groups_never_share_rows(rows, N, K, E):
    """Offsets that fall count as the largest before them: the bits, in every row and every time, of a call with the rising offsets; rows of
    no expert and what lies around C as they were."""
    A, W, _, _ = _case(rows, N, K, E, 21)
    g = np.random.default_rng(E)
    tries = [np.array([0] + [rows, 0] * E)[: E + 1], np.array([rows, 0] * E)[: E + 1], np.array([5, -3] + [rows // 2, 1, 2 ** 31 - 1, -2 ** 31] * E)[: E + 1]]
    tries += [g.integers(-5, rows + 5, E + 1) for _ in range(5)]
    for offsets in tries:
        rising = np.maximum.accumulate(np.clip(offsets, 0, rows))

        def run(o):
            around = torch.full((rows + 2, N), 7.0, device="cuda")
            B.ec_mx_expert_gemm(A, W, torch.from_numpy(o).int().cuda(), dtype=F32, out=around[1:-1])
            return around

        want, got = run(rising), run(offsets)
        assert torch.equal(got, want)
        assert (got[: 1 + rising[0]] == 7.0).all() and (got[1 + rising[-1]:] == 7.0).all()
        assert rising[0] == rising[-1] or not (got[1 + rising[0]: 1 + rising[-1]] == 7.0).all(1).any()


def _layer(n, K, E, d, f, act, seed):
    g = torch.Generator().manual_seed(seed)
    data = dict(choice=torch.randint(-1, E, (n, K), generator=g, dtype=torch.int32).cuda(), X=torch.randn(n, d, generator=g).to(BF16).cuda(),
                weights=torch.rand(n, K, generator=g).cuda())
    W1 = B.ec_mx_quantize((torch.randn(E, d, f, generator=g) * d ** -0.5).cuda(), transposed=True)      # W1's storage
    W2 = B.ec_mx_quantize((torch.randn(E, d, f, generator=g) * f ** -0.5).cuda())                       # W2 [E, d, d'] contracts its rows
    b1, b2 = torch.randn(E, f, generator=g).to(BF16).cuda(), torch.randn(E, d, generator=g).to(BF16).cuda()
    i32 = dict(dtype=torch.int32, device="cuda")
    cfg = B.make_sort_config(n, d, E, K, BF16, F32)
    bufs = dict(plan=B.Sorted(torch.zeros(E + 1, **i32), torch.zeros(n * K, **i32), torch.zeros(n, K, **i32)), rows=B.alloc_mx((n * K, d)),
                H=B.alloc_mx((n * K, f)), Y=torch.zeros(n * K, d, device="cuda"), X_out=torch.zeros(n, d, dtype=BF16, device="cuda"),
                ws=torch.empty(1 << 18, dtype=torch.uint8, device="cuda"))

    def step():
        plan = B.ec_sort_tokens(cfg, data["choice"], out=bufs["plan"], ws=bufs["ws"])
        B.ec_mx_dispatch(cfg, data["X"], plan.place, out=bufs["rows"])
        B.ec_mx_expert_gemm(bufs["rows"], W1, plan.offsets, bias=b1, act=act, out=bufs["H"], ws=bufs["ws"])
        B.ec_mx_expert_gemm(bufs["H"], W2, plan.offsets, bias=b2, out=bufs["Y"], ws=bufs["ws"])
        return B.ec_combine(cfg, bufs["Y"], data["weights"], plan.place, X_out=bufs["X_out"])

    return data, (W1, W2, b1, b2), bufs, step


@pytest.mark.parametrize("n,K,E,d,f,act", [(1, 2, 8, 64, 256, "erf"), (5, 1, 4, 264, 1000, "tanh"), (97, 3, 6, 520, 1096, "erf"), (700, 2, 3, 256, 512, "tanh")])
def test_a_layer_from_tokens_to_tokens(n, K, E, d, f, act):
    """Sort, quantise on the way, product with GeLU to 4 bits, product, combine: each step against 64 bits of what it was given."""
    data, (W1, W2, b1, b2), bufs, step = _layer(n, K, E, d, f, act, n)
    out = step()
    offsets, order, place = R.plan(data["choice"].cpu().numpy(), E)
    m = int(offsets[-1])
    codes, scales = M.encode(_np(data["X"]))
    assert np.array_equal(_np(bufs["rows"].codes)[:m], codes[order // K]) and np.array_equal(_np(bufs["rows"].scales)[:m], scales[order // K])
    wv = [np.stack([M.decode(_np(q.codes[e]), _np(q.scales[e]), q.cols) for e in range(E)]) for q in (W1, W2)]
    rows = M.decode(codes, scales, d)[order // K]
    z, size = M.product(rows, wv[0], offsets, _np(b1))
    H = B.ec_mx_expert_gemm(bufs["rows"], W1, bufs["plan"].offsets, bias=b1, act=act, dtype=F32)
    M.check_product(_np(H)[:m], z, size, d, F32, act)
    hq = M.encode(_np(H)[:m])
    assert np.array_equal(_np(bufs["H"].codes)[:m], hq[0]) and np.array_equal(_np(bufs["H"].scales)[:m, :-(-f // 32)], hq[1][:, :-(-f // 32)])
    z, size = M.product(M.decode(*hq, f), wv[1], offsets, _np(b2))
    M.check_product(_np(bufs["Y"])[:m], z, size, f, F32)
    want, total = R.combine(bufs["Y"], data["weights"], place)
    R.check_sum(out, want, total, K, BF16)


def test_layer_captured_and_from_several_threads():
    """Captured and replayed on other tokens, and beside other calls on other streams: the bits of a call alone."""
    data, _, bufs, step = _layer(300, 2, 8, 512, 1024, "erf", 1)
    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    other = _layer(300, 2, 8, 512, 1024, "erf", 2)[0]
    for k in data:
        data[k].copy_(other[k])
    bufs["X_out"].zero_()
    graph.replay()
    torch.cuda.synchronize()
    got = bufs["X_out"].clone()
    assert torch.equal(step(), got)
    jobs = []
    for i, s in enumerate([(4, 2, 16, 256, 512, "erf"), (500, 2, 4, 512, 264, "tanh"), (60, 4, 8, 1024, 2048, "erf"), (2000, 1, 2, 64, 128, "none")]):
        _, _, bufs, step = _layer(*s, 20 + i)
        jobs.append((step, step().clone()))
    torch.cuda.synchronize()
    start, failed = threading.Barrier(len(jobs)), []

    def work(step, want):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                start.wait()
                for _ in range(100):
                    out = step()
                assert torch.equal(out, want)
        except BaseException as e:
            failed.append(e)

    threads = [threading.Thread(target=work, args=j) for j in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed, failed


def test_expert_choice_slots_through_the_product():
    """The slots of ec_route are groups of k rows: the same product as ec_expert_gemm's, on the values the 4-bit operands stand for."""
    n, d, f, E = 512, 128, 256, 4
    cfg = B.make_config(n, d, f, E, 2.0, BF16)
    g = torch.Generator(device="cuda").manual_seed(3)
    X, Wg = (torch.empty(s, device="cuda").normal_(generator=g).to(BF16) for s in ((n, d), (d, E)))
    W1 = (torch.empty(E, d, f, device="cuda").normal_(generator=g) * d ** -0.5).to(BF16)
    r = B.ec_route(cfg, X, Wg)
    k = B.slots_per_expert(cfg)
    X_in = B.ec_shuffle(cfg, X, r.I).view(E * k, d)
    A, W = B.ec_mx_quantize(X_in), B.ec_mx_quantize(W1, transposed=True)
    offsets = torch.arange(E + 1, dtype=torch.int32, device="cuda") * k
    got = B.ec_mx_expert_gemm(A, W, offsets, dtype=BF16).view(E, k, f)
    values = B.ec_mx_dequantize(A).view(E, k, d), B.ec_mx_dequantize(W).transpose(1, 2).contiguous()
    want = B.ec_expert_gemm(cfg, B.EC_GEMM_XW1, *values)
    size = np.abs(_np(values[0])) @ np.abs(_np(values[1]))
    assert (np.abs(_np(got) - _np(want)) <= 2 * (d + 2) * 2.0 ** -23 * size + 2 * R.HALF_STEP[BF16] * np.abs(_np(want)) + 1e-30).all()


@pytest.mark.parametrize("rows,E", [(1, 1), (2, 8), (5, 2), (20, 1), (37, 4), (3, 64)])
@pytest.mark.parametrize("N,K", [(8, 1032), (136, 2048), (264, 5000), (1096, 8200)])
def test_few_rows_along_a_long_contraction(rows, E, N, K):
    """Few tiles: several CTAs share each, at any length of the contraction, also one that their stretches do not divide.  Every result type."""
    A, W, a, w = _case(rows, N, K, E, rows + N)
    offsets = _groups(rows, E, "any", 3)
    off = torch.from_numpy(offsets).int().cuda()
    bias = torch.randn(E, N, generator=torch.Generator().manual_seed(1)).cuda()
    z, size = M.product(a, w, offsets, _np(bias))
    ws = torch.empty(B.EC_MX_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
    full = B.ec_mx_expert_gemm(A, W, off, bias=bias, act="tanh", dtype=F32, ws=ws)
    assert B.ec_read_status(ws) == B.EC_OK
    M.check_product(_np(full), z, size, K, F32, "tanh")
    for _ in range(20):                                   # the order of the sums does not depend on the CTAs' timing
        assert torch.equal(B.ec_mx_expert_gemm(A, W, off, bias=bias, act="tanh", dtype=F32), full)
    assert torch.equal(B.ec_mx_expert_gemm(A, W, off, bias=bias, act="tanh", dtype=BF16), full.to(BF16))
    q = B.ec_mx_expert_gemm(A, W, off, bias=bias, act="tanh", out=B.alloc_mx((rows, N)))
    codes, scales = M.encode(_np(full))
    assert np.array_equal(_np(q.codes), codes) and np.array_equal(_np(q.scales)[:, :-(-N // 32)], scales[:, :-(-N // 32)])


def test_weights_beyond_the_range_of_32_bit_offsets():
    """Codes of more than 2^32 bytes: the last expert's product is that of its own weights."""
    E, N, K, rows = 72, 16384, 8192, 72
    W = B.alloc_mx((E, N, K))
    assert W.codes.numel() > 2 ** 32
    W.codes.fill_(0x22); W.scales.fill_(127)              # ones
    W.scales[E - 1] = 130                                 # eights
    A = B.ec_mx_quantize(torch.ones(rows, K, device="cuda"))
    out = B.ec_mx_expert_gemm(A, W, torch.arange(E + 1, dtype=torch.int32, device="cuda"), dtype=F32)
    assert (out[:E - 1] == K).all() and (out[E - 1] == 8 * K).all()
    q = B.ec_mx_quantize(torch.ones(1, 32, device="cuda"))
    assert q.codes[0, 0] == 0x66 and q.scales[0, 0] == 125        # 4 x 2^-2
