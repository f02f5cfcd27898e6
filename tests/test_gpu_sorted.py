"""Tokens sorted by expert and back against their definition in 64 bits: the plan bit for bit, the rows moved bit for bit, the
weighted sums and their gradients within what fp32 sums and one rounding allow."""
import threading

import numpy as np
import pytest
import torch

from paper_2202_09368_b200 import binding as B

import _sorted as R

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def _choice(n, K, E, seed, kind="random"):
    g = torch.Generator().manual_seed(seed)
    if kind == "distinct":
        return torch.rand(n, E, generator=g).topk(K, dim=1)[1].int()
    if kind == "one":                                    # everybody names the same expert, several times
        return torch.full((n, K), E - 1, dtype=torch.int32)
    c = torch.randint(0, E, (n, K), generator=g, dtype=torch.int32)
    if kind == "holes":
        bad = torch.tensor([-1, -7, E, E + 5, 2 ** 31 - 1, -2 ** 31], dtype=torch.int64)
        pick = bad[torch.randint(0, len(bad), (n, K), generator=g)]
        c = torch.where(torch.rand(n, K, generator=g) < 0.4, pick, c.long()).int()
    if kind == "none":
        c = torch.full((n, K), -1, dtype=torch.int32)
    return c


def _check_plan(got, choice, E):
    offsets, order, place = R.plan(choice.numpy(), E)
    assert np.array_equal(got.offsets.cpu().numpy(), offsets)
    assert np.array_equal(got.place.cpu().numpy(), place)
    m = int(offsets[-1])
    assert np.array_equal(got.order.cpu().numpy()[:m], order)
    assert (got.order.cpu().numpy()[m:] == -77).all()                  # behind the last expert: as they were


@pytest.mark.parametrize("n,K,E,kind", [
    (0, 2, 8, "random"), (1, 1, 1, "random"), (1, 2, 64, "distinct"), (1, 32, 256, "distinct"), (2, 3, 5, "holes"), (31, 1, 4, "random"),
    (33, 1, 4, "random"), (255, 4, 256, "holes"), (1000, 3, 10, "holes"), (1024, 1, 64, "random"), (1025, 1, 64, "random"), (777, 5, 7, "one"), (500, 2, 16, "none"),
    (8192, 2, 32, "distinct"), (16384, 1, 64, "random"), (16385, 1, 64, "random"), (6079, 3, 10, "holes"), (16384, 2, 64, "distinct"), (65536, 8, 256, "distinct"),
    (4096, 1, 16, "random"), (4097, 1, 16, "holes"), (2048, 1, 16, "holes"), (2049, 1, 200, "holes"), (24576, 1, 64, "random"), (24577, 1, 64, "holes"), (2731, 3, 256, "holes"), (5000, 1, 4, "one"), (32768, 2, 128, "holes"), (65537, 1, 64, "random"), (60000, 1, 1, "one"),
    (100003, 7, 33, "holes"), (151552, 1, 256, "random"), (151553, 1, 256, "one"), (540001, 8, 200, "holes"), (30000, 2, 3, "none"),
])
def test_plan(n, K, E, kind):
    choice = _choice(n, K, E, 3, kind)
    cfg = B.make_sort_config(n, 64, E, K)
    out = B.Sorted(torch.full((E + 1,), -77, dtype=torch.int32, device="cuda"), torch.full((n * K,), -77, dtype=torch.int32, device="cuda"),
                   torch.full((n, K), -77, dtype=torch.int32, device="cuda"))
    _check_plan(B.ec_sort_tokens(cfg, choice.cuda(), out=out), choice, E)


@pytest.mark.parametrize("E", [3, 33, 256])
def test_plans_of_a_cluster_whose_warps_end_unevenly(E):
    """Totals that end inside a warp's round, with choices of no expert: lanes of a warp part before the cluster's last barrier."""
    for total in (2049, 2063, 2080, 4097, 5003, 8191, 8193, 9999, 16383, 20011, 24575):
        choice = _choice(total, 1, E, total, "holes")
        cfg = B.make_sort_config(total, 64, E, 1)
        on = choice.cuda()
        for _ in range(5):
            out = B.Sorted(*(torch.full(s, -77, dtype=torch.int32, device="cuda") for s in ((E + 1,), (total,), (total, 1))))
            _check_plan(B.ec_sort_tokens(cfg, on, out=out), choice, E)


@pytest.mark.parametrize("n,E", [(7, 8), (5000, 8), (40000, 8), (30000, 256)])
def test_status_of_a_plan(n, E):
    """The plan's scratch begins with the status word, as every workspace does: nothing of its own lands there, whatever the memory held."""
    cfg = B.make_sort_config(n, 64, E, 1)
    choice = torch.full((n, 1), 5, dtype=torch.int32)
    choice[: n // 2] = 0
    for fill in (0, 0xA5, 5):
        ws = torch.full((B.ec_sort_workspace_bytes(cfg) + 256,), fill, dtype=torch.uint8, device="cuda")
        out = B.Sorted(*(torch.full(s, -77, dtype=torch.int32, device="cuda") for s in ((E + 1,), (n,), (n, 1))))
        _check_plan(B.ec_sort_tokens(cfg, choice.cuda(), out=out, ws=ws[:-256]), choice, E)
        assert B.ec_read_status(ws) == B.EC_OK and (ws[-256:] == fill).all()


# widths: below, at and beyond the lanes' stretches, odd numbers of 16-byte pieces, one piece
WIDTHS = [(F32, F32, 4), (F32, F32, 36), (F32, F32, 1000), (BF16, BF16, 8), (BF16, BF16, 64), (BF16, BF16, 136), (BF16, BF16, 1000), (BF16, BF16, 4104),
          (BF16, F32, 8), (BF16, F32, 328), (BF16, F32, 2056), (F32, F32, 2052)]


@pytest.mark.parametrize("dtype,y_dtype,d", WIDTHS)
@pytest.mark.parametrize("n,K,E,kind", [(1, 1, 4, "random"), (1, 8, 64, "distinct"), (37, 3, 10, "holes"), (130, 9, 16, "random"), (301, 2, 8, "one"), (19, 32, 256, "holes"),
                                        (40, 2, 8, "none")])
def test_rows_there_and_back(dtype, y_dtype, d, n, K, E, kind):
    g = torch.Generator(device="cuda").manual_seed(5)
    choice = _choice(n, K, E, 11, kind)
    cfg = B.make_sort_config(n, d, E, K, dtype, y_dtype)
    plan = B.ec_sort_tokens(cfg, choice.cuda())
    offsets, order, place = R.plan(choice.numpy(), E)
    m = int(offsets[-1])

    def normal(shape, dt):
        return torch.empty(shape, device="cuda").normal_(generator=g).to(dt)

    X, Y, G, w = normal((n, d), dtype), normal((n * K, d), y_dtype), normal((n, d), dtype), normal((n, K), F32)
    Y[m:] = float("nan")                                                # rows that no choice holds are not read
    w[plan.place < 0] = float("nan")                                    # nor the weights of choices without a row
    X_s = torch.full((n * K, d), 7.0, dtype=dtype, device="cuda")
    B.ec_dispatch(cfg, X, plan.place, X_s=X_s)
    assert torch.equal(X_s[:m].cpu(), X.cpu()[torch.from_numpy(order // K)])
    assert (X_s[m:] == 7.0).all()
    for weights in (w, None):
        want, size = R.combine(Y, weights, place)
        R.check_sum(B.ec_combine(cfg, Y, weights, plan.place), want, size, K, dtype)
    dY, dw = torch.full((n * K, d), 7.0, dtype=y_dtype, device="cuda"), torch.full((n, K), 7.0, device="cuda")
    B.ec_combine_backward(cfg, G, Y, w, plan.place, dY=dY, dweights=dw)
    assert (dY[m:] == 7.0).all()
    G64 = G.cpu().double().numpy()
    w64 = np.nan_to_num(w.cpu().double().numpy().reshape(-1))
    want = w64[order][:, None] * G64[order // K]
    R.check_sum(dY[:m], want, np.abs(want), 1, y_dtype)
    v = R.rows_of(Y, place)
    R.check_sum(dw, (v * G64[:, None]).sum(2), (np.abs(v) * np.abs(G64[:, None])).sum(2), d, F32)
    assert (dw.cpu().numpy()[place < 0] == 0).all()


@pytest.mark.parametrize("dtype,y_dtype,d", [(BF16, BF16, 72), (BF16, BF16, 120), (BF16, BF16, 128), (BF16, F32, 40), (BF16, F32, 64), (F32, F32, 64)])
@pytest.mark.parametrize("n,K,E,kind", [(1, 1, 4, "random"), (37, 1, 10, "holes"), (301, 2, 8, "holes"), (130, 3, 10, "holes"), (55, 4, 16, "random"), (19, 32, 256, "holes")])
def test_rows_of_nine_to_sixteen_pieces(dtype, y_dtype, d, n, K, E, kind):
    """Rows that two tokens of a warp share, by twos and by fours."""
    test_rows_there_and_back(dtype, y_dtype, d, n, K, E, kind)


def test_infinities_and_nan_stay_where_they_belong():
    """A row with NaN or an infinity reaches the tokens that hold it and no others, a weight of zero does not hide it (0 * inf is NaN),
    and what lies in rows without a choice reaches nobody."""
    n, K, E, d = 64, 2, 8, 128
    choice = _choice(n, K, E, 2, "distinct")
    cfg = B.make_sort_config(n, d, E, K, BF16)
    plan = B.ec_sort_tokens(cfg, choice.cuda())
    Y = torch.ones(n * K, d, dtype=BF16, device="cuda")
    w = torch.full((n, K), 0.5, device="cuda")
    Y[int(plan.place[3, 1]), 5] = float("nan")
    Y[int(plan.place[9, 0])] = float("inf")
    w[9, 0] = 0.0
    out = B.ec_combine(cfg, Y, w, plan.place).float().cpu()
    bad = ~torch.isfinite(out)
    want = torch.zeros(n, d, dtype=torch.bool)
    want[3, 5] = True
    want[9] = True
    assert torch.equal(bad, want) and (out[~want] == 1.0).all()


def test_bad_places_are_no_rows():
    """place is the caller's memory: entries outside the rows are choices without a row, whatever they hold."""
    n, K, E, d = 50, 3, 4, 72
    cfg = B.make_sort_config(n, d, E, K, F32)
    place = torch.randint(-5, n * K + 5, (n, K), generator=torch.Generator().manual_seed(1), dtype=torch.int32)
    place[0] = torch.tensor([2 ** 31 - 1, -2 ** 31, n * K], dtype=torch.int32)
    good = torch.where((place >= 0) & (place < n * K), place, -1).numpy()
    Y, G, w = (torch.randn(s, device="cuda") for s in ((n * K, d), (n, d), (n, K)))
    want, size = R.combine(Y, w, good)
    R.check_sum(B.ec_combine(cfg, Y, w, place.cuda()), want, size, K, F32)
    dY, dw = B.ec_combine_backward(cfg, G, Y, w, place.cuda(), dY=torch.zeros_like(Y))
    assert (dw.cpu().numpy()[good < 0] == 0).all()
    held = torch.from_numpy(np.unique(good[good >= 0]))
    rest = torch.ones(n * K, dtype=torch.bool)
    rest[held] = False
    assert (dY.cpu()[rest] == 0).all()
    X_s = B.ec_dispatch(cfg, G, place.cuda(), X_s=torch.zeros(n * K, d, device="cuda"))
    assert (X_s.cpu()[rest] == 0).all() and (X_s.cpu()[held].abs().sum(1) > 0).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_gradients_against_differences(dtype):
    """L = <C, combine(dispatch-shaped Y, w)> is linear in Y and in w, so a central difference has no error but that of the
    calls' arithmetic: each X_out is off by at most its bound, and L is summed in 64 bits.  Steps are powers of two, exact in either type."""
    n, K, E, d = 40, 3, 6, 48
    choice = _choice(n, K, E, 7, "holes")
    cfg = B.make_sort_config(n, d, E, K, dtype, F32)                    # Y in fp32
    if dtype == BF16:
        cfg = B.make_sort_config(n, d, E, K, BF16, F32)
    plan = B.ec_sort_tokens(cfg, choice.cuda())
    g = torch.Generator(device="cuda").manual_seed(1)
    Y, w = torch.randn(n * K, d, generator=g, device="cuda"), torch.randn(n, K, generator=g, device="cuda")
    C = torch.randn(n, d, generator=g, device="cuda").to(dtype)
    dY, dw = B.ec_combine_backward(cfg, C, Y, w, plan.place, dY=torch.zeros_like(Y))
    place = R.plan(choice.numpy(), E)[2]

    def loss(Y, w):
        out = B.ec_combine(cfg, Y, w, plan.place)
        want, size = R.combine(Y, w, place)
        off = (2 * K + 2) * 2.0 ** -24 * size + R.HALF_STEP[dtype] * (np.abs(want) * (1 + 2.0 ** -10) + 2.0 ** -20 * size)
        c = C.double().cpu().numpy()
        return (c * out.double().cpu().numpy()).sum(), off * np.abs(c)

    h = 4.0
    for _ in range(6):
        t, j = int(torch.randint(n, (1,))), int(torch.randint(K, (1,)))
        up, down = w.clone(), w.clone()
        up[t, j] += h; down[t, j] -= h
        (a, ea), (b, eb) = loss(Y, up), loss(Y, down)
        step = float(up[t, j].double() - down[t, j].double())
        # rows of other tokens are the same bits on both sides: only row t's error counts
        assert abs((a - b) / step - float(dw[t, j])) <= (ea[t].sum() + eb[t].sum()) / step + d * 2.0 ** -23 * float((C[t].double().abs() * Y[max(int(plan.place[t, j]), 0)].double().abs()).sum()) + 1e-12
        r, c = int(torch.randint(int(plan.offsets[-1]), (1,))), int(torch.randint(d, (1,)))
        up, down = Y.clone(), Y.clone()
        up[r, c] += h; down[r, c] -= h
        (a, ea), (b, eb) = loss(up, w), loss(down, w)
        step = float(up[r, c].double() - down[r, c].double())
        t = int(plan.order[r]) // K
        assert abs((a - b) / step - float(dY[r, c])) <= (ea[t, c] + eb[t, c]) / step + 2.0 ** -23 * abs(float(dY[r, c])) + 1e-12


@pytest.mark.parametrize("dtype,y_dtype", [(F32, F32), (BF16, F32), (BF16, BF16)])
def test_gradients_against_differences_of_chosen_entries(dtype, y_dtype):
    """As above with entries that are the same in every run: weights of choices that have a row (and one that has none, whose gradient is 0),
    values of rows of every expert.  Y's steps of 4 from small multiples of 1/8 are exact in either type."""
    n, K, E, d, h = 40, 3, 6, 48, 4.0
    choice = _choice(n, K, E, 7, "holes")
    cfg = B.make_sort_config(n, d, E, K, dtype, y_dtype)
    plan = B.ec_sort_tokens(cfg, choice.cuda())
    offsets, order, place = R.plan(choice.numpy(), E)
    g = torch.Generator().manual_seed(11)
    Y = (torch.randint(-16, 17, (n * K, d), generator=g) / 8).to(y_dtype).cuda()
    w, C = torch.randn(n, K, generator=g).cuda(), torch.randn(n, d, generator=g).to(dtype).cuda()
    dY, dw = B.ec_combine_backward(cfg, C, Y, w, plan.place, dY=torch.zeros_like(Y))
    c = C.double().cpu().numpy()

    def loss(Y, w):
        out = B.ec_combine(cfg, Y, w, plan.place)
        want, size = R.combine(Y, w, place)
        sums = (2 * K + 2) * 2.0 ** -24 * size            # the fp32 sums' own error, and the rounding of what they came to
        return c * out.double().cpu().numpy(), (sums + R.HALF_STEP[dtype] * (np.abs(want) + sums)) * np.abs(c)

    held, holes = np.argwhere(place >= 0), np.argwhere(place < 0)
    for t, j in [held[i] for i in (0, len(held) // 3, len(held) // 2, 2 * len(held) // 3, len(held) - 1)] + [holes[len(holes) // 2]]:
        up, down = w.clone(), w.clone()
        up[t, j] += h; down[t, j] -= h
        (a, ea), (b, eb) = loss(Y, up), loss(Y, down)
        assert (np.delete(a, t, 0) == np.delete(b, t, 0)).all()         # the other tokens' rows: the same bits
        if place[t, j] < 0:
            assert (a == b).all() and float(dw[t, j]) == 0
            continue
        step = float(up[t, j].double() - down[t, j].double())
        size = (np.abs(c[t]) * np.abs(Y[int(place[t, j])].double().cpu().numpy())).sum()
        assert abs((a - b)[t].sum() / step - float(dw[t, j])) <= (ea + eb)[t].sum() / step + d * 2.0 ** -23 * size
    for e in range(E):
        r, col = int(offsets[e + 1]) - 1, (7 * e + 3) % d
        assert r >= offsets[e]
        up, down = Y.clone(), Y.clone()
        up[r, col] += h; down[r, col] -= h
        (a, ea), (b, eb) = loss(up, w), loss(down, w)
        t = order[r] // K
        step = float(up[r, col].double() - down[r, col].double())
        assert step == 2 * h
        grad = float(dY[r, col])
        assert abs((a - b).sum() / step - grad) <= (ea + eb)[t, col] / step + 2 * (R.HALF_STEP[y_dtype] + 2.0 ** -24) * abs(grad)


def test_gradient_of_the_dispatch():
    """<C, dispatch(X)> = <combine(C, ones), X> for every X: on small whole numbers every sum is exact, in both types."""
    for dtype in (F32, BF16):
        n, K, E, d = 90, 4, 9, 56
        cfg = B.make_sort_config(n, d, E, K, dtype)
        choice = _choice(n, K, E, 8, "holes")
        plan = B.ec_sort_tokens(cfg, choice.cuda())
        g = torch.Generator(device="cuda").manual_seed(4)
        X = torch.randint(-8, 9, (n, d), generator=g, device="cuda").to(dtype)
        C = torch.randint(-8, 9, (n * K, d), generator=g, device="cuda").to(dtype)
        m = int(plan.offsets[-1])
        X_s, dX = B.ec_dispatch(cfg, X, plan.place), B.ec_combine(cfg, C, None, plan.place)
        assert (X_s[:m].double() * C[:m].double()).sum() == (dX.double() * X.double()).sum()


@pytest.mark.parametrize("dtype,y_dtype", [(F32, F32), (BF16, BF16), (BF16, F32)])
def test_gradient_of_the_dispatch_in_each_pair_of_types(dtype, y_dtype):
    """dX_s has X's type, whatever Y's is: the same identity in exact numbers, with the configuration of the layer, and the bits of a call
    whose configuration has one type for both.  Rows of Y's type are still taken without weights."""
    n, K, E, d = 90, 4, 9, 56
    cfg = B.make_sort_config(n, d, E, K, dtype, y_dtype)
    plan = B.ec_sort_tokens(cfg, _choice(n, K, E, 8, "holes").cuda())
    g = torch.Generator(device="cuda").manual_seed(4)
    X = torch.randint(-8, 9, (n, d), generator=g, device="cuda").to(dtype)
    dX_s = torch.randint(-8, 9, (n * K, d), generator=g, device="cuda").to(dtype)
    m = int(plan.offsets[-1])
    X_s, dX = B.ec_dispatch(cfg, X, plan.place), B.ec_combine(cfg, dX_s, None, plan.place)
    assert dX.dtype is dtype and (X_s[:m].double() * dX_s[:m].double()).sum() == (dX.double() * X.double()).sum()
    assert torch.equal(dX, B.ec_combine(B.make_sort_config(n, d, E, K, dtype), dX_s, None, plan.place))
    assert torch.equal(dX, B.ec_combine(cfg, dX_s.to(y_dtype), None, plan.place))
    if y_dtype is not dtype:                              # with weights it is the layer's combine, and Y of its type
        with pytest.raises(B.EcError):
            B.ec_combine(cfg, dX_s, torch.ones(n, K, device="cuda"), plan.place)


@pytest.mark.parametrize("n,K,E,first", [(50, 3, 10, 1), (3000, 3, 10, 7), (30000, 1, 33, 3)])
def test_slices_of_the_tokens_and_of_a_stack(n, K, E, first):
    """choice[t0:] of an odd number of choices, a plan written into the middle of larger arrays, one layer's offsets of a stack: the results of
    arrays of their own."""
    d, dtype = 72, BF16
    choice = _choice(first + n, K, E, 5, "holes").cuda()[first:]
    assert choice.data_ptr() % 16
    cfg = B.make_sort_config(n, d, E, K, dtype)
    want = B.ec_sort_tokens(cfg, choice.clone())
    stack = torch.full((3, E + 1), -77, dtype=torch.int32, device="cuda")
    order, place = (torch.full((n * K + 2,), -77, dtype=torch.int32, device="cuda") for _ in range(2))
    got = B.ec_sort_tokens(cfg, choice, out=B.Sorted(stack[1], order[1:-1], place[1:-1].view(n, K)))
    m = int(want.offsets[-1])
    assert torch.equal(got.offsets, want.offsets) and torch.equal(got.place, want.place) and torch.equal(got.order[:m], want.order[:m])
    assert (stack[::2] == -77).all() and all((t[[0, -1]] == -77).all() for t in (order, place))
    g = torch.Generator(device="cuda").manual_seed(2)
    X, Y, G, w = (torch.randn(s, generator=g, device="cuda").to(t) for s, t in (((n, d), dtype), ((n * K, d), dtype), ((n, d), dtype), ((n, K), F32)))
    calls = (lambda p: [B.ec_dispatch(cfg, X, p, X_s=torch.zeros_like(Y))], lambda p: [B.ec_combine(cfg, Y, w, p)],
             lambda p: B.ec_combine_backward(cfg, G, Y, w, p, dY=torch.zeros_like(Y)))
    for call in calls:
        for a, b in zip(call(got.place), call(want.place)):
            assert torch.equal(a, b)
    zero = lambda: B.Mx(*(torch.zeros_like(t) for t in (q.codes, q.scales)), d)
    q = B.alloc_mx((n * K, d))
    a, b = (B.ec_mx_dispatch(cfg, X, p.place, out=zero()) for p in (got, want))
    assert torch.equal(a.codes, b.codes) and torch.equal(a.scales, b.scales)
    W = B.ec_mx_quantize(torch.randn(E, 64, d, generator=g, device="cuda"))
    out = [B.ec_mx_expert_gemm(a, W, p.offsets, out=torch.zeros(n * K, 64, device="cuda")) for p in (got, want)]
    assert torch.equal(*out)


def _step(cfg, choice, X, Y, w, G, bufs, ws):
    plan = B.ec_sort_tokens(cfg, choice, out=bufs["plan"], ws=ws)
    B.ec_dispatch(cfg, X, plan.place, X_s=bufs["X_s"])
    B.ec_combine(cfg, Y, w, plan.place, X_out=bufs["X_out"])
    B.ec_combine_backward(cfg, G, Y, w, plan.place, dY=bufs["dY"], dweights=bufs["dw"])
    B.ec_combine(cfg, bufs["dY"], None, plan.place, X_out=bufs["dX"])


def _setup(n, K, E, d, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    cfg = B.make_sort_config(n, d, E, K, dtype)
    data = dict(choice=_choice(n, K, E, seed, "holes").cuda(), X=torch.randn(n, d, generator=g, device="cuda").to(dtype),
                Y=torch.randn(n * K, d, generator=g, device="cuda").to(dtype), w=torch.randn(n, K, generator=g, device="cuda"),
                G=torch.randn(n, d, generator=g, device="cuda").to(dtype))
    i32 = dict(dtype=torch.int32, device="cuda")
    bufs = dict(plan=B.Sorted(torch.zeros(E + 1, **i32), torch.zeros(n * K, **i32), torch.zeros(n, K, **i32)), X_s=torch.zeros_like(data["Y"]),
                X_out=torch.zeros_like(data["X"]), dY=torch.zeros_like(data["Y"]), dw=torch.zeros_like(data["w"]), dX=torch.zeros_like(data["X"]))
    ws = torch.empty(B.ec_sort_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    return cfg, data, bufs, ws


def _flat(bufs):
    return [bufs["plan"].offsets, bufs["plan"].order, bufs["plan"].place] + [bufs[k] for k in ("X_s", "X_out", "dY", "dw", "dX")]


def test_captured_and_replayed_on_new_data():
    """A step captured into a graph, replayed after its inputs changed, gives the bits of the eager calls."""
    for n, K, E, d, dtype in ((700, 3, 12, 264, BF16), (20000, 2, 40, 64, F32)):
        cfg, data, bufs, ws = _setup(n, K, E, d, dtype, 1)
        _step(cfg, **data, bufs=bufs, ws=ws)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            _step(cfg, **data, bufs=bufs, ws=ws)
        _, other, want, _ = _setup(n, K, E, d, dtype, 2)
        _step(cfg, **other, bufs=want, ws=ws)
        for k in data:
            data[k].copy_(other[k])
        for t in _flat(bufs):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(_flat(bufs), _flat(want)):
            assert torch.equal(a, b)


def test_several_threads_and_streams_at_once():
    jobs, failed = [], []
    for i, (n, K, E, d, dtype) in enumerate([(4, 2, 64, 512, BF16), (9000, 2, 16, 128, F32), (30000, 3, 256, 64, BF16), (1500, 8, 32, 1024, BF16)]):
        cfg, data, bufs, ws = _setup(n, K, E, d, dtype, 10 + i)
        _step(cfg, **data, bufs=bufs, ws=ws)
        jobs.append((cfg, data, bufs, ws, [t.clone() for t in _flat(bufs)]))
    torch.cuda.synchronize()
    start = threading.Barrier(len(jobs))

    def work(cfg, data, bufs, ws, want):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                start.wait()
                for _ in range(200):
                    _step(cfg, **data, bufs=bufs, ws=ws)
                for a, b in zip(_flat(bufs), want):
                    assert torch.equal(a, b)
        except BaseException as e:
            failed.append(e)

    threads = [threading.Thread(target=work, args=j) for j in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed, failed


def test_rows_beyond_the_range_of_32_bit_offsets():
    """Row matrices of more than 2^32 bytes and 2^31 values: the last rows are those of the last choices."""
    n, K, E, d = 70001, 8, 4, 4096
    cfg = B.make_sort_config(n, d, E, K, BF16)
    choice = _choice(n, K, E, 3).cuda()
    plan = B.ec_sort_tokens(cfg, choice)
    X = torch.randn(n, d, device="cuda").to(BF16)
    X_s = B.ec_dispatch(cfg, X, plan.place)
    assert X_s.numel() > 2 ** 31
    for r in (0, 1, n * K // 2, 262144, n * K - 2, n * K - 1):
        assert torch.equal(X_s[r], X[int(plan.order[r]) // K])
    out = B.ec_combine(cfg, X_s, None, plan.place)
    assert torch.equal(out, (X.float() * K).to(BF16))                   # K equal rows: a power of two times the token
    dY, dw = B.ec_combine_backward(cfg, X, X_s, torch.full((n, K), 0.5, device="cuda"), plan.place)
    r = n * K - 1
    assert torch.equal(dY[r], X[int(plan.order[r]) // K] * 0.5)
    x = X[n - 1].double()
    assert abs(float(dw[n - 1, K - 1]) - float((x * x).sum())) <= d * 2.0 ** -23 * float((x * x).sum())
