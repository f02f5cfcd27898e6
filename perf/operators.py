"""Tokens sorted by expert and back, and expert products on 4-bit operands: what is timed of them, beside their plain forms.

  sort      ec_sort_tokens, ec_dispatch, ec_combine and, in training, ec_combine_backward and the gradient of the dispatch:
            a layer in which every token picks K experts and none is dropped, for a caller that runs experts of its own
  quantize  ec_mx_quantize and ec_mx_dequantize: a matrix or a stack of weights through the 4-bit format and back
  product   ec_mx_quantize of the rows and ec_mx_expert_gemm: one expert product of a served layer
  ffn       ec_sort_tokens, ec_mx_dispatch, two ec_mx_expert_gemm (the first with GeLU and 4-bit results), ec_combine: the
            feed-forward layer as a served model runs it

The 4-bit format: blocks of 32 along the contraction share a power of two 2^(s - 127), s = max(0, floor(log2 amax) + 125), and
each value is +-{0, 0.5, 1, 1.5, 2, 3, 4, 6} times it, rounded to the nearest (ties to the even code) and held at 6.  A block with
an infinity or a NaN has s = 255 and stands for NaN.  Value 2 i of a row is the low half of byte i.  A row has 16 bytes per block, its
scales a row of their own whose length is a multiple of 16 bytes.

Sizes are in the notation of the layer: n tokens, d model width, f hidden width, E experts, K experts per token.  Buffers that a
program keeps from step to step (outputs, workspace) are part of the prepared state.
"""
import math

import torch

own = False
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def sort(name, n, d, E, K, dtype="bf16", train=False, pad=0.0, skew=0.5):
    case = {"op": "sort", "n": n, "d": d, "E": E, "K": K, "dtype": dtype, "train": train, "pad": pad, "skew": skew}
    return dict(case, name=name) if name else case


def quantize(name, batches, rows, cols, transposed=False, dtype="bf16"):
    case = {"op": "quantize", "batches": batches, "rows": rows, "cols": cols, "transposed": transposed, "dtype": dtype}
    return dict(case, name=name) if name else case


def product(name, n, d, f, E, K, act="none", bias=False, dtype="bf16", skew=0.5):
    case = {"op": "product", "n": n, "d": d, "f": f, "E": E, "K": K, "act": act, "bias": bias, "dtype": dtype, "skew": skew}
    return dict(case, name=name) if name else case


def ffn(name, n, d, f, E, K, act="erf", bias=False, skew=0.5):
    case = {"op": "ffn", "n": n, "d": d, "f": f, "E": E, "K": K, "act": act, "bias": bias, "skew": skew}
    return dict(case, name=name) if name else case


def listed():
    return [
        # a decoding step of four sequences: launches and latency
        sort("sort_decode", 4, 4096, 64, 2),
        # evaluation of the 8B layer with 64 experts, sixteen sequences of 1024 tokens, two experts per token
        sort("sort_8b64e", 16384, 4096, 64, 2),
        # a training step of the 100M layer with 32 experts in fp32 (debugging, reference runs)
        sort("sort_train_f32", 8192, 768, 32, 2, "f32", train=True),
        # nothing a multiple of a tile: ten experts, three per token, the last sixth of the batch is padding
        sort("sort_train_padded", 6079, 1000, 10, 3, train=True, pad=0.17, skew=1.0),
        # many small experts, eight per token: half a million rows, the largest step
        sort("sort_train_wide", 65536, 1024, 256, 8, train=True),
        # activations of a long prompt on their way into a product
        quantize("quantize_rows", 1, 16384, 4096),
        # W1 of sixteen experts laid out for serving: the contraction runs along the matrices' rows
        quantize("quantize_weights", 16, 8192, 4096, transposed=True),
        # decoding with the 8B layer: eight rows, what is read is the weights of their experts
        product("product_decode", 4, 4096, 16384, 64, 2),
        # the first product of the 100M layer, 8192 tokens, with its bias and GeLU
        product("product_100m32e", 8192, 768, 2048, 32, 2, act="erf", bias=True),
        # the first product of the 8B layer, 16384 tokens: the largest product
        product("product_8b64e", 16384, 4096, 16384, 64, 2),
        # a served layer in a few hundred microseconds, uneven experts, ragged widths, tanh GeLU and biases
        ffn("ffn_ragged", 1531, 1096, 4072, 16, 2, act="tanh", bias=True, skew=1.0),
        # decoding a batch of 32 sequences through a whole layer: the weights of most experts are read for a few rows each
        ffn("ffn_decode", 32, 2048, 8192, 32, 2),
    ]


def _log(rng, lo, hi, mult=1):
    """A size spread over the logarithm of [lo, hi], rounded to a multiple of `mult`."""
    v = math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))
    return max(mult, int(round(v / mult)) * mult)


def draw(rng):
    op = rng.choices(["sort", "quantize", "product", "ffn"], [40, 20, 25, 15])[0]
    if op == "quantize":
        cols = _log(rng, 32, 16384, 8)
        rows = _log(rng, 8, min(16384, 2 ** 28 // cols), 8)
        return quantize(None, rng.randint(1, max(1, min(32, 2 ** 28 // (rows * cols)))), rows, cols, rng.random() < 0.5, rng.choice(["bf16", "f32"]))
    E = rng.choice([4, 8, 10, 16, 24, 32, 64, 128, 256])
    K = rng.randint(1, 8) if E >= 8 else rng.randint(1, 4)
    skew = rng.choice([0.0, 0.5, 1.0])
    if op == "sort":
        n = _log(rng, 1, 65536)
        d = _log(rng, 64, min(8192, 2 ** 28 // (n * K)), 8)
        return sort(None, n, d, E, K, rng.choice(["bf16", "bf16", "f32"]), rng.random() < 0.6, rng.choice([0.0, 0.0, 0.1, 0.4]), skew)
    E, K = min(E, 64), min(K, 4)
    n, d = _log(rng, 1, 8192), _log(rng, 256, 4096, 8)
    f = _log(rng, 256, min(16384, 2 ** 30 // (E * d)), 8)
    act, bias = rng.choice(["none", "erf", "tanh"]), rng.random() < 0.4
    if op == "ffn":
        return ffn(None, n, d, f, E, K, act, bias, skew)
    return product(None, n, d, f, E, K, act, bias, rng.choice(["bf16", "bf16", "f32"]), skew)


# ---- inputs -------------------------------------------------------------------------------------------------------


def _choices(gen, n, E, K, pad, skew):
    """K experts for each of n tokens by the gate's score, and those scores; -1 in the padded tokens at the end and, where there are
    any, in one choice of twenty (a choice that a limit on the experts took back)."""
    S = torch.softmax(torch.empty(n, E, device="cuda").normal_(generator=gen) + skew * torch.empty(E, device="cuda").normal_(generator=gen), 1)
    weights, choice = torch.topk(S, K, dim=1)
    choice = choice.int()
    if pad:
        gone = torch.rand(n, K, device="cuda", generator=gen) < 0.05
        gone[n - int(n * pad):] = True
        choice = torch.where(gone, -1, choice)
    return choice.contiguous(), weights.contiguous()


def _pitch(cols):
    return -(-cols // 512) * 16


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(shape, std, dt):
        return torch.empty(shape, dtype=dt, device="cuda").normal_(0.0, std, generator=gen)

    def zeros(shape, dt):
        return torch.zeros(shape, dtype=dt, device="cuda")

    s = dict(case, ws=zeros(1 << 20, torch.uint8), levels=torch.tensor(LEVELS + tuple(-v for v in LEVELS), device="cuda"))
    if case["op"] == "quantize":
        b, r, c, dt = case["batches"], case["rows"], case["cols"], DTYPES[case["dtype"]]
        X = normal((b, c, r) if case["transposed"] else (b, r, c), 1.0, dt)
        X *= torch.exp(normal(X.shape[:-1] + (1,), 1.0, torch.float32)).to(dt)        # rows of very different sizes
        s.update(X=X, codes=zeros((b, r, 16 * -(-c // 32)), torch.uint8), scales=zeros((b, r, _pitch(c)), torch.uint8), back=zeros((b, r, c), dt))
        return s
    n, d, E, K = case["n"], case["d"], case["E"], case["K"]
    choice, weights = _choices(gen, n, E, K, case.get("pad", 0.0), case["skew"])
    s.update(choice=choice, weights=weights, offsets=zeros(E + 1, torch.int32), order=torch.full((n * K,), -1, dtype=torch.int32, device="cuda"),
             place=zeros((n, K), torch.int32))
    if case["op"] == "sort":
        dt = DTYPES[case["dtype"]]
        s.update(X=normal((n, d), 1.0, dt), Y=normal((n * K, d), 1.0, dt), X_s=zeros((n * K, d), dt), X_out=zeros((n, d), dt))
        if case["train"]:
            s.update(dX_out=normal((n, d), 1.0, dt), dX_s=normal((n * K, d), 1.0, dt), dY=zeros((n * K, d), dt),
                     dweights=zeros((n, K), torch.float32), dX=zeros((n, d), dt))
        return s
    f, M = case["f"], n * K
    dims = [("1", f, d)] + ([("2", d, f)] if case["op"] == "ffn" else [])
    for which, N, C in dims:                                                          # weights as they are kept for serving
        codes, scales = zeros((E, N, 16 * -(-C // 32)), torch.uint8), zeros((E, N, _pitch(C)), torch.uint8)
        for e in range(E):
            codes[e], scales[e] = encode(normal((N, C), C ** -0.5, torch.float32))
        s["W" + which], s["S" + which] = codes, scales
        s["b" + which] = normal((E, N), 0.5, torch.bfloat16 if case["op"] == "ffn" else DTYPES[case["dtype"]]) if case["bias"] else None
    if case["op"] == "ffn":
        s.update(X=normal((n, d), 1.0, torch.bfloat16), Xq=zeros((M, 16 * -(-d // 32)), torch.uint8), Xp=zeros((M, _pitch(d)), torch.uint8),
                 Hq=zeros((M, 16 * -(-f // 32)), torch.uint8), Hp=zeros((M, _pitch(f)), torch.uint8), Y=zeros((M, d), torch.float32),
                 X_out=zeros((n, d), torch.bfloat16))
    else:
        s.update(X=normal((M, d), 1.0, torch.bfloat16), Xq=zeros((M, 16 * -(-d // 32)), torch.uint8), Xp=zeros((M, _pitch(d)), torch.uint8),
                 C=zeros((M, f), DTYPES[case["dtype"]]))
        s["offsets"] = _plan(choice, E)[0]                                            # the rows are sorted already
    counts = (choice.reshape(-1, 1) == torch.arange(E, device="cuda")).sum(0)
    s["most"] = max(1, int(counts.max()))                                             # rows of the fullest expert, for the plain form's batches
    return s


# ---- the plain forms ----------------------------------------------------------------------------------------------


def encode(x):
    """x [..., C] in the 4-bit format along its last axis."""
    C = x.shape[-1]
    x = torch.nn.functional.pad(x.float(), (0, -C % 32)).unflatten(-1, (-1, 32))
    size = (x.view(torch.int32) & 0x7FFFFFFF).amax(-1, keepdim=True)                  # bits of the largest magnitude; NaN is above all
    bad = (size >> 23) == 255
    s = torch.where(bad, 255, ((size >> 23) - 2).clamp(min=0))
    y = x.abs() * ((254 - s) << 23).clamp(min=0).view(torch.float32)                  # times 2^(127 - s)
    code = ((y > 0.25).byte() + (y >= 0.75) + (y > 1.25) + (y >= 1.75) + (y > 2.5) + (y >= 3.5) + (y > 5.0)) | (torch.signbit(x).byte() << 3)
    code = torch.where(bad, 0, code).to(torch.uint8).flatten(-2)
    s = s.squeeze(-1).to(torch.uint8)
    return code[..., ::2] | (code[..., 1::2] << 4), torch.nn.functional.pad(s, (0, _pitch(C) - s.shape[-1]))


def decode(codes, scales, C, levels):
    """The values that codes and scales stand for, [..., C] in fp32."""
    v = levels[torch.stack((codes & 15, codes >> 4), -1).flatten(-2).int()].unflatten(-1, (-1, 32))
    s = scales[..., : v.shape[-2]].int()
    p = torch.where(s == 0, 2.0 ** -127, (s << 23).view(torch.float32))
    p = torch.where(s == 255, float("nan"), p)
    return (v * p[..., None]).flatten(-2)[..., :C]


def _plan(choice, E):
    flat = choice.reshape(-1)
    key = torch.where((flat >= 0) & (flat < E), flat, E)
    order = torch.sort(key, stable=True)[1]
    counts = (key[:, None] == torch.arange(E, device=key.device)).sum(0)
    offsets = torch.nn.functional.pad(torch.cumsum(counts, 0), (1, 0)).int()
    r = torch.arange(flat.numel(), device=key.device)
    place = torch.empty_like(r)
    place[order] = r
    place = torch.where(key < E, place, -1).int().view(choice.shape)
    return offsets, torch.where(r < offsets[-1], order, -1).int(), place, order


def _back(rows, place, weights):
    """[n, K, d] in fp32: the rows of each token's choices, times their weights, zeros where there is none."""
    v = rows[place.clamp(min=0).long()].float()
    v = v if weights is None else v * weights[..., None]
    return torch.where(place[..., None] >= 0, v, 0.0)


def _act(z, act):
    if act == "erf":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    return z


def _expert_product(s, rows, which, offsets, act):
    """rows [M, C] in fp32, sorted by expert, times their experts' weights: [M, N] in fp32, zeros behind the last expert's rows."""
    W, E = s["W" + which], s["E"]
    r = torch.arange(rows.shape[0], device=rows.device)
    e = (r[:, None] >= offsets[1:]).sum(1)
    inside, e = e < E, e.clamp(max=E - 1)
    at = torch.where(inside, r - offsets[e], s["most"])
    batch = torch.zeros(E, s["most"] + 1, rows.shape[1], device=rows.device)
    batch[e, at] = rows
    z = torch.bmm(batch, decode(W, s["S" + which], rows.shape[1], s["levels"]).transpose(1, 2))[e, at]
    if s["b" + which] is not None:
        z = z + s["b" + which].float()[e]
    return torch.where(inside[:, None], _act(z, act), 0.0)


def _plain(s):
    if s["op"] == "quantize":
        X = s["X"].transpose(1, 2).contiguous() if s["transposed"] else s["X"]
        return {"back": decode(*encode(X), s["cols"], s["levels"]).to(X.dtype)}
    if s["op"] == "product":
        rows = decode(*encode(s["X"]), s["d"], s["levels"])
        return {"C": _expert_product(s, rows, "1", s["offsets"], s["act"]).to(s["C"].dtype)}
    X, K, dt = s["X"], s["K"], s["X"].dtype
    offsets, order, place, where_from = _plan(s["choice"], s["E"])
    inside = (order >= 0)[:, None]
    if s["op"] == "ffn":
        rows = decode(*encode(X), s["d"], s["levels"])[where_from // K]
        H = decode(*encode(_expert_product(s, rows, "1", offsets, s["act"])), s["f"], s["levels"])
        return {"X_out": _back(_expert_product(s, H, "2", offsets, "none"), place, s["weights"]).sum(1).to(dt)}
    out = {"offsets": offsets, "order": order, "place": place, "X_s": torch.where(inside, X[where_from // K], 0.0),
           "X_out": _back(s["Y"], place, s["weights"]).sum(1).to(dt)}
    if s["train"]:
        g = s["dX_out"].float()
        out["dY"] = torch.where(inside, g[where_from // K] * s["weights"].reshape(-1)[where_from][:, None], 0.0).to(dt)
        out["dweights"] = (_back(s["Y"], place, None) * g[:, None]).sum(2)
        out["dX"] = _back(s["dX_s"], place, None).sum(1).to(dt)
    return out


# ---- the framework's calls ----------------------------------------------------------------------------------------


def _framework(s):
    from paper_2202_09368_b200 import binding as B
    ws = s["ws"]
    if s["op"] == "quantize":
        q = B.ec_mx_quantize(s["X"], transposed=s["transposed"], out=B.Mx(s["codes"], s["scales"], s["cols"]))
        return {"back": B.ec_mx_dequantize(q, out=s["back"])}
    if s["op"] == "product":
        q = B.ec_mx_quantize(s["X"], out=B.Mx(s["Xq"], s["Xp"], s["d"]))
        return {"C": B.ec_mx_expert_gemm(q, B.Mx(s["W1"], s["S1"], s["d"]), s["offsets"], bias=s["b1"], act=s["act"], out=s["C"], ws=ws)}
    X, n, d, E, K = s["X"], s["n"], s["d"], s["E"], s["K"]
    # the second product's rows stay in fp32 until the combine has added them up: one rounding, at the end
    cfg = B.make_sort_config(n, d, E, K, X.dtype, torch.float32 if s["op"] == "ffn" else X.dtype)
    plan = B.ec_sort_tokens(cfg, s["choice"], out=B.Sorted(s["offsets"], s["order"], s["place"]), ws=ws)
    if s["op"] == "ffn":
        rows = B.ec_mx_dispatch(cfg, X, plan.place, out=B.Mx(s["Xq"], s["Xp"], d))
        H = B.ec_mx_expert_gemm(rows, B.Mx(s["W1"], s["S1"], d), plan.offsets, bias=s["b1"], act=s["act"], out=B.Mx(s["Hq"], s["Hp"], s["f"]), ws=ws[-512:-256])
        Y = B.ec_mx_expert_gemm(H, B.Mx(s["W2"], s["S2"], s["f"]), plan.offsets, bias=s["b2"], out=s["Y"], ws=ws[-256:])         # each with a status word of its own
        return {"X_out": B.ec_combine(cfg, Y, s["weights"], plan.place, X_out=s["X_out"])}
    out = {"offsets": plan.offsets, "order": plan.order, "place": plan.place, "X_s": B.ec_dispatch(cfg, X, plan.place, X_s=s["X_s"]),
           "X_out": B.ec_combine(cfg, s["Y"], s["weights"], plan.place, X_out=s["X_out"])}
    if s["train"]:
        out["dY"], out["dweights"] = B.ec_combine_backward(cfg, s["dX_out"], s["Y"], s["weights"], plan.place, dY=s["dY"], dweights=s["dweights"])
        out["dX"] = B.ec_combine(cfg, s["dX_s"], None, plan.place, X_out=s["dX"])
    return out


def run(state):
    return _framework(state) if own else _plain(state)


# ---- the definition in 64 bits ------------------------------------------------------------------------------------


def _through(x):
    """x through the 4-bit format along its last axis, in 64 bits: the block's exponent from frexp, the values by rounding to the
    spacing of their binade."""
    C = x.shape[-1]
    x = torch.nn.functional.pad(x.double(), (0, -C % 32)).unflatten(-1, (-1, 32))
    amax = x.abs().amax(-1, keepdim=True)
    e = (torch.frexp(amax)[1] - 3).clamp(min=-127).double()                           # floor(log2 amax) - 2
    e = torch.where(amax == 0, -127.0, e)
    y = x * torch.exp2(-e)
    step = torch.where(y.abs() < 2, 0.5, torch.where(y.abs() < 4, 1.0, 2.0))
    y = (torch.round(y / step) * step).clamp(-6, 6)
    return torch.where(torch.isfinite(amax), y * torch.exp2(e), float("nan")).flatten(-2)[..., :C]


def _values64(codes, scales, C):
    low, high = codes.int() & 15, codes.int() >> 4
    v = torch.stack((low, high), -1).flatten(-2)
    m, e = (v & 1).double(), (v >> 1) & 3
    size = torch.where(e == 0, m * 0.5, (1 + 0.5 * m) * torch.exp2(e.double() - 1))
    v = torch.where(v >= 8, -size, size).unflatten(-1, (-1, 32))
    return (v * torch.exp2(scales[..., : v.shape[-2]].double() - 127)[..., None]).flatten(-2)[..., :C]


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "quantize":
        return {"back": _through(s["X"].transpose(1, 2) if case["transposed"] else s["X"])}
    gelu = {"none": lambda z: z, "erf": lambda z: torch.nn.functional.gelu(z), "tanh": lambda z: torch.nn.functional.gelu(z, approximate="tanh")}[case["act"]] \
        if "act" in case else None
    n, E, K, d = case["n"], case["E"], case["K"], case["d"]
    flat = s["choice"].reshape(-1)
    lists = [torch.nonzero(flat == e)[:, 0] for e in range(E)]                        # an expert's rows: its choices, in order

    def product64(e, x, which):
        z = x @ _values64(s["W" + which][e], s["S" + which][e], x.shape[1]).T
        return z if s["b" + which] is None else z + s["b" + which][e].double()

    if case["op"] == "product":
        C, first = torch.zeros(n * K, case["f"], dtype=torch.float64, device="cuda"), 0
        for e in range(E):
            last = first + len(lists[e])
            C[first:last] = gelu(product64(e, _through(s["X"][first:last]), "1"))
            first = last
        return {"C": C}
    X = s["X"].double()
    if case["op"] == "ffn":
        out, X = torch.zeros_like(X), _through(X)
        for e in range(E):
            t = lists[e] // K
            y = product64(e, _through(gelu(product64(e, X[t], "1"))), "2")
            out.index_add_(0, t, s["weights"].reshape(-1)[lists[e]].double()[:, None] * y)
        return {"X_out": out}
    out = {"offsets": None, "order": None, "place": None, "X_s": torch.zeros(n * K, d, dtype=torch.float64, device="cuda"), "X_out": torch.zeros_like(X)}
    if case["train"]:
        out.update(dY=torch.zeros_like(out["X_s"]), dweights=torch.zeros(n * K, dtype=torch.float64, device="cuda"), dX=torch.zeros_like(X))
    first = 0
    for e in range(E):
        last, t, w = first + len(lists[e]), lists[e] // K, s["weights"].reshape(-1)[lists[e]].double()[:, None]
        y = s["Y"][first:last].double()
        out["X_s"][first:last] = X[t]
        out["X_out"].index_add_(0, t, w * y)
        if case["train"]:
            g = s["dX_out"].double()[t]
            out["dY"][first:last] = w * g
            out["dweights"][lists[e]] = (g * y).sum(1)
            out["dX"].index_add_(0, t, s["dX_s"][first:last].double())
        first = last
    if case["train"]:
        out["dweights"] = out["dweights"].view(n, K)
    return out


def work(case):
    """Inputs read once, outputs written once.  A 4-bit value is half a byte and its share of a block's scale; of the weights, those of
    the experts that some row is expected to reach (all of them are equally likely here)."""
    size = {"f32": 4, "bf16": 2}
    four = 0.5 + 1 / 32
    if case["op"] == "quantize":
        values = case["batches"] * case["rows"] * case["cols"]
        return {"bytes": values * 2 * size[case["dtype"]], "flops": 4.0 * values}
    n, d, E, K = case["n"], case["d"], case["E"], case["K"]
    M = n * K
    if case["op"] == "sort":
        b, rows = size[case["dtype"]], round(M * (1 - case["pad"]))
        plan = 4 * (3 * M + E + 1)
        moved = (2 * n * d + 2 * rows * d) * b + 4 * M                                # X and X_out, X_s and Y, the weights
        flops = 2.0 * rows * d
        if case["train"]:
            moved += (2 * n * d + 2 * rows * d) * b + 4 * M                           # dX_out and dX, dY and dX_s, the weights' gradient
            flops += 4.0 * rows * d
        return {"bytes": plan + moved, "flops": flops}
    f, reached = case["f"], E * (1 - (1 - 1 / E) ** M)
    bias = reached * 2 * f if case["bias"] else 0
    if case["op"] == "product":
        return {"bytes": 2 * M * d + reached * f * d * four + bias + M * f * size[case["dtype"]], "flops": 2.0 * M * d * f}
    return {"bytes": 4 * n * d + 8 * M + 2 * reached * f * d * four + bias, "flops": 4.0 * M * d * f}
