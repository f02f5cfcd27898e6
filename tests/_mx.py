"""The 4-bit microscaled format restated in numpy from its definition, and expert products on it in 64 bits."""
import math

import numpy as np

import _sorted as S

LEVELS = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def pitches(cols):
    return 16 * -(-cols // 32), 16 * -(-cols // 512)


def encode(x):
    """x [rows, cols], fp32 or less, as (codes, scales) with the padding the quantisation writes."""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    blocks = -(-cols // 32)
    full = np.zeros((rows, 32 * blocks))
    full[:, :cols] = x
    full = full.reshape(rows, blocks, 32)
    amax = np.abs(full).max(-1)                                         # NaN where a block holds one
    bad = ~np.isfinite(amax)
    _, e = np.frexp(np.where(bad, 1.0, amax))                           # amax = m 2^e, m in [1/2, 1)
    s = np.where(amax == 0, 0, np.maximum(e - 1 + 125, 0))
    s = np.where(bad, 255, s)
    with np.errstate(invalid="ignore", over="ignore"):
        y = np.abs(full) * np.ldexp(1.0, 127 - np.where(bad, 127, s))[..., None]
        y = np.where(bad[..., None], 0.0, y)
    gap = np.abs(np.minimum(y, 6.0)[..., None] - LEVELS)                # to the nearest level, ties to the even one
    order = np.where(np.arange(8) % 2 == 0, 0, 1)
    best = gap.min(-1, keepdims=True)
    code = np.where(gap == best, order, 2).argmin(-1)
    code = np.where(bad[..., None], 0, code | (np.signbit(full) << 3)).reshape(rows, -1)
    scales = np.zeros((rows, pitches(cols)[1]), np.uint8)
    scales[:, :blocks] = s
    return (code[:, ::2] | (code[:, 1::2] << 4)).astype(np.uint8), scales


def decode(codes, scales, cols):
    codes = np.asarray(codes)
    code = np.stack((codes & 15, codes >> 4), -1).reshape(codes.shape[0], -1, 32)
    s = np.asarray(scales)[:, : code.shape[1]].astype(np.int64)
    v = np.where(code & 8, -1.0, 1.0) * LEVELS[code & 7] * np.where(s == 255, np.nan, np.ldexp(1.0, s - 127))[..., None]
    return v.reshape(codes.shape[0], -1)[:, :cols]


def erf(z):
    return np.vectorize(math.erf, otypes=[float])(z)


def act(z, kind):
    if kind == "erf":
        return 0.5 * z * (1 + erf(z * math.sqrt(0.5)))
    if kind == "tanh":
        return 0.5 * z * (1 + np.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    return z


def product(a, w, offsets, bias=None):
    """z [rows, N] of the groups' rows in 64 bits and the sum of the magnitudes that went into each; NaN in rows of no expert."""
    z = np.full((a.shape[0], w.shape[1]), np.nan)
    size = np.zeros_like(z)
    for e in range(w.shape[0]):
        r = slice(int(offsets[e]), int(offsets[e + 1]))
        z[r] = a[r] @ w[e].T
        size[r] = np.abs(a[r]) @ np.abs(w[e]).T
        if bias is not None:
            z[r] += bias[e]
            size[r] += np.abs(bias[e])
    return z, size


def check_product(got, z, size, K, dtype, kind="none"):
    """Sums of K exact products in fp32, each of the K additions and the bias's off by at most a whole step (2^-23) of what has gathered,
    which is at most `size`.  GeLU's slope is below 1.13 and its evaluation in fp32 off by at most 2^-20 of |z|; one rounding at the end."""
    want = act(z, kind)
    d = (K + 2) * 2.0 ** -23 * size
    if kind != "none":
        d = 1.13 * d + 2.0 ** -20 * np.abs(z)
    err = np.abs(got - want)
    bound = d + S.HALF_STEP[dtype] * (np.abs(want) + d) + S.TINY[dtype]
    inside = ~np.isnan(z)
    assert (err[inside] <= bound[inside]).all(), float((err - bound)[inside].max())


def form(rows, N, K, E, sms, four_bits=False, gelu=False):
    """How the product cuts its work: rows of a tile and its columns of C (clusters, which are for fewer tiles than CTAs, aside)."""
    mean = rows // E
    if mean <= 90:
        return (32 if mean <= 2 else 64 if mean <= 20 else 128), 128
    tiles, epilogue, stages = rows / 192 + 0.5 * E, 7000 if four_bits else 5200 if gelu else 2700, -(-K // 256)
    rounds = lambda cols: math.ceil(tiles * -(-N // cols) / sms)
    wide = rounds(256) * (stages * 1028 + 2 * epilogue + 1500) < rounds(128) * max(stages * 775 + 700, epilogue + 1100)
    return 192, 256 if wide else 128


def tiles(offsets, N, row_tile, columns):
    return sum(-(-int(n) // row_tile) for n in np.diff(offsets)) * -(-N // columns)
