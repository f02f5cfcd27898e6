"""Tokens sorted by expert, restated in numpy from the definition (64 bits), and what fp32 sums and one rounding may differ from it."""
import numpy as np
import torch

HALF_STEP = {t: torch.finfo(t).eps / 2 for t in (torch.float32, torch.bfloat16)}      # the most one rounding is off, relative
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133}                      # and below the normal range


def plan(choice, E):
    """offsets, order (the m rows) and place of int32 choices [n, K]."""
    flat = np.asarray(choice).reshape(-1)
    lists = [np.flatnonzero(flat == e) for e in range(E)]
    order = np.concatenate(lists) if lists else np.zeros(0, np.int64)
    offsets = np.concatenate([[0], np.cumsum([len(x) for x in lists])])
    place = np.full(flat.shape, -1, np.int64)
    place[order] = np.arange(len(order))
    return offsets, order, place.reshape(choice.shape)


def rows_of(rows, place):
    """[n, K, d] in 64 bits: the rows of each token's choices, zeros where there is none."""
    rows = rows.detach().cpu().double().numpy()
    got = rows[np.maximum(place, 0)]
    return np.where(place[..., None] >= 0, got, 0.0)


def combine(Y, weights, place):
    """X_out, and the sum of the magnitudes that went into each of its values."""
    v = rows_of(Y, place)
    w = np.ones(place.shape) if weights is None else np.where(place >= 0, weights.detach().cpu().double().numpy(), 0.0)
    return (w[..., None] * v).sum(1), (np.abs(w)[..., None] * np.abs(v)).sum(1)


def check_sum(got, want, size, terms, dtype):
    """A sum of `terms` products in fp32 (each product and each addition off by at most half a step of what has gathered so far, which
    is at most `size`), rounded once to dtype."""
    err = np.abs(got.detach().cpu().double().numpy() - want)
    bound = (2 * terms + 2) * 2.0 ** -24 * size + HALF_STEP[dtype] * (np.abs(want) + (2 * terms + 2) * 2.0 ** -24 * size) + TINY[dtype]
    assert (err <= bound).all(), float((err - bound).max())
