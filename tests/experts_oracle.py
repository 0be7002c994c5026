"""The operators of a layer of experts in plain 64-bit numpy, from the definitions in include/dvm_experts.h, and their error bounds."""
from __future__ import annotations

import numpy as np
import torch

EPS = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}   # half a step, relative to the value
BLOCK = 128


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def e4m3_values():
    """Value of every code 0 .. 126 (the positive ones; 127 is NaN): 4 bits of exponent (bias 7), 3 of mantissa."""
    c = np.arange(127)
    e, m = c >> 3, c & 7
    return np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))


def decode(codes):
    """fp64 values of uint8 codes."""
    table = np.append(e4m3_values(), np.nan)
    codes = np.asarray(codes)
    return np.where(codes & 0x80, -1.0, 1.0) * table[codes & 0x7f]


def encode(v):
    """The codes nearest to v, of two the even one; beyond the largest value the largest."""
    table = e4m3_values()
    m = np.minimum(np.abs(v), 448.0)
    hi = np.clip(np.searchsorted(table, m), 1, 126)
    up = (m - table[hi - 1]) - (table[hi] - m)      # exact for 24-bit values near the border; the tests' quotients are rounded to 53 bits
    at = np.where((up > 0) | ((up == 0) & (hi % 2 == 0)), hi, hi - 1)
    return (at | np.where(np.signbit(v), 0x80, 0)).astype(np.uint8)


def routing(logits, top_k, scoring, bias, groups, top_groups, renormalise, factor, positions):
    """ids, weights, places [tokens, top_k], starts [experts + 1]."""
    t, e = logits.shape
    ids, weights, places = np.full((t, top_k), -1), np.zeros((t, top_k)), np.full((t, top_k), -1)
    for i in range(t):
        if positions is not None and positions[i] < 0:
            continue
        z = logits[i]
        with np.errstate(over="ignore", invalid="ignore"):
            if scoring == "softmax":
                p = np.exp(z - (z.max() if not np.isnan(z).any() else np.nan))
                s = p / p.sum()
            else:
                s = 1.0 / (1.0 + np.exp(-z))
        c = s + bias if bias is not None else s
        rank = c if bias is not None else z   # without a bias the order of the scores is that of the logits, ties included
        allowed = np.ones(e, bool)
        if groups > 1:
            of = c.reshape(groups, -1)
            top = np.sort(of, 1)[:, ::-1][:, :2].sum(1)
            keep = np.lexsort((np.arange(groups), np.where(np.isnan(top), np.inf, -top), np.isnan(top)))[:top_groups]
            allowed = np.isin(np.arange(e) // (e // groups), keep)
        order = np.lexsort((np.arange(e), np.where(np.isnan(rank), np.inf, -rank), np.isnan(rank), ~allowed))[:top_k]
        ids[i] = order
        w = s[order]
        weights[i] = (w / w.sum() if renormalise else w) * factor
    counts = np.bincount(ids[ids >= 0], minlength=e)
    starts = np.concatenate([[0], np.cumsum(counts)])
    at = starts[:-1].copy()
    for i in range(t):
        for j in range(top_k):
            if ids[i, j] >= 0:
                places[i, j] = at[ids[i, j]]
                at[ids[i, j]] += 1
    return ids, weights, places, starts


def weights_bound(experts):
    """Relative error of a weight: the exponentials' (2 ulp each and their arguments' rounding, |x| 2^-24 with |x| below 30 in the
    tests), their sum (a rounding per addition at most), quotients and the factor (4 roundings)."""
    return (experts + 4 + 2 * 30 + 4 + 6) * 2.0 ** -24


def scale_of(top):
    """fp32 scales of blocks whose largest magnitudes are `top` (fp32 values): the quotient of two fp32 values in 64 bits rounds to
    fp32 as the exact one does (53 bits are more than 2 x 24 + 2)."""
    return np.maximum((top / 448.0).astype(np.float32), np.float32(2.0 ** -126)).astype(np.float64)


def quantize(v, block_rows=1):
    """codes and scales of v [rows, cols] (fp32 values in 64 bits)."""
    rows, cols = v.shape
    kb, rb = -(-cols // BLOCK), -(-rows // block_rows)
    full = np.zeros((rb * block_rows, kb * BLOCK))
    full[:rows, :cols] = v
    blocks = full.reshape(rb, block_rows, kb, BLOCK)
    bad = ~np.isfinite(blocks).all((1, 3))
    with np.errstate(invalid="ignore"):
        scales = np.where(bad, np.nan, scale_of(np.abs(blocks).max((1, 3))))
    wide = np.where(bad, 1.0, scales)[:, None, :, None]
    codes = encode(np.where(bad[:, None, :, None], 0.0, blocks) / wide).reshape(rb * block_rows, kb * BLOCK)[:rows, :cols]
    return codes, scales


def scaled_bound(exact, magnitude, k_blocks, dtype):
    """Largest error allowed of a scaled product with `magnitude` = the sum of the magnitudes of all its terms: 128 additions of a block
    on the tensor cores, each off by at most 2^-23 of the block's magnitude; the scales' product and each block's multiply-add (or
    the join's addition) a rounding of at most everything so far; the stored value's rounding."""
    fp32 = magnitude * (128 * 2.0 ** -23 + (2 * k_blocks + 2) * 2.0 ** -24)
    return fp32 + EPS[dtype] * (np.abs(exact) + fp32)


def combine(y, places, weights, base):
    """values, magnitudes and whether a token has any row."""
    tokens, k = places.shape
    out = np.zeros((tokens, y.shape[1])) if base is None else base.copy()
    mag, any_row = np.abs(out), np.zeros(tokens, bool)
    for t in range(tokens):
        for j in range(k):
            if 0 <= places[t, j] < y.shape[0]:
                out[t] = out[t] + weights[t, j] * y[places[t, j]]
                mag[t] = mag[t] + np.abs(weights[t, j] * y[places[t, j]])
                any_row[t] = True
    return out, mag, any_row


def combine_bound(exact, magnitude, k, dtype):
    """A rounding of at most everything per multiply-add, and the stored value's."""
    fp32 = magnitude * (k + 1) * 2.0 ** -24
    return fp32 + EPS[dtype] * (np.abs(exact) + fp32)
