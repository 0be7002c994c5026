"""The serving operators in plain 64-bit numpy, from the definitions in include/dvm_serving.h, and their error bounds."""
from __future__ import annotations

import numpy as np
import torch

EPS = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}   # half a step, relative to the value


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def paging(cached, fresh, free, table, page, rows):
    n, width = table.shape
    table = table.copy()
    starts, lengths = np.zeros(n + 1, np.int64), np.zeros(n, np.int64)
    pos, slots = np.full(rows, -1, np.int64), np.full(rows, -1, np.int64)
    k = t = 0
    for i in range(n):
        c, f = max(int(cached[i]), 0), max(int(fresh[i]), 0)
        f = min(f, rows - t)
        starts[i], lengths[i] = t, min(c + f, 2 ** 31 - 1)
        for b in range(-(-c // page), min(-(-int(lengths[i]) // page), width)):
            table[i, b] = free[k] if k < len(free) else -1
            k += 1
        for j in range(f):
            p = min(c + j, 2 ** 31 - 1)
            pos[t] = p
            if p // page < width and table[i, p // page] >= 0:
                slots[t] = table[i, p // page] * page + p % page
            t += 1
    starts[n] = t
    return {"table": table, "starts": starts, "lengths": lengths, "positions": pos, "slots": slots, "taken": np.array([k])}


def turn_head(x, weight, row, rot, eps, interleaved):
    """One head in 64 bits: (value, sum of the magnitudes that went into it)."""
    x = x.astype(np.float64)
    if weight is not None:
        x = x / np.sqrt(np.mean(x * x) + eps) * weight
    y, mag, half = x.copy(), np.abs(x), rot // 2
    for k in range(half):
        i, j = (2 * k, 2 * k + 1) if interleaved else (k, k + half)
        c, s = row[k], row[half + k]
        y[i], y[j] = x[i] * c - x[j] * s, x[j] * c + x[i] * s
        mag[i], mag[j] = abs(x[i] * c) + abs(x[j] * s), abs(x[j] * c) + abs(x[i] * s)
    return y, mag


def attention(q, k, v, table, starts, lengths, scale, window, sinks, max_q=1 << 30):
    """(values, bound weights A = sum p |v|, score magnitudes, seen, row written) of every row and head."""
    rows, hq, d = q.shape
    pages, page, hk, _ = k.shape
    n, width = table.shape
    out, mag = np.zeros((rows, hq, d)), np.zeros((rows, hq, d))
    size, written, seen_n = np.zeros((rows, hq)), np.zeros(rows, bool), np.zeros(rows, np.int64)
    for i in range(n):
        s0 = min(max(int(starts[i]), 0), rows)
        s1 = min(max(int(starts[i + 1]), s0), rows)
        for t in range(s0, min(s1, s0 + max_q)):
            written[t] = True
            p = int(lengths[i]) - (s1 - s0) + (t - s0)
            s = np.arange(0, max(0, min(p + 1, width * page)))
            if window:
                s = s[(s > p - window) | (s < sinks)]
            ids = table[i, s // page] if s.size else s
            s, ids = s[(ids >= 0) & (ids < pages)], ids[(ids >= 0) & (ids < pages)]
            seen_n[t] = s.size
            if not s.size:
                continue
            kk, vv = k[ids, s % page], v[ids, s % page]     # [seen, hk, d]
            for h in range(hq):
                g = h // (hq // hk)
                z = kk[:, g] @ q[t, h] * scale
                with np.errstate(invalid="ignore"):
                    w = np.exp(z - z.max())
                w = w / w.sum()
                out[t, h], mag[t, h] = w @ vv[:, g], w @ np.abs(vv[:, g])
                size[t, h] = (np.abs(kk[:, g]) @ np.abs(q[t, h]) * scale).max()
    return out, mag, size, written, seen_n


def attention_bound(out, mag, size, seen_n, d, out_dtype, tensor_cores):
    """Largest error allowed: the stored value's rounding; each weight's rounding to bf16 for the second product (tensor
    cores); its error from the score, an fp32 sum of d products of size `size` in all (d + 8 roundings: products, the
    scale, the maximum) and from exp2 (2 ulp), in the weight and in the weights' sum; the fp32 sums over the tokens."""
    delta = (d + 8) * 2.0 ** -24 * np.maximum(size, 1.0)[..., None] + 2.0 ** -21
    n = seen_n[:, None, None] + 8.0
    return EPS[out_dtype] * np.abs(out) + ((2.0 ** -8 if tensor_cores else 0.0) + 2 * delta + 2 * n * 2.0 ** -24) * mag * (1 + EPS[out_dtype])
