"""What a decode step does between its packed products, in double precision (test
infrastructure only): the residual sum and norm, the 4-bit cache and the attention
over it, and the choice of a token.  The cache's bytes are read from the layout that
include/vbq.h writes down, position by position.
"""

import numpy as np

from . import quant

PAGE = 64


def round_to(v, dtype):
    """Doubles rounded once to 'f32', 'f16' or 'bf16' (nearest even), as doubles."""
    v = np.asarray(v, dtype=np.float64)
    if dtype == "f32":
        return v.astype(np.float32).astype(np.float64)
    if dtype == "f16":
        with np.errstate(over="ignore"):
            return v.astype(np.float16).astype(np.float64)
    m, e = np.frexp(v)  # bf16: eight significant bits
    return np.ldexp(np.rint(np.ldexp(m, 8)), e - 8)


def add_norm(residual, y, weight, eps, res_type):
    """(x before its rounding, h)."""
    h = np.asarray(residual, dtype=np.float64)
    if y is not None:
        # the sum is an fp32 sum, then residual's type
        h = round_to(round_to(h + y, "f32"), res_type)
    x = h / np.sqrt((h * h).mean(axis=-1, keepdims=True) + eps)
    return (x if weight is None else x * weight), h


# ------------------------------------------------------------------ the cache


def kv_quantize(w):
    """(levels, scales) of rows [..., D] in groups of 64 at 4 bits, both double."""
    w = np.asarray(w, dtype=np.float64)
    flat = w.reshape(-1, w.shape[-1])
    q, s = quant.quantize(flat, np.full((flat.shape[0], flat.shape[1] // 64), 4, dtype=np.uint8))
    scales = np.asarray(s, dtype=np.uint16).view(np.float16).astype(np.float64)
    return np.asarray(q, dtype=np.float64).reshape(w.shape), scales.reshape(w.shape[:-1] + (-1,))


def kv_values(w):
    """Rows [..., D] as the cache holds them."""
    q, s = kv_quantize(w)
    return q * np.repeat(s, 64, axis=-1)


def slot(p):
    """Place of position p (of a page) within its 32-position block."""
    return 8 * ((p % 16) // 4) + 4 * ((p % 32) // 16) + p % 4


def page_position(page, head, D, p):
    """(key levels, key scales, value levels, value scales) of one position of a page
    (uint8 bytes), read code by code."""
    at = page[head * 68 * D:(head + 1) * 68 * D]
    words = at[:64 * D].view(np.uint32)
    scales = at[64 * D:].view(np.float16).astype(np.float64)
    keys, values = np.empty(D), np.empty(D)
    for d in range(D):
        j, g, i = d // 32, (d % 32) // 8, d % 8
        lane = 16 * g + p % 16
        per = D // 32
        word = (p // 16) * 64 * per + (lane * 2 + j if D == 64 else (j // 4) * 256 + lane * 4 + j % 4)
        keys[d] = ((int(words[word]) >> (4 * (i // 2) + 16 * (i % 2))) & 15) - 8
        g, i = slot(p) // 8, slot(p) % 8
        lane = 16 * g + d % 16
        word = 8 * D + (p // 32) * 4 * D + (d // 64) * 256 + lane * 4 + (d // 16) % 4
        values[d] = ((int(words[word]) >> (4 * (i // 2) + 16 * (i % 2))) & 15) - 8
    place = 32 * (p // 32) + slot(p)
    groups = D // 64
    ks = np.array([scales[64 * n + place] for n in range(groups)])
    vs = np.array([scales[64 * (groups + n) + place] for n in range(groups)])
    return keys, ks, values, vs


def attention(q, keys, values, scale, length):
    """q [rows, hq, D] over keys, values [positions, hkv, D]; row r sees positions up to
    length - rows + r.  Returns (out, mean |value| by the same weights)."""
    rows, hq, D = q.shape
    hkv = keys.shape[1]
    out, size = np.zeros(q.shape), np.zeros(q.shape)
    for r in range(rows):
        n = length - rows + r + 1
        if n <= 0:
            continue
        for i in range(hq):
            h = i // (hq // hkv)
            s = scale * (keys[:n, h] @ q[r, i])
            w = np.exp(s - s.max())
            out[r, i] = w @ values[:n, h] / w.sum()
            size[r, i] = w @ np.abs(values[:n, h]) / w.sum()
    return out, size


# ------------------------------------------------------------------ sampling


def sample(z, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, probability, distance of u times the total from the nearest step of the
    running sum, as a share of the total) of one row of logits."""
    z = np.asarray(z, dtype=np.float64)
    cand = ~np.isnan(z) & (z > -np.inf)
    if not cand.any():
        return -1, 0.0, 1.0
    idx = np.nonzero(cand)[0]
    order = idx[np.lexsort((idx, -z[idx]))]
    if not temperature > 0:
        return int(order[0]), 1.0, 1.0
    top = z[order[0]]
    if top == np.inf:
        w = (z[order] == np.inf).astype(np.float64)
    else:
        w = np.exp((z[order] - top) / temperature)
    whole = [int(v) for v in np.rint(np.ldexp(w, 43))]
    n = len(order) if top_k <= 0 else min(top_k, len(order))
    if top_p < 1:
        target, run, keep = max(top_p, 0.0) * sum(whole[:n]), 0, 0
        while keep < n and (keep == 0 or run < target):
            run += whole[keep]
            keep += 1
        n = keep
    floor = min(min_p, 1.0) if min_p > 0 else 0.0
    kept = sorted((int(order[i]), whole[i]) for i in range(n) if w[i] >= floor)
    total = sum(k[1] for k in kept)
    want, run, token, share, near = min(max(u, 0.0), 1.0 - 2.0 ** -53) * total, 0, -1, 0.0, total
    for i, wi in kept:
        run += wi
        near = min(near, abs(run - want))
        if token < 0 and wi and run > want:
            token, share = i, wi / total
    return token, share, near / total
