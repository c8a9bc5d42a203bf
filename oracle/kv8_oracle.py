"""CPU fp64 reference of rotary positions and of the 8-bit paged cache (test infrastructure).

Plain numpy, one page, one head, one query at a time; every quantity from its definition.  States are dicts of
arrays: codes [pages, H, 64, d] and scale [pages, H] for keys and values, sums [batch, H, blocks, d] or None.
"""
from __future__ import annotations

import math

import numpy as np

BLOCK = 64
TOP = 448.0            # largest e4m3 value
SCALE_MIN = -48
STORED_MAX = 2.0 ** 60


# ------------------------------------------------------------------ positions
def frequencies(pairs, base, scaling="none", factor=1.0, trained=4096.0, fast=32.0, slow=1.0):
    """Radians per position of every pair and the amplitude (in 80 bits: positions near 2^31 leave fp64 angles 2^-22 off)."""
    out, wide = [], np.longdouble
    for n in pairs:
        b = wide(base) * wide(factor) ** (wide(n) / (n - 1)) if scaling == "base" and n > 1 else wide(base)
        for i in range(n):
            f = b ** (-wide(i) / n)
            if scaling == "linear":
                f /= factor
            elif scaling == "bands":
                turns = trained * f / (2 * math.pi)
                keep = min(1.0, max(0.0, (turns - slow) / (fast - slow)))
                f *= keep + (1 - keep) / factor
            out.append(f)
    return np.array(out, dtype=wide), (0.1 * math.log(factor) + 1.0 if scaling == "bands" else 1.0)


def rope(x, positions, pairs, freq, amplitude=1.0, layout="half", transpose=False):
    """x [tokens, H, d]; positions [axes, tokens] whole numbers."""
    x = np.asarray(x, dtype=np.float64)
    y = x.copy()
    half = sum(pairs)
    axis = np.repeat(np.arange(len(pairs)), pairs)
    for p in range(half):
        angle = np.asarray(positions[axis[p]]).astype(np.longdouble) * freq[p]
        c, s = np.cos(angle).astype(np.float64)[:, None], np.sin(angle).astype(np.float64)[:, None]
        s = -s if transpose else s
        i, j = (p, p + half) if layout == "half" else (2 * p, 2 * p + 1)
        y[:, :, i] = amplitude * (x[:, :, i] * c - x[:, :, j] * s)
        y[:, :, j] = amplitude * (x[:, :, j] * c + x[:, :, i] * s)
    return y


# ------------------------------------------------------------------ e4m3
def e4m3(x):
    """Nearest e4m3 value, ties to even, of |x| <= 448."""
    x = np.asarray(x, dtype=np.float64)
    _, e = np.frexp(x)                       # |x| = m 2^e, 0.5 <= m < 1
    step = np.ldexp(1.0, np.maximum(e - 1, -6) - 3)
    return np.rint(x / step) * step


def scale_of(top):
    s = SCALE_MIN
    while top > TOP * 2.0 ** s:
        s += 1
    return 2.0 ** s


def storable(x):
    x = np.asarray(x, dtype=np.float64)
    return np.clip(np.where(np.isnan(x), 0.0, x), -STORED_MAX, STORED_MAX)


def append(state, table, held, rows_k, rows_v):
    """Appends rows_k[s], rows_v[s] ([n, H, d], keys already rotated) of every sequence s in place."""
    for s, n0 in enumerate(held):
        n = len(rows_k[s])
        if n == 0:
            continue
        for blk in range(n0 // BLOCK, (n0 + n - 1) // BLOCK + 1):
            lo, hi = max(n0, blk * BLOCK), min(n0 + n, (blk + 1) * BLOCK)
            r0, r1, page = lo - blk * BLOCK, hi - blk * BLOCK, table[s][blk]
            for name, rows in (("k", rows_k[s]), ("v", rows_v[s])):
                for h in range(rows.shape[1]):
                    x = storable(rows[lo - n0:hi - n0, h])
                    codes, scale = state[name + "_codes"][page, h], state[name + "_scale"]
                    new = scale_of(np.abs(x).max())
                    if r0:
                        new = max(new, scale[page, h])
                        codes[:] = e4m3(codes * (scale[page, h] / new))
                    else:
                        codes[:] = 0.0
                    codes[r0:r1] = e4m3(x / new)
                    scale[page, h] = new
                    if name == "k" and state.get("sums") is not None:
                        state["sums"][s, h, blk] = x.sum(0) + codes[:r0].sum(0) * new


# ------------------------------------------------------------------ attention
def attend(q, state, table, lengths, causal, scale=None, sel=None):
    """q: list of [n, Hq, d] per sequence; sel[s][kv head]: block ids, or None.  Returns per sequence (out, lse, spread,
    size), the last two by which rounding errors are measured: the weighted mean of |v| and the sum of |v| over the keys."""
    Hkv, d = state["k_scale"].shape[1], state["k_codes"].shape[-1]
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    res = []
    for s, length in enumerate(lengths):
        x = np.asarray(q[s], dtype=np.float64)
        n, Hq = x.shape[0], x.shape[1]
        out, spread, size = np.zeros((n, Hq, d)), np.zeros((n, Hq, d)), np.zeros((n, Hq, d))
        lse = np.full((n, Hq), -np.inf)
        for h in range(Hkv):
            blocks = list(range((length + BLOCK - 1) // BLOCK)) if sel is None else [int(b) for b in sel[s][h]]
            blocks = [b for b in blocks if b * BLOCK < length]
            if not blocks:
                continue
            page = [table[s][b] for b in blocks]
            k = (state["k_codes"][page, h] * state["k_scale"][page, h][:, None, None]).reshape(-1, d)
            v = (state["v_codes"][page, h] * state["v_scale"][page, h][:, None, None]).reshape(-1, d)
            at = (np.array(blocks)[:, None] * BLOCK + np.arange(BLOCK)).reshape(-1)
            for r in range(h * (Hq // Hkv), (h + 1) * (Hq // Hkv)):
                for i in range(n):
                    see = at < (min(length, length - n + i + 1) if causal else length)
                    if not see.any():
                        continue
                    y = k[see] @ x[i, r] * scale
                    top = y.max()
                    w = np.exp(y - top)
                    total = w.sum()
                    out[i, r] = w @ v[see] / total
                    spread[i, r] = w @ np.abs(v[see]) / total
                    size[i, r] = np.abs(v[see]).sum(0)
                    lse[i, r] = top + math.log(total)
        res.append((out, lse, spread, size))
    return res
