"""The operators on KV caches (include/rserve_attend.h) in 64 bits, from their definitions, one row at a time.

Test infrastructure: shares no code with the library.  Arrays are numpy; what a cache holds is handed over as
the numbers its elements stand for, [tokens, KV heads, d].
"""
from __future__ import annotations

import math

import numpy as np

LIMIT = 2.0 ** 100


# ------------------------------------------------------------------------------------------------ rotary positions
def rotary_frequencies(rotary_dim, theta, scaling="none", factor=1.0, original_max_pos=0, fast_turns=0.0, slow_turns=0.0):
    """f_j of every pair."""
    out = []
    for j in range(rotary_dim // 2):
        f = theta ** (-2.0 * j / rotary_dim)
        if scaling == "linear":
            f = f / factor
        elif scaling == "ramp":
            fast, slow = fast_turns or 32.0, slow_turns or 1.0
            # the pair that turns t times over the original context: original f / (2 pi) = t
            pair = [rotary_dim * math.log(original_max_pos / (t * 2 * math.pi)) / (2 * math.log(theta)) for t in (fast, slow)]
            low, high = max(math.floor(pair[0]), 0), min(math.ceil(pair[1]), rotary_dim - 1)
            share = (j - low) / max(high - low, 1e-3)
            share = 0.0 if share < 0 else 1.0 if share > 1 else share
            f = (1 - share) * f + share * f / factor
        elif scaling == "bands":
            fast, slow = fast_turns or 4.0, slow_turns or 1.0
            turns = original_max_pos * f / (2 * math.pi)
            if turns <= slow:
                f = f / factor
            elif turns < fast:
                s = (turns - slow) / (fast - slow)
                f = (1 - s) * f / factor + s * f
        out.append(f)
    return np.array(out)


def rotary_magnitude(scaling="none", factor=1.0, magnitude=0.0):
    return magnitude if magnitude else 0.1 * math.log(factor) + 1.0 if scaling == "ramp" else 1.0


def rotate(x, positions, rotary_dim, frequencies, layout="halves", magnitude=1.0):
    """[rows, heads, d] with the first rotary_dim features turned by the rows' positions."""
    y = np.array(x, dtype=np.float64)
    half = rotary_dim // 2
    for j in range(half):
        a, b = (j, j + half) if layout == "halves" else (2 * j, 2 * j + 1)
        angle = np.asarray(positions, dtype=np.float64)[:, None] * frequencies[j]
        c, s = np.cos(angle) * magnitude, np.sin(angle) * magnitude
        u, v = np.array(x[..., a], dtype=np.float64), np.array(x[..., b], dtype=np.float64)
        y[..., a], y[..., b] = u * c - v * s, v * c + u * s
    return y


# ------------------------------------------------------------------------------------------------ attention
def attend_row(q, k, v, scale):
    """One head's query [d] over keys and values [n, d]; returns (output, sum of weights times magnitudes of the values).  What is
    not in k and v does not take part."""
    with np.errstate(invalid="ignore", over="ignore"):
        s = k.astype(np.float64) @ q.astype(np.float64) * scale
        w = np.exp(s - s.max())
        w = w / w.sum()
        return w @ v.astype(np.float64), w @ np.abs(v.astype(np.float64))


def attend(q, k, v, first, scale=None, allowed=None):
    """Queries [T, Hq, d] at slots first .. first + T - 1 over keys and values [n, Hkv, d]: (out, magnitudes), both [T, Hq, d].
    allowed(t, KV head): the slots that are seen among those up to the query's own (None: all)."""
    t_n, hq, d = q.shape
    hkv = k.shape[1]
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    out, mag = np.empty(q.shape), np.empty(q.shape)
    for t in range(t_n):
        for h in range(hkv):
            seen = np.arange(first + t + 1)
            if allowed is not None:
                seen = seen[allowed(t, h)[: first + t + 1]]
            for i in range(hq // hkv):
                head = h * (hq // hkv) + i
                out[t, head], mag[t, head] = attend_row(q[t, head], k[seen, h], v[seen, h], scale)
    return out, mag


# ------------------------------------------------------------------------------------------------ bounds and selection
def _limited(x):
    x = np.asarray(x, dtype=np.float64)
    return np.where(np.isnan(x), 0.0, np.clip(x, -LIMIT, LIMIT))


def _unit_exponent(top):
    """The smallest e >= -100 with top <= 127 * 2^e."""
    e = -100
    while top > 127 * 2.0 ** e:
        e += 1
    return e


def block_bounds(k):
    """Keys [64, d] of one block and head: (high codes, low codes, unit)."""
    k = _limited(k)
    high, low = k.max(0), k.min(0)
    unit = 2.0 ** _unit_exponent(max(np.abs(high).max(), np.abs(low).max()))
    return np.ceil(high / unit).astype(np.int64), np.floor(low / unit).astype(np.int64), unit


def query_codes(q):
    """The g heads' queries [g, d] of one token and KV head: (p, n)."""
    g = q.shape[0]
    q = _limited(q)
    codes = np.rint(q / 2.0 ** _unit_exponent(np.abs(q).max())).astype(np.int64)
    halvings = math.ceil(math.log2(g)) if g > 1 else 0
    half = 2 ** halvings // 2
    p = (np.maximum(codes, 0).sum(0) + half) // 2 ** halvings
    n = -((np.maximum(-codes, 0).sum(0) + half) // 2 ** halvings)
    return p, n


def select_blocks(q, bounds, slot, n_blocks, n_first, n_last):
    """Blocks that the token at `slot` attends to, ascending.  q [g, d]; bounds: (high, low, unit) of every finished block."""
    own = slot // 64
    forced = [b for b in range(own + 1) if b < n_first or b > own - n_last]
    rest = [b for b in range(own + 1) if b not in forced]
    take = forced[:n_blocks]
    if rest and len(take) < n_blocks:
        p, n = query_codes(q)
        score = {b: float(int((p * bounds[b][0] + n * bounds[b][1]).sum())) * bounds[b][2] for b in rest}
        take += sorted(rest, key=lambda b: (-score[b], b))[: n_blocks - len(take)]
    return sorted(take)
