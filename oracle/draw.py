"""Tokens of rows of logits from given uniform numbers, with temperature, top-k, top-p and min-p: in whole numbers.

The weights are those of the sampling contract, rint(exp32(l' - max l') 2^40); everything after them is
integer arithmetic of any width."""
import math

import numpy as np

from .sampler import F32, exp32

TWO24, TWO40 = 1 << 24, 1 << 40


def _ceil(x, scale, low, high):
    """ceil(x scale) in [low, high], x a float."""
    x = float(x)
    if not x * scale < high:  # NaN and infinities too
        return high
    return max(math.ceil(x * scale), low)


def kept(logits, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """{id: weight} of the entries that a row's settings (float32 numbers) leave, in the order of the ids."""
    temperature, top_p, min_p = F32(temperature), F32(top_p), F32(min_p)
    x = np.asarray(logits, dtype=F32)
    with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
        if temperature > 0:
            x = x * (F32(1) / temperature)
        else:
            top_k = 1
        at = np.flatnonzero(x > -np.inf)
        if at.size == 0:
            return {}
        x = x[at]
        y = np.where(x == x.max(), F32(0), x - x.max())
        q = np.rint(exp32(np.maximum(y, F32(-31))).astype(np.float64) * TWO40).astype(np.int64)
    order = np.argsort(-x, kind="stable")
    if 0 < top_k < np.asarray(logits).size:
        order = order[:top_k]
    mark = -(-_ceil(top_p, TWO24, 1, TWO24) * sum(int(q[i]) for i in order) // TWO24)
    prefix, run = [], 0
    for i in order:
        if run >= mark:
            break
        prefix.append(i)
        run += int(q[i])
    least = _ceil(min_p, TWO40, 0, TWO40) if min_p > 0 else 0
    return {int(at[i]): int(q[i]) for i in sorted(prefix) if q[i] >= least and q[i] > 0}


def draw(logits, u, **settings):
    """(token, log-probability) of one row; (-1, -inf) where there is nothing to draw from."""
    f = kept(logits, **settings)
    if not f:
        return -1, -math.inf
    total = sum(f.values())
    u = float(u)
    mark = (math.floor(min(u, 1 - 1 / TWO24) * TWO24) if u > 0 else 0) * total // TWO24
    run = 0
    for v, q in f.items():
        run += q
        if run > mark:
            return v, math.log(q / total)
