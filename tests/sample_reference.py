"""Plain definition of the drawing of tokens, one row at a time on the CPU, with
weights in extended precision."""
import math

import numpy as np


def weight_bits(vocab):
    """Weights are whole multiples of 2^-bits."""
    return min(50, 62 - max(vocab - 1, 0).bit_length())


def draw(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(the tokens that may be drawn, {token: log of its share}): more than one token
    only where u lies at a border between two, or a cut of top_p or min_p at one
    between two tokens, as near as the rounding of all weights may move it (half of
    2^-bits a token; at 50 bits two roundings of binary64 more)."""
    x = np.asarray(logits, dtype=np.float64)
    x = np.where(np.isnan(x), -np.inf, x)
    live = x > -np.inf
    if not live.any():
        return {-1}, {-1: math.nan}
    top = x.max()
    if temperature == 0:
        first = int(np.argmax(x))
        return {first}, {first: 0.0}
    near = np.where(x == top, 0.0, x - top) if math.isfinite(top) else np.where(x == top, 0.0, -np.inf)
    if math.isinf(temperature):
        near = np.where(near > -np.inf, 0.0, near)
        temperature = 1.0
    w = np.where(live, np.exp(near.astype(np.longdouble) / np.longdouble(temperature)), 0)
    slack = len(x) * (2.0 ** -(weight_bits(len(x)) + 1) + 2.0 ** -50)
    order = np.lexsort((np.arange(len(x)), -x))
    order = order[live[order]]
    if 0 < top_k < len(order):
        order = order[:top_k]
    cum = np.cumsum(w[order])
    lengths = {len(order)}
    if top_p < 1.0:
        limit = np.longdouble(top_p) * cum[-1]
        before = np.concatenate([[np.longdouble(0)], cum[:-1]])
        lengths = {max(1, int((before < limit - slack).sum())), max(1, int((before < limit + slack).sum()))}
    found, share = set(), {}
    for length in lengths:
        ends = {length}
        if min_p > 0.0:
            kept = w[order[:length]]
            ends = {max(1, int((kept >= min_p * (1 - 1e-12)).sum())), max(1, int((kept >= min_p * (1 + 1e-12)).sum()))}
        for end in ends:
            kept = np.sort(order[:end])
            run = np.cumsum(w[kept])
            target = np.longdouble(min(max(u, 0.0), 1.0 - 2.0 ** -24) if u == u else 0.0) * run[-1]
            for t in (target - slack, target, target + slack):
                at = min(int((run <= t).sum()), len(kept) - 1)
                token = int(kept[at])
                found.add(token)
                share[token] = float(np.log(w[token] / run[-1])) if w[token] > 0 else -math.inf
    return found, share
