"""A language model's steps between two linear layers, in 64 bits on the host, from their definitions in the header."""
import math

import numpy as np

BLOCK = 64
# the largest relative error of one rounding
UNIT_ROUNDOFF = {"float32": 2.0 ** -24, "float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}


def code_places(head_dim):
    """(keys, values): the offset of the code of (token, channel) within a page's codes of one head"""
    m = -(-head_dim // 16)
    t, d = np.arange(BLOCK)[:, None], np.arange(head_dim)[None, :]
    keys = ((t // 16) * m + d // 16) * 256 + (t % 16) * 16 + d % 16
    values = BLOCK * 16 * m + (d // 16) * 1024 + ((t % 16) // 4) * 256 + (d % 16) * 16 + (t // 16) * 4 + t % 4
    return keys, values


def head_bytes(head_dim):
    return 2 * BLOCK * 16 * (-(-head_dim // 16))


def centred(x, p, unit):
    x = np.asarray(x).astype(np.int64)
    return np.where(x > p // 2, x - p, x).astype(np.float64) * unit


def rotate(x, table, positions, interleaved):
    """x (rows, heads, head_dim) at `positions`; table (positions, rot_dim/2, 2)"""
    x = np.array(x, np.float64)
    rot = 2 * table.shape[1]
    first = np.arange(0, rot, 2) if interleaved else np.arange(rot // 2)
    second = first + (1 if interleaved else rot // 2)
    out = x.copy()
    for r, t in enumerate(positions):
        if not 0 <= t < table.shape[0]:
            out[r] = np.nan
            continue
        c, s = table[t, :, 0].astype(np.float64), table[t, :, 1].astype(np.float64)
        out[r][:, first] = x[r][:, first] * c - x[r][:, second] * s
        out[r][:, second] = x[r][:, second] * c + x[r][:, first] * s
    return out


def see(position, length, window, sinks):
    j = np.arange(length)
    seen = j <= position
    if window:
        seen &= (j > position - window) | (j < sinks)
    return seen


def attention(q, k, v, seen, scale, q_bits, w_bits):
    """One query head: (out, bound).  q (dim), k and v (tokens, dim) as the cache stands for them, seen (tokens).  The bound
    follows from what enters the products: queries as whole numbers of q_bits bits of the row's largest (sign and q_bits - 1),
    weights rounded at 2^-w_bits of the largest weight so far, exponents and sums in 32 bits."""
    dim = len(q)
    if not seen.any():
        return np.zeros(dim), np.zeros(dim)
    k, v = k[seen], v[seen]
    s = scale * (k @ q)
    w = np.exp(s - s.max())
    out = (w[:, None] * v).sum(0) / w.sum()
    # of a score: half a step of every channel of the query, and 32-bit roundings of a product of that size
    slack = abs(scale) * np.abs(k).sum(1) * np.abs(q).max() * 2.0 ** -(q_bits - 1) + 2.0 ** -20 * (np.abs(s) + abs(scale) * (np.abs(k) @ np.abs(q)) + np.abs(s).max() + 1)
    rel = np.expm1(2 * slack.max())
    spread = (w[:, None] * np.abs(v)).sum(0) / w.sum()
    bound = 2 * rel * spread + 2 * 2.0 ** -w_bits * np.abs(v).sum(0) / w.sum() + 2.0 ** -18 * spread
    # the weights' own sum is rounded as they are
    bound += 2 * 2.0 ** -w_bits * len(w) / w.sum() * np.abs(out)
    return out, bound


def kept_tokens(z, temperature, top_k, top_p, min_p):
    """(kept (tokens) by index, weights, the least distance of a cut from the next token's edge, as a share of all weight)"""
    z = np.asarray(z, np.float64)
    n = len(z)
    order = np.argsort(-np.where(np.isnan(z), -np.inf, z), kind="stable")
    top = z[order[0]]
    with np.errstate(invalid="ignore"):
        w = np.where(z == top, 1.0, np.exp((z - top) / (temperature if temperature > 0 else 1.0)))
    w = np.where(np.isnan(w), 0.0, w)
    most = 1 if temperature <= 0 else top_k if top_k > 0 else n
    rank = np.empty(n, np.int64)
    rank[order] = np.arange(n)
    kept = rank < most
    margin = math.inf
    if top_p < 1:
        held = w[order] * kept[order]
        before = np.cumsum(held) - held
        edge = top_p * held.sum()
        cut = before < edge
        # nothing lies before the first token, in any precision
        margin = np.abs(before - edge)[0 if edge > 0 else 1:].min(initial=math.inf) / held.sum()
        kept[order] &= cut
    if min_p > 0:
        margin = min(margin, np.abs(w / min(min_p, 1.0) - 1)[w < 1].min() if (w < 1).any() else math.inf)
        kept &= w >= min(min_p, 1.0)
    kept[order[0]] = True
    return kept, w, margin


def attention_in_halves(q, k, v, scales, seen, scale):
    """The same with queries of 16 bits and weights in half precision: each weight times its block's scale of values (`scales`, a
    token each) rounded to 11 bits, or to 2^-25 of the largest of them where that is more; sums in 32 bits."""
    dim = len(q)
    if not seen.any():
        return np.zeros(dim), np.zeros(dim)
    k, v, scales = k[seen], v[seen], scales[seen]
    s = scale * (k @ q)
    w = np.exp(s - s.max())
    out = (w[:, None] * v).sum(0) / w.sum()
    slack = abs(scale) * np.abs(k).sum(1) * np.abs(q).max() * 2.0 ** -15 + 2.0 ** -20 * (np.abs(s) + abs(scale) * (np.abs(k) @ np.abs(q)) + np.abs(s).max() + 1)
    rel = np.expm1(2 * slack.max()) + 2.0 ** -11
    spread = (w[:, None] * np.abs(v)).sum(0) / w.sum()
    return out, 2 * rel * spread + len(w) * 127 * 2.0 ** -25 * (w * scales).max() / w.sum() + 2.0 ** -18 * spread
