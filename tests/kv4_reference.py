"""The 4-bit cache, positions with several axes and the norm in few bits, on the host, from their definitions in the header."""
import math

import numpy as np

BLOCK = 64
MAGNITUDES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
VALUES = np.concatenate([MAGNITUDES, -MAGNITUDES])           # by code


def groups_of(head_dim):
    return -(-head_dim // 32)


def head_bytes(head_dim):
    return BLOCK * (33 * groups_of(head_dim) + 2)


def places(head_dim):
    """(keys' codes, values' codes, exponents, scales): byte offsets by (token, channel), (token, channel), (token, group), (token);
    the half of a code's byte is d % 2 for keys and t % 2 for values"""
    m = groups_of(head_dim)
    t, d, g = np.arange(BLOCK)[:, None], np.arange(32 * m)[None, :], np.arange(m)[None, :]
    keys = ((t // 16) * m + d // 32) * 256 + (t % 16) * 16 + (d % 32) // 2
    values = 1024 * m + (d // 32) * 1024 + ((t % 16) // 4) * 256 + (d % 16) * 16 + (d % 32) // 16 * 8 + (t // 32) * 4 + (t % 32) // 16 * 2 + t % 4 // 2
    exponents = 2048 * m + g * 64 + (t % 16) * 4 + t // 16
    t = t[:, 0]
    scales = 2112 * m + ((t % 16) // 4) * 32 + (t // 16) * 8 + (t % 4) * 2
    return keys, values, exponents, scales


def bf16(x):
    """float32 numbers rounded to bfloat16, ties to even, as float32"""
    bits = np.asarray(x, np.float32).view(np.uint32).astype(np.uint64)
    return ((bits + 0x7fff + (bits >> 16 & 1)) & 0xffff0000).astype(np.uint32).view(np.float32)


def nearest(x):
    """codes of numbers (64 bits): the nearest magnitude, the even code of two"""
    size, code = np.abs(x), np.zeros(np.shape(x), np.uint8)
    for i in range(7):
        border = (MAGNITUDES[i] + MAGNITUDES[i + 1]) / 2
        code += (size >= border) if i % 2 else (size > border)
    return code


def _finite_max(x):
    a = np.abs(x)
    return np.where(np.isfinite(a), a, 0).max(-1)


def _clean(x):
    return np.where(np.isnan(x), 0, x)


def key_codes(x):
    """x (..., head_dim) float32 -> (codes (..., 32 m), exponents + 127 (..., m)); a code's sign is that of its number"""
    dim = x.shape[-1]
    x = np.concatenate([np.asarray(x, np.float64), np.zeros((*x.shape[:-1], -dim % 32))], -1)
    g = _clean(x.reshape(*x.shape[:-1], -1, 32))
    most = _finite_max(g)
    e = np.full(most.shape, -120)
    some = most > 0
    e[some] = [max(-120, min(125, next(k for k in range(math.frexp(v)[1] - 4, 200) if v <= math.ldexp(7, k)))) for v in most[some]]
    with np.errstate(invalid="ignore"):
        scaled = g / np.ldexp(1.0, e)[..., None]
    codes = nearest(np.where(np.isinf(g), 6, scaled)) | (np.signbit(g) << 3).astype(np.uint8)
    return codes.reshape(x.shape), (e + 127).astype(np.uint8)


def value_codes(x):
    """x (..., head_dim) float32 -> (codes (..., 32 m), scales (...) float32 that bfloat16 holds)"""
    dim = x.shape[-1]
    x = np.concatenate([np.asarray(x, np.float32), np.zeros((*x.shape[:-1], -dim % 32), np.float32)], -1)
    x = _clean(x).astype(np.float32)
    scale = bf16(_finite_max(x).astype(np.float32) * np.float32(1 / 6))
    scale = np.where(scale < np.float32(2.0 ** -100), np.float32(0), scale)
    by = np.where(scale > 0, scale, np.float32(1))[..., None]
    with np.errstate(over="ignore"):
        quotient = (x / by).astype(np.float32)
    codes = np.where(scale[..., None] > 0, nearest(np.where(np.isinf(x), 6, quotient)) | (np.signbit(x) << 3).astype(np.uint8), 0)
    return codes.astype(np.uint8), scale


def key_values(codes, exponents, head_dim):
    x = VALUES[codes] * np.repeat(np.ldexp(1.0, exponents.astype(int) - 127), 32, -1)
    return x[..., :head_dim]


def scales_of(page, head_dim):
    """the values' scales of a head's part of a page"""
    s = places(head_dim)[3]
    bits = (page[s].astype(np.uint32) << 16) | (page[s + 1].astype(np.uint32) << 24)
    return np.where((bits & 0x7f800000) == 0x7f800000, np.uint32(0x7fc00000), bits).astype(np.uint32).view(np.float32).astype(np.float64)


def read(page, head_dim):
    """a head's part of a page (head_bytes,) uint8 -> keys and values (64, head_dim), in 64 bits"""
    k, v, e, s = places(head_dim)
    d, t = np.arange(k.shape[1])[None, :], np.arange(BLOCK)[:, None]
    kc, vc = page[k] >> 4 * (d % 2) & 15, page[v] >> 4 * (t % 2) & 15
    scale = scales_of(page, head_dim)
    keys = VALUES[kc] * np.repeat(np.ldexp(1.0, page[e].astype(int) - 127), 32, -1)
    return keys[:, :head_dim], (VALUES[vc] * scale[:, None])[:, :head_dim]


def write(page, t, key, value, head_dim):
    """the codes of one token into a head's part of a page"""
    k, v, e, s = places(head_dim)
    codes, exponents = key_codes(key)
    for d, c in enumerate(codes):
        page[k[t, d]] = page[k[t, d]] & (0xf0 if d % 2 == 0 else 0x0f) | c << 4 * (d % 2)
    page[e[t]] = exponents
    codes, scale = value_codes(value)
    for d, c in enumerate(codes):
        page[v[t, d]] = page[v[t, d]] & (0xf0 if t % 2 == 0 else 0x0f) | c << 4 * (t % 2)
    bits = int(np.float32(scale).view(np.uint32)) >> 16
    page[s[t]], page[s[t] + 1] = bits & 255, bits >> 8


def turn(x, cos, sin, rot, interleaved):
    """x (rows, heads, head_dim) float32 by (rows, rot / 2) cosines and sines, every product and sum rounded to 32 bits"""
    first = np.arange(0, rot, 2) if interleaved else np.arange(rot // 2)
    second = first + (1 if interleaved else rot // 2)
    out, c, s = x.copy(), cos[:, None].astype(np.float32), sin[:, None].astype(np.float32)
    a, b = x[..., first], x[..., second]
    with np.errstate(invalid="ignore"):
        out[..., first], out[..., second] = c * a - s * b, c * b + s * a
    return out


def attention(q, k, v, seen, scale, parts_q, parts_w):
    """One query head: (out, bound).  The bound follows from what enters the products: all of the query where its bits fit 8 * parts_q,
    weights times scales of values rounded at 2^-(8 parts_w) of themselves; products exact, sums in 32 bits in any order."""
    dim = len(q)
    if not seen.any():
        return np.zeros(dim), np.zeros(dim)
    k, v = k[seen], v[seen]
    s = scale * (k @ q)
    w = np.exp(s - s.max())
    out = (w[:, None] * v).sum(0) / w.sum()
    # a score: its terms' sum, one rounding of 32 bits a term and part, and a few of the scaling, the difference to the largest and exp
    u = 2.0 ** -24
    size = abs(scale) * (np.abs(k) @ np.abs(q))
    slack = (dim * parts_q + 8) * u * size.max() + 8 * u * (np.abs(s).max() + 1) + 4 * u
    rel = np.expm1(2 * slack) + 2.0 ** -(8 * parts_w)
    spread = (w[:, None] * np.abs(v)).sum(0) / w.sum()
    return out, 2 * rel * spread + (len(w) * parts_w + 64) * u * spread


def attention_in_halves(q, k, v, scales, seen, scale, parts_q):
    """The same with weights times scales of values (`scales`, a token each) in half precision: rounded by at most 2^-11 of
    themselves, or by half a step of 2^-31 of the largest of them; the scale's logarithm is one more term of a score's sum,
    88 in binary where the scale is 0."""
    dim = len(q)
    if not seen.any():
        return np.zeros(dim), np.zeros(dim)
    k, v, scales = k[seen], v[seen], scales[seen]
    s = scale * (k @ q)
    w = np.exp(s - s.max())
    out = (w[:, None] * v).sum(0) / w.sum()
    u = 2.0 ** -24
    size = abs(scale) * (np.abs(k) @ np.abs(q)).max() + np.abs(np.log(np.where(scales > 0, scales, 2.0 ** -88))).max()
    slack = (dim * parts_q + 16) * u * size + 8 * u * (np.abs(s).max() + 1)
    spread = (w[:, None] * np.abs(v)).sum(0) / w.sum()
    bound = 2 * np.expm1(2 * slack) * spread + 2.0 ** -11 * spread + (len(w) + 64) * u * spread
    return out, bound + len(w) * 6 * 2.0 ** -32 * (w * scales).max() / w.sum()


def rms_norm(x, add, weight, epsilon):
    """(sum, y) in 32 bits, rounded as the header says; sums exactly"""
    s = x.astype(np.float32) if add is None else (x.astype(np.float32) + add.astype(np.float32))
    mean = np.array([math.fsum(r) for r in s.astype(np.float64) ** 2]) / s.shape[1] if np.isfinite(s).all() else (s.astype(np.float64) ** 2).sum(1) / s.shape[1]
    factor = (1.0 / np.sqrt(mean + epsilon)).astype(np.float32)
    with np.errstate(invalid="ignore", over="ignore"):
        return s, s * factor[:, None] * (np.float32(1) if weight is None else weight.astype(np.float32))


def whole(y, limit, group, unit=None):
    """(whole numbers, scales or None) of y (rows, width) float32"""
    rows, width = y.shape
    held = lambda t: np.clip(np.where(np.isnan(t), 0, t), -limit, limit).astype(np.int64)       # noqa: E731
    if unit is not None:
        return held(np.rint(y / np.float32(unit))), None
    group = group or width
    codes, scales = np.zeros(y.shape, np.int64), np.zeros((rows, -(-width // group)), np.float32)
    step = np.float32(1.0 / limit)
    for g in range(scales.shape[1]):
        part = y[:, g * group:(g + 1) * group]
        scales[:, g] = _finite_max(part).astype(np.float32) * step
        with np.errstate(divide="ignore", invalid="ignore", over="ignore"):
            inverse = np.where(scales[:, g] > 0, np.float32(1) / scales[:, g], np.float32(0)).astype(np.float32)
            codes[:, g * group:(g + 1) * group] = held(np.rint(part * inverse[:, None]))
    return codes, scales
