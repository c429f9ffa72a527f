"""Scores beyond 32 bits in attention over the 4-bit cache: above them a query gives NaN, below them a key has no weight."""
import numpy as np
import pytest
import torch

from tests import kv4_reference as ref
from tests.test_gpu_kv4_attention import Case, _many, ctx  # noqa: F401

pytestmark = pytest.mark.gpu


def _case(ctx, kind, new, apart):  # noqa: F811
    c = Case(ctx, [new], [200], _many(new), 2, 64, kind, seed=101)
    c.q = (c.q.abs() * 0.5 + 1).to(c.q.dtype)                    # the sign of a score is the keys'
    k, v, e, s = ref.places(64)
    data = c.cache.data.cpu().numpy().reshape(-1, c.heads, ref.head_bytes(64))
    if apart:                                                    # the divisor has an exponent of its own
        page = data[int(c.table[0, 0])]
        page[:, s[3]], page[:, s[3] + 1] = (100 + 127 << 7) & 255, 100 + 127 >> 1
    c.cache.data.copy_(torch.from_numpy(data).view(c.cache.data.shape))
    return c, data, k, e


def _keys(c, data, k, e, tokens, sign):
    """keys of 6 x 2^125 in all channels: 64 of them times 1 are 2.7e39, times dim^-0.5 3.4e38 and more"""
    for t in tokens:
        page = data[int(c.table[0, t // 64])]
        page[:, k[t % 64]] = 0x77 | (0x88 if sign < 0 else 0)
        page[:, e[t % 64]] = 125 + 127
    c.cache.data.copy_(torch.from_numpy(data).view(c.cache.data.shape))


KINDS = [("bf16", 1), ("f16", 2), ("f32", 2), ("bf16", 150), ("f16", 150)]


@pytest.mark.parametrize("apart", [False, True])
@pytest.mark.parametrize("kind,new", KINDS)
def test_above(ctx, kind, new, apart):  # noqa: F811
    c, data, k, e = _case(ctx, kind, new, apart)
    clean = c.run()
    _keys(c, data, k, e, [199], 1)                               # the last one alone sees it
    out = c.run()
    assert bool(out[-1].isnan().all()) and torch.equal(out[:-1], clean[:-1])
    _keys(c, data, k, e, [0, 70], 1)
    assert bool(c.run().isnan().all())


@pytest.mark.parametrize("kind,new", KINDS)
def test_below(ctx, kind, new):  # noqa: F811
    c, data, k, e = _case(ctx, kind, new, False)
    _keys(c, data, k, e, [0, 64, 65, 190], -1)
    c.check(c.run(), {(0, 0), (0, new - 1)})
    _keys(c, data, k, e, range(200), -1)
    assert bool((c.run() == 0).all())
