"""Attention of prompts over the 4-bit cache in the form that gives a wavefront 32 queries: every row of several groups of queries, contexts of
thousands of tokens, both 16-bit types in and out.  tests/test_kv4_cut_host.py asserts that the cases here take that form."""
import numpy as np
import pytest
import torch

from tests import decode_reference as dref, kv4_reference as ref
from tests.test_gpu_kv4_attention import EPS, PARTS_Q, Case, _plain, ctx  # noqa: F401

pytestmark = pytest.mark.gpu

# new tokens, lengths, heads, queries of a head, channels, types of q and out, window, first tokens
ALL_ROWS = {
    "groups": ([300, 130], [300, 700], 16, 3, 64, "bf16", "bf16", 0, 0),
    "narrow_heads": ([65, 1, 130], [65, 200, 130], 32, 3, 32, "bf16", "bf16", 0, 0),
    "one_sequence": ([600], [1300], 30, 1, 128, "bf16", "bf16", 0, 0),
    "halves": ([257], [400], 40, 2, 80, "f16", "f16", 0, 0),
    "wide_heads": ([140, 33], [500, 600], 16, 2, 256, "bf16", "bf16", 0, 0),
    "window": ([300, 200], [900, 200], 16, 2, 96, "bf16", "bf16", 130, 70),
    "f16_to_bf16": ([200, 60], [200, 300], 24, 2, 64, "f16", "bf16", 0, 0),
    "bf16_to_f16": ([200, 60], [200, 300], 24, 2, 64, "bf16", "f16", 0, 0),
    "bf16_to_f16_wide": ([150], [150], 50, 1, 200, "bf16", "f16", 0, 0),
    "f16_to_bf16_wide": ([150], [150], 60, 1, 192, "f16", "bf16", 0, 0),
}
LONG = {
    "128": ([260], [5000], 44, 2, 128, "bf16", "bf16", 0, 0),
    "64_f16": ([200, 140], [3000, 6100], 32, 4, 64, "f16", "f16", 0, 0),
    "256": ([150], [4100], 60, 1, 256, "bf16", "bf16", 0, 0),
    "window": ([700], [5000], 40, 2, 128, "bf16", "bf16", 2500, 100),
}
RISING = ([140], [4000], 80, 2, 64, "bf16", "bf16", 0, 0)


def case_of(ctx, new, lens, heads, group, dim, kind, out, window, sinks, **more):  # noqa: F811
    c = Case(ctx, new, lens, heads, group, dim, kind, out, seed=dim + sum(new), **more)
    return c, c.run(window=window, sinks=sinks)


def check(c, out, heads):
    """every row of some heads of the queries"""
    data = c.cache.data.cpu().numpy().reshape(-1, c.heads, ref.head_bytes(c.dim))
    got, q = _plain(out), _plain(c.q)
    for b, (n, length) in enumerate(zip(c.new, c.lens)):
        pages = c.table[b].numpy()[:max(1, -(-length // 64))]
        for h in heads:
            with np.errstate(invalid="ignore"):
                k, v = (np.concatenate(x)[:length] for x in zip(*(ref.read(data[p, h // c.group], c.dim) for p in pages)))
            scales = np.concatenate([ref.scales_of(data[p, h // c.group], c.dim) for p in pages])[:length]
            for i in range(n):
                row = c.starts[b] + i
                seen = dref.see(length - n + i, length, c.window, c.sinks)
                want, bound = ref.attention_in_halves(q[row, h], k, v, scales, seen, c.scale, PARTS_Q[c.kind])
                bound = bound + EPS[c.out_kind] * (np.abs(want) + bound) + 2.0 ** -25
                over = np.abs(got[row, h] - want) / bound
                assert over.max() <= 1, (b, i, h, over.max())


@pytest.mark.parametrize("name", list(ALL_ROWS))
def test_every_row(ctx, name):  # noqa: F811
    c, out = case_of(ctx, *ALL_ROWS[name])
    check(c, out, [0, c.group, c.heads * c.group - 1])


@pytest.mark.parametrize("name", list(LONG))
def test_long_contexts(ctx, name):  # noqa: F811
    c, out = case_of(ctx, *LONG[name])
    check(c, out, [c.group + c.group // 2])


def test_bases_that_rise_all_along(ctx):  # noqa: F811
    """Keys grow along the context, so that the largest score so far rises in block after block."""
    c = Case(ctx, *RISING[:6], seed=91, spread=0.5)
    e = ref.places(64)[2]
    data = c.cache.data.cpu().numpy().reshape(-1, c.heads, ref.head_bytes(64))
    for j, page in enumerate(c.table[0].numpy()):
        live = min(64, 4000 - 64 * j)
        data[page][:, e[:live]] = 127 - 6 + j // 8
    c.cache.data.copy_(torch.from_numpy(data).view(c.cache.data.shape))
    check(c, c.run(), [3])
