"""Calls without rows, whose tensors have no address: they do nothing; with rows they are refused (no GPU)."""
import ctypes as C

import pytest

from paper_2105_01827_amd import binding
from tests.test_decode_host import ValuesArg, _struct
from tests.test_kv4_host import CODES, _args4, _cache_and_batch, _norm, _rope_args, ctx  # noqa: F401

# no device here: what is let through ends there
LET_THROUGH = (0, binding.GALA_EHIP)
NOWHERE = {f"{name}__data": 0 for name in ("x", "add", "sum", "out")}


@pytest.mark.parametrize("more", [dict(), dict(out__type=2), dict(out__type=3, how__limit=63), CODES, CODES | dict(how__group=8),
                                  CODES | dict(how__scales=0, how__group=8), CODES | dict(how__scales=0), dict(x__type=2, add__type=3)])
def test_norm(ctx, more):  # noqa: F811
    assert _norm(ctx, rows=0, **NOWHERE, **more) in LET_THROUGH
    for name in ("x", "add", "sum", "out"):
        assert _norm(ctx, rows=1, **more, **{f"{name}__data": 0}) == binding.GALA_EARG
    assert _norm(ctx, rows=0, weight__data=0) == binding.GALA_EARG               # a row for all there are


def _rope(ctx, **change):  # noqa: F811
    a = _rope_args(**change)
    fill = lambda v: (C.c_uint8 * 128)(*v, *[0] * (128 - len(v)))            # noqa: E731
    rope = binding.RopeAxesArg(a["table"], a["positions"], a["columns"], a["rot_dim"], a["interleaved"], a["axes"], a["reserved"], fill(a["axis"]),
                               fill(a["column"]))
    return ctx.lib.gala_rope_apply(ctx.h, None, C.byref(rope), a["at"], a["at_stride"], a["rows"], a["heads"], a["head_dim"],
                                   *(_struct(ValuesArg, a[k]) for k in ("x", "out")))


def test_positions(ctx):  # noqa: F811
    nowhere = dict(at=0, x__data=0, out__data=0)
    assert _rope(ctx, rows=0, **nowhere) in LET_THROUGH
    assert _rope(ctx, rows=0, **nowhere, out__type=2) in LET_THROUGH
    for name in nowhere:
        assert _rope(ctx, rows=1, **{name: 0}) == binding.GALA_EARG


def test_cache(ctx):  # noqa: F811
    def calls(**change):
        a = _args4(**change)
        cache, batch = _cache_and_batch(a)
        q, q_out, k, v = (_struct(ValuesArg, a[n]) for n in ("q", "q_out", "k", "v"))
        yield ctx.lib.gala_kv4_append(ctx.h, None, cache, batch, None, a["heads_q"], q, q_out, k, v)
        yield ctx.lib.gala_kv4_export(ctx.h, None, cache, batch, k, v)
        yield ctx.lib.gala_kv4_attention(ctx.h, None, cache, batch, a["heads_q"], 1.0, 0, 0, q, q_out, 0, 0)
    nowhere = {f"{n}__data": 0 for n in ("q", "q_out", "k", "v")}
    for none in (dict(batch__count=0, batch__lens=0, batch__table=0), dict(batch__max_new=0)):
        assert all(s in LET_THROUGH for s in calls(**none, **nowhere))
    assert all(s == binding.GALA_EARG for s in calls(**nowhere))
