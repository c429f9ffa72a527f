"""A language model's steps between two linear layers: rope tables, sizes and refusals, on the host."""
import ctypes as C
import math

import numpy as np
import pytest

from paper_2105_01827_amd import binding, workloads as wl
from tests import decode_reference as ref

EARG, ENOMEM = binding.GALA_EARG, binding.GALA_ENOMEM


@pytest.fixture(scope="module")
def ctx():
    par = wl.DEFAULT
    return binding.Context(par.n, par.q, par.p, par.gadget_bits)


@pytest.mark.parametrize("scaling", [0, 1, 2])
def test_rope_table(scaling):
    rot, base, factor, original, low, high = 48, 10000.0, 8.0, 512.0, 1.0, 16.0
    got = binding.rope_table(3000, rot, base, scaling, factor, original, low, high)
    f = base ** (-2.0 * np.arange(rot // 2) / rot)
    if scaling == 1:
        f = f / factor
    if scaling == 2:
        kept = np.clip((original * f / (2 * math.pi) - low) / (high - low), 0, 1)
        assert kept.min() == 0 and kept.max() == 1 and ((kept > 0) & (kept < 1)).any()
        f = f * kept + f / factor * (1 - kept)
    angle = np.arange(3000)[:, None] * f
    # half a unit in the last place of 32 bits, and 64-bit roundings of angles up to 3000
    assert np.abs(got[..., 0] - np.cos(angle)).max() <= 2.0 ** -25 + 3000 * 2.0 ** -50
    assert np.abs(got[..., 1] - np.sin(angle)).max() <= 2.0 ** -25 + 3000 * 2.0 ** -50


@pytest.mark.parametrize("change", [dict(rot_dim=0), dict(rot_dim=7), dict(rot_dim=258), dict(positions=-1), dict(base=0.0),
                                    dict(base=math.inf), dict(scaling=3), dict(scaling=1, factor=0.0), dict(scaling=2, original=0.0),
                                    dict(scaling=2, low=4.0, high=4.0), dict(scaling=1, factor=math.nan)])
def test_rope_table_refuses(change):
    args = dict(positions=4, rot_dim=8, base=1e4, scaling=0, factor=2.0, original=64.0, low=1.0, high=2.0) | change
    out = np.zeros((8, 256, 2), np.float32)
    assert binding.load().gala_rope_table(*args.values(), out.ctypes.data_as(C.c_void_p)) == EARG
    assert not out.any()


@pytest.mark.parametrize("head_dim", [1, 15, 16, 17, 64, 80, 128, 200, 256])
def test_code_places_fill_a_page(head_dim):
    size = int(binding.load().gala_kv_cache_bytes(1, 1, head_dim))
    assert size == ref.head_bytes(head_dim)
    keys, values = ref.code_places(head_dim)
    places = np.concatenate([keys.ravel(), values.ravel()])
    assert len(np.unique(places)) == len(places) and places.min() == 0 and places.max() < size
    assert keys.max() < size // 2 <= values.min()
    assert int(binding.load().gala_kv_cache_bytes(5, 3, head_dim)) == 15 * size


def test_sizes_that_do_not_fit_are_zero():
    lib = binding.load()
    for args in [(-1, 1, 64), (1, 0, 64), (1, 1, 0), (1, 1, 257)]:
        assert lib.gala_kv_cache_bytes(*args) == 0
    assert lib.gala_sample_workspace(-1, 10) == 0 and lib.gala_sample_workspace(1, 0) == 0


# Addresses that no call here may touch: every one of these calls has to be refused on the host.
AT = 1 << 20


def _args(**change):
    a = dict(cache=dict(heads=2, head_dim=64, pages=4, codes=AT, scales=AT),
             batch=dict(count=1, max_new=1, max_len=64, table_stride=1, starts=AT, lens=AT, table=AT),
             rope=dict(table=AT, positions=64, rot_dim=64, interleaved=0),
             q=dict(data=AT, stride=256, type=0, unit=1.0), q_out=dict(data=2 * AT, stride=256, type=0, unit=1.0),
             k=dict(data=AT, stride=128, type=0, unit=1.0), v=dict(data=AT, stride=128, type=0, unit=1.0), heads_q=4)
    for key, value in change.items():
        where, _, name = key.partition("__")
        if name:
            a[where] = a[where] | {name: value}
        else:
            a[where] = value
    return a


class ValuesArg(C.Structure):
    _fields_ = [("data", C.c_void_p), ("stride", C.c_int64), ("type", C.c_int32), ("unit", C.c_float)]


class SamplingArg(C.Structure):
    _fields_ = [(k, C.c_void_p) for k in ("temperature", "top_k", "top_p", "min_p", "u")]


def _struct(cls, fields):
    return None if fields is None else C.byref(cls(**fields))


def _append(ctx, a):
    return ctx.lib.gala_kv_append(ctx.h, None, _struct(binding.KvCacheArg, a["cache"]), _struct(binding.KvBatchArg, a["batch"]),
                                  _struct(binding.RopeArg, a["rope"]), a["heads_q"],
                                  *(_struct(ValuesArg, a[k]) for k in ("q", "q_out", "k", "v")))


BAD_CACHE = [dict(cache=None), dict(cache__heads=0), dict(cache__head_dim=0), dict(cache__head_dim=257), dict(cache__pages=-1),
             dict(cache__codes=0), dict(cache__codes=AT + 8), dict(cache__scales=0), dict(cache__scales=AT + 2)]
BAD_BATCH = [dict(batch=None), dict(batch__count=-1), dict(batch__max_new=-1), dict(batch__max_len=-1), dict(batch__table_stride=-1),
             dict(batch__starts=0), dict(batch__lens=0), dict(batch__table=0), dict(batch__max_new=(1 << 30) + 1),
             dict(batch__table_stride=1 << 25)]
BAD_GRID = [dict(batch__max_new=1 << 30, batch__count=4)]          # more rows than a launch has workgroups


@pytest.mark.parametrize("change", BAD_CACHE + BAD_BATCH + BAD_GRID + [
    dict(heads_q=-1), dict(q=None), dict(q_out=None), dict(heads_q=0), dict(k=None), dict(v=None), dict(q__type=4), dict(q__type=-1),
    dict(q__stride=-1), dict(q_out__stride=255), dict(q_out__type=3), dict(q__data=AT + 2), dict(k__type=1), dict(k__type=1, v__type=1),
    dict(k__type=3, v__type=3, q__type=3, k__unit=0.0), dict(k__type=3, v__type=3, q__type=3, v__unit=math.inf),
    dict(q_out__data=AT, q_out__type=1), dict(q_out__data=AT, q_out__stride=512), dict(rope__table=0), dict(rope__table=AT + 4),
    dict(rope__positions=0), dict(rope__rot_dim=0), dict(rope__rot_dim=3), dict(rope__rot_dim=66)])
def test_append_refuses(ctx, change):
    assert _append(ctx, _args(**change)) == EARG


@pytest.mark.parametrize("change", BAD_CACHE + BAD_BATCH + [dict(k=None), dict(v=None), dict(k__stride=127), dict(v__type=1),
                                                            dict(k__type=5, v__type=5)])
def test_export_refuses(ctx, change):
    a = _args(**change)
    assert ctx.lib.gala_kv_export(ctx.h, None, _struct(binding.KvCacheArg, a["cache"]), _struct(binding.KvBatchArg, a["batch"]),
                                  _struct(ValuesArg, a["k"]), _struct(ValuesArg, a["v"])) == EARG


@pytest.mark.parametrize("change", BAD_CACHE + BAD_BATCH + BAD_GRID + [
    dict(heads_q=0), dict(heads_q=3), dict(q=None), dict(q_out=None), dict(q_out__stride=255), dict(q__stride=-1), dict(scale=math.nan),
    dict(scale=math.inf), dict(window=-1), dict(sinks=-1), dict(q_out__data=AT, q_out__type=1), dict(workspace=AT + 8, batch__max_len=1 << 20, batch__table_stride=1 << 14),
    dict(workspace=0, batch__max_len=1 << 20, batch__table_stride=1 << 14)])
def test_attention_refuses(ctx, change):
    a = dict(scale=1.0, window=0, sinks=0, workspace=AT) | _args(**{k: v for k, v in change.items() if k not in ("scale", "window", "sinks", "workspace")})
    a |= {k: v for k, v in change.items() if k in ("scale", "window", "sinks", "workspace")}
    cache, batch = _struct(binding.KvCacheArg, a["cache"]), _struct(binding.KvBatchArg, a["batch"])
    need = ctx.lib.gala_kv_attention_workspace(cache, batch, a["heads_q"], a["window"], a["sinks"])
    assert need or "workspace" not in change
    got = ctx.lib.gala_kv_attention(ctx.h, None, cache, batch, a["heads_q"], a["scale"], a["window"], a["sinks"],
                                    _struct(ValuesArg, a["q"]), _struct(ValuesArg, a["q_out"]), a["workspace"], 1 << 40)
    assert got == EARG


def test_attention_wants_its_workspace(ctx):
    a = _args(batch__max_len=1 << 20, batch__table_stride=1 << 14)
    cache, batch = _struct(binding.KvCacheArg, a["cache"]), _struct(binding.KvBatchArg, a["batch"])
    need = ctx.lib.gala_kv_attention_workspace(cache, batch, 4, 0, 0)
    assert need
    assert ctx.lib.gala_kv_attention(ctx.h, None, cache, batch, 4, 1.0, 0, 0, _struct(ValuesArg, a["q"]),
                                     _struct(ValuesArg, a["q_out"]), AT, need - 1) == ENOMEM


@pytest.mark.parametrize("change", [dict(logits=None), dict(rows=-1), dict(vocab=0), dict(how=None), dict(tokens=0), dict(u=0),
                                    dict(type=9), dict(type=3, unit=0.0), dict(stride=-5), dict(data=AT + 2)])
def test_sample_refuses(ctx, change):
    a = dict(data=AT, stride=100, type=0, unit=1.0, rows=3, vocab=100, u=AT, tokens=AT) | change
    logits = None if "logits" in change else C.byref(ValuesArg(a["data"], a["stride"], a["type"], a["unit"]))
    how = None if "how" in change else C.byref(SamplingArg(0, 0, 0, 0, a["u"]))
    assert ctx.lib.gala_sample(ctx.h, None, logits, a["rows"], a["vocab"], how, a["tokens"], AT, 1 << 40) == EARG


def test_binding_refuses_tensors_that_do_not_fit(ctx):
    import torch
    with pytest.raises(TypeError):
        binding._values(torch.zeros(4, 8, dtype=torch.float64), 1.0)
    with pytest.raises(ValueError):
        binding._values(torch.zeros(4, 8, 6).transpose(1, 2), 1.0)
    v = ValuesArg.from_buffer_copy(binding._values(torch.zeros(4, 24)[:, 8:16].view(4, 2, 4), 0.5))
    assert (v.stride, v.type, v.unit) == (24, 0, 0.5)
    with pytest.raises(TypeError):
        binding.KvBatch(torch.zeros(3, dtype=torch.int64), torch.zeros(2, dtype=torch.int32), torch.zeros(2, 1, dtype=torch.int32), 1, 1)
    with pytest.raises(ValueError):
        binding.KvBatch(torch.zeros(2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.zeros(2, 1, dtype=torch.int32), 1, 1)
    with pytest.raises(ValueError):
        binding.KvCache(ctx, 2, 64, torch.zeros(3, 100, dtype=torch.int8), torch.zeros(3, 2, 2))
    with pytest.raises(ValueError):
        ctx.sample(torch.zeros(3, 10), torch.zeros(2), torch.zeros(3, dtype=torch.int32), 0, 0)


def test_kernels_stay_in_registers():
    """Attention's loops and the appended values are worth having in registers alone."""
    from tests.test_kernel_registers import _kernels
    found = {name: k for (_, name), k in _kernels().items() if any(w in name for w in ("kv_a", "kv_export", "sample_"))}
    assert sum("kv_attention_many" in n for n in found) == 8 and sum("sample_" in n for n in found) == 16
    assert all(k[".private_segment_fixed_size"] == 0 for k in found.values()), {n: k[".private_segment_fixed_size"] for n, k in found.items()}
