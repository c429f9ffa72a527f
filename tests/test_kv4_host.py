"""The 4-bit cache, positions with several axes and the norm in few bits: sizes, layouts and refusals, on the host."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from paper_2105_01827_amd import binding, workloads as wl
from tests import kv4_reference as ref
from tests.test_decode_binding import OnGpu, Unlaunched
from tests.test_decode_host import AT, BAD_BATCH, BAD_GRID, ValuesArg, _args, _struct

EARG, ENOMEM = binding.GALA_EARG, binding.GALA_ENOMEM


@pytest.fixture(scope="module")
def ctx():
    par = wl.DEFAULT
    return binding.Context(par.n, par.q, par.p, par.gadget_bits)


@pytest.mark.parametrize("head_dim", [1, 31, 32, 33, 64, 80, 96, 128, 200, 256])
def test_places_fill_a_page(head_dim):
    size = int(binding.load().gala_kv4_cache_bytes(1, 1, head_dim))
    assert size == ref.head_bytes(head_dim) and int(binding.load().gala_kv4_cache_bytes(5, 3, head_dim)) == 15 * size
    k, v, e, s = ref.places(head_dim)
    t, d = np.arange(64)[:, None], np.arange(k.shape[1])[None, :]
    nibbles = np.concatenate([(2 * k + d % 2).ravel(), (2 * v + t % 2).ravel()] + [(2 * x).ravel() + h for x in (e, s, s + 1) for h in (0, 1)])
    assert np.array_equal(np.sort(nibbles), np.arange(2 * size))


def test_reference_reads_what_it_writes():
    rng = np.random.default_rng(0)
    page = rng.integers(0, 256, ref.head_bytes(80)).astype(np.uint8)
    key, value = (rng.standard_normal(80).astype(np.float32) for _ in range(2))
    before = page.copy()
    ref.write(page, 37, key, value, 80)
    keys, values = ref.read(page, 80)
    old = ref.read(before, 80)
    others = np.arange(64) != 37
    assert np.array_equal(keys[others], old[0][others]) and np.array_equal(values[others], old[1][others], equal_nan=True)
    # half a step of the widest kind, of the largest magnitude's scale
    assert np.abs(keys[37] - key).max() <= 2 * np.abs(key).max() / 3.5 / 2 + 1e-9
    assert np.abs(values[37] - value).max() <= np.abs(value).max() / 6 * 1.01


def test_sizes_that_do_not_fit_are_zero():
    for args in [(-1, 1, 64), (1, 0, 64), (1, 1, 0), (1, 1, 257)]:
        assert binding.load().gala_kv4_cache_bytes(*args) == 0


def _args4(**change):
    a = _args(**{k: v for k, v in change.items() if not k.startswith("cache")})
    a["cache"] = dict(heads=2, head_dim=64, pages=4, reserved=0, data=AT)
    for k, v in change.items():
        if k == "cache":
            a["cache"] = v
        elif k.startswith("cache__"):
            a["cache"] = a["cache"] | {k[7:]: v}
    return a


def _cache_and_batch(a):
    return _struct(binding.Kv4CacheArg, a["cache"]), _struct(binding.KvBatchArg, a["batch"])


BAD_CACHE = [dict(cache=None), dict(cache__heads=0), dict(cache__head_dim=0), dict(cache__head_dim=257), dict(cache__pages=-1),
             dict(cache__data=0), dict(cache__data=AT + 8), dict(cache__reserved=1)]


@pytest.mark.parametrize("change", BAD_CACHE + BAD_BATCH + BAD_GRID + [
    dict(heads_q=-1), dict(q=None), dict(q_out=None), dict(heads_q=0), dict(k=None), dict(v=None), dict(q__type=4), dict(q__type=-1),
    dict(q__stride=-1), dict(q_out__stride=255), dict(q_out__type=3), dict(q__data=AT + 2), dict(k__type=1), dict(k__type=1, v__type=1),
    dict(k__type=3, v__type=3, q__type=3, k__unit=0.0), dict(k__type=3, v__type=3, q__type=3, v__unit=math.inf),
    dict(q_out__data=AT, q_out__type=1), dict(q_out__data=AT, q_out__stride=512), dict(rope__table=0), dict(rope__table=AT + 4),
    dict(rope__positions=0), dict(rope__rot_dim=0), dict(rope__rot_dim=3), dict(rope__rot_dim=66), dict(batch__max_new=1 << 24)])
def test_append_refuses(ctx, change):
    a = _args4(**change)
    assert ctx.lib.gala_kv4_append(ctx.h, None, *_cache_and_batch(a), _struct(binding.RopeArg, a["rope"]), a["heads_q"],
                                   *(_struct(ValuesArg, a[k]) for k in ("q", "q_out", "k", "v"))) == EARG


@pytest.mark.parametrize("change", BAD_CACHE + BAD_BATCH + [dict(k=None), dict(v=None), dict(k__stride=127), dict(v__type=1), dict(k__type=5, v__type=5)])
def test_export_refuses(ctx, change):
    a = _args4(**change)
    assert ctx.lib.gala_kv4_export(ctx.h, None, *_cache_and_batch(a), _struct(ValuesArg, a["k"]), _struct(ValuesArg, a["v"])) == EARG


@pytest.mark.parametrize("change", BAD_CACHE + BAD_BATCH + BAD_GRID + [
    dict(heads_q=0), dict(heads_q=3), dict(q=None), dict(q_out=None), dict(q_out__stride=255), dict(q__stride=-1), dict(scale=math.nan),
    dict(scale=math.inf), dict(window=-1), dict(sinks=-1), dict(q_out__data=AT, q_out__type=1),
    dict(workspace=AT + 8, batch__max_len=1 << 20, batch__table_stride=1 << 14), dict(workspace=0, batch__max_len=1 << 20, batch__table_stride=1 << 14)])
def test_attention_refuses(ctx, change):
    more = {k: v for k, v in change.items() if k in ("scale", "window", "sinks", "workspace")}
    a = dict(scale=1.0, window=0, sinks=0, workspace=AT) | _args4(**{k: v for k, v in change.items() if k not in more}) | more
    cache, batch = _cache_and_batch(a)
    assert ctx.lib.gala_kv4_attention_workspace(cache, batch, a["heads_q"], a["window"], a["sinks"]) or "workspace" not in change
    assert ctx.lib.gala_kv4_attention(ctx.h, None, cache, batch, a["heads_q"], a["scale"], a["window"], a["sinks"], _struct(ValuesArg, a["q"]),
                                      _struct(ValuesArg, a["q_out"]), a["workspace"], 1 << 40) == EARG


def test_attention_wants_its_workspace(ctx):
    a = _args4(batch__max_len=1 << 20, batch__table_stride=1 << 14)
    cache, batch = _cache_and_batch(a)
    need = ctx.lib.gala_kv4_attention_workspace(cache, batch, 4, 0, 0)
    assert need
    assert ctx.lib.gala_kv4_attention(ctx.h, None, cache, batch, 4, 1.0, 0, 0, _struct(ValuesArg, a["q"]), _struct(ValuesArg, a["q_out"]), AT,
                                      need - 1) == ENOMEM


# ---- positions with several axes -----------------------------------------------------------------------------------
def test_axes_layout():
    assert binding.axes_layout([2, 3, 1]) == ([0, 0, 1, 1, 1, 2], list(range(6)))
    assert binding.axes_layout([1, 3, 2], 1) == ([0, 1, 2, 1, 2, 1], list(range(6)))
    assert binding.axes_layout([2, 3], 2) == ([0, 0, 1, 1, 1], [0, 1, 0, 1, 2])
    assert binding.axes_layout([0, 128]) == ([1] * 128, list(range(128)))
    arg = binding.RopeAxesArg()
    assert binding.load().gala_rope_axes_layout(2, np.array([2, 3], np.int32).ctypes.data_as(C.c_void_p), 2, C.byref(arg)) == 0
    assert (arg.columns, arg.rot_dim, arg.axes) == (3, 10, 2)


@pytest.mark.parametrize("sections,order", [([], 0), ([1] * 5, 0), ([-1, 4], 0), ([0, 0], 1), ([100, 29], 0), ([2, 2], 3), ([2, 2], -1), ([2 ** 31 - 1, 2 ** 31 - 1], 0)])
def test_axes_layout_refuses(sections, order):
    with pytest.raises(binding.GalaError):
        binding.axes_layout(sections, order)


def _rope_args(**change):
    a = dict(table=AT, positions=9, columns=8, rot_dim=32, interleaved=0, axes=2, reserved=0, axis=[0, 1] * 8, column=[0, 1, 2, 7] * 4, at=AT, at_stride=2,
             rows=3, heads=2, head_dim=64, x=dict(data=AT, stride=128, type=0, unit=1.0), out=dict(data=2 * AT, stride=128, type=0, unit=1.0))
    for key, value in change.items():
        where, _, name = key.partition("__")
        a[where] = a[where] | {name: value} if name else value
    return a


@pytest.mark.parametrize("change", [
    dict(table=0), dict(table=AT + 4), dict(positions=0), dict(columns=0), dict(columns=257), dict(columns=7), dict(rot_dim=0), dict(rot_dim=31),
    dict(rot_dim=66), dict(axes=0), dict(axes=1), dict(axes=5), dict(reserved=1), dict(at=0), dict(at=AT + 2), dict(at_stride=-1), dict(rows=-1), dict(heads=0),
    dict(heads=(1 << 20) + 1), dict(head_dim=0), dict(head_dim=257), dict(x=None), dict(out=None), dict(x__type=4), dict(out__type=3), dict(out__stride=127),
    dict(x__stride=-1), dict(x__data=AT + 2), dict(out__data=AT, out__type=1), dict(out__data=AT, out__stride=130), dict(rows=1 << 25)])
def test_rope_apply_refuses(ctx, change):
    a = _rope_args(**change)
    fill = lambda v: (C.c_uint8 * 128)(*v, *[0] * (128 - len(v)))            # noqa: E731
    rope = binding.RopeAxesArg(a["table"], a["positions"], a["columns"], a["rot_dim"], a["interleaved"], a["axes"], a["reserved"], fill(a["axis"]),
                               fill(a["column"]))
    assert ctx.lib.gala_rope_apply(ctx.h, None, C.byref(rope), a["at"], a["at_stride"], a["rows"], a["heads"], a["head_dim"],
                                   *(_struct(ValuesArg, a[k]) for k in ("x", "out"))) == EARG


# ---- norm ----------------------------------------------------------------------------------------------------------
class NormArg(C.Structure):
    _fields_ = [("epsilon", C.c_double), ("limit", C.c_int32), ("group", C.c_int32), ("scales", C.c_void_p)]


def _norm(ctx, **change):
    values = lambda n, **more: dict(data=n * AT, stride=128, type=0, unit=1.0) | more        # noqa: E731
    a = dict(how=dict(epsilon=1e-6, limit=0, group=0, scales=0), rows=3, width=128, x=values(1), add=values(2), sum=values(3), weight=values(4), out=values(5))
    for key, value in change.items():
        where, _, name = key.partition("__")
        a[where] = a[where] | {name: value} if name else value
    return ctx.lib.gala_rms_norm(ctx.h, None, _struct(NormArg, a["how"]), a["rows"], a["width"], *(_struct(ValuesArg, a[k]) for k in ("x", "add", "sum", "weight", "out")))


CODES = dict(out__type=4, how__scales=AT, how__limit=127)


@pytest.mark.parametrize("change", [
    dict(how=None), dict(how__epsilon=-1.0), dict(how__epsilon=math.nan), dict(how__epsilon=math.inf), dict(rows=-1), dict(width=0), dict(x=None), dict(out=None),
    dict(x__type=4), dict(add__type=5), dict(weight__type=3), dict(sum__type=3), dict(sum__type=4), dict(out__type=5), dict(out__type=-1), dict(x__stride=-1),
    dict(sum__stride=127), dict(out__stride=127), dict(x__data=AT + 2), dict(out__data=5 * AT + 1), dict(how__limit=-1), dict(how__limit=5), dict(how__group=4),
    dict(how__scales=AT), CODES | dict(how__limit=0), CODES | dict(how__limit=128), CODES | dict(how__group=-1), CODES | dict(how__scales=AT + 2),
    CODES | dict(out__stride=127), CODES | dict(out__data=0), CODES | dict(how__scales=0, out__unit=0.0), CODES | dict(how__scales=0, out__unit=math.inf),
    CODES | dict(how__scales=0, how__group=8), dict(out__type=3, out__stride=128, out__unit=-1.0), dict(out__type=3, how__limit=wl.P // 2 + 1), dict(out__type=3, how__limit=1 << 24),
    dict(out__data=AT, out__type=1), dict(out__data=AT, out__stride=256), dict(sum__data=2 * AT, sum__type=2), dict(out__data=3 * AT), dict(out__data=4 * AT),
    dict(sum__data=4 * AT), dict(rows=1 << 23)])
def test_norm_refuses(ctx, change):
    assert _norm(ctx, **change) == EARG


# ---- binding -------------------------------------------------------------------------------------------------------
def _on_gpu(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnGpu)


class Context(binding.Context):
    def __init__(self):
        self.lib, self.h = Unlaunched(), None

    def close(self):
        pass


@pytest.mark.parametrize("change", [dict(out=_on_gpu(5, 7)), dict(out=_on_gpu(4, 8)), dict(add=_on_gpu(5, 9)), dict(sum_out=_on_gpu(6, 8)), dict(weight=_on_gpu(7)),
                                    dict(weight=_on_gpu(2, 8)), dict(scales=_on_gpu(4), out=_on_gpu(5, 8, dtype=torch.int8), limit=9),
                                    dict(scales=_on_gpu(5, 2), group=3, out=_on_gpu(5, 8, dtype=torch.int8), limit=9), dict(x=_on_gpu(8, 5).t())])
def test_norm_refuses_other_shapes(change):
    with pytest.raises(ValueError):
        Context().rms_norm(**(dict(x=_on_gpu(5, 8), out=_on_gpu(5, 8)) | change))


def test_norm_refuses_a_row_that_is_no_row():
    for x in (_on_gpu(8), _on_gpu(8)[0]):
        with pytest.raises(ValueError):
            Context().rms_norm(x, x)


@pytest.mark.parametrize("change", [dict(x=torch.zeros(5, 8)), dict(add=torch.zeros(5, 8)), dict(add=_on_gpu(5, 8, dtype=torch.int8)), dict(x=_on_gpu(5, 8, dtype=torch.float64)),
                                    dict(scales=torch.zeros(5), out=_on_gpu(5, 8, dtype=torch.int8)), dict(scales=_on_gpu(5, dtype=torch.float64), out=_on_gpu(5, 8, dtype=torch.int8))])
def test_norm_refuses_other_tensors(change):
    with pytest.raises(TypeError):
        Context().rms_norm(**(dict(x=_on_gpu(5, 8), out=_on_gpu(5, 8)) | change))


def test_axes_refuse_other_tensors():
    table = _on_gpu(9, 4, 2)
    for bad in (dict(axis=[0] * 5), dict(axis=[0, 0, 4, 0]), dict(column=[0, 1, 2, 4]), dict(axis=[], column=[]), dict(axis=[-1, 0, 0, 0]), dict(table=_on_gpu(9, 8))):
        with pytest.raises(ValueError):
            binding.AxesRope(**(dict(table=table, axis=[0, 0, 1, 1], column=[0, 1, 2, 3]) | bad))
    with pytest.raises(TypeError):
        binding.AxesRope(torch.zeros(9, 4, 2), [0] * 4, [0] * 4)
    rope = binding.AxesRope(table, [0, 0, 1, 1], [0, 1, 2, 3])
    good = dict(rope=rope, at=_on_gpu(5, 2, dtype=torch.int32), x=_on_gpu(5, 3, 8), out=_on_gpu(5, 3, 8))
    for bad in (dict(at=_on_gpu(4, 2, dtype=torch.int32)), dict(at=_on_gpu(5, 1, dtype=torch.int32)), dict(out=_on_gpu(5, 2, 8)), dict(x=_on_gpu(5, 24), out=_on_gpu(5, 24)),
                dict(at=_on_gpu(2, 5, dtype=torch.int32).t())):
        with pytest.raises(ValueError):
            Context().rope_apply(**(good | bad))
    for bad in (dict(at=_on_gpu(5, 2)), dict(at=torch.zeros(5, 2, dtype=torch.int32)), dict(x=torch.zeros(5, 3, 8))):
        with pytest.raises(TypeError):
            Context().rope_apply(**(good | bad))


def test_cache_refuses_other_tensors(ctx):
    with pytest.raises(ValueError):
        binding.Kv4Cache(ctx, 2, 64, _on_gpu(3, 100, dtype=torch.uint8))
    with pytest.raises(TypeError):
        binding.Kv4Cache(ctx, 2, 64, torch.zeros(3, 2 * ref.head_bytes(64), dtype=torch.uint8))
    with pytest.raises(TypeError):
        binding.Kv4Cache(ctx, 2, 64, _on_gpu(3, 2 * ref.head_bytes(64), dtype=torch.int8))
    cache = binding.Kv4Cache(ctx, 2, 64, _on_gpu(3, 2 * ref.head_bytes(64), dtype=torch.uint8))
    with pytest.raises(ValueError):
        cache.append(None, _on_gpu(5, 2, 64), _on_gpu(4, 2, 64))


def test_kernels_stay_in_registers():
    from tests.test_kernel_registers import _kernels
    found = {name: k for (_, name), k in _kernels().items() if any(w in name for w in ("kv4_", "rope_apply", "rms_norm"))}
    assert sum("kv4_attention" in n for n in found) >= 8 and sum("rms_norm" in n for n in found) >= 2
    assert all(k[".private_segment_fixed_size"] == 0 for k in found.values()), {n: k[".private_segment_fixed_size"] for n, k in found.items()}
