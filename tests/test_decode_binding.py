"""The binding refuses tensors that a call would read or write beyond, on the host and before anything is launched."""
import pytest
import torch

from paper_2105_01827_amd import binding, workloads as wl

HEADS, DIM = 2, 16


@pytest.fixture(scope="module")
def ctx():
    par = wl.DEFAULT
    return binding.Context(par.n, par.q, par.p, par.gadget_bits)


class Unlaunched:
    """Entry points that must not be reached"""

    def __getattr__(self, name):
        raise AssertionError(f"{name} was called")


class Batch:
    ref = None


def _cache():
    """a cache whose memory is of no matter: its calls go nowhere"""
    cache = object.__new__(binding.KvCache)
    cache.heads, cache.head_dim, cache.ref, cache._lib, cache._ctx = HEADS, DIM, None, Unlaunched(), None
    return cache


class OnGpu(torch.Tensor):
    """a tensor that says that it lies on the GPU, so that all else about it is looked at without one"""
    is_cuda = True


def _on_gpu(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnGpu)


GOOD = dict(k=(5, HEADS, DIM), v=(5, HEADS, DIM), q=(5, 6, DIM), q_out=(5, 6, DIM))


def _append(make, **change):
    shapes = GOOD | change
    return _cache().append(Batch(), *(make(*shapes[n]) for n in ("k", "v")), **{n: make(*shapes[n]) for n in ("q", "q_out")})


@pytest.mark.parametrize("change", [dict(k=(5, HEADS, DIM - 1)), dict(k=(5, HEADS - 1, DIM)), dict(v=(5, HEADS + 1, DIM)),
                                    dict(v=(5, HEADS * DIM // 2)), dict(v=(4, HEADS, DIM)), dict(q_out=(5, 5, DIM)),
                                    dict(q_out=(4, 6, DIM)), dict(q=(5, 6, DIM - 1)), dict(q=(5, 7 * DIM)), dict(q=(5, 7, DIM))])
def test_append_refuses_other_shapes(change):
    with pytest.raises(ValueError):
        _append(_on_gpu, **change)


def test_append_takes_what_fits():
    for change in (dict(), dict(k=(5, HEADS * DIM)), dict(q=(5, 6 * DIM)), dict(q_out=(9, 6, DIM)), dict(q=(5, 1, 6 * DIM))):
        with pytest.raises(AssertionError, match="gala_kv_append was called"):
            _append(_on_gpu, **change)


@pytest.mark.parametrize("k,v", [((5, HEADS, DIM), (4, HEADS, DIM)), ((5, HEADS, 8), (5, HEADS, 8)), ((5, 1, DIM), (5, 1, DIM))])
def test_export_refuses_other_shapes(k, v):
    with pytest.raises(ValueError):
        _cache().export(Batch(), _on_gpu(*k), _on_gpu(*v))


@pytest.mark.parametrize("q,out,bytes_", [((5, 6, DIM), (5, 6, DIM - 1), 64), ((5, 6, DIM), (4, 6, DIM), 64), ((5, 6, DIM), (5, 5, DIM), 64),
                                          ((5, 6, DIM - 1), (5, 6, DIM - 1), 64), ((5, 6, DIM), (5, 6, DIM), 65)])
def test_attention_refuses_other_shapes(q, out, bytes_):
    with pytest.raises(ValueError):
        _cache().attention(Batch(), _on_gpu(*q), _on_gpu(*out), 1.0, _on_gpu(64, dtype=torch.uint8), bytes_)


def test_sample_refuses_a_workspace_that_is_too_small(ctx):
    with pytest.raises(ValueError):
        ctx.sample(_on_gpu(3, 10), _on_gpu(3), _on_gpu(3, dtype=torch.int32), _on_gpu(63, dtype=torch.uint8), 64)


def test_a_rope_table_of_another_shape():
    for shape in [(10, 8), (10, 8, 3), (10, 8, 2, 1)]:
        with pytest.raises(ValueError):
            binding.Rope(_on_gpu(*shape))


def test_memory_of_the_host_is_refused(ctx):
    host, words = torch.zeros, dict(dtype=torch.int32)
    scratch = torch.zeros(64, dtype=torch.uint8)
    with pytest.raises(TypeError, match="GPU"):
        _append(host)
    with pytest.raises(TypeError, match="GPU"):
        _cache().export(Batch(), host(5, HEADS, DIM), host(5, HEADS, DIM))
    with pytest.raises(TypeError, match="GPU"):
        _cache().attention(Batch(), host(5, 6, DIM), host(5, 6, DIM), 1.0, scratch, 64)
    with pytest.raises(TypeError, match="GPU"):
        _cache().attention(Batch(), _on_gpu(5, 6, DIM), _on_gpu(5, 6, DIM), 1.0, scratch, 64)
    with pytest.raises(TypeError, match="GPU"):
        binding.Rope(host(10, 8, 2))
    with pytest.raises(TypeError, match="GPU"):
        binding.KvBatch(host(3, **words), host(2, **words), host(2, 1, **words), 1, 1)
    with pytest.raises(TypeError, match="GPU"):
        binding.KvCache(ctx, HEADS, DIM, torch.zeros(3, binding.KvCache.page_bytes(HEADS, DIM), dtype=torch.int8), host(3, HEADS, 2))
    with pytest.raises(TypeError, match="GPU"):
        ctx.sample(host(3, 10), host(3), host(3, **words), scratch, 64)
