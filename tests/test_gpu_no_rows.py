"""Empty tensors in the calls around the 4-bit cache: a batch of nothing does nothing."""
import pytest
import torch

from paper_2105_01827_amd import binding
from tests.test_gpu_kv4_attention import ctx  # noqa: F401

pytestmark = pytest.mark.gpu


def _empty(*shape, dtype=torch.float32):
    return torch.empty(0, *shape, dtype=dtype, device="cuda")


def test_norm(ctx):  # noqa: F811
    x, weight = _empty(128), torch.ones(128, device="cuda")
    ctx.rms_norm(x, _empty(128))
    ctx.rms_norm(x, _empty(128, dtype=torch.bfloat16), add=_empty(128, dtype=torch.int64), sum_out=_empty(128), weight=weight)
    ctx.rms_norm(x, _empty(128, dtype=torch.int64), limit=63)
    for group in (0, 8):
        ctx.rms_norm(x, _empty(128, dtype=torch.int8), weight=weight, limit=127, scales=_empty(-(-128 // (group or 128))), group=group)
    some = torch.zeros(3, 128, device="cuda")
    ctx.rms_norm(some[:0], some[3:], add=some[1:1])
    torch.cuda.synchronize()


def test_positions(ctx):  # noqa: F811
    axis, column = binding.axes_layout([8, 8])
    rope = binding.AxesRope(torch.from_numpy(binding.rope_table(9, 32)).cuda(), axis, column)
    x = _empty(2, 32)
    ctx.rope_apply(rope, _empty(2, dtype=torch.int32), x, x)
    ctx.rope_apply(rope, _empty(2, dtype=torch.int32), x, _empty(2, 32, dtype=torch.bfloat16))
    torch.cuda.synchronize()


def test_cache(ctx):  # noqa: F811
    cache = binding.Kv4Cache(ctx, 2, 64, pages=1)
    before = cache.data.clone()
    words = dict(dtype=torch.int32, device="cuda")
    none = binding.KvBatch(torch.zeros(1, **words), torch.empty(0, **words), torch.empty(0, 1, **words), 1, 1)
    no_new = binding.KvBatch(torch.zeros(2, **words), torch.ones(1, **words), torch.zeros(1, 1, **words), 0, 1)
    for batch in (none, no_new):
        q, k = _empty(4, 64), _empty(2, 64)
        cache.append(batch, k, k, q=q, q_out=torch.empty_like(q))
        cache.export(batch, k, torch.empty_like(k))
        need = cache.attention_workspace_bytes(batch, 4)
        cache.attention(batch, q, torch.empty_like(q), 1.0, torch.empty(max(need, 16), dtype=torch.uint8, device="cuda"), need)
    assert torch.equal(cache.data, before)
