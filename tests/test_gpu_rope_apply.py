"""Rotary positions with several axes: bit for bit what the definition gives when every product and sum is rounded to 32 bits."""
import numpy as np
import pytest
import torch

from paper_2105_01827_amd import binding, workloads as wl
from tests import decode_reference as dref, kv4_reference as ref

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "residue": torch.int64}
UNIT = 2.0 ** -12


@pytest.fixture(scope="module")
def ctx():
    par = wl.DEFAULT
    return binding.Context(par.n, par.q, par.p, par.gadget_bits)


def _case(seed, kind, rows, heads, dim, sections, order, interleaved, positions=50):
    gen = torch.Generator().manual_seed(seed)
    axis, column = binding.axes_layout(sections, order)
    table = torch.from_numpy(binding.rope_table(positions, 2 * (max(column) + 1)))
    at = torch.randint(0, positions, (rows, len(sections)), generator=gen, dtype=torch.int32)
    x = torch.randn(rows, heads, dim, generator=gen)
    x = torch.round(x / UNIT).to(torch.int64).remainder(wl.P) if kind == "residue" else x.to(TYPES[kind])
    return binding.AxesRope(table.cuda(), axis, column, interleaved), table.numpy(), np.array(axis), np.array(column), at, x


def _want(x, table, axis, column, at, interleaved):
    plain = dref.centred(x.numpy(), wl.P, UNIT).astype(np.float32) if x.dtype == torch.int64 else x.float().numpy()
    inside = ((at >= 0) & (at < table.shape[0])).all(1).numpy()
    a = table[np.where(inside[:, None], at.numpy()[:, axis], 0), column]
    out = ref.turn(plain, a[..., 0], a[..., 1], 2 * len(axis), interleaved)
    out[~inside] = np.nan
    return torch.from_numpy(out)


@pytest.mark.parametrize("kind,out,dim,sections,order,interleaved", [
    ("f32", "f32", 64, [8, 12, 12], 0, False), ("bf16", "bf16", 128, [16, 24, 24], 1, False), ("f16", "f16", 80, [20, 20], 2, False),
    ("residue", "f32", 128, [64], 0, True), ("residue", "bf16", 64, [4, 12], 2, True), ("bf16", "f32", 256, [32, 32, 32, 32], 1, True),
    ("f32", "f16", 33, [3, 5, 8], 0, False), ("f16", "bf16", 96, [5, 7], 1, False), ("f32", "f32", 200, [1], 0, False), ("f16", "f16", 2, [1], 0, True),
    ("bf16", "bf16", 40, [0, 20], 0, False), ("bf16", "bf16", 72, [16, 16], 0, False), ("f16", "f16", 48, [4, 4], 0, True)])
@pytest.mark.parametrize("rows,heads", [(1, 1), (7, 5), (300, 3)])
def test_types_and_layouts(ctx, kind, out, dim, sections, order, interleaved, rows, heads):
    rope, table, axis, column, at, x = _case(dim + rows, kind, rows, heads, dim, sections, order, interleaved)
    got = torch.full((rows, heads, dim), 7.0, dtype=TYPES[out], device="cuda")
    ctx.rope_apply(rope, at.cuda(), x.cuda(), got, unit=UNIT)
    assert torch.equal(got.cpu(), _want(x, table, axis, column, at, interleaved).to(TYPES[out]))


@pytest.mark.parametrize("heads", [1, 40, 131])
def test_many_rows(ctx, heads):
    """Enough that a thread turns several heads by the same angles."""
    rope, table, axis, column, at, x = _case(heads, "bf16", 40000 // heads + 3, heads, 128, [16, 24, 24], 0, False)
    got = torch.empty_like(x, device="cuda")
    ctx.rope_apply(rope, at.cuda(), x.cuda(), got)
    assert torch.equal(got.cpu(), _want(x, table, axis, column, at, False).bfloat16())


def test_one_axis_is_append_s_rotation(ctx):
    """A token's position on every axis: the same bits as queries get on their way into a cache."""
    table = torch.from_numpy(binding.rope_table(90, 64)).cuda()
    x = torch.randn(90, 4, 64, generator=torch.Generator().manual_seed(4)).bfloat16().cuda()
    starts, lens, pages = (torch.tensor(v, dtype=torch.int32, device="cuda") for v in ([0, 90], [90], [[0, 1]]))
    want, got = torch.empty_like(x), torch.empty_like(x)
    cache = binding.Kv4Cache(ctx, 1, 64, pages=2)
    cache.append(binding.KvBatch(starts, lens, pages, 90, 90), None, None, q=x, q_out=want, rope=binding.Rope(table))
    axis, column = binding.axes_layout([8, 12, 12], 1)
    at = torch.arange(90, dtype=torch.int32, device="cuda")[:, None].expand(-1, 3)
    ctx.rope_apply(binding.AxesRope(table, axis, column), at.contiguous(), x, got)
    assert torch.equal(got, want)


@pytest.mark.parametrize("dim,sections", [(64, [16, 16]), (33, [8, 8])])
def test_positions_that_the_table_does_not_have(ctx, dim, sections):
    rope, table, axis, column, at, x = _case(5, "f32", 9, 2, dim, sections, 0, False)
    at[1, 0], at[3, 1], at[5, 0], at[8, 1] = -1, 50, 2 ** 31 - 1, -2 ** 31
    got = torch.empty_like(x, device="cuda")
    ctx.rope_apply(rope, at.cuda(), x.cuda(), got)
    want = _want(x, table, axis, column, at, False)
    assert torch.equal(got.cpu().isnan(), want.isnan()) and torch.equal(got.cpu().nan_to_num(9), want.nan_to_num(9))
    assert int(got.isnan().any(-1).any(-1).sum()) == 4


@pytest.mark.parametrize("dim", [64, 33])
def test_in_place_rows_apart_and_part_of_a_projection(ctx, dim):
    """Queries and keys of a fused projection in place; the values behind them, and what lies between rows, are left alone."""
    rope, table, axis, column, at, x = _case(6, "bf16", 50, 8, dim, [8, 8], 0, False)
    wide = torch.full((50, 8 * dim + 8), 3.0, dtype=torch.bfloat16, device="cuda")
    rows = wide[:, :8 * dim].view(50, 8, dim)
    rows.copy_(x)
    ctx.rope_apply(rope, at.cuda(), rows[:, :6], rows[:, :6])
    assert torch.equal(rows[:, :6].cpu(), _want(x[:, :6], table, axis, column, at, False).bfloat16())
    assert torch.equal(rows[:, 6:].cpu(), x[:, 6:]) and bool((wide[:, 8 * dim:] == 3).all())


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16", "residue"])
def test_rows_that_begin_anywhere(ctx, kind):
    rope, table, axis, column, at, x = _case(7, kind, 21, 3, 64, [16, 16], 2, False)
    out = torch.float32 if kind == "residue" else TYPES[kind]
    want = torch.empty(x.shape, dtype=out, device="cuda")
    ctx.rope_apply(rope, at.cuda(), x.cuda(), want, unit=UNIT)
    shifted = torch.empty(x.numel() + 8, dtype=x.dtype, device="cuda")[1:1 + x.numel()].view(x.shape).copy_(x)
    got = torch.empty(x.numel() + 8, dtype=out, device="cuda")[3:3 + x.numel()].view(x.shape)
    ctx.rope_apply(rope, at.cuda(), shifted, got, unit=UNIT)
    assert torch.equal(got, want)


def test_one_position_for_all_rows_and_none(ctx):
    rope, table, axis, column, at, x = _case(8, "f32", 12, 2, 32, [8, 8], 0, False)
    one = at[:1].expand(12, -1)
    got = torch.empty_like(x, device="cuda")
    ctx.rope_apply(rope, at.cuda()[:1].expand(12, -1), x.cuda(), got)
    assert torch.equal(got.cpu(), _want(x, table, axis, column, one, False))
    none = torch.empty(0, 2, 32, device="cuda")
    if none.data_ptr():
        ctx.rope_apply(rope, at.cuda()[:0], none, none)


def test_another_stream_and_a_graph(ctx):
    rope, table, axis, column, at, x = _case(9, "f16", 70, 4, 80, [20, 20], 2, False)
    at, x = at.cuda(), x.cuda()
    want, out = torch.empty_like(x), torch.empty_like(x)
    ctx.rope_apply(rope, at, x, want)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        ctx.rope_apply(rope, at, x, out, stream=torch.cuda.current_stream())
    for _ in range(3):
        out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
