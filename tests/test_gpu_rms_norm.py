"""Residual and root-mean-square norm in few bits: bit for bit what the definition gives with its roundings to 32 bits."""
import numpy as np
import pytest
import torch

from paper_2105_01827_amd import binding, workloads as wl
from tests import decode_reference as dref, kv4_reference as ref

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "residue": torch.int64, "codes": torch.int8}
UNIT = 2.0 ** -12


@pytest.fixture(scope="module")
def ctx():
    par = wl.DEFAULT
    return binding.Context(par.n, par.q, par.p, par.gadget_bits)


def _values(gen, kind, *shape):
    x = torch.randn(*shape, generator=gen) * (1 + 9 * (torch.rand(shape[-1], generator=gen) < 0.05))
    return torch.round(x / UNIT).to(torch.int64).remainder(wl.P) if kind == "residue" else x.to(TYPES[kind])


def _plain(x):
    return None if x is None else dref.centred(x.cpu().numpy(), wl.P, UNIT).astype(np.float32) if x.dtype == torch.int64 else x.cpu().float().numpy()


def _residues(codes):
    return torch.from_numpy(codes).remainder(wl.P)


class Case:
    def __init__(self, rows, width, kind="f32", add="f32", out="codes", weight="f32", seed=0):
        gen = torch.Generator().manual_seed(seed + width)
        self.x = _values(gen, kind, rows, width).cuda()
        self.add = _values(gen, add, rows, width).cuda() if add else None
        self.weight = (1 + 0.3 * torch.randn(width, generator=gen)).to(TYPES[weight]).cuda() if weight else None
        self.out = torch.full((rows, width), 7, dtype=TYPES[out], device="cuda")
        self.sum = torch.full((rows, width), 7, dtype=torch.float32 if kind == "residue" else TYPES[kind], device="cuda")

    def run(self, ctx, limit=0, group=0, unit=None, epsilon=1e-6, scaled=None, stream=None):
        rows, width = self.x.shape
        whole = self.out.dtype in (torch.int8, torch.int64)
        scaled = whole and unit is None if scaled is None else scaled
        self.scales = torch.full((rows, -(-width // (group or width))), -1.0, device="cuda") if scaled else None
        ctx.rms_norm(self.x, self.out, add=self.add, sum_out=self.sum, weight=self.weight, epsilon=epsilon, limit=limit, scales=self.scales, group=group,
                     unit=unit or 1.0, x_unit=UNIT, add_unit=UNIT, stream=stream)
        return self

    def check(self, limit=0, group=0, unit=None, epsilon=1e-6):
        s, y = ref.rms_norm(_plain(self.x), _plain(self.add), _plain(self.weight), epsilon)
        if self.sum is not None:
            assert torch.equal(self.sum.cpu(), torch.from_numpy(s).to(self.sum.dtype))
        if self.out.dtype not in (torch.int8, torch.int64):
            assert torch.equal(self.out.cpu(), torch.from_numpy(y).to(self.out.dtype))
            return
        codes, scales = ref.whole(y, limit or wl.P // 2, group, unit)
        assert torch.equal(self.out.cpu(), _residues(codes) if self.out.dtype == torch.int64 else torch.from_numpy(codes).to(torch.int8))
        if scales is not None:
            assert np.array_equal(self.scales.cpu().numpy(), scales)


WIDTHS = [1, 7, 8, 63, 64, 65, 128, 511, 512, 513, 520, 1000, 2047, 2048, 2049, 2056, 4095, 4096, 4104, 5121, 8192, 8193, 8200, 16383, 16384, 16385, 16392, 20000]


@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("out", ["codes", "f32"])
def test_widths(ctx, width, out):
    for rows in (1, 5):
        c = Case(rows, width, out=out)
        limit = 127 if out == "codes" else 0
        c.run(ctx, limit).check(limit)


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16", "residue"])
@pytest.mark.parametrize("add", [None, "f32", "f16", "bf16", "residue"])
@pytest.mark.parametrize("out", ["f32", "f16", "bf16", "codes", "residue"])
def test_types(ctx, kind, add, out):
    limit = {"codes": 127, "residue": 63}.get(out, 0)
    for width, weight in ((136, "bf16"), (137, "f16"), (1040, None)):
        Case(6, width, kind, add, out, weight, seed=3).run(ctx, limit).check(limit)


@pytest.mark.parametrize("width,group", [(256, 32), (256, 64), (4096, 128), (300, 128), (1000, 8), (1000, 24), (1000, 1), (129, 128), (512, 512), (500, 600), (8192, 8),
                                         (16384, 1), (16384, 2), (20000, 128), (20000, 1), (20000, 20000), (9000, 4500)])
@pytest.mark.parametrize("out", ["codes", "residue"])
def test_groups(ctx, width, group, out):
    Case(3, width, "bf16", "residue", out, seed=4).run(ctx, 127, group).check(127, group)


@pytest.mark.parametrize("limit", [1, 7, 63, 127])
@pytest.mark.parametrize("width", [200, 201, 17000])
def test_limits(ctx, limit, width):
    for out in ("codes", "residue"):
        Case(4, width, out=out, seed=5).run(ctx, limit).check(limit)
        Case(4, width, out=out, seed=5).run(ctx, limit, unit=2.0 ** -5).check(limit, unit=2.0 ** -5)


def test_large_limits_of_residues(ctx):
    Case(4, 256, out="residue").run(ctx, 300000).check(300000)
    Case(4, 256, out="residue").run(ctx).check()                         # every number that there is
    Case(4, 256, out="residue").run(ctx, unit=2.0 ** -16).check(unit=2.0 ** -16)
    Case(4, 256, out="residue").run(ctx, unit=2.0 ** -30).check(unit=2.0 ** -30)        # all held to p / 2
    # a modulus whose half has more than 24 bits
    wide = binding.Context(64, 1152921504606844417, 2147473409, 20)
    c = Case(4, 256, add=None, out="residue").run(wide, unit=2.0 ** -30)
    _, y = ref.rms_norm(_plain(c.x), None, _plain(c.weight), 1e-6)
    most = int(np.nextafter(np.float32(2147473409 // 2), np.float32(0))) if int(np.float32(2147473409 // 2)) > 2147473409 // 2 else int(np.float32(2147473409 // 2))
    codes, _ = ref.whole(y, most, 0, 2.0 ** -30)
    assert torch.equal(c.out.cpu(), torch.from_numpy(codes).remainder(2147473409))


@pytest.mark.parametrize("width", [96, 97, 17000])
def test_no_numbers_and_zeros(ctx, width):
    """A row of zeros, NaN, infinities, and rows so large and so small that a square leaves 32 bits."""
    for out, limit in (("codes", 127), ("residue", 127), ("f32", 0)):
        c = Case(8, width, add=None, out=out, seed=6)
        c.x[0] = 0
        c.x[1, 5], c.x[2, 3], c.x[3, 4] = float("nan"), float("inf"), float("-inf")
        c.x[4] *= 1e30
        c.x[5] *= 1e-25
        c.x[6, 1:] = 0
        c.run(ctx, limit, epsilon=0.0)
        with np.errstate(all="ignore"):
            s, y = ref.rms_norm(_plain(c.x), None, _plain(c.weight), 0.0)
            assert torch.equal(c.sum.cpu().nan_to_num(9), torch.from_numpy(s).nan_to_num(9))
            if out == "f32":
                y = torch.from_numpy(y)
                assert torch.equal(c.out.cpu().isnan(), y.isnan()) and torch.equal(c.out.cpu().nan_to_num(9), y.nan_to_num(9))
            else:
                codes, scales = ref.whole(y, limit, 0)
                assert torch.equal(c.out.cpu(), _residues(codes) if out == "residue" else torch.from_numpy(codes).to(torch.int8))
                assert np.array_equal(c.scales.cpu().numpy(), scales)
    c = Case(2, width, add=None, out="codes", seed=6)                    # zeros with an epsilon: zeros
    c.x[0] = 0
    c.run(ctx, 127).check(127)
    assert bool((c.out[0] == 0).all()) and float(c.scales[0, 0]) == 0
    c = Case(3, width, add=None, out="codes", seed=6)                    # a fixed unit
    c.x[0, 1], c.x[1, 2] = float("nan"), float("inf")
    c.run(ctx, 100, unit=0.25)
    assert bool((c.out[:2] == 0).all()) and bool((c.out[2] != 0).any())


@pytest.mark.parametrize("rows", [1, 2, 3, 4, 5, 1000])
def test_rows_that_share_a_workgroup(ctx, rows):
    for width in (128, 100):
        Case(rows, width, "bf16", "bf16", seed=7).run(ctx, 127).check(127)


@pytest.mark.parametrize("width", [256, 257, 17000])
def test_in_place(ctx, width):
    """The stream in place, the sum over the added numbers, the output over either."""
    for kind in ("f32", "bf16"):
        want = Case(5, width, kind, kind, kind, seed=8).run(ctx)
        for sum_at, out_at in (("x", None), ("add", None), (None, "x"), (None, "add"), ("x", "add"), ("add", "x")):
            c = Case(5, width, kind, kind, kind, seed=8)
            c.sum = getattr(c, sum_at) if sum_at else c.sum
            c.out = getattr(c, out_at) if out_at else c.out
            c.run(ctx)
            assert torch.equal(c.sum, want.sum) and torch.equal(c.out, want.out)


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16", "residue"])
def test_rows_that_begin_anywhere_and_apart(ctx, kind):
    """Rows on 16 bytes, and the same rows elsewhere: the same bits, and nothing between the rows."""
    for out in ("codes", "residue", "f32"):
        limit = {"codes": 127, "residue": 127}.get(out, 0)
        want = Case(9, 264, kind, kind, out, seed=9).run(ctx, limit)
        c = Case(9, 264, kind, kind, out, seed=9)
        wide = torch.full((9, 271), 5, dtype=c.out.dtype, device="cuda")
        c.out = wide[:, 3:267]
        for name in ("x", "add"):
            t = getattr(c, name)
            setattr(c, name, torch.zeros(9, 265, dtype=t.dtype, device="cuda")[:, 1:].copy_(t))
        c.run(ctx, limit)
        assert torch.equal(c.out, want.out) and torch.equal(c.sum, want.sum)
        assert bool((wide[:, :3] == 5).all()) and bool((wide[:, 267:] == 5).all())


def test_one_row_for_all_and_no_sum(ctx):
    c = Case(6, 128, "f32", "bf16", "codes", seed=10)
    c.add = c.add[:1].expand(6, -1)
    c.sum = None
    c.run(ctx, 127).check(127)
    none = Case(1, 16, add=None)
    ctx.rms_norm(none.x[:0], none.out[:0], limit=127, scales=torch.empty(1, device="cuda")) if none.x[:0].data_ptr() else None


def test_another_stream_and_a_graph(ctx):
    c = Case(33, 2000, "bf16", "residue", "residue", seed=11).run(ctx, 127, 40)
    want = [t.clone() for t in (c.out, c.sum, c.scales)]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        ctx.rms_norm(c.x, c.out, add=c.add, sum_out=c.sum, weight=c.weight, limit=127, scales=c.scales, group=40, add_unit=UNIT, stream=torch.cuda.current_stream())
    for _ in range(3):
        for t in (c.out, c.sum, c.scales):
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((c.out, c.sum, c.scales), want))
