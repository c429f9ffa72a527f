"""Attention over the paged 8-bit cache against the definition in 64 bits on the values that the cache stands for.  The bounds
come from what the header says of the products' operands (tests/decode_reference.py)."""
import numpy as np
import pytest
import torch

from paper_2105_01827_amd import binding, workloads as wl
from tests import decode_reference as ref

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "residue": torch.int64}
UNIT = 2.0 ** -12


@pytest.fixture(scope="module")
def ctx():
    par = wl.DEFAULT
    return binding.Context(par.n, par.q, par.p, par.gadget_bits)


def _int32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _plain(x):
    return ref.centred(x.cpu().numpy(), wl.P, UNIT) if x.dtype == torch.int64 else x.cpu().double().numpy()


class Case:
    def __init__(self, ctx, new, lens, heads, group, dim, kind="bf16", out=None, seed=0, spread=2.0, most=None, layout_gap=0):
        gen = torch.Generator().manual_seed(seed)
        self.new, self.lens, self.heads, self.group, self.dim, self.kind = new, lens, heads, group, dim, kind
        blocks = max(1, max(-(-n // 64) for n in lens))
        pages = len(lens) * blocks + 1
        self.cache = binding.KvCache(ctx, heads, dim, pages=pages)
        # codes everywhere, also behind the ends; only channels beyond the head's size are 0
        codes = torch.randint(-127, 128, (pages, heads, ref.head_bytes(dim)), generator=gen).to(torch.int8).numpy()
        self.k, self.v = (codes[:, :, p] for p in ref.code_places(dim))          # [page, head, token, channel]
        live = np.zeros(ref.head_bytes(dim), bool)
        for p in ref.code_places(dim):
            live[p] = True
        codes[:, :, ~live] = 0
        self.cache.codes.copy_(torch.from_numpy(codes).view(pages, -1))
        self.cache.scales.copy_((torch.rand(pages, heads, 2, generator=gen) + 0.5) / 73)
        self.table = torch.randperm(pages, generator=gen)[:len(lens) * blocks].view(len(lens), blocks).to(torch.int32)
        self.starts = np.concatenate([[0], np.cumsum(new)])
        q = torch.randn(int(self.starts[-1]), heads * group + layout_gap, dim, generator=gen) * spread
        q = torch.round(q / UNIT).to(torch.int64).remainder(wl.P) if kind == "residue" else q.to(TYPES[kind])
        self.q = q.cuda()[:, :heads * group]
        self.out_kind = out or kind
        self.most = most

    def run(self, scale=None, window=0, sinks=0, stream=None, out=None):
        self.scale, self.window, self.sinks = self.dim ** -0.5 if scale is None else scale, window, sinks
        most = self.most or (max(self.new), max(self.lens))
        batch = binding.KvBatch(_int32(self.starts.tolist()), _int32(self.lens), self.table.cuda(), *most)
        out = torch.full(self.q.shape, 7, dtype=TYPES[self.out_kind], device="cuda") if out is None else out
        need = self.cache.attention_workspace_bytes(batch, self.heads * self.group, window, sinks)
        self.workspace = torch.full((max(need, 16),), 0xff, dtype=torch.uint8, device="cuda")
        self.cache.attention(batch, self.q, out, self.scale, self.workspace, need, window=window, sinks=sinks, unit=UNIT, stream=stream)
        self.keep = batch
        return out

    def check(self, out, rows=None):
        got, q = _plain(out), _plain(self.q)
        scales = self.cache.scales.cpu().double().numpy()
        fine = self.kind in ("f32", "residue") or self.out_kind in ("f32", "residue")
        worst = 0.0
        max_new, max_len = self.most or (max(self.new), max(self.lens))
        for b, (n, length) in enumerate(zip(self.new, self.lens)):
            end = min(length, max_len)
            pages = self.table[b].numpy()
            ok = (pages >= 0) & (pages < scales.shape[0])
            at = np.where(ok, pages, 0)
            k = (self.k[at].astype(np.float64) * scales[at][..., 0, None, None]).transpose(1, 0, 2, 3).reshape(self.heads, -1, self.dim)
            v = (self.v[at].astype(np.float64) * scales[at][..., 1, None, None]).transpose(1, 0, 2, 3).reshape(self.heads, -1, self.dim)
            there = np.repeat(ok, 64)[:end]
            for i in range(n):
                row = self.starts[b] + i
                if rows is not None and (b, i) not in rows:
                    continue
                if i >= max_new:
                    assert (out[row].cpu() == 7).all()
                    continue
                tokens = min(end, k.shape[1])
                seen = ref.see(length - n + i, tokens, self.window, self.sinks) & there[:tokens]
                for h in range(self.heads * self.group):
                    if not np.isfinite(q[row, h]).all():
                        assert np.isnan(got[row, h]).all()
                        continue
                    at_scale = np.repeat(scales[at][:, h // self.group, 1], 64)[:tokens]
                    halves = not fine and min(max(self.new), max_new) * self.group >= 64
                    want, bound = ref.attention_in_halves(q[row, h], k[h // self.group, :tokens], v[h // self.group, :tokens], at_scale, seen,
                                                          self.scale) if halves else ref.attention(q[row, h], k[h // self.group, :tokens], v[h // self.group, :tokens], seen, self.scale,
                                                *((24, 23) if fine else (16, 15)))
                    eps = ref.UNIT_ROUNDOFF.get({"f16": "float16", "bf16": "bfloat16", "f32": "float32"}.get(self.out_kind), 0)
                    bound = bound + eps * (np.abs(want) + bound) + (UNIT / 2 if self.out_kind == "residue" else 0) + 2.0 ** -24
                    over = np.abs(got[row, h] - want) / bound
                    worst = max(worst, over.max())
                    assert over.max() <= 1, (b, i, h, over.max())
        return worst


@pytest.mark.parametrize("dim", [1, 15, 16, 33, 48, 64, 80, 96, 128, 129, 192, 200, 256])
@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_head_sizes(ctx, dim, kind):
    c = Case(ctx, [1, 1, 1], [200, 63, 1], 2, 3, dim, kind, seed=dim)
    c.check(c.run())


@pytest.mark.parametrize("kind,out", [("f32", "f32"), ("f16", "f16"), ("bf16", "bf16"), ("residue", "residue"), ("residue", "f32"),
                                      ("f32", "residue"), ("bf16", "f32"), ("f32", "bf16"), ("f16", "residue")])
def test_types(ctx, kind, out):
    c = Case(ctx, [1, 5], [300, 129], 2, 4, 64, kind, out, seed=3)
    c.check(c.run())


@pytest.mark.parametrize("heads,group", [(1, 1), (3, 1), (1, 5), (2, 8), (1, 16), (2, 17), (1, 40), (7, 2)])
def test_groups(ctx, heads, group):
    c = Case(ctx, [1, 3], [150, 70], heads, group, 64, seed=heads * 100 + group)
    c.check(c.run())


@pytest.mark.parametrize("length", [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 255, 256, 257, 1000, 4095, 4097])
def test_lengths(ctx, length):
    c = Case(ctx, [1], [length], 2, 2, 64, "f32", seed=length)
    c.check(c.run())


def test_many_lengths_in_one_batch(ctx):
    lens = [0, 1, 64, 65, 700, 3000, 128, 5, 2049, 1]
    c = Case(ctx, [0] + [1] * 8 + [0], lens, 3, 4, 128, seed=11)
    c.check(c.run())


@pytest.mark.parametrize("new,lens", [([64], [64]), ([65, 1, 130], [65, 200, 130]), ([100], [1000]), ([17, 33], [400, 33])])
@pytest.mark.parametrize("group", [1, 3, 8])
def test_prompts(ctx, new, lens, group):
    c = Case(ctx, new, lens, 2, group, 64, seed=sum(new) + group)
    c.check(c.run())


@pytest.mark.parametrize("dim,kind,group", [(128, "bf16", 4), (256, "f16", 2), (80, "f32", 5), (200, "residue", 1)])
def test_long_prompts(ctx, dim, kind, group):
    """some rows of each: the first, around the edges of tiles, the last"""
    c = Case(ctx, [600, 450], [600, 1300], 1, group, dim, kind, seed=dim)
    rows = {(0, i) for i in (0, 1, 15, 16, 63, 64, 255, 256, 599)} | {(1, i) for i in (0, 31, 32, 449)}
    c.check(c.run(), rows)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 0), (63, 4), (64, 64), (65, 100), (100, 0), (1000, 4), (5000, 5000)])
@pytest.mark.parametrize("new", [1, 90])
def test_windows(ctx, window, sinks, new):
    c = Case(ctx, [new, 1, new], [600, 50, new], 2, 2, 64, "f32", seed=window + sinks)
    rows = None if new == 1 else {(0, i) for i in (0, 1, 40, 89)} | {(2, i) for i in (0, 15, 16, 70, 89)} | {(1, 0)}
    c.check(c.run(window=window, sinks=sinks), rows)


def test_scales_far_apart(ctx):
    """Scores that rise and fall by hundreds, blocks whose values are a million times another's, a negative scale."""
    c = Case(ctx, [1, 4], [500, 300], 2, 2, 64, "f32", seed=21)
    c.cache.scales.mul_(torch.logspace(-3, 3, c.cache.scales.numel(), device="cuda").view_as(c.cache.scales)[torch.randperm(c.cache.scales.shape[0], device="cuda")])
    c.check(c.run())
    c.check(c.run(scale=-0.3))
    c.check(c.run(scale=0.0))


def test_zero_scales_and_zero_queries(ctx):
    c = Case(ctx, [1, 2], [200, 100], 2, 2, 64, seed=22)
    c.cache.scales[::2, :, 0] = 0
    c.cache.scales[::3, :, 1] = 0
    c.q[1, 2] = 0
    c.check(c.run())


def test_rows_that_see_nothing(ctx):
    """No tokens, positions before the first token, pages given back."""
    c = Case(ctx, [1, 5, 1, 2], [0, 3, 130, 70], 2, 3, 64, seed=23)
    c.table[2, :] = -1
    c.table[3, 1] = c.cache.codes.shape[0]
    out = c.run()
    c.check(out)
    assert bool((out[0] == 0).all() and (out[1:3] == 0).all() and (out[6] == 0).all())


def test_pages_behind_a_window_are_not_needed(ctx):
    c = Case(ctx, [1], [1000], 2, 2, 64, seed=24)
    want = c.run(window=200, sinks=3)
    c.table[0, 1:12] = -1                                        # 800 is in block 12
    assert torch.equal(c.run(window=200, sinks=3), want)


def test_scales_of_pages_nobody_sees_may_be_anything(ctx):
    """A block behind the end, one behind the window and one of nobody hold NaN: no row comes near them."""
    c = Case(ctx, [1, 1], [100, 400], 2, 2, 64, seed=25)
    seen = {int(c.table[0, 0]), int(c.table[0, 1])} | {int(p) for p in c.table[1, 4:7]}
    unseen = [p for p in range(c.cache.codes.shape[0]) if p not in seen]
    c.cache.scales[unseen] = float("nan")
    assert bool(c.run(window=140)[:2].isfinite().all())
    c.lens = [100, 400]
    c.check(c.run(window=140))


def test_a_query_with_nan_or_infinity_spoils_its_own_head_alone(ctx):
    c = Case(ctx, [1, 3], [100, 90], 2, 3, 64, "f32", seed=26)
    clean = c.run()
    c.q[0, 1, 5], c.q[2, 4, 63], c.q[3, 0, 0] = float("nan"), float("inf"), float("-inf")
    out = c.run()
    bad = torch.zeros(4, 6, dtype=torch.bool, device="cuda")
    bad[0, 1] = bad[2, 4] = bad[3, 0] = True
    assert bool(out[bad].isnan().all()) and torch.equal(out[~bad], clean[~bad])


def test_bounds_that_the_host_gives(ctx):
    """Rows beyond max_new are left alone, keys beyond max_len are not seen."""
    c = Case(ctx, [3, 6], [200, 90], 2, 2, 64, seed=27, most=(4, 150))
    c.check(c.run())
    c = Case(ctx, [1, 1], [200, 90], 2, 2, 64, seed=28, most=(1, 100000))
    c.check(c.run())


def test_rows_apart_and_in_place(ctx):
    c = Case(ctx, [2, 3], [200, 90], 2, 2, 48, seed=29, layout_gap=3)
    want = c.run()
    c.check(want)
    c.q = c.q.clone()
    assert torch.equal(c.run(out=c.q), want)


def test_a_long_sequence(ctx):
    """One query over 70000 tokens, split over the whole card and joined; twice the same bits."""
    c = Case(ctx, [1], [70001], 1, 4, 128, "f16", seed=30)
    out = c.run()
    c.check(out, {(0, 0)})
    for _ in range(3):
        assert torch.equal(c.run(), out)


def test_offsets_beyond_32_bits(ctx):
    """Pages that lie more than 4 GiB into the codes."""
    heads, dim, blocks = 1, 128, 300000
    free, _ = torch.cuda.mem_get_info()
    if free < 8 << 30:
        pytest.skip("needs 8 GiB")
    c = Case(ctx, [1], [130], heads, 2, dim, seed=31)
    want = c.run()
    big = binding.KvCache(ctx, heads, dim, pages=blocks)
    at = torch.tensor([blocks - 1, 7, blocks - 3])
    for i in range(3):
        big.codes[at[i]] = c.cache.codes[int(c.table[0, i])]
        big.scales[at[i]] = c.cache.scales[int(c.table[0, i])]
    assert big.codes.numel() > 1 << 32
    c.cache, c.table = big, at.view(1, 3).to(torch.int32)
    assert torch.equal(c.run(), want)


def test_another_stream_and_a_graph(ctx):
    c = Case(ctx, [1, 1], [5000, 300], 2, 4, 64, seed=32)
    want = c.run()
    out = torch.empty_like(want)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    batch, need, ws = c.keep, c.workspace.numel(), c.workspace
    with torch.cuda.graph(graph, stream=stream):
        c.cache.attention(batch, c.q, out, c.scale, ws, need, stream=torch.cuda.current_stream())
    for _ in range(3):
        out.zero_(), ws.fill_(0xff)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_after_append(ctx):
    """The order of codes that append writes is the order that attention reads."""
    heads, group, dim, n = 2, 4, 96, 150
    c = Case(ctx, [n], [n], heads, group, dim, "f32", seed=33)
    k, v = (torch.randn(n, heads, dim, generator=torch.Generator().manual_seed(s)).cuda() for s in (1, 2))
    c.run()
    c.cache.append(c.keep, k, v)
    codes = c.cache.codes.cpu().numpy().reshape(c.cache.codes.shape[0], heads, -1)
    c.k, c.v = (codes[:, :, p] for p in ref.code_places(dim))
    c.check(c.run(), {(0, i) for i in (0, 1, 64, 100, 149)})


@pytest.mark.parametrize("dim", [1, 16, 40, 64, 72, 80, 96, 112, 128, 160, 192, 200, 256])
@pytest.mark.parametrize("kind,group", [("bf16", 3), ("f16", 8)])
def test_prompts_of_every_head_size(ctx, dim, kind, group):
    c = Case(ctx, [180, 1, 77], [180, 300, 200], 32, group, dim, kind, seed=dim, spread=1.0)
    out = c.run()
    c.check(out, {(0, 0), (0, 63), (0, 179), (1, 0), (2, 5), (2, 76)} if dim < 100 else {(0, 179), (2, 5)})


@pytest.mark.parametrize("window,sinks", [(1, 0), (16, 4), (100, 0), (65, 70), (1000, 4)])
def test_windows_of_prompts(ctx, window, sinks):
    c = Case(ctx, [200, 50, 130], [500, 50, 131], 32, 4, 64, "bf16", seed=window)
    c.check(c.run(window=window, sinks=sinks), {(0, i) for i in (0, 17, 199)} | {(1, 0), (1, 49), (2, 0), (2, 129)})


def test_prompts_with_scales_far_apart(ctx):
    c = Case(ctx, [150, 3], [400, 90], 32, 4, 64, "f16", seed=41)
    n = c.cache.scales.numel()
    c.cache.scales.mul_(torch.logspace(-2, 2, n, device="cuda")[torch.randperm(n, device="cuda")].view_as(c.cache.scales))
    rows = {(0, 0), (0, 70), (0, 149), (1, 2)}
    c.check(c.run(scale=0.02), rows)
    c.check(c.run(scale=-0.02), rows)
    c.check(c.run(scale=0.0), rows)
    c.cache.scales[::2, :, 0] = 0
    c.cache.scales[::3, :, 1] = 0
    c.check(c.run(scale=0.02), rows)


def test_prompts_that_see_little(ctx):
    """Rows before the first token, pages given back, bounds of the host, rows apart, a NaN in one head's query."""
    c = Case(ctx, [140, 200, 10], [100, 260, 300], 32, 4, 64, "bf16", seed=42, layout_gap=1, most=(180, 250))
    c.table[1, 1], c.table[2, :] = -1, c.cache.codes.shape[0]
    c.q[150, 7, 3], c.q[151, 8, 0] = float("nan"), float("inf")
    out = c.run()
    c.check(out, {(0, 0), (0, 39), (0, 40), (0, 139), (1, 0), (1, 10), (1, 11), (1, 179), (1, 199), (2, 4)})
    assert bool((out[:40] == 0).all()) and bool((out[340:] == 0).all())
    again = c.run()
    assert torch.equal(out.nan_to_num(9), again.nan_to_num(9))


def test_prompts_into_other_types(ctx):
    for kind, out in (("bf16", "f16"), ("f16", "bf16")):
        c = Case(ctx, [130], [300], 64, 2, 96, kind, out, seed=43)
        c.check(c.run(), {(0, 0), (0, 77), (0, 129)})


@pytest.mark.parametrize("kind,new", [("bf16", 1), ("f32", 3), ("f16", 150), ("residue", 2)])
def test_rows_that_begin_anywhere(ctx, kind, new):
    """Rows on 16 bytes, and the same rows an element further on: the same bits."""
    c = Case(ctx, [new, 1], [300, 90], 32, 4, 64, kind, seed=50)
    want, q = c.run(), c.q
    c.q = torch.empty(q.numel() + 8, dtype=q.dtype, device="cuda")[1:1 + q.numel()].view(q.shape).copy_(q)
    out = torch.empty(q.numel() + 8, dtype=want.dtype, device="cuda")[3:3 + q.numel()].view(q.shape)
    assert torch.equal(c.run(out=out), want)


@pytest.mark.parametrize("window,sinks", [(2 ** 31 - 1, 0), (2 ** 31 - 1, 2 ** 31 - 1), (5, 2 ** 31 - 1), (2 ** 30, 3)])
def test_windows_without_end(ctx, window, sinks):
    for new in (2, 130):
        c = Case(ctx, [new, 10], [200, 4], 32, 4, 64, seed=51)
        want = c.run()
        assert torch.equal(c.run(window=window, sinks=sinks), want)


def test_in_place_for_prompts(ctx):
    c = Case(ctx, [150, 1], [300, 90], 32, 4, 64, "bf16", seed=52)
    want = c.run()
    c.q = c.q.clone()
    assert torch.equal(c.run(out=c.q), want)


def test_prompts_are_the_same_bits_again(ctx):
    c = Case(ctx, [300, 200], [400, 200], 32, 4, 96, "f16", seed=53)
    want = c.run()
    for _ in range(3):
        assert torch.equal(c.run(), want)
