"""Attention over the paged 4-bit cache against the definition in 64 bits on the values that the cache stands for.  The bounds
come from what the header says of the products' operands (tests/kv4_reference.py)."""
import numpy as np
import pytest
import torch

from paper_2105_01827_amd import binding, workloads as wl
from tests import decode_reference as dref, kv4_reference as ref

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "residue": torch.int64}
UNIT = 2.0 ** -12
EPS = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
PARTS_Q = {"bf16": 1, "f16": 2, "f32": 3, "residue": 3}


@pytest.fixture(scope="module")
def ctx():
    par = wl.DEFAULT
    return binding.Context(par.n, par.q, par.p, par.gadget_bits)


def _int32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _plain(x):
    return dref.centred(x.cpu().numpy(), wl.P, UNIT) if x.dtype == torch.int64 else x.cpu().double().numpy()


def _many(new):
    """heads that make enough groups of queries for the form of whole prompts, where there are 128 of them"""
    return 32 if new >= 128 else 2


class Case:
    def __init__(self, ctx, new, lens, heads, group, dim, kind="bf16", out=None, seed=0, spread=2.0, most=None, layout_gap=0, exponents=(-3, 0)):
        gen = torch.Generator().manual_seed(seed)
        self.new, self.lens, self.heads, self.group, self.dim, self.kind = new, lens, heads, group, dim, kind
        blocks = max(1, max(-(-n // 64) for n in lens))
        pages = len(lens) * blocks + 1
        self.cache = binding.Kv4Cache(ctx, heads, dim, pages=pages)
        self.table = torch.randperm(pages, generator=gen)[:len(lens) * blocks].view(len(lens), blocks).to(torch.int32)
        k, v, e, s = ref.places(dim)
        # codes everywhere, also behind the ends; exponents and scales of 255, which are no numbers, where no token is
        data = torch.randint(0, 256, (pages, heads, ref.head_bytes(dim)), generator=gen).numpy().astype(np.uint8)
        pad = np.arange(k.shape[1]) >= dim
        for t in range(64):
            for d in np.nonzero(pad)[0]:
                data[:, :, k[t, d]] &= 0xf0 if d % 2 == 0 else 0x0f
                data[:, :, v[t, d]] &= 0xf0 if t % 2 == 0 else 0x0f
        data[:, :, 2048 * e.shape[1]:] = 255
        scales = ref.bf16(((torch.rand(pages, heads, 64, generator=gen) + 0.5) / 3).numpy()).view(np.uint32) >> 16
        some = torch.randint(*exponents, (pages, heads, 64, e.shape[1]), generator=gen).numpy() + 127
        for b, n in enumerate(lens):
            for j in range(-(-n // 64)):
                page, live = int(self.table[b, j]), min(64, n - 64 * j)
                data[page][:, e[:live]] = some[page][:, :live]
                data[page][:, s[:live]], data[page][:, s[:live] + 1] = scales[page][:, :live] & 255, scales[page][:, :live] >> 8
        self.cache.data.copy_(torch.from_numpy(data).view(pages, -1))
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
        data = self.cache.data.cpu().numpy().reshape(-1, self.heads, ref.head_bytes(self.dim))
        fine = bool({self.kind, self.out_kind} & {"f32", "residue"})
        max_new, max_len = self.most or (max(self.new), max(self.lens))
        for b, (n, length) in enumerate(zip(self.new, self.lens)):
            end = min(length, max_len)
            pages = self.table[b].numpy()
            ok = (pages >= 0) & (pages < data.shape[0])
            with np.errstate(invalid="ignore"):
                held = [[ref.read(data[p if fine else 0, h], self.dim) for p, fine in zip(pages, ok)] for h in range(self.heads)]
            k, v = (np.stack([np.concatenate([x[i] for x in of]) for of in held]) for i in range(2))
            scales = np.stack([np.concatenate([ref.scales_of(data[p if fine else 0, h], self.dim) for p, fine in zip(pages, ok)]) for h in range(self.heads)])
            there = np.repeat(ok, 64)[:end]
            for i in range(n):
                row = self.starts[b] + i
                if rows is not None and (b, i) not in rows:
                    continue
                if i >= max_new:
                    assert (out[row].cpu() == 7).all()
                    continue
                tokens = min(end, k.shape[1])
                seen = dref.see(length - n + i, tokens, self.window, self.sinks) & there[:tokens]
                for h in range(self.heads * self.group):
                    if not np.isfinite(q[row, h]).all():
                        assert np.isnan(got[row, h]).all()
                        continue
                    of = k[h // self.group, :tokens], v[h // self.group, :tokens]
                    parts_q = 3 if fine else PARTS_Q[self.kind]
                    if not fine:
                        want, bound = ref.attention_in_halves(q[row, h], *of, scales[h // self.group, :tokens], seen, self.scale, parts_q)
                    else:
                        want, bound = ref.attention(q[row, h], *of, seen, self.scale, parts_q, 3)
                    # one rounding to the output's type; half precision's smallest step
                    bound = bound + EPS.get(self.out_kind, 0) * (np.abs(want) + bound) + (UNIT / 2 if self.out_kind == "residue" else 0) + 2.0 ** -25
                    over = np.abs(got[row, h] - want) / bound
                    assert over.max() <= 1, (b, i, h, over.max())


@pytest.mark.parametrize("dim", [1, 15, 32, 33, 48, 64, 80, 96, 128, 129, 160, 192, 200, 224, 256])
@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_head_sizes(ctx, dim, kind):
    c = Case(ctx, [1, 1, 1], [200, 63, 1], 2, 3, dim, kind, seed=dim)
    c.check(c.run())


@pytest.mark.parametrize("kind,out", [("f32", "f32"), ("f16", "f16"), ("bf16", "bf16"), ("residue", "residue"), ("residue", "f32"),
                                      ("f32", "residue"), ("bf16", "f32"), ("f32", "bf16"), ("f16", "residue"), ("bf16", "f16"), ("f16", "bf16")])
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
    c = Case(ctx, [0] + [1] * 8 + [0], [0, 1, 64, 65, 700, 3000, 128, 5, 2049, 1], 3, 4, 128, seed=11)
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
    c.check(c.run(), {(0, i) for i in (0, 1, 15, 16, 63, 64, 255, 256, 599)} | {(1, i) for i in (0, 31, 32, 449)})


@pytest.mark.parametrize("dim", [1, 16, 40, 64, 72, 80, 96, 112, 128, 160, 192, 200, 224, 256])
@pytest.mark.parametrize("kind,group", [("bf16", 3), ("f16", 8), ("f32", 2)])
def test_prompts_of_every_head_size(ctx, dim, kind, group):
    c = Case(ctx, [180, 1, 77], [180, 300, 200], 8 if group > 3 else 16, group, dim, kind, seed=dim, spread=1.0)
    c.check(c.run(), {(0, 0), (0, 63), (0, 179), (1, 0), (2, 5), (2, 76)} if dim < 100 else {(0, 179), (2, 5)})


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 0), (63, 4), (64, 64), (65, 100), (100, 0), (1000, 4), (5000, 5000)])
@pytest.mark.parametrize("new", [1, 90])
def test_windows(ctx, window, sinks, new):
    c = Case(ctx, [new, 1, new], [600, 50, new], 2, 2, 64, "f32", seed=window + sinks)
    rows = None if new == 1 else {(0, i) for i in (0, 1, 40, 89)} | {(2, i) for i in (0, 15, 16, 70, 89)} | {(1, 0)}
    c.check(c.run(window=window, sinks=sinks), rows)


@pytest.mark.parametrize("window,sinks", [(1, 0), (16, 4), (100, 0), (65, 70), (1000, 4)])
def test_windows_of_prompts(ctx, window, sinks):
    c = Case(ctx, [200, 50, 130], [500, 50, 131], 8, 4, 64, "bf16", seed=window)
    c.check(c.run(window=window, sinks=sinks), {(0, i) for i in (0, 17, 199)} | {(1, 0), (1, 49), (2, 0), (2, 129)})


@pytest.mark.parametrize("window,sinks", [(2 ** 31 - 1, 0), (2 ** 31 - 1, 2 ** 31 - 1), (5, 2 ** 31 - 1), (2 ** 30, 3)])
def test_windows_without_end(ctx, window, sinks):
    for new in (2, 130):
        c = Case(ctx, [new, 10], [200, 4], 8 if new < 128 else 32, 4, 64, seed=51)
        want = c.run()
        assert torch.equal(c.run(window=window, sinks=sinks), want)


@pytest.mark.parametrize("kind,new", [("f32", 1), ("bf16", 140)])
def test_exponents_and_scales_far_apart(ctx, kind, new):
    """Keys of all sizes, so that scores rise and fall by hundreds; values a million times another's; a negative scale, none."""
    c = Case(ctx, [new, 4], [500, 300], _many(new), 2, 64, kind, seed=21, exponents=(-9, 4))
    k, v, e, s = ref.places(64)
    data = c.cache.data.view(-1, c.heads, ref.head_bytes(64)).cpu().numpy()
    rng = np.random.default_rng(1)
    for p in range(data.shape[0]):
        for h in range(c.heads):
            data[p, h, s + 1] = np.where(data[p, h, s + 1] < 255, 0x30 + rng.integers(0, 21, 64), 255)       # from 6e-10 to 500
    c.cache.data.copy_(torch.from_numpy(data).view(c.cache.data.shape))
    rows = None if new == 1 else {(0, 0), (0, 77), (0, 139), (1, 3)}
    for scale in (None, -0.3, 0.0):
        c.check(c.run(scale=scale), rows)


@pytest.mark.parametrize("kind,new,length", [("bf16", 1, 500), ("bf16", 140, 500), ("f16", 1, 7000), ("f32", 2, 500)])
@pytest.mark.parametrize("some", [(-99,), (110,), (110, -60), (100, 60, -30, -99)])
def test_scales_further_apart_than_32_bits(ctx, kind, new, length, some):
    """Scales of 2^some, none and ordinary ones, in any order: a token's weight counts in the divisor whatever its value's scale is."""
    c = Case(ctx, [new, 4], [length, 300], _many(new), 2, 64, kind, "f32" if kind == "f32" else "bf16", seed=71, spread=0.5)
    k, v, e, s = ref.places(64)
    data = c.cache.data.view(-1, c.heads, ref.head_bytes(64)).cpu().numpy()
    rng = np.random.default_rng(len(some) + new)
    choice = np.array([0] + [x + 127 << 7 for x in (0, -3) + some])
    for p in range(data.shape[0]):
        for h in range(c.heads):
            live = (data[p, h, s + 1] < 255).copy()
            bits = choice[rng.integers(0, len(choice), 64)]
            if p % 3 == 0:
                bits = choice[rng.integers(0, 3, 64)]           # blocks with ordinary scales alone, before and behind the others
            data[p, h, s] = np.where(live, bits & 255, data[p, h, s])
            data[p, h, s + 1] = np.where(live, bits >> 8, data[p, h, s + 1])
    c.cache.data.copy_(torch.from_numpy(data).view(c.cache.data.shape))
    c.check(c.run(), None if new < 3 else {(0, 0), (0, 77), (0, 139), (1, 3)})


def test_many_small_weights_beside_a_large_one(ctx):
    """The first key has nearly all weight and a value of nothing; thousands of others share the rest."""
    for kind in ("bf16", "f16", "f32"):
        for new in (1, 40):
            c = Case(ctx, [new], [8192], 1, 4, 64, kind, seed=60, exponents=(-8, -7))
            k, v, e, s = ref.places(64)
            data = c.cache.data.view(-1, ref.head_bytes(64)).cpu().numpy()
            first = data[int(c.table[0, 0])]
            for d in range(64):
                first[k[0, d]] = first[k[0, d]] & (0xf0 if d % 2 == 0 else 0x0f) | 2 << 4 * (d % 2)          # 1
                first[v[0, d]] &= 0xf0
            first[e[0]] = 127
            c.cache.data.copy_(torch.from_numpy(data).view(c.cache.data.shape))
            c.q = (c.q.abs() * 0.5 + 0.2).to(c.q.dtype)
            c.check(c.run(), {(0, 0), (0, new - 1)})


def test_zero_codes_and_zero_queries(ctx):
    c = Case(ctx, [1, 2], [200, 100], 2, 2, 64, seed=22)
    c.cache.data[::2, :2048] = 0
    c.q[1, 2] = 0
    c.check(c.run())


def test_rows_that_see_nothing(ctx):
    """No tokens, positions before the first token, pages given back."""
    for group in (3, 70):
        c = Case(ctx, [1, 5, 1, 2], [0, 3, 130, 70], 2, group, 64, seed=23)
        c.table[2, :] = -1
        c.table[3, 1] = c.cache.data.shape[0]
        out = c.run()
        c.check(out)
        assert bool((out[0] == 0).all() and (out[1:3] == 0).all() and (out[6] == 0).all())


def test_pages_behind_a_window_are_not_needed(ctx):
    c = Case(ctx, [1], [1000], 2, 2, 64, seed=24)
    want = c.run(window=200, sinks=3)
    c.table[0, 1:12] = -1                                        # 800 is in block 12
    assert torch.equal(c.run(window=200, sinks=3), want)


@pytest.mark.parametrize("new", [1, 130])
def test_what_nobody_sees_may_be_anything(ctx, new):
    """Pages behind the end, behind the window and of nobody, and the first page, which stands for missing ones, are no numbers."""
    c = Case(ctx, [new, new], [300, 500], _many(new), 2, 64, seed=25)
    c.table[c.table == 0] = c.cache.data.shape[0] - 1            # page 0 is nobody's
    c.table[1, 2] = -1
    want = c.run(window=240)
    seen = {int(p) for p in c.table.flatten() if p >= 0}
    c.cache.data[[p for p in range(c.cache.data.shape[0]) if p not in seen]] = 255
    out = c.run(window=240)
    assert torch.equal(out, want) and bool(out.isfinite().all())
    if new == 1:
        c.table[1, 0] = -1                                       # 500 - 240 is in block 4
        assert torch.equal(c.run(window=240), want)


def test_a_query_with_nan_or_infinity_spoils_its_own_head_alone(ctx):
    for kind, new in (("f32", 3), ("bf16", 140)):
        c = Case(ctx, [1, new], [100, 190], _many(new), 3, 64, kind, seed=26)
        clean = c.run()
        c.q[0, 1, 5], c.q[2, 4, 63], c.q[3, 0, 0] = float("nan"), float("inf"), float("-inf")
        out = c.run()
        bad = torch.zeros(out.shape[:2], dtype=torch.bool, device="cuda")
        bad[0, 1] = bad[2, 4] = bad[3, 0] = True
        assert bool(out[bad].isnan().all()) and torch.equal(out[~bad], clean[~bad])


def test_bounds_that_the_host_gives(ctx):
    """Rows beyond max_new are left alone, keys beyond max_len are not seen."""
    c = Case(ctx, [3, 6], [200, 90], 2, 2, 64, seed=27, most=(4, 150))
    c.check(c.run())
    c = Case(ctx, [1, 1], [200, 90], 2, 2, 64, seed=28, most=(1, 100000))
    c.check(c.run())
    c = Case(ctx, [140, 200, 10], [100, 260, 300], 8, 4, 64, "bf16", seed=42, layout_gap=1, most=(180, 250))
    out = c.run()
    c.check(out, {(0, 0), (0, 39), (0, 40), (0, 139), (1, 0), (1, 179), (1, 199), (2, 4)})
    assert bool((out[:40] == 0).all())


def test_rows_apart_and_in_place(ctx):
    for new in ([2, 3], [150, 1]):
        c = Case(ctx, new, [200, 90], _many(new[0]), 2, 48, seed=29, layout_gap=3)
        want = c.run()
        c.check(want, {(0, 0), (0, new[0] - 1), (1, 0)})
        c.q = c.q.clone()
        assert torch.equal(c.run(out=c.q), want)


def test_a_long_sequence(ctx):
    """One query over 70000 tokens, split over the whole card and joined; twice the same bits."""
    c = Case(ctx, [1], [70001], 1, 4, 128, "f16", seed=30)
    out = c.run()
    c.check(out, {(0, 0)})
    for _ in range(3):
        assert torch.equal(c.run(), out)


@pytest.mark.parametrize("count", [33, 64, 65, 100])
def test_prompts_of_many_sequences(ctx, count):
    """As many as a wavefront has lanes, more, and a number that is no power of two; lengths of all kinds, some without new tokens."""
    new = [(b * 53) % 140 if b % 7 else 0 for b in range(count)]
    new[5] = 140
    c = Case(ctx, new, [n + (b * 29) % 200 for b, n in enumerate(new)], 4, 2, 32, "bf16", seed=count)
    c.check(c.run(), {(b, i) for b in range(count) for i in (0, new[b] - 1) if new[b]})


def test_prompts_are_the_same_bits_again(ctx):
    c = Case(ctx, [300, 200], [400, 200], 8, 4, 96, "f16", seed=53)
    want = c.run()
    for _ in range(3):
        assert torch.equal(c.run(), want)


def test_offsets_beyond_32_bits(ctx):
    """Pages that lie more than 4 GiB into the cache."""
    if torch.cuda.mem_get_info()[0] < 8 << 30:
        pytest.skip("needs 8 GiB")
    for new in (1, 130):
        heads = 1 if new < 128 else 64
        c = Case(ctx, [new], [130], heads, 2, 128, seed=31)
        want = c.run()
        pages = (1 << 32) // (heads * ref.head_bytes(128)) + 9
        big = binding.Kv4Cache(ctx, heads, 128, pages=pages)
        assert big.data.numel() > 1 << 32
        at = torch.tensor([pages - 1, 7, pages - 3])
        for i in range(3):
            big.data[at[i]] = c.cache.data[int(c.table[0, i])]
        c.cache, c.table = big, at.view(1, 3).to(torch.int32)
        assert torch.equal(c.run(), want)


@pytest.mark.parametrize("new,lens", [([1, 1], [5000, 300]), ([140, 3], [200, 300])])
def test_another_stream_and_a_graph(ctx, new, lens):
    c = Case(ctx, new, lens, _many(new[0]), 4, 64, seed=32)
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


@pytest.mark.parametrize("kind,new", [("bf16", 1), ("f32", 3), ("f16", 150), ("residue", 2)])
def test_rows_that_begin_anywhere(ctx, kind, new):
    """Rows on 16 bytes, and the same rows an element further on: the same bits."""
    c = Case(ctx, [new, 1], [300, 90], 8 if new < 128 else 32, 4, 64, kind, seed=50)
    want, q = c.run(), c.q
    c.q = torch.empty(q.numel() + 8, dtype=q.dtype, device="cuda")[1:1 + q.numel()].view(q.shape).copy_(q)
    out = torch.empty(q.numel() + 8, dtype=want.dtype, device="cuda")[3:3 + q.numel()].view(q.shape)
    assert torch.equal(c.run(out=out), want)


def test_after_append(ctx):
    """The order of codes that append writes is the order that attention reads."""
    heads, group, dim, n = 2, 4, 96, 150
    c = Case(ctx, [n], [n], heads, group, dim, "f32", seed=33)
    k, v = (torch.randn(n, heads, dim, generator=torch.Generator().manual_seed(s)).cuda() for s in (1, 2))
    c.run()
    c.cache.append(c.keep, k, v)
    c.check(c.run(), {(0, i) for i in (0, 1, 64, 100, 149)})
