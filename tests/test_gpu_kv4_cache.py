"""Appending to the paged 4-bit cache with positions rotated in, and reading it back: every byte by the definition, which rounds
in 32 bits where the header says so."""
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


def _values(gen, kind, *shape):
    x = torch.randn(*shape, generator=gen)
    if kind == "residue":
        return torch.round(x / UNIT).to(torch.int64).remainder(wl.P).cuda()
    return x.to(TYPES[kind]).cuda()


def _plain(x):
    """as float32, exactly"""
    return dref.centred(x.cpu().numpy(), wl.P, UNIT).astype(np.float32) if x.dtype == torch.int64 else x.cpu().float().numpy()


def _int32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class Sequences:
    """A cache of its own, and every byte that it should hold."""

    def __init__(self, ctx, heads, dim, batch, blocks, seed, spare=2):
        self.gen = torch.Generator().manual_seed(seed)
        self.heads, self.dim, self.batch = heads, dim, batch
        pages = batch * blocks + spare
        self.cache = binding.Kv4Cache(ctx, heads, dim, pages=pages)
        garbage = torch.randint(0, 256, self.cache.data.shape, generator=self.gen).to(torch.uint8)
        self.cache.data.copy_(garbage)                   # what lies behind a sequence's end is nobody's
        self.want = garbage.numpy().reshape(pages, heads, ref.head_bytes(dim)).copy()
        self.table = torch.randperm(pages, generator=self.gen)[:batch * blocks].view(batch, blocks).to(torch.int32)
        self.lens = [0] * batch

    def step(self, new):
        self.lens = [a + n for a, n in zip(self.lens, new)]
        starts = np.concatenate([[0], np.cumsum(new)])
        return starts, binding.KvBatch(_int32(starts.tolist()), _int32(self.lens), self.table.cuda(), max(new), max(self.lens))

    def expect(self, starts, k, v):
        """k (rotated) and v (rows, heads, dim) float32 into the expected bytes; the cache has to hold them, and nothing else"""
        for b in range(self.batch):
            n = starts[b + 1] - starts[b]
            for i in range(n):
                t = self.lens[b] - n + i
                page = int(self.table[b, t // 64])
                for h in range(self.heads):
                    ref.write(self.want[page, h], t % 64, k[starts[b] + i, h], v[starts[b] + i, h], self.dim)
        got = self.cache.data.cpu().numpy().reshape(self.want.shape)
        assert np.array_equal(got, self.want), np.argwhere(got != self.want)[:8]

    def rows(self, b, n):
        """keys and values of the first n tokens of a sequence, as the expected bytes stand for them"""
        both = [np.concatenate(x) for x in zip(*[[np.stack(y, 1) for y in zip(*[ref.read(self.want[int(p), h], self.dim) for h in range(self.heads)])]
                                                 for p in self.table[b, :-(-n // 64)]])] if n else [np.zeros((0, self.heads, self.dim))] * 2
        return [x[:n] for x in both]


@pytest.mark.parametrize("kind,dim,rot,interleaved,heads,group", [
    ("f32", 64, 64, False, 3, 2), ("bf16", 128, 128, False, 2, 4), ("f16", 80, 40, True, 2, 1), ("residue", 128, 64, True, 1, 3),
    ("residue", 33, 32, False, 1, 1), ("bf16", 256, 256, True, 1, 2), ("f32", 200, 2, False, 1, 3), ("f16", 1, 0, False, 2, 1),
    ("f16", 16, 16, False, 1, 8), ("bf16", 96, 96, False, 2, 5), ("residue", 64, 0, False, 3, 1), ("f16", 192, 96, False, 1, 2)])
def test_append_and_export(ctx, kind, dim, rot, interleaved, heads, group):
    """Prompts of several lengths, then single tokens, then a few at once, over block edges; part of a fused projection."""
    s = Sequences(ctx, heads, dim, 3, 5, seed=dim + rot)
    rope = table = None
    if rot:
        table = binding.rope_table(320, rot)
        rope = binding.Rope(torch.from_numpy(table).cuda(), interleaved)
    for new in [(70, 1, 64), (1, 1, 1), (0, 62, 3), (5, 64, 1), (1, 1, 130), (130, 0, 0)]:
        before = list(s.lens)
        starts, batch = s.step(new)
        total = int(starts[-1])
        fused = _values(s.gen, kind, total, group * heads + 2 * heads, dim)
        q, k, v = fused.split([group * heads, heads, heads], 1)
        out = torch.float32 if kind == "residue" else TYPES[kind]
        q_out = torch.full((total, group * heads, dim), 7.0, dtype=out, device="cuda")
        s.cache.append(batch, k, v, q=q, q_out=q_out, rope=rope, unit=UNIT)
        at = np.concatenate([np.arange(a, a + n) for a, n in zip(before, new)])
        turned = [ref.turn(_plain(x), table[at, :, 0], table[at, :, 1], rot, interleaved) if rot else _plain(x) for x in (q, k)]
        assert torch.equal(q_out.cpu(), torch.from_numpy(turned[0]).to(out))
        s.expect(starts, turned[1], _plain(v))
    # everything back, whole sequences, as the values that the codes stand for
    lens = s.lens
    starts = np.concatenate([[0], np.cumsum(lens)])
    whole = binding.KvBatch(_int32(starts.tolist()), _int32(lens), s.table.cuda(), max(lens), max(lens))
    want = [np.concatenate(x) for x in zip(*[s.rows(b, n) for b, n in enumerate(lens)])]
    for kind_out in ("f32", "f16", "bf16", "residue"):
        back = [torch.zeros(int(starts[-1]), heads, dim, dtype=TYPES[kind_out], device="cuda") for _ in range(2)]
        s.cache.export(whole, *back, unit=UNIT)
        for x, y in zip(back, want):
            y = torch.from_numpy(y)
            if kind_out == "residue":
                assert torch.equal(x.cpu(), torch.round(y / UNIT).to(torch.int64).remainder(wl.P))
            else:                                        # a code times its scale has 11 bits: exact in 32
                assert torch.equal(x.cpu(), y.float().to(TYPES[kind_out]))


def test_every_border_between_two_codes(ctx):
    """Numbers on the borders, next to them, and of all sizes: exponents at both ends, scales too small for a value."""
    tiny, u = np.float32(2.0 ** -126), np.float32(2.0 ** -23)
    borders = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 6, 7, 7.5], np.float32)
    row = np.concatenate([b * np.array([1 - u, 1, 1 + u], np.float32) for b in borders] + [[0, -0.0]]).astype(np.float32)
    rows = [row * s for s in (1, -1, 3e-3, 2.0 ** -60, 2.0 ** 100)] + [row * 2.0 ** k for k in (-100, -118, -121, -125, -149, 124)]
    for largest in (6.99999, 7, 7.000001, 3.4e38, 1e-45, 2.0 ** -100 * 6, 2.0 ** -100 * 5.9, 2.0 ** -120 * 7, 2.0 ** 127):
        x = np.zeros(32, np.float32)
        x[:4] = np.float32(largest) * np.array([1, -0.5, 0.3, -0.1], np.float32)
        rows.append(x)
    rows.append(np.full(32, tiny))
    x = np.stack([np.concatenate([r, rows[(i + 3) % len(rows)]]) for i, r in enumerate(rows)]).astype(np.float32)[:, None]
    s = Sequences(ctx, 1, 64, 1, 1, seed=1)
    starts, batch = s.step((len(x),))
    k = torch.from_numpy(x).cuda()
    s.cache.append(batch, k, k.flip(0))
    s.expect(starts, x, x[::-1])


def test_values_of_16_bits_meet_borders_of_their_scale(ctx):
    """Multiples of a scale of 16-bit numbers: quotients that a reciprocal would put on the other side of a border."""
    for kind in ("f16", "bf16"):
        s = Sequences(ctx, 4, 128, 1, 2, seed=2)
        starts, batch = s.step((128,))
        x = torch.randint(-48, 49, (128, 4, 128), generator=s.gen) * (torch.randint(1, 256, (128, 4, 1), generator=s.gen) / 1024)
        x = x.to(TYPES[kind]).cuda()
        s.cache.append(batch, x, x)
        s.expect(starts, _plain(x), _plain(x))


def test_infinities_and_nan(ctx):
    s = Sequences(ctx, 2, 64, 1, 1, seed=8)
    starts, batch = s.step((20,))
    k = _values(s.gen, "f32", 20, 2, 64)
    k[3, 0, 5], k[4, 0, 6], k[5, 1, 7] = float("inf"), float("-inf"), float("nan")
    k[6], k[7], k[8, :, 32:] = float("nan"), float("inf"), 0
    v = k.flip(2).contiguous()
    s.cache.append(batch, k, v)
    s.expect(starts, _plain(k), _plain(v))
    back = [torch.empty_like(k) for _ in range(2)]
    s.cache.export(batch, *back)
    assert all(bool(x.isfinite().all()) for x in back)


def test_single_tokens_leave_their_neighbours(ctx):
    """Token by token through a block and into the next: two tokens of a value share a byte."""
    s = Sequences(ctx, 2, 48, 2, 2, seed=3)
    for i in range(70):
        starts, batch = s.step((1, i % 2))
        x = _values(s.gen, "bf16", int(starts[-1]), 4, 48)
        s.cache.append(batch, x[:, :2], x[:, 2:])
        s.expect(starts, _plain(x[:, :2]), _plain(x[:, 2:]))


@pytest.mark.parametrize("new", [15, 16, 17, 63, 64, 65])
def test_token_counts_at_launch_shapes(ctx, new):
    for first in (0, 1, 60):
        s = Sequences(ctx, 1, 160, 2, 4, seed=new)
        if first:
            starts, batch = s.step((first, first))
            x = _values(s.gen, "f16", 2 * first, 2, 160)
            s.cache.append(batch, x[:, :1], x[:, 1:])
            s.expect(starts, _plain(x[:, :1]), _plain(x[:, 1:]))
        starts, batch = s.step((new, new - 1))
        x = _values(s.gen, "f16", 2 * new - 1, 2, 160)
        s.cache.append(batch, x[:, :1], x[:, 1:])
        s.expect(starts, _plain(x[:, :1]), _plain(x[:, 1:]))


def test_queries_alone_and_in_place(ctx):
    s = Sequences(ctx, 2, 64, 2, 3, seed=5)
    starts, batch = s.step((90, 17))
    rope = binding.Rope(torch.from_numpy(binding.rope_table(100, 32)).cuda(), True)
    x = _values(s.gen, "bf16", 107, 6, 64)
    out = torch.empty_like(x)
    data = s.cache.data.clone()
    s.cache.append(batch, None, None, q=x, q_out=out, rope=rope)
    assert torch.equal(data, s.cache.data)
    same = x.clone()
    s.cache.append(batch, None, None, q=same, q_out=same, rope=rope)
    assert torch.equal(same, out) and not torch.equal(same, x)


def test_one_row_for_all_and_rows_apart(ctx):
    """A row stride of zero repeats one row; a stride beyond the row leaves the gap alone."""
    s = Sequences(ctx, 2, 48, 1, 2, seed=6)
    starts, batch = s.step((70,))
    one = _values(s.gen, "f32", 1, 2, 48).expand(70, -1, -1)
    wide = torch.full((70, 2 * 48 + 5), 3.0, device="cuda")
    q_out = wide[:, :96].view(70, 2, 48)
    s.cache.append(batch, one, one, q=one, q_out=q_out)
    s.expect(starts, _plain(one), _plain(one))
    assert torch.equal(q_out, one) and bool((wide[:, 96:] == 3).all())


def test_tokens_without_a_place_are_skipped(ctx):
    """Pages that are not there, positions that the rope table does not have, rows beyond max_new, more rows than tokens."""
    s = Sequences(ctx, 1, 32, 3, 3, seed=7)
    s.table[0, 1], s.table[1, 0] = -1, s.cache.data.shape[0]
    batch = binding.KvBatch(_int32([0, 150, 220, 320]), _int32([150, 70, 90]), s.table.cuda(), 140, 150)
    table = binding.rope_table(60, 32)
    k, v = (_values(s.gen, "f32", 320, 1, 32) for _ in range(2))
    q_out = torch.full((320, 1, 32), 7.0, device="cuda")
    s.cache.append(batch, k, v, q=k, q_out=q_out, rope=binding.Rope(torch.from_numpy(table).cuda()))
    at = np.concatenate([np.arange(150), np.arange(70), np.arange(-10, 90)])
    inside, taken = (at >= 0) & (at < 60), np.ones(320, bool)
    taken[140:150] = False
    got = q_out.cpu().numpy()
    assert np.isnan(got[~inside & taken]).all() and not np.isnan(got[inside]).any() and (got[140:150] == 7).all()
    keys = ref.turn(_plain(k), table[at.clip(0, 59), :, 0], table[at.clip(0, 59), :, 1], 32, False)
    keys[~inside] = np.nan                                # stored as 0
    for row, t in enumerate(at):
        b = 0 if row < 150 else 1 if row < 220 else 2
        page = int(s.table[b, t // 64]) if t >= 0 else -1
        if taken[row] and 0 <= page < s.cache.data.shape[0]:
            ref.write(s.want[page, 0], t % 64, keys[row, 0], _plain(v)[row, 0], 32)
    assert np.array_equal(s.cache.data.cpu().numpy().reshape(s.want.shape), s.want)
    back = [torch.full((320, 1, 32), 7.0, device="cuda") for _ in range(2)]
    s.cache.export(batch, *back)
    absent = np.zeros(320, bool)
    absent[64:128] = absent[150:214] = absent[220:230] = True
    for x in back:
        x = x.cpu().numpy()
        assert (x[absent & taken] == 0).all() and (x[140:150] == 7).all() and np.isfinite(x).all()
    assert (back[1].cpu().numpy()[~absent & taken] != 0).any(-1).all()


def test_empty_calls(ctx):
    s = Sequences(ctx, 1, 16, 2, 1, seed=10)
    starts, batch = s.step((0, 0))
    nobody = binding.KvBatch(_int32([0]), _int32([]), torch.empty(0, 1, dtype=torch.int32, device="cuda"), 0, 0)
    one = torch.ones(1, 1, 16, device="cuda")
    s.cache.append(nobody, one, one)
    s.cache.append(batch, one, one)
    s.cache.export(batch, one, one.clone())
    s.expect(starts, _plain(one), _plain(one))
    assert bool((one == 1).all())


def test_another_stream_and_a_graph(ctx):
    s = Sequences(ctx, 4, 128, 2, 2, seed=11)
    starts, batch = s.step((65, 64))
    rope = binding.Rope(torch.from_numpy(binding.rope_table(128, 128)).cuda())
    x = _values(s.gen, "bf16", 129, 12, 128)
    q, k, v = x.split(4, 1)
    out, start = torch.empty_like(q.contiguous()), s.cache.data.clone()
    s.cache.append(batch, k, v, q=q, q_out=out, rope=rope)
    want, data = out.clone(), s.cache.data.clone()
    back, kept = ([torch.zeros(129, 4, 128, device="cuda") for _ in range(2)] for _ in range(2))
    s.cache.export(batch, *kept)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        s.cache.append(batch, k, v, q=q, q_out=out, rope=rope, stream=torch.cuda.current_stream())
        s.cache.export(batch, *back, stream=torch.cuda.current_stream())
    for _ in range(3):
        out.zero_(), s.cache.data.copy_(start), back[0].zero_(), back[1].zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(s.cache.data, data) and all(torch.equal(a, b) for a, b in zip(back, kept))


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16", "residue"])
@pytest.mark.parametrize("new", [(70, 3), (1, 1)])
def test_rows_that_begin_anywhere(ctx, kind, new):
    """Rows on 16 bytes, and the same rows an element further on: the same bits."""
    heads, dim = 2, 64
    results = []
    for shift in (0, 1):
        s = Sequences(ctx, heads, dim, 2, 2, seed=12)
        rope = binding.Rope(torch.from_numpy(binding.rope_table(128, 64)).cuda())
        out = torch.float32 if kind == "residue" else TYPES[kind]
        for step in (new, (2, 5)):
            starts, batch = s.step(step)
            total = int(starts[-1])
            row = 4 * heads * dim
            wide = torch.zeros(total * (row + 1) + 8, dtype=TYPES[kind], device="cuda")
            rows = wide[shift:shift + total * (row + shift)].view(total, row + shift)[:, :row].view(total, 4 * heads, dim)
            rows.copy_(_values(s.gen, kind, total, 4 * heads, dim))
            q, k, v = rows.split([2 * heads, heads, heads], 1)
            q_out = torch.zeros(total * 2 * heads * dim + 8, dtype=out, device="cuda")[shift:shift + total * 2 * heads * dim].view(total, 2 * heads, dim)
            s.cache.append(batch, k, v, q=q, q_out=q_out, rope=rope, unit=UNIT)
        back = [torch.zeros(total * heads * dim + 8, dtype=out, device="cuda")[shift:shift + total * heads * dim].view(total, heads, dim) for _ in range(2)]
        s.cache.export(batch, *back)
        results.append([q_out.clone(), s.cache.data.clone()] + [b.clone() for b in back])
    for a, b in zip(*results):
        assert torch.equal(a, b)


@pytest.mark.parametrize("rot,interleaved", [(6, True), (12, True), (24, False), (40, False), (8, True), (48, False)])
def test_pairs_of_odd_counts(ctx, rot, interleaved):
    """Rotations that end inside a piece of eight channels."""
    s = Sequences(ctx, 1, 48, 1, 2, seed=rot)
    table = binding.rope_table(100, rot)
    starts, batch = s.step((70,))
    k, v = (_values(s.gen, "f32", 70, 1, 48) for _ in range(2))
    s.cache.append(batch, k, v, rope=binding.Rope(torch.from_numpy(table).cuda(), interleaved))
    s.expect(starts, ref.turn(_plain(k), table[:70, :, 0], table[:70, :, 1], rot, interleaved), _plain(v))


def test_offsets_beyond_32_bits(ctx):
    """A page more than 4 GiB into the cache."""
    if torch.cuda.mem_get_info()[0] < 8 << 30:
        pytest.skip("needs 8 GiB")
    s = Sequences(ctx, 1, 128, 1, 1, seed=13)
    starts, batch = s.step((64,))
    x = _values(s.gen, "bf16", 64, 2, 128)
    s.cache.append(batch, x[:, :1], x[:, 1:])
    pages = (1 << 32) // ref.head_bytes(128) + 5
    big = binding.Kv4Cache(ctx, 1, 128, pages=pages)
    assert big.data.numel() > 1 << 32
    far = binding.KvBatch(batch.tensors[0], batch.tensors[1], _int32([[pages - 1]]), 64, 64)
    big.append(far, x[:, :1], x[:, 1:])
    assert torch.equal(big.data[-1], s.cache.data[int(s.table[0, 0])])
    back, want = ([torch.empty(64, 1, 128, device="cuda") for _ in range(2)] for _ in range(2))
    big.export(far, *back), s.cache.export(batch, *want)
    assert all(torch.equal(a, b) for a, b in zip(back, want))
