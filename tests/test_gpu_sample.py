"""Tokens from logits and given uniform numbers against the definition in 64 bits.  The uniform numbers are put in the middle of
tokens' shares, and cuts away from tokens' edges, so that 32-bit weights (off by 2^-20 of themselves at most) leave one answer."""
import numpy as np
import pytest
import torch

from paper_2105_01827_amd import binding, workloads as wl
from tests import decode_reference as ref

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
UNIT = 2.0 ** -10
MARGIN = 2.0 ** -18


@pytest.fixture(scope="module")
def ctx():
    par = wl.DEFAULT
    return binding.Context(par.n, par.q, par.p, par.gadget_bits)


def _run(ctx, logits, u, **how):
    rows, vocab = logits.shape
    tokens = torch.full((rows,), -7, dtype=torch.int32, device="cuda")
    need = ctx.sample_workspace_bytes(rows, vocab)
    ws = torch.full((max(need, 16),), 0xff, dtype=torch.uint8, device="cuda")
    args = {k: torch.tensor(np.asarray(v), dtype=torch.int32 if k == "top_k" else torch.float32, device="cuda") for k, v in how.items()}
    ctx.sample(logits, torch.tensor(np.asarray(u), dtype=torch.float32, device="cuda"), tokens, ws, need, unit=UNIT, **args)
    return tokens.cpu().numpy()


def _logits(rows, vocab, kind, seed, spread=2.0):
    gen = torch.Generator().manual_seed(seed)
    rank = torch.rand(rows, vocab, generator=gen).argsort(-1).float()
    z = 6 - torch.log1p(rank) + spread * 0.3 * torch.randn(rows, vocab, generator=gen)
    if kind == "residue":
        return torch.round(z / UNIT).to(torch.int64).remainder(wl.P)
    return z.to(TYPES[kind])


def _plain(z):
    return ref.centred(z.numpy(), wl.P, UNIT) if z.dtype == torch.int64 else z.double().numpy()


def _choose(z, temperature, top_k, top_p, min_p, pick):
    """(u, the token it has to give): the middle of the share of one of the likelier kept tokens"""
    kept, w, margin = ref.kept_tokens(z, temperature, top_k, top_p, min_p)
    share = np.where(kept, w, 0.0)
    places = np.flatnonzero(share > share.sum() * 1e-4)
    token = places[int(pick * len(places))]
    run = np.cumsum(share)
    u = np.float32((run[token] - share[token] / 2) / run[-1])
    assert run[token - 1] / run[-1] + MARGIN < u < run[token] / run[-1] - MARGIN if token else u < run[0] / run[-1] - MARGIN
    return u, token, margin


def _away(z, how):
    """`how` with top_p and min_p moved until their cuts are far enough from every token's edge"""
    temperature, top_k, top_p, min_p = how
    for _ in range(200):
        if ref.kept_tokens(z, temperature, top_k, top_p, min_p)[2] > MARGIN:
            return temperature, top_k, float(np.float32(top_p)), float(np.float32(min_p))
        top_p, min_p = np.float32(top_p * (0.9971 if top_p < 1 else 1)), np.float32(min_p * 1.0031)
    raise AssertionError("no cut")


HOW = [(1.0, 0, 1.0, 0.0), (0.7, 0, 0.9, 0.0), (1.3, 50, 1.0, 0.0), (0.9, 40, 0.8, 0.0), (1.0, 0, 1.0, 0.05), (0.5, 300, 0.97, 0.01),
       (0.0, 5, 0.5, 0.5), (2.0, 1, 1.0, 0.0), (1.0, 10 ** 9, 0.5, 0.3), (0.01, 0, 0.999, 0.0), (1.0, 0, 0.0, 0.0), (1.0, 0, 0.6, 1.0)]


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16", "residue"])
@pytest.mark.parametrize("vocab", [1, 2, 3, 63, 64, 65, 1000, 1024, 1025, 5003, 33001])
def test_every_cut(ctx, vocab, kind):
    logits = _logits(len(HOW), vocab, kind, seed=vocab)
    plain = _plain(logits)
    how = [_away(z, h) if vocab > 1 else h for z, h in zip(plain, HOW)]
    chosen = [_choose(z, *h, pick=(0.37 + 0.61 * r) % 1) for r, (z, h) in enumerate(zip(plain, how))]
    t, k, p, m = zip(*how)
    got = _run(ctx, logits.cuda(), [c[0] for c in chosen], temperature=t, top_k=k, top_p=p, min_p=m)
    assert got.tolist() == [c[1] for c in chosen]


@pytest.mark.parametrize("rows,vocab", [(1, 131072), (3, 100003), (300, 777), (70, 20000), (2, 200001)])
def test_sizes(ctx, rows, vocab):
    logits = _logits(rows, vocab, "f32", seed=rows)
    plain = _plain(logits)
    for how in [(0.8, 0, 1.0, 0.0), (0.8, 50, 0.9, 0.0), (0.6, 0, 0.95, 0.0)]:
        hows = [_away(z, how) for z in plain]
        chosen = [_choose(z, *h, pick=(0.11 + 0.41 * r) % 1) for r, (z, h) in enumerate(zip(plain, hows))]
        t, k, p, m = zip(*hows)
        got = _run(ctx, logits.cuda(), [c[0] for c in chosen], temperature=t, top_k=k, top_p=p, min_p=m)
        assert got.tolist() == [c[1] for c in chosen]


def test_all_defaults_and_strides(ctx):
    logits = _logits(5, 300, "f32", seed=1)
    wide = torch.full((5, 320), 1e30)
    wide[:, :300] = logits
    chosen = [_choose(z, 1.0, 0, 1.0, 0.0, pick=0.2 * r) for r, z in enumerate(_plain(logits))]
    got = _run(ctx, wide.cuda()[:, :300], [c[0] for c in chosen])
    assert got.tolist() == [c[1] for c in chosen]
    same = logits[:1].cuda().expand(5, -1)                       # one row for all
    got = _run(ctx, same, [0.0, 0.1, 0.5, 0.9, 1.0 - 2.0 ** -24])
    run = np.cumsum(np.exp(_plain(logits[0]) - _plain(logits[0]).max()))
    for u, token in zip([0.0, 0.1, 0.5, 0.9, 1.0 - 2.0 ** -24], got):
        below = run[token - 1] if token else 0.0
        assert below / run[-1] - MARGIN <= u <= run[token] / run[-1] + MARGIN


@pytest.mark.parametrize("vocab", [5, 64, 3001, 70000])
def test_equal_logits(ctx, vocab):
    """Ties go to the lowest index: of equal logits the first are kept."""
    logits = torch.zeros(6, vocab)
    k = max(1, vocab // 3)
    how = dict(temperature=[1.0] * 6, top_k=[0, k, 0, k, 0, 1], top_p=[1.0, 1.0, 0.5, 0.5, 1.0, 1.0], min_p=[0.0, 0.0, 0.0, 0.0, 1.0, 0.0])
    u = np.float32(0.999)
    got = _run(ctx, logits.cuda(), [u] * 6, **how)
    kept = [vocab, k, -(-vocab // 2), -(-k // 2), vocab, 1]
    assert got.tolist() == [min(int(float(u) * n), n - 1) for n in kept]
    # both zeros are equal too
    logits[:, 1::2] = -0.0
    assert _run(ctx, logits.cuda(), [u] * 6, **how).tolist() == got.tolist()


def test_two_values(ctx):
    """More equal logits at the cut than are kept of them."""
    logits = torch.full((4, 9000), 1.0)
    logits[:, 100::7] = 2.0
    high = torch.arange(100, 9000, 7)
    low = torch.tensor([i for i in range(9000) if i < 100 or (i - 100) % 7])
    for k in (10, len(high), len(high) + 500, 8999):
        kept = torch.cat([high[:k], low[:max(0, k - len(high))]]).sort().values
        w = torch.where(logits[0, kept] == 2, 1.0, float(np.exp(-1.0))).double().cumsum(0)
        places = [0, len(kept) // 3, len(kept) // 2, len(kept) - 1]
        u = [float((w[i] - (w[i] - (w[i - 1] if i else 0)) / 2) / w[-1]) for i in places]
        got = _run(ctx, logits.cuda(), u, top_k=[k] * 4)
        assert got.tolist() == [int(kept[i]) for i in places]


def test_infinities_and_nan(ctx):
    inf, nan = float("inf"), float("nan")
    rows = [[-inf, -inf, -inf, -inf], [nan, nan, nan, nan], [nan, -inf, nan, -inf], [1.0, nan, nan, -inf], [nan, -inf, 3.0, -inf],
            [0.0, inf, 5.0, inf], [inf, nan, inf, -inf], [-3e38, -inf, -inf, -3e38], [3e38, -3e38, 0.0, 3e38]]
    n = len(rows)
    for how in [{}, dict(top_k=[2] * n), dict(top_p=[0.99] * n), dict(min_p=[0.1] * n), dict(temperature=[0.5] * n, top_k=[3] * n, top_p=[0.9] * n)]:
        low, high = (_run(ctx, torch.tensor(rows).cuda(), [u] * n, **how) for u in (0.0, 0.9999))
        assert low.tolist() == [-1, -1, -1, 0, 2, 1, 0, 0, 0]
        assert high.tolist() == [-1, -1, -1, 0, 2, 3, 2, 3, 3]
    assert _run(ctx, torch.tensor(rows).cuda(), [0.9999] * n, temperature=[0.0] * n).tolist() == [-1, -1, -1, 0, 2, 1, 0, 0, 0]


def test_numbers_outside_their_ranges(ctx):
    logits = _logits(1, 500, "f32", seed=9).expand(8, -1).contiguous()
    first = int(logits[0].argmax())
    got = _run(ctx, logits.cuda(), [0.5] * 8, top_p=[-1.0, 0.0, 1.0, 2.0, float("nan"), 1.0, 1.0, 1.0],
               min_p=[0.0, 0.0, 0.0, 0.0, 0.0, 2.0, -1.0, float("nan")], top_k=[0, 0, 0, -5, 0, 0, 0, 0])
    assert got[0] == got[1] == first and got[5] == first
    assert len(set(got[[2, 3, 4, 6, 7]].tolist())) == 1
    last = _run(ctx, logits.cuda(), [1.0, 7.0, -1.0, float("nan"), 0.0, 1e30, -0.0, float("inf")])
    assert set(last[[0, 1, 5, 7]].tolist()) == {499} and set(last[[2, 3, 4, 6]].tolist()) == {0}


def test_a_sharp_peak_and_a_flat_field(ctx):
    """Temperatures that leave one token, and a hundred thousand tokens of almost the same weight."""
    z = torch.randn(2, 100000, generator=torch.Generator().manual_seed(4)) * 1e-3
    z[0, 77] = 30.0
    got = _run(ctx, z.cuda(), [0.9999, 0.25], temperature=[0.1, 1.0])
    w = np.cumsum(np.exp(z[1].double().numpy()))
    assert got[0] == 77
    assert w[got[1] - 1] / w[-1] - MARGIN <= 0.25 <= w[got[1]] / w[-1] + MARGIN


def test_no_rows(ctx):
    _run(ctx, torch.zeros(0, 10, device="cuda").view(0, 10), []) if torch.zeros(0, 10, device="cuda").data_ptr() else None
    ws = torch.zeros(16, dtype=torch.uint8, device="cuda")
    t = torch.zeros(1, dtype=torch.int32, device="cuda")
    z = torch.zeros(1, 10, device="cuda")
    how = binding._pack_sampling(0, 0, 0, 0, z.data_ptr())
    assert ctx.lib.gala_sample(ctx.h, None, binding._values(z, 1.0), 0, 10, how, t.data_ptr(), ws.data_ptr(), 16) == 0


def test_another_stream_and_a_graph(ctx):
    logits = _logits(4, 20000, "bf16", seed=12).cuda()
    u = torch.tensor([0.1, 0.4, 0.7, 0.95], device="cuda")
    p = torch.full((4,), 0.9, device="cuda")
    tokens = torch.zeros(4, dtype=torch.int32, device="cuda")
    need = ctx.sample_workspace_bytes(4, 20000)
    ws = torch.zeros(max(need, 16), dtype=torch.uint8, device="cuda")
    ctx.sample(logits, u, tokens, ws, need, top_p=p)
    want = tokens.clone()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        ctx.sample(logits, u, tokens, ws, need, top_p=p, stream=torch.cuda.current_stream())
    for _ in range(3):
        tokens.zero_(), ws.fill_(0xff)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(tokens, want)


@pytest.mark.parametrize("rows,vocab,kind", [(2, 3000001, "f32"), (600, 300, "bf16"), (1, 1100000, "f16"), (40, 4097, "residue")])
def test_many_rows_and_many_tokens(ctx, rows, vocab, kind):
    """Chunks of more tokens than usual, and more rows than the card has workgroups."""
    logits = _logits(rows, vocab, kind, seed=vocab)
    plain = _plain(logits)
    for how in [(0.8, 0, 1.0, 0.0), (0.8, 100, 0.9, 0.0), (0.6, 0, 0.5, 0.0)]:
        hows = [_away(z, how) for z in plain]
        chosen = [_choose(z, *h, pick=(0.07 + 0.37 * r) % 1) for r, (z, h) in enumerate(zip(plain, hows))]
        t, k, p, m = zip(*hows)
        got = _run(ctx, logits.cuda(), [c[0] for c in chosen], temperature=t, top_k=k, top_p=p, min_p=m)
        assert got.tolist() == [c[1] for c in chosen]


def test_cuts_among_many_close_logits(ctx):
    """A bin that holds more tokens than a list: the cut is searched over the whole row."""
    z = (torch.randn(3, 60000, generator=torch.Generator().manual_seed(8)) * 1e-3).float()
    plain = _plain(z)
    hows = [_away(p, h) for p, h in zip(plain, [(1.0, 20000, 1.0, 0.0), (1.0, 0, 0.3, 0.0), (1.0, 30000, 0.6, 0.999)])]
    for row, (p, h) in enumerate(zip(plain, hows)):
        kept, w, _ = ref.kept_tokens(p, *h)
        run = np.cumsum(np.where(kept, w, 0.0))
        for u in (0.1, 0.5, 0.9):
            t, k, q, m = h
            token = int(_run(ctx, z[row:row + 1].cuda(), [u], temperature=[t], top_k=[k], top_p=[q], min_p=[m])[0])
            assert kept[token]
            # a share of 1 / 20000 is as small as the weights' rounding can be told apart from
            assert run[token] / run[-1] - w[token] / run[-1] - MARGIN <= u <= run[token] / run[-1] + MARGIN


def test_logits_that_begin_anywhere(ctx):
    z = _logits(3, 5000, "f16", seed=77).cuda()
    u = [0.2, 0.5, 0.8]
    want = _run(ctx, z, u, top_p=[0.9] * 3)
    for shift in (1, 3, 7):
        moved = torch.empty(3, 5009, dtype=torch.float16, device="cuda").flatten()[shift:shift + 3 * 5001].view(3, 5001)[:, :5000]
        moved.copy_(z)
        assert _run(ctx, moved, u, top_p=[0.9] * 3).tolist() == want.tolist()
