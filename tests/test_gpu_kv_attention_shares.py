"""Attention over the paged 8-bit cache where few keys have most of the weight and thousands share the rest: what those give
must come out within a few roundings of the output, however many they are.  Values have a mean far from zero, so that what is
lost does not average out.

Queries are whole multiples of 1/64 with a largest of 127/64, so that whole numbers of 16 bits hold them exactly and the bounds
need no allowance for the queries' rounding."""
import numpy as np
import pytest
import torch

from tests import decode_reference as ref
from tests.test_gpu_kv_attention import TYPES, UNIT, Case, _plain, ctx  # noqa: F401

pytestmark = pytest.mark.gpu
FIRST = 127.0 / 64                # the first channel of every query, and of the first key


def _case(ctx, new, lens, heads, group, dim, kind, out, share, spread, seed):
    """Every sequence's first token has no value and about `share` of the last query's weight; `spread` scales the other keys'
    scores apart, 0 leaves them equal.  Returns (case, scale of the scores)."""
    c = Case(ctx, new, lens, heads, group, dim, kind, out, seed=seed)
    rng = np.random.default_rng(seed)
    k = rng.integers(-127, 128, c.k.shape).astype(np.int8)
    v = rng.integers(20, 128, c.v.shape).astype(np.int8)
    k[..., 0] = 0
    for pages in c.table.numpy():
        k[pages[0], :, 0] = 0
        k[pages[0], :, 0, 0] = 127
        v[pages[0], :, 0] = 0
    codes = np.zeros((*k.shape[:2], ref.head_bytes(dim)), np.int8)
    for part, place in zip((k, v), ref.code_places(dim)):
        codes[:, :, place] = part
    c.k, c.v = k, v
    c.cache.codes.copy_(torch.from_numpy(codes).view(codes.shape[0], -1))
    c.cache.scales[..., 0] = 1.0 / 64
    scale = float(np.float32(np.log(share / (1 - share) * (max(lens) - 1)) / FIRST ** 2))
    q = rng.integers(-3, 4, tuple(c.q.shape)) * (spread / 64)
    q[..., 0] = FIRST
    q = torch.from_numpy(q)
    c.q = (torch.round(q / UNIT).to(torch.int64).remainder(1032193) if kind == "residue" else q.to(TYPES[kind])).cuda()
    return c, scale


def _check(c, out, rows, of_block, halves=False):
    """of_block: the largest error of a weight as a share of the largest weight in its block of 64 keys; halves: weights times
    their block's scale of values in half precision instead, with steps of 2^-31 of the largest at the most where they are small."""
    got, q, scales = _plain(out), _plain(c.q), c.cache.scales.cpu().double().numpy()
    eps = ref.UNIT_ROUNDOFF.get(str(out.dtype).replace("torch.", ""), 0)
    tiny = UNIT / 2 if c.out_kind == "residue" else 2.0 ** -24
    for b, i in rows:
        pages, n = c.table[b].numpy(), c.lens[b] - c.new[b] + i + 1
        for h in range(c.heads * c.group):
            head = h // c.group
            k, v = ((x[pages, head].astype(np.float64) * scales[pages, head, w][:, None, None]).reshape(-1, c.dim)[:n]
                    for w, x in enumerate((c.k, c.v)))
            x = q[c.starts[b] + i, h]
            s = c.scale * (k @ x)
            w = np.exp(s - s.max())
            want, mean = (w[:, None] * v).sum(0) / w.sum(), (w[:, None] * np.abs(v)).sum(0) / w.sum()
            # exponents and sums in 32 bits, of the numerator and of the weights' sum
            slack = 2.0 ** -20 * (np.abs(s) + c.scale * (np.abs(k) @ np.abs(x)) + np.abs(s).max() + 1)
            bound = (2 * np.expm1(slack.max()) + 2.0 ** -18) * mean
            if halves:
                of_scale = np.repeat(scales[pages, head, 1], 64)[:n]
                bound += 2.0 ** -11 * mean + n * 127 * 2.0 ** -32 * (w * of_scale).max() / w.sum()
            else:
                edges = np.arange(0, n, 64)
                bound += of_block * (np.maximum.reduceat(w, edges)[:, None] * np.add.reduceat(np.abs(v), edges)).sum(0) / w.sum()
            bound += eps * (np.abs(want) + bound) + tiny
            if n > 64:
                assert (bound < 0.03 * np.abs(want)).all() or c.out_kind == "residue"          # nothing, or half, would not do
                assert (bound < 0.2 * np.abs(want)).all()
            over = (np.abs(got[c.starts[b] + i, h] - want) / bound).max()
            assert over <= 1, (b, i, h, over, float(np.median(got[c.starts[b] + i, h] / want)))


# (new tokens, lengths, heads, query heads of each): one workgroup a head; more than 256 workgroups; keys split over workgroups;
# short prompts beside a long history
SHAPES = [([1], [900], 2, 3), ([1] * 20, [1500] * 20, 16, 1), ([1], [8192], 2, 2), ([1, 1], [30001, 20000], 2, 2), ([20, 3], [3000, 2500], 2, 4)]


@pytest.mark.parametrize("kind,out", [("f16", "f16"), ("bf16", "bf16"), ("f32", "f32"), ("residue", "f32"), ("f32", "residue")])
@pytest.mark.parametrize("share,spread", [(0.9, 0), (0.95, 1), (0.98, 0), (0.98, 1)])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_a_first_token_without_a_value(ctx, shape, share, spread, kind, out):
    new, lens, heads, group = SHAPES[shape]
    c, scale = _case(ctx, new, lens, heads, group, 64, kind, out, share, spread, seed=shape)
    rows = {(0, 0), (0, new[0] - 1), (len(new) - 1, new[-1] - 1)}
    _check(c, c.run(scale=scale), rows, 2.0 ** -32)


# prompts long enough for weights in half precision: few keys, or many groups of queries
PROMPTS = [([150, 40], [1000, 700], 16, 4), ([260, 200], [8192, 6000], 16, 8)]


@pytest.mark.parametrize("kind,out", [("f16", "f16"), ("bf16", "bf16"), ("f16", "bf16")])
@pytest.mark.parametrize("share,spread", [(0.9, 0), (0.98, 0), (0.98, 1), (0.995, 0), (0.998, 0)])
@pytest.mark.parametrize("shape", range(len(PROMPTS)))
def test_a_first_token_without_a_value_in_prompts(ctx, shape, share, spread, kind, out):
    new, lens, heads, group = PROMPTS[shape]
    c, scale = _case(ctx, new, lens, heads, group, 64, kind, out, share, spread, seed=10 + shape)
    _check(c, c.run(scale=scale), {(0, 0), (0, new[0] - 1), (1, new[1] - 1)}, None, halves=True)


@pytest.mark.parametrize("new", [1, 150])
@pytest.mark.parametrize("large", [1.0, 2.0 ** 20, 2.0 ** 50])
def test_blocks_of_zeros_beside_large_values(ctx, new, large):
    """Every second block holds nothing but zeros: its keys count in the weights' sum whatever the others' values are."""
    c, scale = _case(ctx, [new], [640], 32, 4, 64, "bf16", "bf16", 0.5, 0, seed=40)
    c.cache.scales[..., 1] *= large
    zero = c.table[0, ::2].long()
    c.cache.scales[zero.cuda(), :, 1] = 0
    _check(c, c.run(scale=0.0), {(0, 0), (0, new - 1)}, 2.0 ** -32, halves=new > 1)
    c.cache.codes.view(c.cache.codes.shape[0], c.heads, -1)[zero.cuda(), :, ref.head_bytes(64) // 2:] = 0
    c.v[zero.numpy()] = 0
    _check(c, c.run(scale=scale), {(0, 0), (0, new - 1)}, 2.0 ** -32, halves=new > 1)


def test_long_prompts_as_exact_sums(ctx):
    """Few groups of queries over many keys: weights are not in half precision there, whatever the types."""
    for kind in ("f16", "bf16"):
        c, scale = _case(ctx, [600, 450], [600, 1300], 1, 4, 128, kind, kind, 0.98, 1, seed=50)
        _check(c, c.run(scale=scale), {(0, i) for i in (0, 15, 16, 63, 64, 255, 256, 599)} | {(1, i) for i in (0, 31, 32, 449)}, 2.0 ** -32)


def test_a_token_beside_a_prompt(ctx):
    """The call's bound on new tokens decides for all of its sequences: one token is worked out as the prompt's are."""
    c, scale = _case(ctx, [150, 1, 1], [1000, 900, 70], 16, 4, 64, "f16", "f16", 0.98, 0, seed=51)
    _check(c, c.run(scale=scale), {(0, 149), (1, 0), (2, 0)}, None, halves=True)
