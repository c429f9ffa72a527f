"""The new operators together, as they are used: a small language model over a cache in 4 bits, and a decoder block's steps
with positions on several axes, captured into a graph and replayed."""
import dataclasses

import numpy as np
import pytest
import torch

from paper_2105_01827_amd import binding, private_decode as pd, workloads as wl
from tests import decode_reference as dref, kv4_reference as ref

pytestmark = pytest.mark.gpu


def test_tokens_on_ciphertexts_and_in_the_clear():
    shape = pd.Shape(steps=3, bits=4)
    prompts = pd.prompts_for(shape)
    private, clear = (pd.Model(shape, private=p).answer(prompts) for p in (True, False))
    assert torch.equal(private, clear)
    assert private.min() >= 0 and private.max() < shape.vocab and len(private.unique()) > 2


def test_token_by_token_is_the_prompt_at_once():
    """A token's codes depend on no other token, so logits after a prompt given as a whole and token by token differ by the
    roundings of attention alone."""
    shape = pd.Shape(batch=1, bits=4)
    prompt = pd.prompts_for(shape)[0][:20]
    whole, single = (pd.Model(shape, private=False) for _ in range(2))
    a = whole.step(torch.tensor(prompt, device="cuda"), [len(prompt)])
    for token in prompt:
        b = single.step(torch.tensor([token], device="cuda"), [1])
    used = whole.cache.data[whole.table[0, 0]]
    k, v, e, s = ref.places(shape.head_dim)
    live = np.unique(np.concatenate([x[:20].ravel() for x in (k, e, s[:, None], s[:, None] + 1)]))
    both = [c.data[int(m.table[0, 0])].cpu().numpy().reshape(shape.heads_kv, -1) for m, c in ((whole, whole.cache), (single, single.cache))]
    assert used.numel() and np.array_equal(both[0][:, live], both[1][:, live])
    a, b = (torch.where(x > wl.P // 2, x - wl.P, x).double() for x in (a, b))
    assert float(torch.nn.functional.cosine_similarity(a, b)) > 0.9999


def test_four_bits_are_near_eight():
    """Logits of the same prompt over both caches: e2m1 keeps a value to within a quarter, most far better."""
    prompt = pd.prompts_for(pd.Shape(batch=1))[0][:40]
    a, b = (pd.Model(dataclasses.replace(pd.Shape(batch=1), bits=bits), private=False).step(torch.tensor(prompt, device="cuda"), [len(prompt)]) for bits in (8, 4))
    a, b = (torch.where(x > wl.P // 2, x - wl.P, x).double() for x in (a, b))
    assert float(torch.nn.functional.cosine_similarity(a, b)) > 0.9


class Block:
    """norm -> (a projection of fixed numbers) -> positions -> append -> attention, for `counts` new tokens of each sequence"""
    width, heads, heads_kv, dim = 96, 4, 2, 32

    def __init__(self, counts, lens, seed=0):
        par = wl.DEFAULT
        self.ctx = binding.Context(par.n, par.q, par.p, par.gadget_bits)
        gen = torch.Generator().manual_seed(seed)
        rows = sum(counts)
        self.x, self.add = (torch.randn(rows, self.width, generator=gen).cuda() for _ in range(2))
        self.project = (torch.randint(-3, 4, (self.width, (self.heads + 2 * self.heads_kv) * self.dim), generator=gen) / 8).cuda()
        axis, column = binding.axes_layout([4, 6, 6], 1)
        self.rope = binding.AxesRope(torch.from_numpy(binding.rope_table(300, self.dim)).cuda(), axis, column)
        self.at = torch.randint(0, 300, (rows, 3), generator=gen, dtype=torch.int32).cuda()
        blocks = -(-max(lens) // 64)
        self.cache = binding.Kv4Cache(self.ctx, self.heads_kv, self.dim, pages=len(lens) * blocks)
        self.cache.data.zero_()
        self.table = torch.randperm(len(lens) * blocks, generator=gen).view(len(lens), blocks).to(torch.int32).cuda()
        starts = [0] + list(np.cumsum(counts))
        self.batch = binding.KvBatch(torch.tensor(starts, dtype=torch.int32, device="cuda"), torch.tensor(lens, dtype=torch.int32, device="cuda"), self.table,
                                     max(counts), max(lens))
        self.codes, self.scales = torch.empty(rows, self.width, dtype=torch.int8, device="cuda"), torch.empty(rows, 1, device="cuda")
        self.sum, self.out = torch.empty_like(self.x), torch.empty(rows, self.heads, self.dim, device="cuda")
        self.qkv = torch.empty(rows, self.heads + 2 * self.heads_kv, self.dim, device="cuda")
        need = self.cache.attention_workspace_bytes(self.batch, self.heads)
        self.need, self.workspace = need, torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")

    def step(self, stream=None):
        self.ctx.rms_norm(self.x, self.codes, add=self.add, sum_out=self.sum, limit=127, scales=self.scales, stream=stream)
        torch.matmul(self.codes.float() * self.scales, self.project, out=self.qkv.view(-1, self.project.shape[1]))
        q, k, v = self.qkv.split([self.heads, self.heads_kv, self.heads_kv], 1)
        both = self.qkv[:, :self.heads + self.heads_kv]
        self.ctx.rope_apply(self.rope, self.at, both, both, stream=stream)
        self.cache.append(self.batch, k, v, stream=stream)
        self.cache.attention(self.batch, q, self.out, self.dim ** -0.5, self.workspace, self.need, stream=stream)
        return self.out


@pytest.mark.parametrize("counts,lens", [([70, 3], [70, 40]), ([1, 1, 1], [130, 1, 64])])
def test_a_block_in_a_graph(counts, lens):
    c = Block(counts, lens)
    want = [t.clone() for t in (c.step(), c.sum, c.codes, c.qkv, c.cache.data)]
    assert bool(want[0].isfinite().all())
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        c.step(torch.cuda.current_stream())
    for _ in range(4):
        for t in (c.out, c.sum, c.codes, c.qkv, c.cache.data):
            t.zero_()
        c.x.mul_(1.0)                                    # eager work between the replays
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((c.out, c.sum, c.codes, c.qkv, c.cache.data), want))


def test_a_block_against_the_definition():
    """One sequence from its first token: every step of the block by its definition, attention in 64 bits."""
    c = Block([50], [50], seed=3)
    out = c.step().cpu().double().numpy()
    s, y = ref.rms_norm(c.x.cpu().numpy(), c.add.cpu().numpy(), None, 1e-6)
    codes, scales = ref.whole(y, 127, 0)
    assert np.array_equal(c.codes.cpu().numpy(), codes) and np.array_equal(c.sum.cpu().numpy(), s) and np.array_equal(c.scales.cpu().numpy(), scales)
    qkv = c.qkv.cpu().numpy()                            # queries and keys turned, values as the projection gave them
    q, k, v = qkv[:, :4], qkv[:, 4:6], qkv[:, 6:]
    codes, exponents = ref.key_codes(k)
    keys = ref.key_values(codes, exponents, c.dim)
    codes, scale = ref.value_codes(v)
    values = ref.VALUES[codes][..., :c.dim] * scale[..., None].astype(np.float64)
    for i in range(50):
        seen = dref.see(i, 50, 0, 0)
        for h in range(4):
            want, bound = ref.attention(q[i, h].astype(np.float64), keys[:, h // 2], values[:, h // 2], seen, c.dim ** -0.5, 3, 3)
            assert (np.abs(out[i, h] - want) <= bound + 2.0 ** -24 * np.abs(want) + 2.0 ** -30).all()


def test_two_calls_at_once():
    """Two caches on two streams, each with a workspace of its own."""
    a, b = Block([1, 1], [5000, 300], seed=1), Block([1, 1], [4000, 100], seed=2)
    for c in (a, b):
        c.cache.data.random_(0, 256)
        c.cache.data.bitwise_and_(0x77)                  # exponents and scales that are numbers
    torch.cuda.synchronize()
    want = [c.step().clone() for c in (a, b)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        for c, st in zip((a, b), streams):
            with torch.cuda.stream(st):
                c.step(st)
        torch.cuda.synchronize()
        assert all(torch.equal(c.out, w) for c, w in zip((a, b), want))
