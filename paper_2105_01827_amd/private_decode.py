"""A small language model answered privately: ``python -m paper_2105_01827_amd.private_decode``.

The server holds the weights and evaluates every linear layer on ciphertexts (``he_fc``); the client holds the tokens, the
activations and the cache, and runs what lies between two linear layers on the values that its share and the server's add
up to: the residual stream and its norm in 8 bits, positions, the paged cache of 8 or 4 bits, attention and the choice of the
next token.  Both ends run in this process, on
one device.  Weights are random, as small whole numbers; activations travel as fixed-point numbers modulo p.
What hides one end's numbers from the other -- keys, encryption, the server's shares and masks -- is drawn afresh from the
system's random source at every use, whatever the model's seed.

One decoder block, several sequences at once: prompts of different lengths first, then token by token.
"""
import argparse
import dataclasses
import secrets

import numpy as np
import torch

from . import binding, devmem, workloads as wl


@dataclasses.dataclass(frozen=True)
class Shape:
    vocab: int = 500
    width: int = 128
    heads: int = 4
    heads_kv: int = 2
    head_dim: int = 32
    batch: int = 3
    steps: int = 6
    context: int = 256               # tokens that a sequence may have, its answer's included
    bits: int = 8                    # of a number in the cache: 8 or 4
    unit_x: float = 2.0 ** -5        # what one unit of an activation stands for
    unit_w: float = 2.0 ** -6        # ... and of a weight


def _fresh(*shape):
    """64-bit words that nobody else knows"""
    return np.frombuffer(secrets.token_bytes(8 * int(np.prod(shape))), np.uint64).reshape(shape).copy()


class Linear:
    """y = W x on ciphertexts, or (private=False) in the clear by the same whole numbers: both give the same residues."""

    def __init__(self, ctx, keys, weights, private):
        self.ctx, self.sk, self.private = ctx, keys, private
        self.n_o, self.n_i = weights.shape
        residues = (weights % wl.P).astype(np.uint64)
        if private:
            self.plan = ctx.fc_plan(residues)
            self.plan.bind(ctx.galois_keygen(keys, self.plan.rotations(), seed=secrets.randbits(64)))
            # where a packed input keeps what: slot -> 1 + index of the input, 0 for none
            self.places = devmem.to_dev(self.plan.pack_input(np.arange(1, self.n_i + 1, dtype=np.uint64)))
        self.weights = torch.from_numpy(weights.astype(np.float64)).cuda()

    def __call__(self, x):
        """x (rows, n_i) residues -> (rows, n_o) residues"""
        rows, n = x.shape[0], self.ctx.n
        if not self.private:
            centred = torch.where(x > wl.P // 2, x - wl.P, x).double()
            return (centred @ self.weights.t()).to(torch.int64).remainder(wl.P)
        # client: copies into slots, encryption with randomness of its own for each row
        slots = torch.nn.functional.pad(x, (1, 0))[:, self.places].contiguous()
        seeds = devmem.to_dev(_fresh(rows))
        ct, out = devmem.dev_empty(rows * 2 * n), devmem.dev_empty(rows * 2 * n)
        self.ctx.encrypt_batch(self.sk, slots, seeds, rows, ct)
        # server: the layer, masked by its share, and the other slots by masks from a seed that the client does not know: without
        # them they hold partial inner products of the weights
        r = devmem.to_dev(_fresh(rows, self.n_o) % np.uint64(wl.P))
        need = self.plan.workspace_bytes(rows)
        self.plan.he_fc(ct, rows, r, secrets.randbits(64), out, torch.empty(need, dtype=torch.uint8, device="cuda"), need)
        # client: its share, and the server's
        share = torch.empty(rows, self.n_o, dtype=torch.int64, device="cuda")
        self.ctx.decrypt_batch(self.sk, out, rows, slots)
        self.plan.unpack_share_batch(slots, rows, share)
        return (share + r).remainder(wl.P)


class Model:
    def __init__(self, shape, seed=0, private=True):
        self.shape, s = shape, shape
        par = wl.DEFAULT
        self.ctx = binding.Context(par.n, par.q, par.p, par.gadget_bits)
        rng = np.random.default_rng(seed)
        keys = self.ctx.keygen(secrets.randbits(64)) if private else None
        qkv = (s.heads + 2 * s.heads_kv) * s.head_dim

        def linear(n_o, n_i):
            return Linear(self.ctx, keys, rng.integers(-15, 16, (n_o, n_i)), private)

        self.embedding = torch.from_numpy(rng.standard_normal((s.vocab, s.width))).float().cuda()
        self.qkv, self.merge, self.head = linear(qkv, s.width), linear(s.width, s.heads * s.head_dim), linear(s.vocab, s.width)
        self.blocks = -(-s.context // 64)
        self.cache = {8: binding.KvCache, 4: binding.Kv4Cache}[s.bits](self.ctx, s.heads_kv, s.head_dim, pages=s.batch * self.blocks)
        # pages in any order
        self.table = torch.from_numpy(rng.permutation(s.batch * self.blocks).astype(np.int32).reshape(s.batch, self.blocks)).cuda()
        table = binding.rope_table(64 * self.blocks, s.head_dim)
        self.rope = binding.Rope(torch.from_numpy(table).cuda())
        self.lens = [0] * s.batch

    def normed(self, x, merged=None):
        """The stream x, a layer's output added if there is one, as the next layer takes it: its norm as whole numbers of 8 bits"""
        out = torch.empty(x.shape, dtype=torch.int64, device="cuda")
        self.ctx.rms_norm(x, out, add=merged, limit=127, unit=self.shape.unit_x, add_unit=self.shape.unit_x * self.shape.unit_w)
        return out

    def step(self, tokens, counts):
        """`tokens`: new ones of all sequences, counts[b] of sequence b; returns the logits after each sequence's last, as residues"""
        s, unit = self.shape, self.shape.unit_x * self.shape.unit_w
        if min(counts) < 1:
            raise ValueError("logits come after a sequence's last new token: each has to bring one")
        if max(a + b for a, b in zip(self.lens, counts)) > s.context:
            raise ValueError(f"a sequence has room for {s.context} tokens")
        self.lens = [a + b for a, b in zip(self.lens, counts)]
        starts = torch.tensor([0] + list(np.cumsum(counts)), dtype=torch.int32, device="cuda")
        batch = binding.KvBatch(starts, torch.tensor(self.lens, dtype=torch.int32, device="cuda"), self.table, max(counts), max(self.lens))
        x = self.embedding[tokens]
        qkv = self.qkv(self.normed(x)).view(-1, s.heads + 2 * s.heads_kv, s.head_dim)
        q, k, v = qkv.split([s.heads, s.heads_kv, s.heads_kv], 1)
        turned = torch.empty(q.shape, dtype=torch.float32, device="cuda")
        self.cache.append(batch, k, v, q=q, q_out=turned, rope=self.rope, unit=unit)
        # attention straight into the next layer's fixed point
        mixed = torch.empty(q.shape, dtype=torch.int64, device="cuda")
        need = self.cache.attention_workspace_bytes(batch, s.heads)
        self.cache.attention(batch, turned, mixed, s.head_dim ** -0.5, torch.empty(max(need, 16), dtype=torch.uint8, device="cuda"),
                             need, unit=s.unit_x)
        merged = self.merge(mixed.view(-1, s.heads * s.head_dim))
        last = (starts[1:] - 1).long()
        return self.head(self.normed(x[last], merged[last]))

    def answer(self, prompts, temperature=0.8, top_k=40, top_p=0.95, seed=0):
        """Prompts (lists of tokens) -> the tokens that follow, (steps, batch); sequences begin anew"""
        s, rows = self.shape, len(prompts)
        # the last token drawn needs no place
        if max(map(len, prompts)) + s.steps - 1 > s.context:
            raise ValueError(f"a sequence has room for {s.context} tokens, its answer's included")
        self.lens = [0] * s.batch
        gen = torch.Generator().manual_seed(seed)
        need = self.ctx.sample_workspace_bytes(rows, s.vocab)
        workspace = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
        settings = dict(temperature=torch.full((rows,), temperature, device="cuda"), top_p=torch.full((rows,), top_p, device="cuda"),
                        top_k=torch.full((rows,), top_k, dtype=torch.int32, device="cuda"))
        tokens, counts, answer = torch.tensor(sum(prompts, []), device="cuda"), [len(p) for p in prompts], []
        for _ in range(s.steps):
            logits = self.step(tokens, counts)
            drawn = torch.empty(rows, dtype=torch.int32, device="cuda")
            self.ctx.sample(logits, torch.rand(rows, generator=gen).cuda(), drawn, workspace, need, unit=s.unit_x * s.unit_w, **settings)
            answer.append(drawn)
            tokens, counts = drawn.long(), [1] * rows
        return torch.stack(answer).cpu()


def prompts_for(shape, seed=0):
    rng = np.random.default_rng([seed, 7])
    return [rng.integers(0, shape.vocab, int(n)).tolist() for n in rng.integers(3, 90, shape.batch)]


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=Shape.steps)
    ap.add_argument("--batch", type=int, default=Shape.batch)
    ap.add_argument("--bits", type=int, default=Shape.bits, choices=(8, 4), help="of a number in the cache")
    a = ap.parse_args()
    shape = Shape(steps=a.steps, batch=a.batch, bits=a.bits)
    prompts = prompts_for(shape)
    shape = dataclasses.replace(shape, context=max(map(len, prompts)) + shape.steps)
    for private in (True, False):
        answer = Model(shape, private=private).answer(prompts)
        for b, p in enumerate(prompts):
            print(f"{'on ciphertexts' if private else 'in the clear  '}  sequence {b} ({len(p)} tokens): {answer[:, b].tolist()}", flush=True)


if __name__ == "__main__":
    main()
