"""What the operators of a language model on the client's side are timed on.

In private inference the server holds the weights and evaluates the linear layers on ciphertexts; what lies between
two linear layers has no weights and runs with the client: the keys and values of its tokens go into its cache with
their positions rotated in, its queries attend to that cache, and at the end it draws the next token from the logits.
Every case is one pass through one of these three operators:

  append     queries, keys and values of new tokens -> rotated queries; keys (rotated) and values in a paged cache of
             8-bit codes with one scale for each block of 64 tokens, head, and keys or values.  A pass then reads the
             blocks that it touched back as the values they stand for.
  attention  queries of a batch of sequences over such a cache: causal, with or without a sliding window and first
             tokens that stay visible, from one query to a whole prompt for each sequence.
  sample     one token a row from logits and given uniform numbers, with temperature, top-k, top-p and min-p.

Values are floats, or residues modulo p: fixed-point numbers as a decrypted share holds them.
"""
import math

import torch

own = False

BLOCK = 64                 # tokens of a page of the cache, which share a scale
P = 1032193                # plaintext modulus of the residues
UNIT = 2.0 ** -12          # what one unit of a residue stands for
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "residue": torch.int64}
WEIGHT_ONE = 2.0 ** 40     # sampling weights are whole multiples of 2^-40 of the largest


# ---- cases ------------------------------------------------------------------------------------------------------
def _append(batch, new, length, heads_q, heads_kv, dim, rot, layout, type_, ragged=0.0):
    return {"kind": "append", "batch": batch, "new": new, "length": length, "heads_q": heads_q, "heads_kv": heads_kv,
            "dim": dim, "rot": rot, "layout": layout, "type": type_, "ragged": ragged}


def _attention(batch, new, length, heads_q, heads_kv, dim, type_, window=0, sinks=0, ragged=0.0):
    return {"kind": "attention", "batch": batch, "new": new, "length": length, "heads_q": heads_q,
            "heads_kv": heads_kv, "dim": dim, "type": type_, "window": window, "sinks": sinks, "ragged": ragged}


def _sample(rows, vocab, type_, temperature, top_k, top_p, min_p):
    return {"kind": "sample", "rows": rows, "vocab": vocab, "type": type_, "temperature": temperature, "top_k": top_k,
            "top_p": top_p, "min_p": min_p}


def listed():
    named = {
        # one user's next token, from the shares of a decrypted projection: latency
        "append_1tok_b1_residue": _append(1, 1, 500, 16, 16, 64, 64, "half", "residue"),
        # the next token of 64 users at once, histories of all lengths
        "append_1tok_b64_bf16": _append(64, 1, 4096, 32, 8, 128, 128, "half", "bf16", 0.9),
        # four prompts behind a shared beginning, part of each head rotated, pairs side by side, from shares
        "append_prompts_b4_residue": _append(4, 2000, 2300, 16, 4, 128, 64, "interleaved", "residue", 0.7),
        # one long prompt, a head size that fills no power of two
        "append_prompt_b1_f16": _append(1, 8191, 8191, 24, 24, 80, 80, "half", "f16"),
        # one user's next token over a short history: latency
        "attend_1tok_b1_len1000_bf16": _attention(1, 1, 1000, 16, 16, 64, "bf16"),
        # one user's next token over a very long history: the whole card works on one sequence
        "attend_1tok_b1_len131072_f16": _attention(1, 1, 131072, 32, 4, 128, "f16"),
        # the next token of 64 users, histories up to 8192 tokens: the cache is streamed once
        "attend_1tok_b64_len8192_bf16": _attention(64, 1, 8192, 64, 8, 128, "bf16", ragged=0.5),
        # a window over long histories with a few first tokens visible, in 32 bits
        "attend_window_b32_f32": _attention(32, 1, 30001, 20, 4, 96, "f32", window=1024, sinks=4, ragged=0.9),
        # prompts that attend to themselves and to an earlier part of their sequences
        "attend_prompts_b2_bf16": _attention(2, 2000, 5207, 32, 8, 128, "bf16", ragged=0.6),
        # one user's token from a small vocabulary: latency
        "sample_b1_v32000_f32": _sample(1, 32000, "f32", 0.8, 50, 0.95, 0.0),
        # 64 users' tokens, top-p alone, from 16-bit logits
        "sample_b64_v100003_bf16": _sample(64, 100003, "bf16", 0.7, 0, 0.9, 0.0),
        # a large batch's tokens from decrypted logits, the whole tail but what min-p takes
        "sample_b256_v131072_residue": _sample(256, 131072, "residue", 1.0, 0, 1.0, 0.02),
    }
    return [dict(case, name=name) for name, case in named.items()]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of any size between the listed ones."""
    while True:
        kind = rng.choice(["append", "attention", "attention", "sample"])
        if kind == "sample":
            c = _sample(_log_int(rng, 1, 256), _log_int(rng, 100, 131072), rng.choice(["f32", "f16", "bf16", "residue"]),
                        rng.choice([0.0, 0.3, 0.7, 1.0, 1.3]), rng.choice([0, 0, 1, 20, 50, 400]),
                        rng.choice([1.0, 1.0, 0.95, 0.9, 0.5]), rng.choice([0.0, 0.0, 0.02, 0.1]))
            return c
        heads_kv = rng.choice([1, 2, 4, 5, 8, 16])
        heads_q = heads_kv * rng.choice([1, 2, 3, 4, 8])
        dim = rng.choice([32, 64, 64, 80, 96, 128, 128, 128, 192, 256])
        batch = _log_int(rng, 1, 64)
        new = rng.choice([1, 1, 1, _log_int(rng, 2, 16), _log_int(rng, 16, 4096)])
        if kind == "append":
            c = _append(batch, new, new + rng.choice([0, _log_int(rng, 1, 8192)]), heads_q, heads_kv, dim,
                        rng.choice([dim, dim // 2]), rng.choice(["half", "interleaved"]),
                        rng.choice(["f32", "f16", "bf16", "residue"]), rng.choice([0.0, 0.5, 0.9]))
            if batch * new * (heads_q + 2 * heads_kv) * dim <= 8191 * 72 * 80:
                return c
        else:
            length = new + rng.choice([0, _log_int(rng, 1, 100000)])
            window = rng.choice([0, 0, 0, _log_int(rng, 16, 4096)])
            c = _attention(batch, new, length, heads_q, heads_kv, dim, rng.choice(["f32", "f16", "bf16", "bf16"]), window,
                           rng.choice([0, 1, 4, 70]) if window else 0, rng.choice([0.0, 0.5, 0.9]))
            w = work(c)
            plain = 4 * batch * heads_q * new * length * dim      # products of the plain form
            if w["bytes"] <= 0.9e9 and w["flops"] <= 1.6e11 and plain <= 3.4e11 and batch * heads_kv * length * dim <= 64 * 8 * 8192 * 128:
                return c


def _spread(most, least, count, ragged):
    """count whole numbers up to `most`, the first equal to it, the others down to a share of 1 - ragged"""
    return [max(least, int(round(most * (1 - ragged * (b * 0.618034 % 1.0))))) for b in range(count)]


def _lengths(case):
    """(new tokens, tokens with the new ones) of each sequence"""
    new = _spread(case["new"], 1, case["batch"], case["ragged"] if case["new"] > 1 else 0.0)
    before = _spread(case["length"] - case["new"], 0, case["batch"], case["ragged"])
    return new, [n + b for n, b in zip(new, before)]


# ---- inputs -----------------------------------------------------------------------------------------------------
_kept = {}


def _context():
    """The framework's context, one for all passes, as a client's program keeps one."""
    from paper_2105_01827_amd import binding, workloads as wl
    if "ctx" not in _kept:
        par = wl.DEFAULT
        assert par.p == P
        _kept["ctx"] = binding.Context(par.n, par.q, par.p, par.gadget_bits)
    return _kept["ctx"]


def _values(gen, type_, *shape, spread=1.0):
    x = torch.randn(*shape, generator=gen, device="cuda") * spread
    return torch.round(x / UNIT).to(torch.int64).remainder(P) if type_ == "residue" else x.to(TYPES[type_])


def _int32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _starts(counts):
    return _int32([sum(counts[:b]) for b in range(len(counts) + 1)])


def _rope_table(positions, rot):
    """cos and sin of every position's angles, 10000^(-2i/rot) radians a position"""
    inv = 10000.0 ** (-torch.arange(rot // 2, device="cuda", dtype=torch.float64) * 2 / rot)
    a = torch.arange(positions, device="cuda", dtype=torch.float64)[:, None] * inv
    return torch.stack([a.cos(), a.sin()], -1).float().contiguous()


def _cache(gen, case, lens):
    """pages in any order; codes [page, head, token, value] of keys and of values, scales [page, head, keys or values]"""
    blocks = [-(-n // BLOCK) for n in lens]
    pages, heads, dim = sum(blocks) + 3, case["heads_kv"], case["dim"]
    order = torch.randperm(pages - 1, generator=gen, device="cuda").to(torch.int32)     # the last page is nobody's
    table = torch.full((len(lens), max(blocks)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(blocks):
        table[b, :n] = order[at:at + n]
        at += n
    codes = []
    for _ in range(2):
        c = torch.empty(pages, heads, BLOCK, dim, dtype=torch.int8, device="cuda")
        for part in c.split(2048):
            part.copy_((torch.randn(part.shape, generator=gen, device="cuda", dtype=torch.float32) * 33).round_().clamp_(-127, 127))
        codes.append(c)
    scales = (torch.rand(pages, heads, 2, generator=gen, device="cuda") + 0.5) / 33
    return table, codes[0], codes[1], scales


def _packed(k, v):
    """The same codes in the framework's order: of each page and head the keys, then the values, heads padded to a
    multiple of 16.  Keys lie in runs of 16 channels of 16 tokens, values in runs of 16 tokens of 16 channels."""
    pages, heads, _, dim = k.shape
    m = -(-dim // 16)
    k, v = (torch.nn.functional.pad(t, (0, 16 * m - dim)) for t in (k, v))
    k = k.view(pages, heads, 4, 16, m, 16).permute(0, 1, 2, 4, 3, 5).reshape(pages, heads, 1, -1)
    v = v.view(pages, heads, 4, 4, 4, m, 16).permute(0, 1, 5, 3, 6, 2, 4).reshape(pages, heads, 1, -1)
    return torch.cat([k, v], 2).contiguous()


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    s = dict(case)
    if case["kind"] == "sample":
        rows, vocab = case["rows"], case["vocab"]
        # a few likely tokens and a long tail, in any order
        rank = torch.rand(rows, vocab, generator=gen, device="cuda").argsort(-1).float()
        z = 12 - 1.1 * torch.log1p(rank) + 0.4 * torch.randn(rows, vocab, generator=gen, device="cuda")
        s["logits"] = torch.round(z / UNIT).to(torch.int64).remainder(P) if case["type"] == "residue" else z.to(TYPES[case["type"]])
        s["u"] = torch.rand(rows, generator=gen, device="cuda")
        for name in ("temperature", "top_p", "min_p"):
            s["of_" + name] = torch.full((rows,), case[name], device="cuda")
        s["of_top_k"] = torch.full((rows,), case["top_k"], dtype=torch.int32, device="cuda")
        s["tokens"] = torch.empty(rows, dtype=torch.int32, device="cuda")
        if own:      # the handle and the workspace that a client's program keeps
            s["ctx"] = _context()
            s["workspace_bytes"] = s["ctx"].sample_workspace_bytes(rows, vocab)
            s["workspace"] = torch.empty(s["workspace_bytes"], dtype=torch.uint8, device="cuda")
        return s
    new, lens = _lengths(case)
    heads_q, heads, dim, total = case["heads_q"], case["heads_kv"], case["dim"], sum(new)
    s["starts"], s["lens"], s["total"] = _starts(new), _int32(lens), total
    s["max_new"], s["max_len"] = max(new), max(lens)
    s["table"], s["k_codes"], s["v_codes"], s["scales"] = _cache(gen, case, lens)
    if own:          # the cache as earlier calls left it, in the framework's order
        from paper_2105_01827_amd import binding
        s["ctx"] = _context()
        s["codes"] = _packed(s.pop("k_codes"), s.pop("v_codes"))
        s["cache"] = binding.KvCache(s["ctx"], heads, dim, s["codes"], s["scales"])
        s["step"] = binding.KvBatch(s["starts"], s["lens"], s["table"], s["max_new"], s["max_len"])
    if case["kind"] == "append":
        fused = _values(gen, case["type"], total, heads_q + 2 * heads, dim)       # one projection's outputs
        s["q"], s["k"], s["v"] = fused.split([heads_q, heads, heads], 1)
        s["rope"] = _rope_table(max(lens), case["rot"])
        out = torch.float32 if case["type"] == "residue" else TYPES[case["type"]]
        s["q_out"] = torch.empty(total, heads_q, dim, dtype=out, device="cuda")
        back = [n - (n - m) // BLOCK * BLOCK for n, m in zip(lens, new)]          # tokens of the touched blocks
        s["back_starts"], s["back_total"], s["back_most"] = _starts(back), sum(back), max(back)
        s["k_back"], s["v_back"] = (torch.empty(sum(back), heads, dim, dtype=out, device="cuda") for _ in range(2))
        if own:
            s["rotation"] = binding.Rope(s["rope"], case["layout"] == "interleaved")
            s["back"] = binding.KvBatch(s["back_starts"], s["lens"], s["table"], s["back_most"], s["max_len"])
    else:
        s["q"] = _values(gen, case["type"], total, heads_q, dim, spread=2.0)
        s["out"] = torch.empty_like(s["q"])
        if own:
            s["workspace_bytes"] = s["cache"].attention_workspace_bytes(s["step"], heads_q, case["window"], case["sinks"])
            s["workspace"] = torch.empty(max(s["workspace_bytes"], 8), dtype=torch.uint8, device="cuda")
    return s


# ---- the plain forms --------------------------------------------------------------------------------------------
def _float(x):
    """A value in 32 bits: of a residue, its representative nearest to zero times the unit."""
    return torch.where(x > P // 2, x - P, x).float() * UNIT if x.dtype == torch.int64 else x.float()


def _rows(starts, total):
    """(sequence, row within it) of every row of a ragged batch"""
    counts = (starts[1:] - starts[:-1]).long()
    seq = torch.repeat_interleave(torch.arange(len(counts), device="cuda"), counts, output_size=total)
    return seq, torch.arange(total, device="cuda") - starts[seq]


def _rotated(x, cos, sin, rot, layout):
    if layout == "half":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        return torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., rot:]], -1)
    a, b = x[..., 0:rot:2], x[..., 1:rot:2]
    return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), x[..., rot:]], -1)


def _store(s, codes, which, x, first, touched):
    """New values x [sequence, block, token, head, value] with their places `touched` [sequence, block, token] into the
    pages: the block's scale grows where a new value needs it, and codes that are there are then rounded to it."""
    any_new = touched.any(2)
    blocks = first[:, None] // BLOCK + torch.arange(touched.shape[1], device="cuda")
    page = torch.where(any_new, s["table"].gather(1, blocks.clamp(max=s["table"].shape[1] - 1)).long(), codes.shape[0] - 1)
    held = (blocks * BLOCK < first[:, None])[..., None]                                  # has earlier tokens
    old = torch.where(held, s["scales"][page][..., which], 0.0)
    scale = torch.maximum(old, x.abs().amax((2, 4)) * (1.0 / 127.0))                     # [sequence, block, head]
    inverse = torch.where(scale > 0, scale.reciprocal(), 0.0)
    fresh = torch.round(x * inverse[:, :, None, :, None]).clamp(-127, 127)
    before = torch.round(codes[page].float() * (old * inverse)[..., None, None]).transpose(2, 3)
    codes[page] = torch.where(touched[..., None, None], fresh, before).transpose(2, 3).to(torch.int8)
    s["scales"][page, :, which] = scale


def _append_plain(s):
    seq, row = _rows(s["starts"], s["total"])
    new = s["starts"][1:] - s["starts"][:-1]
    first = (s["lens"] - new).long()
    pos = first[seq] + row
    cos, sin = (s["rope"][pos][:, None, :, i] for i in range(2))
    q = _rotated(_float(s["q"]), cos, sin, s["rot"], s["layout"]).to(s["q_out"].dtype)
    k = _rotated(_float(s["k"]), cos, sin, s["rot"], s["layout"])
    # the new tokens laid out by blocks: as many as the longest row of new tokens can touch
    place = (first // BLOCK * BLOCK)[:, None] + torch.arange(((s["max_new"] + BLOCK - 2) // BLOCK + 1) * BLOCK, device="cuda")
    touched = ((place >= first[:, None]) & (place < s["lens"][:, None])).view(len(new), -1, BLOCK)
    source = (s["starts"][:-1, None] + place - first[:, None]).clamp(0, s["total"] - 1)
    for codes, which, x in ((s["k_codes"], 0, k), (s["v_codes"], 1, _float(s["v"]))):
        laid = x[source].view(*touched.shape, *x.shape[1:]) * touched[..., None, None]
        _store(s, codes, which, laid, first, touched)
    seq, row = _rows(s["back_starts"], s["back_total"])
    pos = first[seq] // BLOCK * BLOCK + row
    page = s["table"][seq, pos // BLOCK].long()
    back = [(codes[page, :, pos % BLOCK].float() * s["scales"][page][..., which, None]).to(s["q_out"].dtype)
            for codes, which in ((s["k_codes"], 0), (s["v_codes"], 1))]
    return {"q": q, "k": back[0], "v": back[1]}


def _attention_plain(s):
    seq, row = _rows(s["starts"], s["total"])
    new = s["starts"][1:] - s["starts"][:-1]
    batch, most, heads, dim = len(new), s["max_new"], s["heads_kv"], s["dim"]
    group = s["heads_q"] // heads
    at = (s["lens"] - new)[:, None] + torch.arange(most, device="cuda")                  # positions of the queries
    # the blocks that some query can see: all, or those of the first tokens and of the window
    first, near = -(-s["sinks"] // BLOCK), (s["window"] + most + BLOCK - 2) // BLOCK + 1
    whole = not s["window"] or first + near >= s["table"].shape[1]
    block = torch.arange(s["table"].shape[1] if whole else first + near, device="cuda").expand(batch, -1)
    begin = block[:, :1] * 0 if whole else ((at[:, :1] + 1 - s["window"]).clamp(min=0) // BLOCK)
    block = block if whole else torch.where(block < first, block, block - first + begin)
    there = (block[..., None] * BLOCK + torch.arange(BLOCK, device="cuda")).flatten(1)
    twice = torch.zeros_like(there, dtype=torch.bool)                                     # a first block within the window too
    if not whole:
        twice[:, :first * BLOCK] = there[:, :first * BLOCK] >= begin * BLOCK
    page = s["table"].gather(1, block.clamp(max=s["table"].shape[1] - 1)).clamp(min=0).long()
    k, v = ((codes[page].float() * s["scales"][page][..., which, None, None]).transpose(1, 2).reshape(batch, heads, -1, dim)
            for codes, which in ((s["k_codes"], 0), (s["v_codes"], 1)))
    q = torch.zeros(batch, most, heads, group, dim, device="cuda")
    q[seq, row] = _float(s["q"]).view(-1, heads, group, dim)
    q = q.permute(0, 2, 3, 1, 4).reshape(batch, heads, group * most, dim)
    score = (torch.matmul(q, k.transpose(2, 3).contiguous()) * dim ** -0.5).view(batch, heads, group, most, -1)
    there, at = there[:, None], at[..., None]
    seen = (there <= at) & (there < s["lens"][:, None, None]) & ~twice[:, None]
    if s["window"]:
        seen &= (there > at - s["window"]) | (there < s["sinks"])
    score = score.masked_fill(~seen[:, None, None], -torch.inf)
    top = score.amax(-1, keepdim=True)
    weight = torch.exp(score - torch.where(top > -torch.inf, top, 0.0))
    total = weight.sum(-1, keepdim=True)
    out = torch.matmul(weight.view(batch, heads, group * most, -1), v).view(batch, heads, group, most, dim)
    out = (out / torch.where(total > 0, total, 1.0)).permute(0, 3, 1, 2, 4)[seq, row]
    return out.reshape(s["q"].shape).to(s["q"].dtype)


def _sample_plain(s):
    z = _float(s["logits"])
    order = torch.sort(z, dim=-1, descending=True, stable=True)
    greedy = s["of_temperature"] <= 0
    rate = torch.where(greedy, 1.0, s["of_temperature"]).reciprocal()[:, None]
    w = torch.exp((order.values - order.values[:, :1]) * rate)
    weight = (w.double() * WEIGHT_ONE).to(torch.int64)                                   # sums in any order are the same
    most = torch.where(greedy, 1, torch.where(s["of_top_k"] > 0, s["of_top_k"], z.shape[1]))
    kept = torch.arange(z.shape[1], device="cuda") < most[:, None]
    weight = weight * kept
    before = weight.cumsum(-1) - weight
    kept &= before.double() < (s["of_top_p"].double() * weight.sum(-1).double())[:, None]
    kept &= w >= s["of_min_p"][:, None]
    kept[:, 0] = True
    weight = weight * kept
    total = weight.sum(-1)
    target = torch.minimum((s["u"].double() * total.double()).to(torch.int64), total - 1)
    by_index = torch.zeros_like(weight).scatter_(1, order.indices, weight).cumsum(-1)
    return (by_index <= target[:, None]).sum(-1).to(torch.int32)


def run(s):
    if own:
        if s["kind"] == "append":
            s["cache"].append(s["step"], s["k"], s["v"], q=s["q"], q_out=s["q_out"], rope=s["rotation"], unit=UNIT)
            s["cache"].export(s["back"], s["k_back"], s["v_back"])
            return {"q": s["q_out"], "k": s["k_back"], "v": s["v_back"]}
        if s["kind"] == "attention":
            s["cache"].attention(s["step"], s["q"], s["out"], s["dim"] ** -0.5, s["workspace"], s["workspace_bytes"],
                                 window=s["window"], sinks=s["sinks"])
            return s["out"]
        s["ctx"].sample(s["logits"], s["u"], s["tokens"], s["workspace"], s["workspace_bytes"], unit=UNIT,
                        temperature=s["of_temperature"], top_k=s["of_top_k"], top_p=s["of_top_p"], min_p=s["of_min_p"])
        return s["tokens"]
    return {"append": _append_plain, "attention": _attention_plain, "sample": _sample_plain}[s["kind"]](s)


# ---- what a pass cannot do without ------------------------------------------------------------------------------
def _size(type_):
    return {"f32": 4, "f16": 2, "bf16": 2, "residue": 8}[type_]


def _seen(case):
    """(pairs of a query and a key that it sees, keys that some query sees), summed over the sequences"""
    pairs = keys = 0
    for new, length in zip(*_lengths(case)):
        window, sinks = case["window"] or length, case["sinks"]
        at = torch.arange(length - new, length)
        pairs += int((at.add(1).clamp(max=window) + at.add(1 - window).clamp(0, sinks)).sum())
        begin = max(0, length - new + 1 - window)
        keys += length - begin + min(begin, sinks)
    return pairs, keys


def work(case):
    """Bytes: every input once, every output once, of the cache what the call has to touch.  Operations: two for each
    product of a query with a key and of a weight with a value; one each for the other operators' values."""
    if case["kind"] == "sample":
        n = case["rows"] * case["vocab"]
        return {"bytes": n * _size(case["type"]) + case["rows"] * 24, "flops": n}
    new, lens = _lengths(case)
    heads, dim, heads_q = case["heads_kv"], case["dim"], case["heads_q"]
    if case["kind"] == "append":
        out = 4 if case["type"] == "residue" else _size(case["type"])
        row = (heads_q + 2 * heads) * dim
        back = sum(n - (n - m) // BLOCK * BLOCK for n, m in zip(lens, new))
        total = sum(new)
        return {"bytes": total * (row * _size(case["type"]) + heads_q * dim * out + 2 * heads * dim + case["rot"] * 4) +
                         (back - total) * 2 * heads * dim + back * 2 * heads * dim * out + (back // BLOCK + 1) * heads * 8,
                "flops": 3 * total * row}
    pairs, keys = _seen(case)
    blocks = keys // BLOCK + len(lens)
    return {"bytes": 2 * keys * heads * dim + blocks * heads * 8 + 2 * sum(new) * heads_q * dim * _size(case["type"]),
            "flops": 4 * pairs * heads_q * dim}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------
def _exact_float(x):
    if x.dtype != torch.int64:
        return x.double()
    x = x.double()
    return (x - P * (2 * x > P)) * UNIT


def _exact_append(s):
    """Sequence by sequence; each pair of a head as a complex number, turned by its position's angle."""
    out = {"q": [], "k": [], "v": []}
    starts, lens, rot = s["starts"].tolist(), s["lens"].tolist(), s["rot"]

    def turned(x, turn):
        pairs = x[..., :rot].unflatten(-1, (2, -1) if s["layout"] == "half" else (-1, 2))
        axis = -2 if s["layout"] == "half" else -1
        z = torch.complex(pairs.select(axis, 0), pairs.select(axis, 1)) * turn
        return torch.cat([torch.stack([z.real, z.imag], axis).flatten(-2), x[..., rot:]], -1)

    for b, length in enumerate(lens):
        lo, hi = starts[b], starts[b + 1]
        first = length - (hi - lo)
        turn = torch.complex(*s["rope"][first:length].double().unbind(-1))[:, None]
        out["q"].append(turned(_exact_float(s["q"][lo:hi]), turn))
        fresh = {"k": turned(_exact_float(s["k"][lo:hi]), turn), "v": _exact_float(s["v"][lo:hi])}
        for block in range(first // BLOCK, -(-length // BLOCK)):
            page, begin, end = int(s["table"][b, block]), max(first, block * BLOCK), min(length, block * BLOCK + BLOCK)
            for which, (name, x) in enumerate(fresh.items()):
                x = x[begin - first:end - first]
                there = begin - block * BLOCK
                codes = (s["k_codes"], s["v_codes"])[which][page, :, :there].double().transpose(0, 1)
                old = s["scales"][page, :, which].double() * (there > 0)
                scale = torch.maximum(old, x.abs().amax((0, 2)) / 127)[:, None]
                least = scale.clamp(min=1e-300)
                rows = torch.cat([codes * old[:, None] / least, x / least]).round().clamp(-127, 127)
                out[name].append(rows * scale)
    return {name: torch.cat(rows) for name, rows in out.items()}


def _exact_attention(s):
    """Sequence by sequence and head by head over the keys it sees."""
    starts, lens, group = s["starts"].tolist(), s["lens"].tolist(), s["heads_q"] // s["heads_kv"]
    out = torch.zeros(s["total"], s["heads_q"], s["dim"], dtype=torch.float64, device="cuda")
    for b, length in enumerate(lens):
        lo, hi = starts[b], starts[b + 1]
        page = s["table"][b, :-(-length // BLOCK)].long()
        at = torch.arange(length - (hi - lo), length, device="cuda")[:, None]
        there = torch.arange(length, device="cuda")[None]
        hidden = there > at
        if s["window"]:
            hidden |= (at - there >= s["window"]) & (there >= s["sinks"])
        for h in range(s["heads_kv"]):
            k, v = ((c[page, h].double() * s["scales"][page, h, which].double()[:, None, None]).reshape(-1, s["dim"])[:length]
                    for which, c in enumerate((s["k_codes"], s["v_codes"])))
            for g in range(h * group, h * group + group):
                score = s["q"][lo:hi, g].double() @ k.t() / math.sqrt(s["dim"])
                out[lo:hi, g] = torch.softmax(score.masked_fill(hidden, -math.inf), -1) @ v
    return out


def _exact_sample(s):
    tokens = []
    for r in range(s["rows"]):
        z = _exact_float(s["logits"][r])
        if s["temperature"] <= 0:
            tokens.append(int((z == z.max()).nonzero()[0]))
            continue
        chance = torch.softmax(z / float(s["of_temperature"][r]), -1)
        order = torch.argsort(z, descending=True, stable=True)[:s["top_k"] or None]
        likely = chance[order]
        kept = (likely.cumsum(0) - likely < float(s["of_top_p"][r]) * likely.sum()) & (likely >= float(s["of_min_p"][r]) * likely[0])
        kept[0] = True
        places, by = torch.sort(order[kept])
        run_ = likely[kept][by].cumsum(0)
        tokens.append(int(places[min(int((run_ <= float(s["u"][r]) * run_[-1]).sum()), len(places) - 1)]))
    return torch.tensor(tokens, dtype=torch.int32)


def exact(case, seed):
    assert not own
    s = prepare(case, seed)
    return {"append": _exact_append, "attention": _exact_attention, "sample": _exact_sample}[case["kind"]](s)
