"""Scales of values at places that no query sees - behind a sequence's end, in front of its window, in the first page, which stands for
missing ones - decide nothing: not a result's bits, whatever numbers they are."""
import numpy as np
import pytest
import torch

from tests import kv4_reference as ref
from tests.test_gpu_kv4_attention import Case, _many, ctx  # noqa: F401

pytestmark = pytest.mark.gpu
WINDOW, SINKS = 240, 3
# none that is a number; beyond what 32 bits let share a sum with ordinary ones, on either side; ordinary; mixed by token
SCALES = {"none": [0xffff], "large": [100 + 127 << 7], "small": [-95 + 127 << 7], "ordinary": [127 << 7],
          "mixed": [100 + 127 << 7, 0, -95 + 127 << 7, 0xffff, 126 << 7]}


def _unseen(c, first):
    """(page, token) of everything that no query sees from position first[b] of sequence b on, but for the first tokens"""
    seen = set()
    for b, n in enumerate(c.lens):
        for t in [*range(SINKS), *range(first[b], n)]:
            page = int(c.table[b, t // 64])
            if page >= 0:
                seen.add((page, t % 64))
    return [(p, t) for p in range(c.cache.data.shape[0]) for t in range(64) if (p, t) not in seen]


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("new", [1, 60, 130])
@pytest.mark.parametrize("window", [0, WINDOW])
def test_unseen_scales_decide_nothing(ctx, kind, new, window):  # noqa: F811
    c = Case(ctx, [new, new], [300, 500], _many(new), 2, 64, kind, seed=81)
    c.table[c.table == 0] = c.cache.data.shape[0] - 1            # page 0 is nobody's
    c.table[1, 3] = -1
    s = ref.places(64)[3]
    unseen = np.array(_unseen(c, [max(0, n - new - window + 1) if window else 0 for n in c.lens]))
    assert len(set(unseen[:, 0])) > 3 and (unseen[:, 0] == 0).any()
    clean, out = c.cache.data.cpu().numpy().reshape(-1, c.heads, ref.head_bytes(64)), {}
    for name, bits in SCALES.items():
        data = clean.copy()
        bits = np.array(bits)[np.arange(len(unseen)) % len(bits)][:, None]
        data[unseen[:, 0], :, s[unseen[:, 1]]], data[unseen[:, 0], :, s[unseen[:, 1]] + 1] = bits & 255, bits >> 8
        c.cache.data.copy_(torch.from_numpy(data).view(c.cache.data.shape))
        out[name] = c.run(window=window, sinks=SINKS)
        assert bool(out[name].isfinite().all())
    assert all(torch.equal(o, out["none"]) for o in out.values()), [n for n, o in out.items() if not torch.equal(o, out["none"])]
    c.check(out["mixed"], {(0, 0), (0, new - 1), (1, 0), (1, new - 1)})
