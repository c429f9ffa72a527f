"""The longest vocabulary that sampling takes: sums of 2^24 weights of 2^40 would not fit 64 bits."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2105_01827_amd import binding, workloads as wl
from tests.test_decode_host import AT, EARG, SamplingArg, ValuesArg

LONGEST = (1 << 24) - 1


@pytest.fixture(scope="module")
def ctx():
    par = wl.DEFAULT
    return binding.Context(par.n, par.q, par.p, par.gadget_bits)


@pytest.mark.parametrize("vocab", [LONGEST + 1, LONGEST + 2, 1 << 25, 1 << 30, 2 ** 31 - 1])
def test_longer_vocabularies_are_refused(ctx, vocab):
    logits, how = ValuesArg(AT, 0, 0, 1.0), SamplingArg(0, 0, 0, 0, AT)
    assert ctx.lib.gala_sample(ctx.h, None, C.byref(logits), 1, vocab, C.byref(how), AT, AT, 1 << 40) == EARG
    assert ctx.lib.gala_sample_workspace(1, vocab) == 0
    assert ctx.lib.gala_sample_workspace(1, LONGEST) > 0


@pytest.mark.gpu
@pytest.mark.parametrize("how,kept", [({}, LONGEST), (dict(top_k=LONGEST // 3), LONGEST // 3), (dict(top_p=0.5), LONGEST // 2 + 1),
                                      (dict(temperature=1e30, min_p=0.5), LONGEST)])
def test_equal_logits_of_the_longest(ctx, how, kept):
    """Sums next to 2^64, exact all the way: the token is the share of the kept ones that u says."""
    logits = torch.zeros(1, LONGEST, dtype=torch.float16, device="cuda").expand(2, -1)
    args = {k: torch.full((2,), v, dtype=torch.int32 if k == "top_k" else torch.float32, device="cuda") for k, v in how.items()}
    u = np.float32([0.25, 0.9999])
    need = ctx.sample_workspace_bytes(2, LONGEST)
    tokens = torch.full((2,), -7, dtype=torch.int32, device="cuda")
    ctx.sample(logits, torch.from_numpy(u).cuda(), tokens, torch.empty(need, dtype=torch.uint8, device="cuda"), need, **args)
    assert tokens.tolist() == [int(float(x) * kept) for x in u]
