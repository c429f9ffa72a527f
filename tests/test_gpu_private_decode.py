"""The small language model whose linear layers run on ciphertexts: whole numbers all the way between the client's steps, so
its tokens are those of the same model with the same whole-number products in the clear."""
import pytest
import torch

from paper_2105_01827_amd import private_decode as pd

pytestmark = pytest.mark.gpu


def test_tokens_on_ciphertexts_and_in_the_clear():
    shape = pd.Shape(steps=4)
    prompts = pd.prompts_for(shape)
    private, clear = (pd.Model(shape, private=p).answer(prompts) for p in (True, False))
    assert torch.equal(private, clear)
    assert private.min() >= 0 and private.max() < shape.vocab and len(private.unique()) > 3


def test_token_by_token_is_the_prompt_at_once():
    """Logits after a prompt given as a whole, and token by token: the codes of a growing block are rounded again when its
    scale grows, a code's step at most for each growth."""
    shape = pd.Shape(batch=1)
    prompt = pd.prompts_for(shape)[0][:20]
    whole, single = (pd.Model(shape, private=False) for _ in range(2))
    a = whole.step(torch.tensor(prompt, device="cuda"), [len(prompt)])
    for token in prompt:
        b = single.step(torch.tensor([token], device="cuda"), [1])
    a, b = (torch.where(x > pd.wl.P // 2, x - pd.wl.P, x).double() for x in (a, b))
    assert float(torch.nn.functional.cosine_similarity(a, b)) > 0.98
