"""The small language model's sequences: as many tokens as they have room for, and from the beginning for each answer."""
import pytest
import torch

from paper_2105_01827_amd import private_decode as pd

pytestmark = pytest.mark.gpu


def test_no_more_tokens_than_there_is_room_for():
    model = pd.Model(pd.Shape(batch=2, steps=61, context=100), private=False)
    with pytest.raises(ValueError):
        model.answer([[1] * 41, [2]])
    assert model.answer([[1] * 40, [2]]).shape == (61, 2) and model.lens == [100, 61]
    tokens = torch.tensor([3, 4], device="cuda")
    with pytest.raises(ValueError):
        model.step(tokens, [1, 1])
    assert model.lens == [100, 61]


def test_answers_begin_anew():
    shape = pd.Shape(batch=2, steps=5, context=64)
    model, other = (pd.Model(shape, private=False) for _ in range(2))
    first = model.answer([[1, 2, 3] * 10, [4] * 20])
    second = model.answer([[5] * 40, [6, 7]])
    assert torch.equal(second, other.answer([[5] * 40, [6, 7]]))
    assert torch.equal(first, other.answer([[1, 2, 3] * 10, [4] * 20]))


def test_as_long_as_the_context():
    """A context beyond the default, over the whole rope table and the last page."""
    model = pd.Model(pd.Shape(batch=1, steps=3, context=300), private=False)
    logits = model.step(torch.arange(300, device="cuda"), [300])
    assert model.blocks == 5 and int(logits.unique().numel()) > 100


def test_a_sequence_without_new_tokens():
    """There is no last token of its own whose logits it could get."""
    model = pd.Model(pd.Shape(batch=2, steps=1), private=False)
    with pytest.raises(ValueError):
        model.answer([[1, 2], []])
    assert model.lens == [0, 0]
