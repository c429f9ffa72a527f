"""What hides one end's numbers from the other in the private model: never the same twice, whatever the model's seed."""
import pytest
import torch

from paper_2105_01827_amd import binding, private_decode as pd

pytestmark = pytest.mark.gpu


def test_nothing_that_hides_is_drawn_twice(monkeypatch):
    drawn = {"keys": [], "rows": [], "shares": [], "masks": []}
    keygen, galois, encrypt, he_fc = (binding.Context.keygen, binding.Context.galois_keygen, binding.Context.encrypt_batch,
                                      binding.FcPlan.he_fc)

    def spy_keygen(self, seed):
        drawn["keys"].append(seed)
        return keygen(self, seed)

    def spy_galois(self, sk, rots, seed):
        drawn["keys"].append(seed)
        return galois(self, sk, rots, seed)

    def spy_encrypt(self, sk, slots, seeds, *args, **kw):
        drawn["rows"] += seeds.cpu().view(torch.int64).tolist()
        return encrypt(self, sk, slots, seeds, *args, **kw)

    def spy_fc(self, ct, batch, r, mask_seed, *args, **kw):
        drawn["masks"].append(mask_seed)
        drawn["shares"] += [tuple(row) for row in r.cpu().view(torch.int64).tolist()]
        return he_fc(self, ct, batch, r, mask_seed, *args, **kw)

    monkeypatch.setattr(binding.Context, "keygen", spy_keygen)
    monkeypatch.setattr(binding.Context, "galois_keygen", spy_galois)
    monkeypatch.setattr(binding.Context, "encrypt_batch", spy_encrypt)
    monkeypatch.setattr(binding.FcPlan, "he_fc", spy_fc)
    shape = pd.Shape(batch=2, steps=2)
    answers = []
    for _ in range(2):
        torch.cuda.manual_seed(5)                       # nor does what the program seeds for itself matter
        answers.append(pd.Model(shape, seed=3).answer([[1, 2, 3], [4, 5]]))
    assert torch.equal(*answers)
    assert len(drawn["keys"]) == 8 and len(drawn["masks"]) == 12 and len(drawn["rows"]) == 2 * (5 + 5 + 2 + 2 + 2 + 2)
    for what, words in drawn.items():
        assert len(set(words)) == len(words), what
    # words of 64 bits: one below 2^32 would be a chance of one in four thousand million
    assert all(abs(w) >= 1 << 32 for what in ("keys", "rows", "masks") for w in drawn[what])
