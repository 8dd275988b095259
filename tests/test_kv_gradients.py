"""A cache passes no gradients on: it says so instead of dropping them (on the CPU, before a device is touched)."""
import pytest
import torch

import paper_2609_36601_amd as saki
from paper_2609_36601_amd import speculative
from tests.test_rollout_cached_host import model
from tests.test_rollout_driver_host import fakes  # noqa: F401


def test_tensors_with_a_history_are_refused():
    c = saki.PagedKV.alloc(3, 4, 8, 2, 2, 8, 16, device="cpu")
    x = torch.zeros(3, 2, 16, dtype=torch.bfloat16)
    leaf = torch.zeros(3, 2, 16, dtype=torch.bfloat16, requires_grad=True)
    made = leaf * 2
    for bad in (leaf, made):
        for call in (lambda: c.append(0, bad, x, n_new=1), lambda: c.append(0, x, bad, n_new=1),
                     lambda: c.append(0, x, x, q=bad, n_new=1), lambda: c.attention(0, bad, n_new=1)):
            with pytest.raises(ValueError, match="no_grad"):
                call()


def test_a_rollout_of_networks_that_train_records_nothing(fakes):  # noqa: F811
    def run(m):
        return speculative.rollout(m, [4, 9, 4], 3, 8, 0.3, 5, dtype=torch.float32)[0]

    want = run(model(3))
    m = model(3)
    for w in m.weights:
        for x in [w["embed"], *w["qkv"], *w["out"], w["logits"]]:
            x.requires_grad_(True)
    got = run(m)
    assert torch.equal(got["tokens"], want["tokens"]) and not any(t.requires_grad for t in got.values())
    assert torch.is_grad_enabled()
