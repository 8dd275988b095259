"""Which of the two kinds a model of the rollout driver is, on the CPU."""
import numpy as np
import pytest
import torch

from paper_2609_36601_amd import speculative
from paper_2609_36601_amd.workloads import SyntheticARTorch
from tests.test_rollout_cached_host import model as cached_model
from tests.test_rollout_driver_host import fakes  # noqa: F401


@pytest.mark.parametrize("caches", [None, {"logits": 3}, [torch.zeros(2), torch.zeros(2)], torch.zeros(3), "hits", 7])
def test_a_models_own_caches_do_not_change_its_rollout(fakes, caches):  # noqa: F811
    args = (np.arange(5), 3, 7, 0.2, 5)
    want, waves = speculative.rollout(SyntheticARTorch(12, seed=3, device="cpu"), *args, dtype=torch.float32)
    m = SyntheticARTorch(12, seed=3, device="cpu")
    m.caches = caches
    got, n = speculative.rollout(m, *args, dtype=torch.float32)
    assert n == waves and all(torch.equal(got[f], want[f]) for f in ("tokens", "length", "done", "corrected"))


def test_a_model_with_the_calls_and_no_caches_is_of_the_first_kind(fakes):  # noqa: F811
    args = (np.arange(5), 3, 7, 0.2, 5)
    want, _ = speculative.rollout(SyntheticARTorch(12, seed=3, device="cpu"), *args, dtype=torch.float32)
    for caches in (None, (), []):
        m = SyntheticARTorch(12, seed=3, device="cpu")
        m.start = m.draft_into = m.verify_into = lambda *a: pytest.fail("not this kind")
        m.caches = caches
        got, _ = speculative.rollout(m, *args, dtype=torch.float32)
        assert torch.equal(got["tokens"], want["tokens"])


@pytest.mark.parametrize("k", [1, 4])
def test_rows_of_a_table_that_hold_just_enough(fakes, k):  # noqa: F811
    """prompt + max_len + k - 2 tokens a sequence are enough; with k = 1, whose waves commit one token each, one less is not."""
    m = cached_model(2)
    prompt, page, pages = max(len(m.prompt(p)) for p in (4, 9)), 8, 3
    for lack in (0, 1):
        m = cached_model(2)
        L = pages * page - prompt - k + 2 + lack
        for c in m.caches:
            c.t.pages = c.t.pages[:, :pages].copy()
        if not lack:
            tr, _ = speculative.rollout(m, [4, 9], k, L, 0.3, 1, dtype=torch.float32)
            assert (tr["length"] == L).all()
        elif k == 1:
            with pytest.raises(RuntimeError, match="too few pages"):
                speculative.rollout(m, [4, 9], k, L, 0.3, 1, dtype=torch.float32)
