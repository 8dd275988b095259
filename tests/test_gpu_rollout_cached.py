"""Speculative rollouts of a pair of networks with paged key-value caches: reserve, append, attention, fork and
commit as a rollout calls them, with sampling, verification and commit between.

Every committed token's log p and log pi are checked against the networks evaluated in 64 bits on the whole
committed sequence, without a cache: a wrong page, position, rollback or shared prompt changes them.
Bound (32 bits): a hidden row passes about ten sums of at most 128 products (128 2^-24 relative to their
sizes, each), logits are at most 32 in size: 10 * 2^-17 * 32 = 2.4e-3, twice that for log p with its
normaliser."""
import numpy as np
import pytest
import torch

from paper_2609_36601_amd import binding
from paper_2609_36601_amd.workloads import SyntheticAttentionPair
from tests.test_rollout_cached_host import dense_logits

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def logp(row, token):
    return row[token] - (row.max() + np.log(np.exp(row - row.max()).sum()))


def check(m, prompts, tr, tol):
    worst, n = 0.0, 0
    for b, p in enumerate(prompts):
        L = int(tr["length"][b])
        text = list(m.prompt(p)) + tr["tokens"][b, :L].tolist()
        for net, key in ((0, "logp_token"), (1, "logt_token")):
            rows = dense_logits(m, net, text)[len(text) - L - 1:-1]
            assert np.abs(rows).max() < 32
            want = np.array([logp(rows[i], text[len(text) - L + i]) for i in range(L)])
            got = tr[key][b, :L].double().cpu().numpy()
            worst = max(worst, float(np.abs(got - want).max()))
            n += L
    print(f"{n} log-probabilities, worst difference {worst:.2g}", flush=True)
    assert worst <= tol
    return n


@pytest.mark.parametrize("k,page,windows,sinks", [(4, 8, (0, 0), 0), (8, 16, (24, 0), 2), (1, 8, (0, 16), 0)])
def test_rollout_with_caches(saki_lib, k, page, windows, sinks):
    prompts = [3, 3, 3, 8, 5, 8, 8, 3]
    L, eps = 40, 0.2
    m = SyntheticAttentionPair(500, len(prompts), 16, 90, page_size=page, windows=windows, sinks=sinks, seed=1, device=DEV)
    timing = {}
    tr, waves = saki_lib.rollout(m, prompts, k, L, eps, 77, dtype=torch.float32, timing=timing)
    assert (tr["length"] == L).all() and (tr["done"] == binding.SEQ_FINISHED).all()
    assert len(timing["cache"]) == 4 * waves
    if k > 1:
        assert waves < 40 and bool(tr["corrected"].any()) and not bool(tr["corrected"].all())
    assert check(m, prompts, tr, 5e-3) == 2 * 8 * L
    for c in m.caches:
        assert int(c.refs.abs().sum()) == 0 and int(c.held.sum()) == 0 and (c.pages == -1).all()


def test_rollout_with_bf16_caches_ends_and_returns_its_pages(saki_lib):
    """bf16 networks and logits, an end token: sequences end at different waves."""
    prompts = list(range(12)) * 2
    m = SyntheticAttentionPair(50, 24, 40, 400, page_size=8, dtype=torch.bfloat16, seed=2, device=DEV)
    tr, _ = saki_lib.rollout(m, prompts, 5, 120, 0.2, 5, eos_id=7, dtype=torch.bfloat16, check_every=4)
    assert (tr["done"] == binding.SEQ_FINISHED).all() and len(set(tr["length"].tolist())) > 3
    ends = tr["tokens"].gather(1, (tr["length"].long() - 1)[:, None])[:, 0]
    assert ((ends == 7) | (tr["length"] == 120)).all()
    assert all(int(c.refs.abs().sum()) == 0 for c in m.caches)


def test_a_cache_too_small_is_reported(saki_lib):
    m = SyntheticAttentionPair(50, 6, 40, 30, page_size=8, seed=2, device=DEV)
    with pytest.raises(RuntimeError, match="too few pages"):
        saki_lib.rollout(m, range(6), 4, 200, 0.2, 5, dtype=torch.float32)
