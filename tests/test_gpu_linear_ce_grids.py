"""saki_linear_ce on so many rows and tokens that one launch could not hold a thread for each (2^32 threads)."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_more_tiles_than_a_launch_takes(saki_lib):
    """262,400 rows x 2,097,152 tokens: rows of it alone have the same log-probabilities."""
    n, V, D = 262400, 1 << 21, 8
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    x, w = torch.randn(n, D, generator=g, device=DEV).bfloat16(), torch.randn(V, D, generator=g, device=DEV).bfloat16()
    token = torch.randint(0, V, (n,), generator=g, dtype=torch.int32, device=DEV)
    valid = torch.ones(n, dtype=torch.uint8, device=DEV)
    valid[5:60] = 0
    for mask in (None, valid):
        out = saki_lib.linear_ce(x, w, token, valid_mask=mask, train=False)
        torch.cuda.synchronize()
        assert not out["row_status"].any()
        for a, z in ((0, 300), (n // 2, n // 2 + 300), (n - 300, n)):
            part = saki_lib.linear_ce(x[a:z], w, token[a:z], valid_mask=None if mask is None else mask[a:z], train=False)
            assert torch.equal(out["logp_token"][a:z], part["logp_token"])
        # and by the definition
        at = torch.arange(100, 110, device=DEV)
        logits = x[at].double() @ w.double().t()
        want = logits.gather(1, token[at].long()[:, None])[:, 0] - torch.logsumexp(logits, 1)
        assert float((out["logp_token"][at] - want).abs().max()) < 1e-4
        del out, part


def test_more_tiles_than_a_launch_takes_in_32_bits(saki_lib):
    """790,000 rows x 698,880 tokens: the weight in one piece, its product in two launches."""
    n, V, D = 790000, 698880, 8
    g = torch.Generator(device=DEV)
    g.manual_seed(2)
    x, w = torch.randn(n, D, generator=g, device=DEV), torch.randn(V, D, generator=g, device=DEV)
    token = torch.randint(0, V, (n,), generator=g, dtype=torch.int32, device=DEV)
    out = saki_lib.linear_ce(x, w, token, train=False)
    torch.cuda.synchronize()
    assert not out["row_status"].any()
    for a in (0, n // 2, n - 1000):
        part = saki_lib.linear_ce(x[a:a + 1000], w, token[a:a + 1000], train=False)
        assert torch.equal(out["logp_token"][a:a + 1000], part["logp_token"])
