"""saki_distill_top: the same bits for the same call, and for the same rows in calls of other sizes."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("direction", [0, 1])
@pytest.mark.parametrize("V,k,dtype", [(4096, 200, torch.float32), (4096, 255, torch.bfloat16), (3000, 130, torch.bfloat16),
                                       (3001, 256, torch.float32), (40000, 200, torch.float32), (4096, 40, torch.bfloat16)])
def test_the_same_bits(saki_lib, V, k, dtype, direction):
    """Lists over several waves, more rows than the card has places for, divergences near 0 and of usual size."""
    n = 3000
    g = torch.Generator(device=DEV)
    g.manual_seed(V + k)
    x = saki_lib.alloc_rows(n, V, dtype, DEV)
    x.copy_(2 * torch.randn(n, V, generator=g, device=DEV))
    top = saki_lib.top_logits(x, k)
    noise = torch.logspace(-6, 0, n, device=DEV)[:, None]
    logit = top["top_logit"] + noise * torch.randn(n, k, generator=g, device=DEV)

    def call(a=0, z=n):
        return saki_lib.distill_top(x[a:z], top["top_token"][a:z], logit[a:z], top["rest_logit"][a:z], direction=direction, grad_scale=0.3)

    want = call()
    assert not want["row_status"].any()
    for _ in range(4):
        got = call()
        for name in want:
            assert torch.equal(got[name], want[name]), name
    for step in (700, 129, 1):  # (1: some rows alone)
        for a in range(0, n, step) if step > 1 else range(0, n, 97):
            got = call(a, min(a + step, n))
            for name in ("row_loss", "grad"):
                assert torch.equal(got[name], want[name][a:a + step]), (name, a, step)
