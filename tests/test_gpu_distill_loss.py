"""saki_distill_top without a gradient: the losses, their sum and the status of the call with one, and the oracle's."""
import numpy as np
import pytest
import torch

from oracle import distill as oracle

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("direction", [0, 1])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,V,k", [(1, 1, 1), (5, 700, 256), (7, 4099, 30), (3, 60001, 64), (3, 151936, 200), (2600, 1025, 17)])
def test_losses_alone(saki_lib, n, V, k, dtype, direction):
    rng = np.random.default_rng(n + V + k)
    x = saki_lib.alloc_rows(n, V, dtype, DEV)
    x.copy_(torch.as_tensor(rng.normal(size=(n, V)) * 3))
    teacher = torch.as_tensor(rng.normal(size=(n, V)) * 3, device=DEV).float()
    list_of = saki_lib.alloc_rows(n, V, torch.float32, DEV)
    list_of.copy_(teacher)
    top = saki_lib.top_logits(list_of, k)
    token, logit, rest = top["top_token"], top["top_logit"], top["rest_logit"]
    valid = torch.as_tensor(rng.random(n) < 0.8, device=DEV).to(torch.uint8)
    if n > 2:
        x[0, V // 2], token[1, 0] = float("nan"), V  # (a row that is not finite, a list that cannot be used)
        valid[:3] = 1
    tau, scale = 1.7, 0.3
    args = (x, token, logit, rest, tau, direction, valid, scale)
    alone = saki_lib.distill_top(*args, grad_dtype=None)
    again = saki_lib.distill_top(*args, grad_dtype=None)
    both = saki_lib.distill_top(*args)
    torch.cuda.synchronize()
    assert alone["grad"] is None and torch.equal(alone["row_status"], both["row_status"])
    codes, loss, other = (t.cpu().numpy() for t in (alone["row_status"], alone["row_loss"], both["row_loss"]))
    if n > 2:
        assert codes[:3].tolist() == [1, 4, 0] and np.isnan(loss[:2]).all() and np.isnan(alone["loss_sum"].item())
    for name in ("row_loss", "loss_sum"):
        assert torch.equal(alone[name].view(torch.int32), again[name].view(torch.int32))
    # Shares' logarithms are off by d = (2 a + 20 + log V) 2^-24, a <= 30; the loss by 4 d (1 + |l|), reverse's by d times the
    # shares' logarithms, some 100, and its rounding.
    d = (80 + np.log(V)) * 2.0**-24
    xs, total, slack = x.float().cpu().numpy().astype(np.float64), 0.0, 0.0
    for r in range(n):
        if not valid[r]:
            assert loss[r] == 0 and codes[r] == 0
        elif codes[r] == 0:
            want = oracle.distill_row(xs[r], token[r].cpu().numpy(), logit[r].cpu().numpy(), rest[r].item(), tau, direction == 1)[0]
            tol = 4 * d * (1 + abs(want)) * (100 if direction else 1) + abs(want) * 2.0**-24
            assert abs(loss[r] - want) <= tol and abs(other[r] - loss[r]) <= 2 * tol
            total, slack = total + scale * want, slack + scale * tol
    if not np.isnan(loss).any():
        assert abs(alone["loss_sum"].item() - total) <= slack
