"""saki_linear_ce on rows that are certain of their token: loss and gradient are of the size of what the other tokens
have left, and as exact as that, not as 1.

The head: the token's weight is the first unit vector, every other's one of the others.  So logits are elements of the hidden state,
exactly, and grad_hidden's elements are a gradient of the token's logit by itself and sums of the others'.
"""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HALF = {torch.float32: 2.0**-24, torch.bfloat16: 2.0**-8}


def problem(n, V, D, least, dtype, rng):
    """Hidden states (as dtype, in 64 bits), the token, each other token's element; 1 - p from 1e-3 down to `least`."""
    token = int(rng.integers(V))
    at = 1 + np.arange(V) % (D - 1)
    at[token] = 0
    x = rng.normal(size=(n, D)) + rng.uniform(-15, 15, (n, 1))
    others = np.log(np.sum(np.exp(x[:, at[at > 0]]), 1))
    x[:, 0] = others - np.log(np.logspace(-3, np.log10(least), n))
    return torch.as_tensor(x).to(dtype).double().numpy(), token, at


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,V,D", [(9, 1000, 64), (70, 1000, 64), (40, 32000, 24), (300, 32000, 64), (300, 5000, 1024), (800, 1000, 64),
                                   (2100, 9000, 72)])
@pytest.mark.parametrize("least", [1e-8, 1e-20])
def test_certain_rows(saki_lib, n, V, D, least, dtype):
    rng = np.random.default_rng(n + V)
    x, token, at = problem(n, V, D, least, dtype, rng)
    w = torch.zeros(V, D, dtype=dtype, device=DEV)
    w[torch.arange(V), torch.as_tensor(at)] = 1.0
    weight = rng.normal(size=n).astype(np.float32)
    out = saki_lib.linear_ce(torch.as_tensor(x, device=DEV).to(dtype), w, torch.full((n,), token, dtype=torch.int32, device=DEV),
                             torch.as_tensor(weight, device=DEV))
    torch.cuda.synchronize()
    assert not out["row_status"].any()
    share = np.exp(x[:, at] - x[:, :1])  # relative to the token's
    share[:, token] = 0.0
    u = share.sum(1)
    rest, loss = u / (1 + u), np.log1p(u)
    # A logit in units of log2 is rounded (a 2^-24 of a size a), its difference from a maximum and the maxima's from each other
    # are (2 a 2^-24 each, and log2 e itself is off by 2^-25 of the difference): 7 a 2^-24 ln 2 of a share.  Two exponentials are
    # off by 2^-23, a wave's sum is of 128 numbers, 32 of them one behind the other and two exchanges: 34 2^-24.
    a = np.abs(x).max(1) * 1.4427
    rel = (7 * a * 0.6932 + 4 + 34) * 2.0**-24
    got = out["logp_token"].double().cpu().numpy()
    assert np.all(np.abs(got + loss) <= loss * (rel + 2.0**-24)), np.max(np.abs(got + loss) / loss)
    got = out["row_loss"].double().cpu().numpy()
    assert np.all(np.abs(got - weight * loss) <= np.abs(weight) * loss * (rel + 2.0**-23))
    # the token's own gradient: the weight's product with it and the inputs' type round once each (f32: 24 bits in parts),
    # the result too
    dx = out["grad_hidden"].double().cpu().numpy()
    want = -weight * rest
    tol = np.abs(want) * (rel + 2.0**-23 + 2 * HALF[dtype]) + 1e-37
    assert np.all(np.abs(dx[:, 0] - want) <= tol), np.max(np.abs(dx[:, 0] - want) / np.abs(want))
    # the others', of one sign, in sums over V
    shares = np.zeros((n, D))
    np.add.at(shares.T, at, share.T)
    want = weight[:, None] * (shares / (1 + u[:, None]))
    want[:, 0] = 0.0
    tol = np.abs(want) * (rel[:, None] + 2.0**-23 + 2 * HALF[dtype] + 2 * (V / 8 + 8 + V // 256) * 2.0**-24) + 1e-37
    assert np.all(np.abs(dx - want)[:, 1:] <= tol[:, 1:])
    # and the token's row of grad_weight: a sum over the rows
    dw = out["grad_weight"][token].double().cpu().numpy()
    each = np.abs(weight * rest)[:, None] * np.abs(x)
    tol = np.sum(each * (rel[:, None] + 2.0**-23 + HALF[dtype] + 2 * (n / 8 + 8) * 2.0**-24), 0)
    want = np.sum((-weight * rest)[:, None] * x, 0)
    assert np.all(np.abs(dw - want) <= tol + HALF[dtype] * np.abs(want) + 1e-37)
