"""saki_linear_ce on vocabularies of several pieces (the gradient of a piece's logits takes at most 256 MiB), against the
definition in 64 bits."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HALF = {torch.float32: 2.0**-24, torch.bfloat16: 2.0**-8}


def definition(x, w, token, weight, take, scale, dtype):
    """Loss, log-probability and both gradients in 64 bits, and what rounding allows of each: a logit is a sum of D products,
    (D / 8 + 8) 2^-24 of their sizes (f32: twice that, for the parts); the log-sum-exp is off by the largest such error and 80 2^-24; a
    gradient of a logit by twice both, and half a step of the inputs' type; its sums over V (over the rows) by (V / 8 + 8) 2^-24
    and one more for each addition of a piece or a split."""
    n, D = x.shape
    V = w.shape[0]
    f = 2 if dtype == torch.float32 else 1
    at = torch.arange(n, device=DEV)
    logits = x @ w.t()
    lse = torch.logsumexp(logits, 1)
    logp = logits[at, token] - lse
    p = logits.sub_(lse[:, None]).exp_()
    part = torch.where(take, weight, 0.0)
    el = f * (D / 8 + 8) * 2.0**-24 * (x.abs() @ w.abs().t()).amax(1) + 80 * 2.0**-24
    error = p * (2 * el * part.abs())[:, None]
    error[at, token] += 2.0**-24 * part.abs()
    p[at, token] -= 1.0
    p *= part[:, None]
    size = p.abs()
    error += HALF[dtype] * size
    dx, dw = scale * (p @ w), scale * (p.t() @ x)
    ex = scale * (error @ w.abs() + f * (V / 8 + 8 + V // 256) * 2.0**-24 * (size @ w.abs())) + HALF[dtype] * dx.abs() + 1e-38
    ew = scale * (error.t() @ x.abs() + f * (n / 8 + 8) * 2.0**-24 * (size.t() @ x.abs())) + HALF[dtype] * dw.abs() + 1e-38
    return logp, 2 * el + logp.abs() * 2.0**-24, dx, ex, dw, ew


def within(got, want, tol):
    return bool(((got.double() - want).abs() <= tol).all())


# dtype, rows, tokens, elements: pieces; logits kept for the gradient, or computed again
CASES = [(torch.bfloat16, 2900, 49999, 72), (torch.bfloat16, 2900, 49999, 1032),      # 2, again; 2, kept
         (torch.bfloat16, 2900, 150001, 24),                                        # 4, again
         (torch.bfloat16, 20, 600001, 24), (torch.bfloat16, 20, 600001, 80),        # 2 for few rows, again; kept
         (torch.float32, 800, 50001, 40), (torch.float32, 800, 50001, 264),         # 2, the weight in parts, again; kept
         (torch.float32, 700, 60001, 40), (torch.float32, 700, 60001, 264),         # 2, the weight as it is, again; kept
         (torch.float32, 1500, 90001, 136)]                                         # 4, the weight in parts, kept


@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("dtype,n,V,D", CASES)
def test_pieces(saki_lib, dtype, n, V, D, masked):
    g = torch.Generator(device=DEV)
    g.manual_seed(n + V + D)
    rand = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    x, w = rand(n, D).to(dtype), (rand(V, D) * (2.0 / D**0.5)).to(dtype)
    token = torch.randint(0, V, (n,), generator=g, dtype=torch.int32, device=DEV)
    token[:3] = torch.tensor([0, V // 2, V - 1], dtype=torch.int32)
    weight, scale = rand(n), 0.37
    valid = (torch.rand(n, generator=g, device=DEV) < 0.6).to(torch.uint8) if masked else None
    if masked:
        x[valid == 0], token[valid == 0] = float("nan"), -7
    out = saki_lib.linear_ce(x, w, token, weight, valid, scale)
    torch.cuda.synchronize()
    assert not out["row_status"].any()
    take = torch.ones(n, dtype=torch.bool, device=DEV) if valid is None else valid != 0
    logp, tol, dx, ex, dw, ew = definition(torch.where(take[:, None], x.double(), 0.0), w.double(), token.clamp(min=0).long(),
                                           weight.double(), take, scale, dtype)
    logp = torch.where(take, logp, 0.0)
    assert within(out["logp_token"], logp, tol)
    assert within(out["row_loss"], -weight.double() * logp, weight.abs() * tol + (weight * logp).abs() * 2.0**-24)
    assert within(out["grad_hidden"], dx, ex) and not out["grad_hidden"][~take].any()
    assert within(out["grad_weight"], dw, ew)
    # one gradient alone
    for name, like in (("grad_hidden", x), ("grad_weight", w)):
        one = torch.empty_like(like)
        kinds = {"grad_hidden": False, "grad_weight": False, name: True}
        ws = torch.empty(saki_lib.linear_ce_workspace_bytes(x, w, **kinds), dtype=torch.uint8, device=DEV)
        saki_lib.saki_linear_ce(x, w, token, weight, valid, scale, workspace=ws, **{name: one})
        assert torch.equal(one, out[name]), name
