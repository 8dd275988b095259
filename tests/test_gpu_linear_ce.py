"""saki_linear_ce against the float64 oracle."""
import numpy as np
import pytest
import torch

from oracle import distill as oracle

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HALF = {torch.float32: 2.0**-24, torch.bfloat16: 2.0**-8}


def matrix(x, dtype, pad=0):
    """x on the device, `pad` elements of NaN behind each row."""
    t = torch.full((x.shape[0], x.shape[1] + pad), float("nan"), dtype=dtype, device=DEV)
    t[:, :x.shape[1]] = torch.as_tensor(x, device=DEV).to(dtype)
    return t[:, :x.shape[1]]


def f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def bounds(x, w, token, weight, take, scale, dtype):
    """What rounding allows, from the magnitudes of the terms.  A logit is a sum of D products in 32 bits, 32 of which a
    matrix instruction adds in one rounding each for the first of 4 k groups: (D / 8 + 8) 2^-24 sum |x w| (f32: six products
    of parts and the parts dropped, twice that).  The log-sum-exp is off by the largest logit error and (2 a + 20) 2^-24 of
    its own, a <= 30.  A gradient of a logit is w_r (p - 1[..]), with p off relatively by twice that, then rounded to the
    inputs' type; the gradients' sums over v (r) are in 32 bits, K / 8 + 8 roundings, and are rounded once."""
    D, V, n = x.shape[1], len(w), len(x)
    f = 2 if dtype == torch.float32 else 1
    el = f * (D / 8 + 8) * 2.0**-24 * (np.abs(x) @ np.abs(w).T)
    dl = el.max(1) + 80 * 2.0**-24
    logits = x @ w.T
    p = np.exp(logits - np.array([oracle._lse(l) for l in logits])[:, None])
    d = p.copy()
    hot = np.zeros_like(p)
    hot[np.arange(n)[take], token[take]] = 1
    d = np.abs(p - hot) * np.abs(weight)[:, None] * take[:, None]
    ed = (p * 2 * dl[:, None] + hot * 2.0**-24) * np.abs(weight)[:, None] * take[:, None] + d * HALF[dtype]
    dx = scale * (ed @ np.abs(w) + f * (V / 8 + 8 + V // 256) * 2.0**-24 * (d @ np.abs(w)))
    dw = scale * (ed.T @ np.abs(x) + f * (n / 8 + 8) * 2.0**-24 * (d.T @ np.abs(x)))
    return dl, dx, dw


def check(x, w, token, dtype, weight=None, valid=None, scale=1.0, pads=(0, 0), **kw):
    import paper_2609_36601_amd as saki

    xd, wd = matrix(x, dtype, pads[0]), matrix(w, dtype, pads[1])
    x, w = f64(xd), f64(wd)
    n = len(x)
    dev = lambda a, t: None if a is None else torch.as_tensor(a, device=DEV).to(t)  # noqa: E731
    out = saki.linear_ce(xd, wd, dev(token, torch.int32), dev(weight, torch.float32), dev(valid, torch.uint8), scale, **kw)
    torch.cuda.synchronize()
    wt = np.ones(n) if weight is None else np.asarray(weight, dtype=np.float32).astype(np.float64)
    ok = np.ones(n, dtype=bool) if valid is None else np.asarray(valid) != 0
    bad = ok & ((token < 0) | (token >= len(w)) | ~np.isfinite(wt))
    take = ok & ~bad
    x = np.where(take[:, None], x, 0.0)
    loss, logp, dx, dw = oracle.linear_ce(x, w, token, wt, ok, scale)
    wt = np.where(take, wt, 0.0)  # (rows without a loss have no error)
    codes = np.where(bad, 4, 0)
    np.testing.assert_array_equal(out["row_status"].cpu().numpy(), codes)
    el, ex, ew = bounds(x, w, np.where(take, token, 0), wt, take, abs(scale), dtype)
    got = f64(out["logp_token"])
    np.testing.assert_array_equal(np.isnan(got), bad)
    assert np.all(np.abs(got - logp)[~bad] <= (2 * el + np.abs(logp) * 2.0**-24)[~bad])
    got = f64(out["row_loss"])
    assert np.all(np.abs(got - loss)[~bad] <= (2 * el * np.abs(wt) + np.abs(loss) * 2.0**-23)[~bad]) and np.all(np.isnan(got[bad]))
    if not bad.any():
        assert abs(out["loss_sum"].item() - scale * loss.sum()) <= abs(scale) * np.sum(2 * el * np.abs(wt) + np.abs(loss) * 2.0**-23)
    if out["grad_hidden"] is not None:
        got = f64(out["grad_hidden"])
        assert np.all(np.isnan(got[bad]))
        tol = ex + HALF[dtype] * np.abs(dx) + 1e-38
        assert np.all(np.abs(got - dx)[~bad] <= tol[~bad]), np.max((np.abs(got - dx) / tol)[~bad])
        got = f64(out["grad_weight"])
        tol = ew + HALF[dtype] * np.abs(dw) + 1e-38
        assert np.all(np.abs(got - dw) <= tol), np.max(np.abs(got - dw) / tol)
    return out


def problem(n, V, D, rng, spread=2.0):
    return rng.normal(size=(n, D)), rng.normal(size=(V, D)) * spread / np.sqrt(D), rng.integers(0, V, n)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,V,D", [(1, 1, 8), (1, 300, 64), (3, 7, 8), (17, 65, 72), (64, 1000, 128), (65, 1001, 136),
                                   (100, 257, 64), (130, 5000, 200), (257, 511, 520), (513, 999, 256), (5, 40001, 64),
                                   (1000, 130, 24)])
def test_sizes(saki_lib, n, V, D, dtype):
    rng = np.random.default_rng(n + V + D)
    check(*problem(n, V, D, rng), dtype, scale=0.37)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,V,D", [(128, 700, 264), (129, 700, 8), (768, 300, 328), (769, 300, 328), (769, 300, 16), (3, 2, 1024)])
def test_the_forms_of_a_call(saki_lib, n, V, D, dtype):
    """Both sides of: f32 weights as they are or in parts, logits kept or computed again, the rows of grad_weight's sums in splits."""
    rng = np.random.default_rng(n + D)
    check(*problem(n, V, D, rng), dtype, valid=rng.random(n) < 0.7)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_the_large_tiles(saki_lib, dtype):
    """Sizes of which the products fill the card with their largest tiles, none of them whole."""
    rng = np.random.default_rng(3)
    check(*problem(4400, 4001, 72, rng), dtype, scale=0.5)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_the_large_tiles_of_the_gradients(saki_lib, dtype):
    rng = np.random.default_rng(4)
    x, w, token = problem(2100, 4500, 4104, rng)
    check(x, w, token, dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,V,D", [(40, 300, 64), (300, 2000, 136), (2000, 300, 64)])
@pytest.mark.parametrize("share", [0.0, 0.05, 0.6, 1.0])
def test_masks_and_weights(saki_lib, n, V, D, dtype, share):
    """Rows that take no part hold NaN and tokens of no meaning."""
    rng = np.random.default_rng(n)
    x, w, token = problem(n, V, D, rng)
    valid = rng.random(n) < share
    if share == 0.05:
        valid[-1] = True
    weight = rng.normal(size=n)
    weight[::7] = 0.0
    x[~valid], token[~valid], weight[~valid] = np.nan, 10**9, np.nan
    out = check(x, w, token, dtype, weight, valid, scale=1.0 / n)
    if share == 0.0:
        assert not out["grad_weight"].any() and not out["grad_hidden"].any()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("masked", [False, True])
def test_strides(saki_lib, dtype, masked):
    """Rows with NaN behind them, whole tiles of k and not."""
    rng = np.random.default_rng(8)
    for D in (64, 104):
        x, w, token = problem(70, 333, D, rng)
        check(x, w, token, dtype, valid=rng.random(70) < 0.7 if masked else None, pads=(8, 24))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_that_cannot_be_used(saki_lib, dtype):
    rng = np.random.default_rng(9)
    x, w, token = problem(90, 500, 64, rng)
    weight = np.ones(90)
    token[3], token[40], token[89] = -1, 500, 2**31 - 1
    weight[17], weight[18] = np.nan, np.inf
    check(x, w, token, dtype, weight)
    check(x, w, token, dtype, weight, valid=rng.random(90) < 0.5)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_a_row_that_is_not_finite(saki_lib, dtype):
    rng = np.random.default_rng(10)
    for bad in (np.nan, np.inf):
        x, w, token = problem(70, 300, 64, rng)
        x[5, 3] = bad
        out = saki_lib.linear_ce(matrix(x, dtype), matrix(w, dtype), torch.as_tensor(token, device=DEV).int())
        torch.cuda.synchronize()
        status = out["row_status"].cpu().numpy()
        assert status[5] == 1 and status.sum() == 1
        assert np.isnan(out["row_loss"][5].item()) and bool(out["grad_hidden"][5].isnan().all())
        keep = np.arange(70) != 5
        assert bool(out["grad_hidden"][torch.as_tensor(keep, device=DEV)].isfinite().all())
        assert bool(out["grad_weight"].isnan().any()) and np.isnan(out["loss_sum"].item())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,D", [(8, 512), (70, 64), (800, 24)])
def test_rows_of_no_use_among_others(saki_lib, n, D, dtype):
    """Logits kept and computed again: a row without a token adds nothing though its logits are infinite; a row that is not
    finite leaves the other rows' outputs alone."""
    rng = np.random.default_rng(13)
    x, w, token = problem(n, 300, D, rng)
    x[3] = 3e38 * np.sign(w[7])
    token[3] = -1
    xd, wd, td = matrix(x, dtype), matrix(w, dtype), torch.as_tensor(token, device=DEV).int()
    out = saki_lib.linear_ce(xd, wd, td)
    x[3] = 0
    plain = saki_lib.linear_ce(matrix(x, dtype), wd, td)
    xd[5, 3] = float("nan")
    td[3] = 2
    none = saki_lib.linear_ce(xd, wd, td)
    torch.cuda.synchronize()
    assert out["row_status"].tolist() == [4 if r == 3 else 0 for r in range(n)]
    assert bool(out["grad_weight"].isfinite().all()) and torch.equal(out["grad_weight"], plain["grad_weight"])
    assert bool(out["grad_hidden"][3].isnan().all())
    others = [r for r in range(n) if r not in (3, 5)]
    assert torch.equal(out["grad_hidden"][others], plain["grad_hidden"][others])
    assert none["row_status"].tolist() == [1 if r in (3, 5) else 0 for r in range(n)]
    assert torch.equal(none["grad_hidden"][others], out["grad_hidden"][others]) and torch.equal(none["row_loss"][others], out["row_loss"][others])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_logits_of_all_sizes(saki_lib, dtype):
    """Rows that are certain (log p near 0), rows whose logits are near 1e30, rows of logits that are all alike."""
    rng = np.random.default_rng(11)
    x, w, token = problem(64, 400, 64, rng)
    x[:16] = 40 * w[token[:16]]
    x[32:] = 0.0
    out = check(x, w, token, dtype)
    assert bool((out["logp_token"][32:] + np.log(400)).abs().max() < 1e-6)
    x = np.zeros((4, 64))
    w = np.zeros((400, 64))
    x[:, 0], w[:, 0] = 1e15, np.arange(400) * -1e15
    out = saki_lib.linear_ce(matrix(x, dtype), matrix(w, dtype), torch.tensor([0, 0, 1, 399], dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()
    logp = out["logp_token"].cpu().numpy()
    assert not out["row_status"].any() and logp[0] == 0 and logp[1] == 0 and abs(logp[2] + 1e30) < 1e28 and logp[3] < -3e32


def test_one_gradient_or_none(saki_lib):
    rng = np.random.default_rng(12)
    x, w, token = problem(200, 3000, 128, rng)
    for dtype in (torch.bfloat16, torch.float32):
        xd, wd, t = matrix(x, dtype), matrix(w, dtype), torch.as_tensor(token, device=DEV).int()
        want = saki_lib.linear_ce(xd, wd, t)
        alone = saki_lib.linear_ce(xd, wd, t, train=False)
        assert alone["grad_hidden"] is None
        assert torch.allclose(alone["row_loss"], want["row_loss"], rtol=0, atol=1e-4)
        for name, like in (("grad_hidden", xd), ("grad_weight", wd)):
            out = torch.full((like.shape[0], like.shape[1] + 8), 3.0, dtype=dtype, device=DEV)
            kinds = {"grad_hidden": False, "grad_weight": False, name: True}
            ws = torch.empty(saki_lib.linear_ce_workspace_bytes(xd, wd, **kinds), dtype=torch.uint8, device=DEV)
            saki_lib.saki_linear_ce(xd, wd, t, workspace=ws, **{name: out[:, :like.shape[1]]})
            assert torch.equal(out[:, :like.shape[1]], want[name]) and bool((out[:, like.shape[1]:] == 3).all())


def test_no_rows(saki_lib):
    w = torch.ones(50, 16, dtype=torch.bfloat16, device=DEV)
    out = saki_lib.linear_ce(torch.empty(0, 16, dtype=torch.bfloat16, device=DEV), w, torch.empty(0, dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()
    assert not out["grad_weight"].any() and out["loss_sum"].item() == 0


def test_the_routed_objective(saki_lib):
    """With row weights from the events of a coupling, the gradients are those of the routed loss on the logits."""
    rng = np.random.default_rng(14)
    n, V, D = 96, 1000, 64
    x, w, token = problem(n, V, D, rng)
    xd, wd = matrix(x, torch.float32), matrix(w, torch.float32)
    logits = f64(xd) @ f64(wd).T
    s = saki_lib.alloc_rows(n, V, torch.float32, DEV)
    s.copy_(torch.as_tensor(logits, device=DEV))
    corrected = torch.as_tensor(rng.random(n) < 0.3, device=DEV).to(torch.uint8)
    mode = torch.as_tensor(rng.integers(0, V, n), device=DEV).int()
    tok = torch.as_tensor(token, device=DEV).int()
    adv = torch.as_tensor(rng.normal(size=n), device=DEV).float()
    valid = torch.as_tensor(rng.random(n) < 0.8, device=DEV).to(torch.uint8)
    want = saki_lib.route_loss(s, tok, corrected, mode, adv, valid, 1.0 / n)
    target, part = torch.where(corrected != 0, mode, tok), torch.where(corrected != 0, 1.0, adv)
    got = saki_lib.linear_ce(xd, wd, target, part, valid, 1.0 / n)
    torch.cuda.synchronize()
    g = f64(want["grad"])
    # the logits given to route_loss are rounded to 32 bits (2^-24 of up to 10), and both sides' logarithms are off by some 100 2^-24
    np.testing.assert_allclose(f64(got["row_loss"]), f64(want["row_loss"]), atol=3e-5 * float(part.abs().max()))
    np.testing.assert_allclose(f64(got["grad_hidden"]), g @ f64(wd), atol=3e-5 * np.abs(g).sum(1).max() * np.abs(f64(wd)).max())
    np.testing.assert_allclose(f64(got["grad_weight"]), g.T @ f64(xd), atol=3e-5 * np.abs(g).sum(0).max() * np.abs(f64(xd)).max())
