"""saki_distill_top against the float64 oracle."""
import numpy as np
import pytest
import torch

from oracle import distill as oracle
from tests.test_gpu_top_logits import rows

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
FORWARD, REVERSE = 0, 1


def lists(x, k, rng, short=False, tau=1.0):
    """A teacher's lists for rows x [n, V] (float64): top logits of a perturbed copy, some entries left out."""
    n, V = x.shape
    t = 0.7 * x + rng.normal(size=x.shape) * 1.5
    logit, token, rest = oracle.top_logits(t, min(k, V), tau)
    if k > V:
        token = np.concatenate([token, np.full((n, k - V), -1)], 1)
        logit = np.concatenate([logit, np.zeros((n, k - V))], 1)
    if short:
        gone = rng.random(token.shape) < 0.4
        for r in range(n):
            lost = [rest[r] / tau] + list(logit[r][gone[r] & (token[r] >= 0)] / tau)
            rest[r] = tau * oracle._lse(np.array(lost))
        token, logit = np.where(gone, -1, token), np.where(gone, np.nan, logit)
    return token.astype(np.int32), logit.astype(np.float32), rest.astype(np.float32)


def check(x_dev, token, logit, rest, direction=FORWARD, tau=1.0, valid=None, grad_dtype=torch.float32, scale=1.0, status=None):
    import paper_2609_36601_amd as saki

    n, V = x_dev.shape
    d = lambda a, t: None if a is None else torch.as_tensor(a, device=DEV).to(t)  # noqa: E731
    out = saki.distill_top(x_dev, d(token, torch.int32), d(logit, torch.float32), d(rest, torch.float32), tau, direction,
                           d(valid, torch.uint8), scale, grad_dtype)
    torch.cuda.synchronize()
    x = x_dev.float().cpu().numpy().astype(np.float64)
    loss, grad = out["row_loss"].cpu().numpy().astype(np.float64), out["grad"].float().cpu().numpy().astype(np.float64)
    codes = out["row_status"].cpu().numpy()
    # An exponential's argument of size a is off by a 2^-23 and its value by 2^-23 more, sums of 16 by 16 2^-24, and the
    # temperature by 2^-24: logarithms of shares by d = (2 a + 20 + log V) 2^-24, with a <= 30 where weights matter
    # (e^-30 of a sum is below its rounding), logits to double exactly.
    dl = (60 + 20 + np.log(V)) * 2.0**-24
    half = {torch.float32: 2.0**-24, torch.bfloat16: 2.0**-8}[grad_dtype]
    total = 0.0
    for r in range(n):
        if valid is not None and not valid[r]:
            assert loss[r] == 0 and not grad[r].any() and codes[r] == 0
            continue
        want = oracle.distill_row(x[r], token[r], logit[r], None if rest is None else rest[r], tau, direction == REVERSE)
        if want is None:
            assert codes[r] == 4 and np.isnan(loss[r]) and np.all(np.isnan(grad[r]))
            continue
        assert codes[r] == 0
        l, g = want
        p = np.exp(x[r] / tau - oracle._lse(x[r] / tau))
        kept = token[r] >= 0
        # the loss adds shares t, p (each sums to 1) times logarithms that are off by d, and reverse's shares by d
        # themselves, times logarithms; gradients are shares times such sums
        big = 1.0
        if direction == REVERSE and kept.any():
            big = 1 + abs(l) + np.max(np.abs(np.append(g * tau / np.maximum(p, 1e-300), 0))[: V])
        assert abs(loss[r] - l) <= 4 * dl * (1 + abs(l)) * (1 if direction == FORWARD else big) + abs(l) * 2.0**-24
        share = p + 0.0
        if direction == FORWARD:
            share = np.maximum(share, np.abs(share - g * tau))  # p_j and what the teacher's side takes from it
        a = 2 * np.abs(x[r] - x[r].max()) / tau  # a token's own exponential
        tol = scale / tau * share * (4 * dl * big + (a + 4) * 2.0**-24) + half * scale * np.abs(g) + 1e-38
        assert np.all(np.abs(grad[r] - scale * g) <= tol), (r, np.max(np.abs(grad[r] - scale * g) / tol))
        total += scale * l
    if not np.isnan(loss).any():
        assert abs(out["loss_sum"].item() - total) <= np.sum(4 * dl * scale * (1 + np.abs(loss)) * (1 if direction == FORWARD else 100))
    return out


@pytest.mark.parametrize("direction", [FORWARD, REVERSE])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,V,k", [(1, 1, 1), (3, 8, 3), (4, 65, 20), (3, 1000, 256), (5, 1024, 1), (3, 4099, 64),
                                   (2, 50001, 100), (2, 151936, 64), (1, 300001, 33)])
def test_rows(saki_lib, n, V, k, dtype, direction):
    rng = np.random.default_rng(n * V + k)
    x = rows(rng.normal(size=(n, V)) * 3, dtype)
    token, logit, rest = lists(x.float().cpu().numpy().astype(np.float64), k, rng)
    check(x, token, logit, rest, direction, grad_dtype=torch.float32 if k % 2 else torch.bfloat16, scale=0.37)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("k,V", [(1, 500), (17, 3001), (40, 20)])
def test_without_a_rest(saki_lib, dtype, k, V):
    rng = np.random.default_rng(5 + k)
    x = rows(rng.normal(size=(4, V)) * 2, dtype)
    token, logit, _ = lists(x.float().cpu().numpy().astype(np.float64), k, rng)
    check(x, token, logit, None)


@pytest.mark.parametrize("direction", [FORWARD, REVERSE])
@pytest.mark.parametrize("tau", [0.5, 3.3])
@pytest.mark.parametrize("n", [7, 1500])
def test_short_lists_masks_and_temperatures(saki_lib, n, tau, direction):
    rng = np.random.default_rng(n)
    V = 2777
    x = rng.normal(size=(n, V)) * 2
    valid = rng.random(n) < 0.6
    token, logit, rest = lists(x.astype(np.float32).astype(np.float64), 30, rng, short=True, tau=tau)
    x[~valid] = np.nan
    token[~valid] = 10**9  # rows that take no part are not looked at
    x = rows(x, torch.float32)
    check(x, token, logit, rest, direction, tau, valid, torch.bfloat16 if n == 7 else torch.float32, 1.0 / n)


def test_rows_that_list_nothing(saki_lib):
    rng = np.random.default_rng(23)
    x = rows(rng.normal(size=(3, 700)), torch.float32)
    none = np.full((3, 4), -1, dtype=np.int32)
    logit = np.full((3, 4), np.nan, dtype=np.float32)
    out = check(x, none, logit, None)
    assert not out["row_loss"].any() and not out["grad"].any()
    low = np.full(3, -np.inf, dtype=np.float32)
    assert not check(x, none, logit, low)["grad"].any()
    for direction in (FORWARD, REVERSE):  # one bucket on both sides
        assert not check(x, none, logit, np.zeros(3, dtype=np.float32), direction)["row_loss"].any()
    # listed tokens without a share
    out = check(x, np.array([[1, 2, 3, 4]] * 3, dtype=np.int32), np.full((3, 4), -np.inf, dtype=np.float32), None)
    assert not out["grad"].any()
    check(x, np.array([[1, 2, 3, 4]] * 3, dtype=np.int32), np.array([[0.5, -np.inf, 0.25, -np.inf]] * 3, dtype=np.float32), None)


def test_lists_that_cannot_be_used(saki_lib):
    rng = np.random.default_rng(29)
    V = 2000
    x = rows(rng.normal(size=(8, V)), torch.bfloat16)
    token = np.tile(np.array([5, 100, 1999], dtype=np.int32), (8, 1))
    logit = np.zeros((8, 3), dtype=np.float32)
    rest = np.zeros(8, dtype=np.float32)
    token[1, 2], token[2, 0], token[3] = V, -2, [7, 9, 7]
    logit[4, 1], logit[5, 2], rest[6] = np.nan, np.inf, np.nan
    for direction in (FORWARD, REVERSE):
        out = check(x, token, logit, rest, direction)
        assert out["row_status"].cpu().tolist() == [0, 4, 4, 4, 4, 4, 4, 0]
    # infinite divergences
    token = np.tile(np.arange(4, dtype=np.int32), (2, 1))
    small = rows(rng.normal(size=(2, 4)), torch.float32)
    logit = np.zeros((2, 4), dtype=np.float32)
    out = check(small, token, logit, np.array([0.0, -np.inf], dtype=np.float32))
    assert out["row_status"].cpu().tolist() == [4, 0]
    logit[0, 0] = -np.inf
    out = check(small, token, logit, np.array([0.0, 0.0], dtype=np.float32), REVERSE)
    assert out["row_status"].cpu().tolist() == [4, 0]
    out = check(small, token[:, :3], logit[:, 1:], np.array([0.0, -np.inf], dtype=np.float32), REVERSE)
    assert out["row_status"].cpu().tolist() == [0, 4]


@pytest.mark.parametrize("V", [600, 9000])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_rows_that_are_not_finite(saki_lib, V, bad):
    rng = np.random.default_rng(31)
    x = rng.normal(size=(6, V))
    token, logit, rest = lists(x, 8, rng)
    x[0, 3] = bad
    x[2, V - 1] = bad
    x[3, token[3, 2]] = bad
    x[4] = bad
    import paper_2609_36601_amd as saki
    d = lambda a: torch.as_tensor(a, device=DEV)  # noqa: E731
    out = saki.distill_top(rows(x, torch.float32), d(token), d(logit), d(rest))
    torch.cuda.synchronize()
    assert out["row_status"].cpu().tolist() == [1, 0, 1, 1, 1, 0]
    for r in (0, 2, 3, 4):
        assert np.isnan(out["row_loss"][r].item()) and bool(out["grad"][r].isnan().all())
    assert bool(out["grad"][[1, 5]].isfinite().all()) and np.isnan(out["loss_sum"].item())


@pytest.mark.parametrize("direction", [FORWARD, REVERSE])
def test_shares_far_below_one(saki_lib, direction):
    """The student leaves e^-300 to the tokens that are not listed, or to the listed ones."""
    rng = np.random.default_rng(37)
    V = 3000
    x = rng.normal(size=(4, V))
    token = np.tile(np.array([2, 1500, 2999], dtype=np.int32), (4, 1))
    x[:2, token[0]] += 300.0
    x[2:, token[0]] -= 300.0
    logit = rng.normal(size=(4, 3)).astype(np.float32)
    check(rows(x, torch.float32), token, logit, np.zeros(4, dtype=np.float32), direction)


def test_the_gradient_in_the_students_buffer(saki_lib):
    rng = np.random.default_rng(41)
    for dtype, V in ((torch.bfloat16, 5003), (torch.float32, 151936)):
        x = rows(rng.normal(size=(5, V)), dtype)
        token, logit, rest = (torch.as_tensor(a, device=DEV) for a in lists(x.float().cpu().numpy().astype(np.float64), 20, rng))
        want = saki_lib.distill_top(x, token, logit, rest, grad_dtype=dtype)
        ws = torch.empty(saki_lib.workspace_bytes(saki_lib.SAKI_OP_DISTILL_TOP, 5, V), dtype=torch.uint8, device=DEV)
        saki_lib.saki_distill_top(x, token, logit, rest, grad=x, workspace=ws)
        assert torch.equal(x, want["grad"])


def test_a_strided_list_and_outputs_left_alone(saki_lib):
    rng = np.random.default_rng(43)
    x = rows(rng.normal(size=(6, 3000)), torch.bfloat16)
    token, logit, rest = (torch.as_tensor(a, device=DEV) for a in lists(x.float().cpu().numpy().astype(np.float64), 24, rng))
    want = saki_lib.distill_top(x, token[:, :9].contiguous(), logit[:, :9].contiguous(), rest)
    grad = torch.full((6, 3016), 5.0, device=DEV)
    ws = torch.empty(saki_lib.workspace_bytes(saki_lib.SAKI_OP_DISTILL_TOP, 6, 3000), dtype=torch.uint8, device=DEV)
    saki_lib.saki_distill_top(x, token[:, :9], logit[:, :9], rest, grad=grad[:, :3000], workspace=ws)
    assert torch.equal(grad[:, :3000], want["grad"]) and bool((grad[:, 3000:] == 5).all())


def test_the_teachers_own_list(saki_lib):
    """top_logits of a teacher, then distill_top of a student: the way the two are used; the student's own list has
    divergence 0."""
    rng = np.random.default_rng(47)
    t = rows(rng.normal(size=(40, 20000)) * 3, torch.bfloat16)
    s = rows(rng.normal(size=(40, 20000)) * 3, torch.bfloat16)
    top = saki_lib.top_logits(t, 64)
    args = (top["top_token"], top["top_logit"], top["rest_logit"])
    check(s, *(a.cpu().numpy() for a in args))
    for direction in (FORWARD, REVERSE):
        out = saki_lib.distill_top(t, *args, direction=direction)
        assert float(out["row_loss"].abs().max()) < 1e-5 and float(out["grad"].abs().max()) < 1e-5
