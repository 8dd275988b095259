"""saki_top_logits against the float64 oracle: values and tokens exactly, the others' log-sum-exp to what 32-bit
exponentials allow."""
import numpy as np
import pytest
import torch

from oracle import distill as oracle

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def rows(x, dtype):
    """x as rows of this type with a pitch of whole 16 bytes; what lies behind a row is NaN."""
    per = 16 // torch.tensor([], dtype=dtype).element_size()
    t = torch.full((x.shape[0], (x.shape[1] + per - 1) // per * per + per), float("nan"), dtype=dtype, device=DEV)
    t[:, :x.shape[1]] = torch.as_tensor(x, device=DEV).to(dtype)
    return t[:, :x.shape[1]]


def rest_tolerance(x, tok, tau, want):
    """An exponential's argument (x - L) c, of size a, is off by a 2^-23 (two roundings) and its value by 2^-23 more; 16 are
    added in 32 bits (16 2^-24); c is off by 2^-24, which moves tau log sum by at most tau log V 2^-24; the
    result is rounded.  In natural units, with a the mean of |x - L| / tau under the weights."""
    V = x.shape[1]
    a = np.zeros(len(x))
    for r in range(len(x)):
        m = np.ones(V, dtype=bool)
        m[tok[r]] = False
        if m.any():
            d = (x[r][m] - x[r][tok[r][-1]]) / tau
            w = np.exp(d - d.max())
            a[r] = np.sum(w * np.abs(d)) / w.sum()
    return tau * (2 * a + 2 + 16 + np.log(V)) * 2.0**-24 + np.abs(np.where(np.isfinite(want), want, 0)) * 2.0**-24


def check(x_dev, k, tau=1.0, **kw):
    import paper_2609_36601_amd as saki

    out = saki.top_logits(x_dev, k, temperature=tau, **kw)
    torch.cuda.synchronize()
    x = x_dev.float().cpu().numpy().astype(np.float64)
    logit, tok, rest = oracle.top_logits(x, k, tau)
    np.testing.assert_array_equal(out["top_token"].cpu().numpy(), tok)
    np.testing.assert_array_equal(out["top_logit"].cpu().numpy(), logit.astype(np.float32))
    got = out["rest_logit"].cpu().numpy().astype(np.float64)
    np.testing.assert_array_equal(np.isfinite(got), np.isfinite(rest))
    fine = np.isfinite(rest)
    assert np.all(np.abs(got - rest)[fine] <= rest_tolerance(x, tok, tau, rest)[fine])
    assert not out["row_status"].any()
    return out


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,V,k", [(1, 1, 1), (3, 7, 7), (5, 63, 20), (2, 256, 256), (4, 1000, 1), (3, 1023, 256),
                                   (2, 1025, 64), (6, 4099, 33), (3, 20000, 256), (1, 49999, 100), (2, 151936, 64),
                                   (600, 3001, 17), (515, 9000, 256)])
def test_rows(saki_lib, n, V, k, dtype):
    rng = np.random.default_rng(n * V + k)
    check(rows(rng.normal(size=(n, V)) * 3, dtype), k)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("tau", [0.25, 1.7, 50.0])
def test_temperatures(saki_lib, dtype, tau):
    rng = np.random.default_rng(7)
    check(rows(rng.normal(size=(3, 30001)) * 4, dtype), 50, tau)


@pytest.mark.parametrize("n", [2, 600])
@pytest.mark.parametrize("kind", ["equal", "two_values", "rising", "falling", "zeros", "blocks", "peak", "sampled", "sampled_ties"])
def test_orders_and_ties(saki_lib, kind, n):
    V = 20011
    i = np.arange(V)
    x = {"equal": np.full(V, 2.5), "two_values": (i % 3 == 0) * 1.0, "rising": i * 0.125, "falling": -i * 0.125,
         "zeros": np.where(i % 2 == 0, 0.0, -0.0), "blocks": np.floor(i / 700) % 5, "peak": np.where(i == 15000, 30.0, 0.0),
         # (a first chunk whose 64 lanes each hold a large entry: a threshold guessed from it leaves fewer than 90)
         "sampled": np.where((i < 512) & (i % 8 == 0), 5.0 + i / 64, i * -0.001),
         "sampled_ties": np.where((i < 512) & (i % 8 == 0), 5.0, (i % 11) * 0.25)}[kind]
    for dtype in (torch.bfloat16, torch.float32):
        check(rows(np.tile(x, (n, 1)), dtype), 90)


@pytest.mark.parametrize("V,k", [(5000, 4), (30000, 200)])
def test_a_rest_far_below_the_list(saki_lib, V, k):
    """Masked tokens of the type's lowest value, and a rest of e^-500 of the row."""
    rng = np.random.default_rng(9)
    for low in (-3.0e38, -500.0):
        x = np.full((3, V), low)
        for r in range(3):
            x[r, rng.permutation(V)[:k]] = rng.normal(size=k)
        check(rows(x, torch.float32), k)
        x[:, 17] += 1.0  # (one of them listed, or the largest of the rest)
        check(rows(x, torch.float32), k)


@pytest.mark.parametrize("V", [900, 30000])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_rows_that_are_not_finite(saki_lib, V, bad):
    rng = np.random.default_rng(11)
    x = rng.normal(size=(6, V))
    x[1, 0] = bad
    x[3, V - 1] = bad
    x[4, :] = bad
    out = saki_lib.top_logits(rows(x, torch.float32), 5)
    torch.cuda.synchronize()
    status = out["row_status"].cpu().numpy()
    assert status.tolist() == [0, 1, 0, 1, 1, 0]
    for r in (1, 3, 4):
        assert np.all(np.isnan(out["top_logit"][r].cpu().numpy())) and np.isnan(out["rest_logit"][r].item())
        assert out["top_token"][r].cpu().tolist() == [-1] * 5
    good = [0, 2, 5]
    _, tok, _ = oracle.top_logits(x[good].astype(np.float32), 5)
    np.testing.assert_array_equal(out["top_token"].cpu().numpy()[good], tok)


def test_strided_outputs_and_missing_ones(saki_lib):
    rng = np.random.default_rng(13)
    x = rows(rng.normal(size=(9, 12345)), torch.bfloat16)
    full = saki_lib.top_logits(x, 40)
    logit = torch.full((9, 50), 7.0, device=DEV)
    token = torch.full((9, 50), 7, dtype=torch.int32, device=DEV)
    ws = torch.empty(saki_lib.workspace_bytes(saki_lib.SAKI_OP_TOP_LOGITS, 9, 12345), dtype=torch.uint8, device=DEV)
    saki_lib.saki_top_logits(x, 40, logit[:, :40], token[:, :40], workspace=ws)
    assert torch.equal(logit[:, :40], full["top_logit"]) and torch.equal(token[:, :40], full["top_token"])
    assert bool((logit[:, 40:] == 7).all()) and bool((token[:, 40:] == 7).all())


def test_many_rows_in_one_call_and_split(saki_lib):
    rng = np.random.default_rng(17)
    x = rows(rng.normal(size=(2500, 2049)), torch.bfloat16)
    whole = saki_lib.top_logits(x, 12)
    parts = [saki_lib.top_logits(x[a:a + 700], 12) for a in range(0, 2500, 700)]
    for f in ("top_logit", "top_token"):
        assert torch.equal(whole[f], torch.cat([p[f] for p in parts]))
    # (few rows are read in parts, whose sums are added in another order)
    assert torch.allclose(whole["rest_logit"], torch.cat([p["rest_logit"] for p in parts]), rtol=2.0**-20, atol=2.0**-20)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,V,k", [(1, 98305, 1), (3, 110003, 256), (40, 98304, 20), (40, 98311, 20), (255, 100001, 7), (256, 100001, 7),
                                   (1, 600001, 64)])
def test_long_rows_in_few_and_many(saki_lib, n, V, k, dtype):
    """Both sides of what is read in parts."""
    rng = np.random.default_rng(n + V + k)
    check(rows(rng.normal(size=(n, V)) * 3, dtype), k, 1.3)


@pytest.mark.parametrize("kind", ["equal", "two_values", "rising", "falling", "blocks", "peak", "sampled", "sampled_ties"])
def test_orders_and_ties_of_long_rows(saki_lib, kind):
    V = 120011
    i = np.arange(V)
    x = {"equal": np.full(V, 2.5), "two_values": (i % 3 == 0) * 1.0, "rising": i * 0.0625, "falling": -i * 0.0625,
         "blocks": np.floor(i / 700) % 5, "peak": np.where(i == 75000, 30.0, 0.0),
         "sampled": np.where((i % 16384 < 512) & (i % 8 == 0), 5.0 + i / 4096, i * -0.001),
         "sampled_ties": np.where((i % 16384 < 512) & (i % 8 == 0), 5.0, (i % 11) * 0.25)}[kind]
    for dtype in (torch.bfloat16, torch.float32):
        check(rows(np.tile(x, (2, 1)), dtype), 90)


def test_long_rows_far_below_the_list(saki_lib):
    test_a_rest_far_below_the_list(saki_lib, 120000, 200)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_long_rows_that_are_not_finite(saki_lib, bad):
    test_rows_that_are_not_finite(saki_lib, 120000, bad)
