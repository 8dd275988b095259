"""Token ranges that are not in order: each counts as empty by itself, the others keep their rows, in the append and in
the attention alike."""
import numpy as np
import pytest
import torch

from tests.kv_cases import filled, to_cache

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def rows_of(offsets, n_tokens):
    """The ranges by the rule alone: {row: (sequence, place in its range)}."""
    rows = {}
    for b, (a, z) in enumerate(zip(offsets, offsets[1:])):
        if 0 <= a < z <= n_tokens:
            rows.update({i: (b, i - a) for i in range(a, z)})
    return rows


CASES = [[0, 5, -3, 12], [-1, 2, 2, 2], [0, 0, 99, 99], [4, 2, 4, 4], [0, 99, 0, 4], [9, 9, 3, 12], [12, 0, 0, 12],
         [0, 12, 0, -5], [13, 4, 12, 3], [2, 6, 6, 10], [5, 5, 5, 5], [2**31 - 1, -2**31, 7, 9]]


@pytest.mark.parametrize("offsets", CASES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_ranges_out_of_order(saki_lib, offsets, dtype):
    print(f"ranges {offsets} {dtype}", flush=True)
    check(saki_lib, offsets, 12, [6, 8, 3], dtype)


@pytest.mark.parametrize("n", [300, 3000])
def test_among_many_sequences(saki_lib, n):
    """Ranges of one row each, some of them out of order: a search that trusts the order loses their neighbours."""
    rng = np.random.default_rng(n)
    offsets = np.arange(n + 1)
    broken = rng.integers(1, n, n // 10)
    offsets[broken] = np.where(rng.random(n // 10) < 0.5, rng.integers(-n, 0, n // 10), rng.integers(n + 1, 2 * n, n // 10))
    assert len(rows_of(offsets.tolist(), n)) > n // 2
    check(saki_lib, offsets.tolist(), n, rng.integers(0, 20, n).tolist(), torch.float32)


def check(saki, offsets, n_tokens, lengths, dtype):
    rng = np.random.default_rng(3)
    hq, hk, dim, page = 4, 2, 16, 8
    n = len(lengths)
    t = filled(lengths, page, sum(-(-(L + 12) // page) for L in lengths) + 2, 6, rng, extra=12)
    g = torch.Generator(device=DEV).manual_seed(9)
    k, v = (torch.randn(1, t.refs.size, hk, page, dim, generator=g, device=DEV).to(dtype) for _ in range(2))
    c = to_cache(saki, t, k, v)
    x = torch.randn(n_tokens, hq + 2 * hk, dim, generator=g, device=DEV).to(dtype)
    rows = rows_of(offsets, n_tokens)
    assert len(offsets) == n + 1
    off = torch.tensor(offsets, dtype=torch.int32, device=DEV)
    q = torch.full((n_tokens, hq, dim), 3.0, dtype=dtype, device=DEV)
    wk, wv, wq = k.clone(), v.clone(), q.clone()
    for i, (b, j) in rows.items():
        pos = lengths[b] + j
        at = int(t.pages[b, pos // page]) if pos // page < t.held[b] else -1
        wq[i] = x[i, :hq] if at >= 0 else float("nan")
        if at >= 0:
            wk[0, at, :, pos % page], wv[0, at, :, pos % page] = x[i, hq:hq + hk], x[i, hq + hk:]
    c.append(0, x[:, hq:hq + hk], x[:, hq + hk:], q=x[:, :hq], q_out=q, offsets=off)
    torch.testing.assert_close(q, wq, rtol=0, atol=0, equal_nan=True)
    assert torch.equal(k, wk) and torch.equal(v, wv)
    # attention: the same rows, as alone in a call that has them in order; the others are left as they are
    out, lse = torch.full_like(q, 3.0), torch.full((n_tokens, hq), 3.0, device=DEV)
    c.attention(0, x[:, :hq], out=out, lse=lse, offsets=off)
    count = np.bincount([b for b, _ in rows.values()], minlength=n)
    order = sorted(rows, key=lambda i: rows[i])
    sorted_off = torch.tensor(np.concatenate([[0], np.cumsum(count)]), dtype=torch.int32, device=DEV)
    wout, wlse = torch.full_like(out, 3.0), torch.full_like(lse, 3.0)
    if order:
        at = torch.tensor(order, device=DEV)
        part = torch.empty(len(order), hq, device=DEV)
        wout[at] = c.attention(0, x[at, :hq].contiguous(), lse=part, offsets=sorted_off)
        wlse[at] = part
    torch.testing.assert_close(out, wout, rtol=0, atol=0, equal_nan=True)
    torch.testing.assert_close(lse, wlse, rtol=0, atol=0, equal_nan=True)
