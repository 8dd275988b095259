"""The cache oracle against its own invariants and independent formulas."""
import numpy as np
import pytest
import torch

from oracle import cache as ocache
from tests.kv_cases import filled


def _sound(t):
    count = np.zeros_like(t.refs)
    for b in range(t.pages.shape[0]):
        held = t.pages[b, :t.held[b]]
        assert (held >= 0).all() and len(set(held)) == len(held) and (t.pages[b, t.held[b]:] == -1).all()
        assert 0 <= t.length[b] <= t.held[b] * t.page_size
        np.add.at(count, held, 1)
    np.testing.assert_array_equal(count, t.refs)


@pytest.mark.parametrize("seed", range(6))
def test_pages_stay_consistent_through_random_steps(seed):
    rng = np.random.default_rng(seed)
    n, P = 7, 8
    t = ocache.Table(n, 9, 40, P)
    content = {}  # what every (page, slot) holds: the token's history
    hist = [[] for _ in range(n)]
    for step in range(60):
        if rng.random() < 0.3:
            empty = [b for b in range(n) if t.held[b] == 0]
            other = [b for b in range(n) if t.held[b] and t.length[b]]
            if empty and other:
                s, d = int(rng.choice(other)), empty[0]
                assert t.fork([s], [d]) == [ocache.OK]
                hist[d] = list(hist[s])
        want = rng.integers(0, 12, n)
        before = t.copy()
        status, copies = t.reserve(want)
        for a, z, slots in copies:
            for i in range(slots):
                content[z, i] = content[a, i]
        if ocache.NO_PAGES in status:
            for f in ("pages", "length", "held", "refs"):
                np.testing.assert_array_equal(getattr(t, f), getattr(before, f))
        delta = np.zeros(n, dtype=int)
        for b in range(n):
            if status[b] == ocache.OK and want[b]:
                for i in range(want[b]):  # every token of the wave is written, then some are taken back
                    at = t.length[b] + i
                    page = t.pages[b, at // P]
                    assert t.refs[page] == 1
                    content[page, at % P] = (step, b, i)
                delta[b] = rng.integers(0, want[b] + 1)
                hist[b] += [(step, b, i) for i in range(delta[b])]
        done = rng.random(n) < 0.05
        assert set(t.commit(delta, done)) == {ocache.OK}
        for b in np.nonzero(done)[0]:
            hist[b] = []
        _sound(t)
        for b in range(n):  # every sequence still holds its own tokens
            got = [content[t.pages[b, i // P], i % P] for i in range(t.length[b])]
            assert got == hist[b]
        if step % 9 == 8:
            n_live, moves = t.compact()
            for a, z in moves:
                for i in range(P):
                    if (a, i) in content:
                        content[z, i] = content.pop((a, i))
            assert (t.refs[:n_live] > 0).all() and (t.refs[n_live:] == 0).all()
            _sound(t)


def test_last_writer_keeps_a_page_that_all_holders_write():
    t = filled([5, 0, 0], 8, 10, 4, np.random.default_rng(0))
    t.fork([0, 0], [1, 2])
    page = t.pages[0, 0]
    two = t.copy()
    status, copies = t.reserve([1, 1, 1])
    assert status == [0, 0, 0] and [c[0] for c in copies] == [page, page] and t.pages[2, 0] == page
    status, copies = two.reserve([1, 1, 0])  # the third holds it too and does not write
    assert len(copies) == 2 and two.pages[2, 0] == page and two.refs[page] == 1


def test_rope_and_attention_against_torch():
    rng = np.random.default_rng(3)
    d, r = 12, 8
    freq = 100.0 ** (-np.arange(0, r, 2) / r) / (2 * np.pi)
    x = rng.normal(size=d)
    for inter in (0, 1):
        for pos in (0, 1, 12345):
            pairs = x[:r].reshape(-1, 2) if inter else x[:r].reshape(2, -1).T
            z = (pairs[:, 0] + 1j * pairs[:, 1]) * 0.7 * np.exp(2j * np.pi * freq * pos)
            want = np.stack([z.real, z.imag], 1).reshape(-1) if inter else np.concatenate([z.real, z.imag])
            np.testing.assert_allclose(ocache.rope(x, pos, freq, r, inter, 0.7)[:r], want, rtol=1e-9, atol=1e-9)
            np.testing.assert_array_equal(ocache.rope(x, pos, freq, r, inter, 0.7)[r:], x[r:])
    q, k, v = rng.normal(size=(3, 4, d)), rng.normal(size=(20, 2, d)), rng.normal(size=(20, 2, d))
    pos = np.array([17, 18, 19])
    out, lse = ocache.attention(q, k, v, pos, 0.3, window=6, sinks=2)
    for i in range(3):
        seen = torch.tensor([j <= pos[i] and (j > pos[i] - 6 or j < 2) for j in range(20)])
        for h in range(4):
            s = 0.3 * torch.tensor(k[:, h // 2]) @ torch.tensor(q[i, h])
            s = s.masked_fill(~seen, -torch.inf)
            np.testing.assert_allclose(lse[i, h], torch.logsumexp(s, 0), rtol=1e-12)
            np.testing.assert_allclose(out[i, h], torch.softmax(s, 0) @ torch.tensor(v[:, h // 2]), rtol=1e-12)


def test_hidden_tokens_have_no_influence_and_empty_rows_are_zero():
    rng = np.random.default_rng(4)
    q, k, v = rng.normal(size=(1, 2, 8)), rng.normal(size=(9, 1, 8)), rng.normal(size=(9, 1, 8))
    a, la = ocache.attention(q, k, v, [5], 1.0, window=3)
    k[6:], v[:3] = np.nan, np.inf
    b, lb = ocache.attention(q, k, v, [5], 1.0, window=3)
    np.testing.assert_array_equal(a, b)
    k[:] = -np.inf
    c, lc = ocache.attention(np.abs(q), k, v, [5], 1.0)
    assert (c == 0).all() and (lc == -np.inf).all()
