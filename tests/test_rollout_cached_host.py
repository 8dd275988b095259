"""The rollout driver with caches, on the CPU: the library's calls are replaced by stand-ins built on the oracle
(oracle/cache.py for the caches), and its trajectories must equal the oracle rollout's with a model that
computes every logit row from the whole prefix, without a cache."""
import numpy as np
import pytest
import torch

from oracle import cache as ocache
from oracle import rollout as orollout
from paper_2609_36601_amd import binding, speculative
from paper_2609_36601_amd.workloads import SyntheticAttentionPair
from tests.test_rollout_driver_host import fakes  # noqa: F401


class OracleCache:
    """PagedKV's methods on the CPU."""

    def __init__(self, real):
        self.n_seq, self.real = real.n_seq, real
        n_seq, width = real.pages.shape
        self.t = ocache.Table(n_seq, width, real.n_pages, real.page_size)
        shape = (real.n_layers, real.n_pages, real.page_size, real.n_kv_heads, real.head_dim)
        self.k, self.v = np.full(shape, np.nan), np.full(shape, np.nan)
        self.most = 0

    def reserve(self, n_new):
        status, copies = self.t.reserve(n_new.tolist())
        for a, z, n in copies:
            for x in (self.k, self.v):
                x[:, z, :n] = x[:, a, :n]
        self.most = max(self.most, int((self.t.refs > 0).sum()))
        return torch.tensor(status, dtype=torch.uint8)

    def commit(self, delta=None, done=None):
        return torch.tensor(self.t.commit(None if delta is None else delta.tolist(), None if done is None else done.tolist()))

    def fork(self, src, dst):
        assert set(self.t.fork(src.tolist(), dst.tolist())) == {0}

    def _rows(self, n_new, offsets, shift):
        for b in range(self.n_seq):
            a, z = (b * n_new, b * n_new + n_new) if offsets is None else (int(offsets[b]), int(offsets[b + 1]))
            yield b, a, z, int(self.t.length[b]) + shift

    def append(self, layer, k, v, q, rope, n_new=None, offsets=None, shift=0):
        out = q.double().numpy().copy()
        turn = dict(freq=rope["freq"].numpy(), rotary_dim=rope["rotary_dim"], interleaved=rope["interleaved"],
                    amplitude=rope["amplitude"])
        P = self.t.page_size
        for b, a, z, start in self._rows(n_new, offsets, shift):
            for i in range(a, z):
                pos = start + i - a
                if pos // P >= self.t.held[b]:
                    out[i] = np.nan
                    continue
                page = self.t.pages[b, pos // P]
                assert self.t.refs[page] == 1
                for h in range(k.shape[1]):
                    self.k[layer, page, pos % P, h] = ocache.rope(k[i, h].double().numpy(), pos, **turn)
                self.v[layer, page, pos % P] = v[i].double().numpy()
                for h in range(q.shape[1]):
                    out[i, h] = ocache.rope(out[i, h], pos, **turn)
        return torch.as_tensor(out).to(q.dtype)

    def attention(self, layer, q, window, sinks, n_new=None, offsets=None, shift=0):
        out = np.full(q.shape, np.nan)
        P = self.t.page_size
        for b, a, z, start in self._rows(n_new, offsets, shift):
            if z == a or start + z - a > self.t.held[b] * P:
                continue
            pages = self.t.pages[b, :self.t.held[b]]
            k, v = (x[layer, pages].reshape(-1, *x.shape[3:])[:start + z - a] for x in (self.k, self.v))
            out[a:z] = ocache.attention(q[a:z].double().numpy(), k, v, start + np.arange(z - a), q.shape[2] ** -0.5, window,
                                        sinks)[0]
        return torch.as_tensor(out).to(q.dtype)


class WholePrefix:
    """The same networks without caches, for the oracle's rollout: a state is a number that stands for a prefix."""

    def __init__(self, model):
        self.m, self.prefixes = model, []

    def _state(self, prefix):
        self.prefixes.append(prefix)
        return len(self.prefixes) - 1

    def initial(self, ids):
        return np.array([self._state(list(self.m.prompt(int(p)))) for p in ids])

    def advance(self, states, tokens):
        return np.array([self._state(self.prefixes[int(s)] + [int(t)]) for s, t in
                         zip(np.atleast_1d(states), np.atleast_1d(tokens))])

    def logits(self, states):
        rows = [[dense_logits(self.m, net, self.prefixes[int(s)])[-1] for s in np.atleast_1d(states)] for net in range(2)]
        return tuple(np.stack(r).astype(np.float32) for r in rows)


def dense_logits(m, net, prefix):
    """Logits behind every token of a sequence, by attention over the whole of it, in 64 bits."""
    pos = np.arange(len(prefix))
    w = {k: [x.double().cpu() for x in v] if isinstance(v, list) else v.double().cpu() for k, v in m.weights[net].items()}
    freq = m.rope["freq"].cpu().numpy()

    def attend(i, q, k, v):
        q, k = (torch.as_tensor(np.stack([[ocache.rope(x[p, h].numpy(), p, freq, m.head_dim, False, 1.0) for h in
                                           range(x.shape[1])] for p in pos])) for x in (q, k))
        return torch.as_tensor(ocache.attention(q.numpy(), k.numpy(), v.numpy(), pos, m.head_dim ** -0.5, m.windows[net],
                                                m.sinks)[0])

    keep, m.weights = m.weights, {net: w}
    h = m._hidden(net, torch.as_tensor(np.asarray(prefix)), attend)
    m.weights = keep
    return (h @ w["logits"]).numpy()


def model(B, n_pages=60, **kw):
    m = SyntheticAttentionPair(14, B, 8, n_pages, page_size=8, layers=2, heads=2, kv_heads=1, head_dim=8, width=16,
                               most_prompt=12, device="cpu", seed=3, **kw)
    m.caches = tuple(OracleCache(c) for c in m.caches)
    return m


@pytest.mark.parametrize("k,eos,kw", [(3, -1, {}), (4, 5, dict(windows=(6, 0), sinks=1)), (1, -1, {})])
def test_cached_rollout_equals_the_rollout_without_caches(fakes, k, eos, kw):  # noqa: F811
    prompts, L, eps, seed = [4, 4, 9, 4, 2, 9], 10, 0.3, 11
    m = model(len(prompts), **kw)
    tr, waves = speculative.rollout(m, prompts, k, L, eps, seed, eos_id=eos, dtype=torch.float32)
    want = orollout.rollout(WholePrefix(m), np.array(prompts), k, L, eps, seed, eos_id=eos)
    assert waves == want["waves"]
    for key in ("tokens", "corrected", "length", "done"):
        np.testing.assert_array_equal(tr[key].numpy(), want[key], err_msg=key)
    for c in m.caches:  # finished sequences have given back everything
        assert (c.t.refs == 0).all() and (c.t.held == 0).all() and c.most > 0
    # responses of one prompt shared its pages
    assert len(m.prompt(4)) > 8 and (want["length"] > 0).all()


def test_a_cache_too_small_is_reported(fakes):  # noqa: F811
    m = model(6, n_pages=7)
    with pytest.raises(RuntimeError, match="too few pages"):
        speculative.rollout(m, [4, 9, 2, 1, 0, 5], 3, 30, 0.3, 1, dtype=torch.float32)


def test_a_model_with_caches_takes_no_stream(fakes):  # noqa: F811
    with pytest.raises(ValueError, match="current stream"):
        speculative.rollout(model(2), [1, 2], 3, 4, 0.3, 1, stream=object())
    tr, waves = speculative.rollout(model(2), [1, 2], 3, 0, 0.3, 1)
    assert waves == 0 and (tr["done"] == binding.SEQ_FINISHED).all()
