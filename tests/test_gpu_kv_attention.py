"""Attention over the paged cache on the GPU against the oracle in 64 bits.

Bound of an output element, with w the softmax weights: a score is a sum of d products in 32 bits, off by at
most e = (d + 8) 2^-24 scale sum |q_i k_i| (the products of bf16 elements are exact, the sum is not; scaling
and the exponential's argument add a few steps, whose size goes by the score, which the sum bounds).  A
weight is then off by 2 e + 2^-21 relative, and sums over n keys by n 2^-24.  bf16: each weight is
rounded once more (2^-8) for its product with the value, and the output.  Every term multiplies sum w |v|."""
import numpy as np
import pytest
import torch

from oracle import cache as ocache
from tests.kv_cases import filled, to_cache, token_major

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NAN = float("nan")


def make(saki, dtype, lengths, new, group, hk, dim, page, seed, order="heads", shift=0, scale_q=1.0, spare=0):
    """A cache that holds lengths + shift + new tokens; every slot that holds none is NaN."""
    rng = np.random.default_rng(seed)
    lengths, new = np.asarray(lengths), np.asarray(new)
    total = lengths + shift + new
    t = filled(list(total), page, int(sum(-(-total // page))) + 3, int(max(-(-total // page))) + 2, rng)
    shape = (2, t.refs.size, hk, page, dim)
    k, v = (token_major(*shape, dtype, DEV) if order == "tokens" else torch.empty(shape, dtype=dtype, device=DEV)
            for _ in range(2))
    k.fill_(NAN)
    v.fill_(NAN)
    g = torch.Generator(device=DEV).manual_seed(seed)
    dense = []
    for b in range(len(lengths)):
        kb, vb = (torch.randn(int(total[b]), hk, dim, generator=g, device=DEV).to(dtype) for _ in range(2))
        dense.append((kb, vb))
        put(t, b, k, v, kb, vb)
    t.length[:] = lengths
    off = np.concatenate([[0], np.cumsum(new)])
    q = (scale_q * torch.randn(int(off[-1]) + spare, group * hk, dim, generator=g, device=DEV)).to(dtype)
    return t, to_cache(saki, t, k, v), q, off, dense


def put(t, b, k, v, kb, vb, layer=1):
    pos = torch.arange(kb.shape[0], device=DEV)
    ids = torch.as_tensor(t.pages[b], device=DEV)[pos // t.page_size]
    k[layer, ids, :, pos % t.page_size] = kb
    v[layer, ids, :, pos % t.page_size] = vb


def check(out, lse, q, off, dense, t, scale, window, sinks, shift=0, rows=None):
    bf = out.dtype == torch.bfloat16
    qd = q.double().cpu().numpy()
    for b in range(len(off) - 1):
        if off[b + 1] == off[b]:
            continue
        kb, vb = (x.double().cpu().numpy() for x in dense[b])
        pos = t.length[b] + shift + np.arange(off[b + 1] - off[b])
        pick = np.arange(len(pos)) if rows is None or len(pos) <= rows else \
            np.unique(np.concatenate([[0, len(pos) - 1], np.random.default_rng(b).integers(0, len(pos), rows)]))
        qb = qd[off[b]:off[b + 1]][pick]
        want, wl = ocache.attention(qb, kb, vb, pos[pick], scale, window, sinks)
        size, _ = ocache.attention(qb, kb, np.abs(vb), pos[pick], scale, window, sinks)
        d, n = q.shape[2], kb.shape[0]
        seen = kb[:pos.max() + 1]
        finite = np.where(np.isfinite(seen), np.abs(seen), 0)
        e = np.abs(scale) * (d + 8) * 2.0**-24 * np.einsum("ihd,d->ih", np.nan_to_num(np.abs(qb)), finite.max((0, 1)))
        rel = 2 * e + 2.0**-21 + (n + 16) * 2.0**-24 + (2.0**-8 if bf else 0)
        tol = rel[..., None] * size + (2.0**-8 if bf else 2.0**-24) * np.abs(want) + 1e-30
        got = out[off[b]:off[b + 1]].double().cpu().numpy()[pick]
        np.testing.assert_array_equal(np.isnan(got), np.isnan(want))
        bad = ~(np.abs(got - want) <= tol) & ~np.isnan(want) & ~(got == want)
        assert not bad.any(), (b, np.abs(got - want)[bad][:5], tol[bad][:5], np.argwhere(bad)[:5])
        if lse is not None:
            gl = lse[off[b]:off[b + 1]].double().cpu().numpy()[pick]
            same = (gl == wl) | (np.isnan(gl) & np.isnan(wl))
            assert (same | (np.abs(gl - wl) <= e + (n + 16) * 2.0**-24 + 2.0**-20 * (1 + np.abs(wl)))).all()


def run(saki, t, c, q, off, dense, scale=None, window=0, sinks=0, shift=0, uniform=None, rows=None, **kw):
    scale = q.shape[2] ** -0.5 if scale is None else scale
    lse = torch.full(q.shape[:2], 7.0, device=DEV)
    out = torch.full_like(q, 7.0)
    how = dict(n_new=uniform) if uniform is not None else dict(
        offsets=torch.as_tensor(off, dtype=torch.int32, device=DEV))
    c.attention(1, q, out=out, lse=lse, scale=scale, window=window, sinks=sinks, shift=shift, **how, **kw)
    check(out, lse, q, off, dense, t, scale, window, sinks, shift, rows)
    assert (out[off[-1]:] == 7.0).all() and (lse[off[-1]:] == 7.0).all()
    return out, lse


BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("dim,group,hk,page,order", [(128, 2, 3, 16, "heads"), (64, 1, 2, 8, "tokens"),
                                                     (80, 7, 1, 32, "heads"), (8, 3, 2, 8, "heads"),
                                                     (256, 4, 1, 64, "tokens"), (136, 17, 1, 16, "heads"),
                                                     (112, 40, 2, 128, "heads")])
def test_single_tokens(saki_lib, dtype, dim, group, hk, page, order):
    lengths = [0, 1, 7, 31, 32, 33, 130, 517]
    print(f"single tokens: {dtype} dim {dim} group {group}", flush=True)
    run(saki_lib, *make(saki_lib, dtype, lengths, [1] * 8, group, hk, dim, page, dim + group, order), uniform=1)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (5, 3), (40, 4), (64, 70), (1000, 1), (100, 0)])
def test_ragged_verification_with_windows(saki_lib, dtype, window, sinks):
    print(f"ragged: {dtype} window {window} sinks {sinks}", flush=True)
    run(saki_lib, *make(saki_lib, dtype, [0, 90, 200, 45, 333], [3, 8, 0, 1, 17], 4, 2, 64, 16, window + sinks,
                        spare=2), window=window, sinks=sinks)


@pytest.mark.parametrize("dtype,dim,group,window,sinks", [(BF, 128, 2, 0, 0), (BF, 64, 5, 0, 0), (F32, 64, 3, 0, 0),
                                                          (BF, 96, 4, 60, 5), (F32, 128, 2, 33, 0), (BF, 256, 1, 0, 0),
                                                          (BF, 128, 1, 200, 130)])
def test_prompts(saki_lib, dtype, dim, group, window, sinks):
    print(f"prompts: {dtype} dim {dim} group {group} window {window}", flush=True)
    run(saki_lib, *make(saki_lib, dtype, [0, 0, 37, 0], [1, 300, 129, 513], group, 2, dim, 32, dim + window, "tokens"),
        window=window, sinks=sinks, rows=12)


@pytest.mark.parametrize("dtype,new", [(BF, 1), (F32, 1), (BF, 8), (F32, 5)])
def test_one_long_sequence_is_split(saki_lib, dtype, new):
    print(f"long: {dtype} {new}", flush=True)
    run(saki_lib, *make(saki_lib, dtype, [20011], [new], 4, 1, 64, 16, new), uniform=new)
    run(saki_lib, *make(saki_lib, dtype, [20011, 3, 900], [new] * 3, 4, 2, 128, 64, new), uniform=new, rows=3)


@pytest.mark.parametrize("dtype,rows", [(BF, 256), (F32, 128)])
def test_tables_too_short_for_a_split(saki_lib, dtype, rows):
    """A table of 8 blocks a sequence: nothing is split and nothing joined, whatever the window."""
    new = 10
    t, c, q, off, dense = make(saki_lib, dtype, [rows - new], [new], 4, 2, 64, 16, 31)
    c = saki_lib.PagedKV(c.k, c.v, c.pages[:, :rows // 16].contiguous(), c.length, c.held, c.refs)
    for window in (0, rows - 56, rows // 2, 33):
        run(saki_lib, t, c, q, off, dense, uniform=new, window=window, sinks=3)


@pytest.mark.parametrize("dim,page,order,lengths,new", [
    (64, 8, "heads", [3001], [100]), (128, 8, "heads", [2500, 0], [70, 200]), (128, 16, "tokens", [0, 5000], [65, 130]),
    (40, 16, "heads", [700, 30, 0], [90, 0, 129]), (128, 256, "heads", [1, 257], [128, 255])])
def test_prompts_behind_long_caches(saki_lib, dim, page, order, lengths, new):
    """Many rows whose keys are split and joined, in pages shorter and longer than a tile."""
    print(f"long prompts: dim {dim} page {page} {lengths} {new}", flush=True)
    args = make(saki_lib, BF, lengths, new, 3, 2, dim, page, dim + page, order, spare=3)
    run(saki_lib, *args, rows=9)
    run(saki_lib, *args, rows=9, window=333, sinks=70)


def test_shift_and_large_scores(saki_lib):
    """Tokens behind the committed ones (a draft position), and scores far from 0: the running maximum moves."""
    t, c, q, off, dense = make(saki_lib, BF, [60, 5, 300], [1, 1, 1], 2, 2, 64, 8, 3, shift=4)
    run(saki_lib, t, c, q, off, dense, shift=4, uniform=1)
    t, c, q, off, dense = make(saki_lib, F32, [260, 15, 300], [2, 2, 2], 2, 2, 64, 8, 4, scale_q=30.0)
    for b in range(3):  # scores that grow along the sequence
        kb, vb = dense[b]
        kb *= torch.linspace(0.1, 6, kb.shape[0], device=DEV)[:, None, None]
        put(t, b, c.k, c.v, kb, vb)
    run(saki_lib, t, c, q, off, dense, uniform=2)
    run(saki_lib, t, c, q, off, dense, uniform=2, scale=-0.3)
    run(saki_lib, t, c, q, off, dense, uniform=2, scale=0.0)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_hidden_tokens_have_no_influence(saki_lib, dtype):
    """NaN and infinities in keys and values that a token does not see: later drafts, tokens before the window,
    other sequences' slots; and rows whose every score is -infinity."""
    t, c, q, off, dense = make(saki_lib, dtype, [50, 70], [6, 6], 3, 2, 64, 8, 21)
    for b, L in ((0, 50), (1, 70)):
        kb, vb = dense[b]
        kb[L + 3], vb[L + 3] = NAN, float("inf")   # seen by drafts 3, 4, 5 alone
        vb[L + 5] = NAN
        kb[10], vb[10] = float("inf"), -float("inf")  # before the window
        put(t, b, c.k, c.v, kb, vb)
    out, lse = run(saki_lib, t, c, q, off, dense, uniform=6, window=20, sinks=2)
    assert torch.isfinite(out.view(2, 6, -1)[:, :3]).all()
    low = torch.finfo(dtype).min
    t, c, q, off, dense = make(saki_lib, dtype, [9, 40], [1, 1], 2, 1, 64, 8, 22)
    q.abs_()
    dense[0][0].fill_(-float("inf"))  # every score -infinity
    dense[1][0][:35] = low            # the lowest finite keys: scores of -infinity or nearly so
    for b in range(2):
        put(t, b, c.k, c.v, *dense[b])
    lse = torch.empty(2, 2, device=DEV)
    out = c.attention(1, q, lse=lse, n_new=1)
    assert (out[0] == 0).all() and (lse[0] == -float("inf")).all()
    assert torch.isfinite(out[1]).all()


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("window,sinks", [(0, 0), (90, 3)])
def test_hidden_tokens_in_prompts(saki_lib, dim, window, sinks):
    """The same where one workgroup holds rows that see a token and rows that do not."""
    t, c, q, off, dense = make(saki_lib, BF, [100, 0], [200, 150], 2, 2, dim, 32, dim + window)
    for b, (kb, vb) in enumerate(dense):
        kb[30], vb[30] = float("inf"), -float("inf")
        vb[110] = NAN
        kb[140] = NAN
        vb[-1] = float("inf")
        put(t, b, c.k, c.v, kb, vb)
    out, lse = run(saki_lib, t, c, q, off, dense, window=window, sinks=sinks)
    assert torch.isfinite(out[200:230]).all() and torch.isfinite(lse[200:230]).all()  # before token 30
    t, c, q, off, dense = make(saki_lib, BF, [0, 0], [150, 130], 2, 1, dim, 8, 22)
    q.abs_()
    dense[0][0].fill_(-float("inf"))
    put(t, 0, c.k, c.v, *dense[0])
    lse = torch.empty(280, 2, device=DEV)
    out = c.attention(1, q, lse=lse, offsets=torch.as_tensor([0, 150, 280], dtype=torch.int32, device=DEV))
    assert (out[:150] == 0).all() and (lse[:150] == -float("inf")).all() and torch.isfinite(out[150:]).all()


def test_prompts_without_pages_and_in_place(saki_lib):
    t, c, q, off, dense = make(saki_lib, BF, [50, 70, 20, 1500], [100] * 4, 3, 2, 64, 8, 23)
    want = c.attention(1, q, n_new=100)
    wide = torch.zeros(400, 11, 64, dtype=BF, device=DEV)
    wide[:, 2:8] = q
    got = c.attention(1, wide[:, 2:8], out=wide[:, 2:8], n_new=100)
    assert torch.equal(got, want) and (wide[:, :2] == 0).all() and (wide[:, 8:] == 0).all()
    c.held[0] -= 1
    c.pages[1, 3] = -1
    c.pages[3, 100] = c.k.shape[1]
    c.length[2] = -7
    lse = torch.empty(q.shape[:2], device=DEV)
    out = c.attention(1, q, lse=lse, n_new=100)
    assert torch.isnan(out).all() and torch.isnan(lse).all()


def test_calls_at_once_on_two_streams(saki_lib):
    """Calls on two streams with workspaces of their own do not disturb each other."""
    a = make(saki_lib, BF, [9000, 5], [3, 3], 4, 2, 128, 16, 40)
    b = make(saki_lib, BF, [300, 2000], [120, 120], 2, 2, 64, 32, 41)
    want = [a[1].attention(1, a[2], n_new=3), b[1].attention(1, b[2], n_new=120)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(10):
        for i, (x, new) in enumerate(((a, 3), (b, 120))):
            with torch.cuda.stream(streams[i]):
                got[i].append(x[1].attention(1, x[2], n_new=new))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(g, want[i]) for g in got[i])


@pytest.mark.parametrize("new", [3, 70])
def test_ranges_that_overlap_stay_in_bounds(saki_lib, new):
    """Not allowed, and what the rows get is open; no row behind the tokens is written."""
    t, c, q, off, dense = make(saki_lib, BF, [3000] * 40, [new] * 40, 4, 2, 64, 16, 42)
    offsets = torch.as_tensor([0, new] * 20 + [0], dtype=torch.int32, device=DEV)
    out = torch.full_like(q, 7.0)
    c.attention(1, q[:new], out=out[:new], offsets=offsets)
    torch.cuda.synchronize()
    assert (out[new:] == 7.0).all()


def test_sequences_without_pages_get_nan(saki_lib):
    t, c, q, off, dense = make(saki_lib, BF, [50, 70, 20], [2, 2, 2], 3, 2, 64, 8, 23)
    want = c.attention(1, q, n_new=2)
    c.held[0] -= 1
    c.pages[1, 3] = -1
    lse = torch.empty(q.shape[:2], device=DEV)
    out = c.attention(1, q, lse=lse, n_new=2)
    assert torch.isnan(out[:4]).all() and torch.isnan(lse[:4]).all() and torch.equal(out[4:], want[4:])
    c.length[2] = -7
    assert torch.isnan(c.attention(1, q, n_new=2)).all()


def test_in_place_strided_rows_and_another_stream(saki_lib):
    t, c, q, off, dense = make(saki_lib, BF, [500, 7, 3000], [2, 2, 2], 3, 2, 64, 16, 24)
    want = c.attention(1, q, n_new=2)
    wide = torch.zeros(6, 11, 64, dtype=BF, device=DEV)
    wide[:, 2:8] = q
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = c.attention(1, wide[:, 2:8], out=wide[:, 2:8], n_new=2, stream=s)
    s.synchronize()
    assert torch.equal(got, want) and (wide[:, :2] == 0).all() and (wide[:, 8:] == 0).all()
    heads_first = torch.zeros(6, 6, 64, dtype=BF, device=DEV)
    c.attention(1, q, out=heads_first.transpose(0, 1), n_new=2)
    assert torch.equal(heads_first.transpose(0, 1), want)


def test_results_do_not_depend_on_the_run(saki_lib):
    t, c, q, off, dense = make(saki_lib, BF, [9000, 40], [4, 4], 4, 2, 128, 16, 25)
    first = c.attention(1, q, n_new=4)
    for _ in range(5):
        assert torch.equal(c.attention(1, q, n_new=4), first)


def test_captured_calls_replay(saki_lib):
    """Two graphs of append and attention on one cache, replayed in turn with eager work between."""
    t, c, q, off, dense = make(saki_lib, BF, [800, 30], [3, 3], 4, 2, 64, 16, 26)
    rope = saki_lib.rope(64, device=DEV)
    g_ = torch.Generator(device=DEV).manual_seed(5)
    x = torch.randn(6, 8 + 4, 64, generator=g_, device=DEV).to(BF)

    def step(window):
        r = c.append(1, x[:, 8:10], x[:, 10:], q=x[:, :8], rope=rope, n_new=3)
        return c.attention(1, r, n_new=3, window=window)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graphs = []
    with torch.cuda.stream(s):
        step(0)
        torch.cuda.synchronize()
        for window in (0, 100):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                out = step(window)
            graphs.append((g, out, window))
    torch.cuda.synchronize()
    for i in range(4):
        x.copy_(torch.randn(x.shape, generator=g_, device=DEV))
        for g, out, window in graphs:
            g.replay()
            torch.cuda.synchronize()
            got = out.clone()
            assert torch.equal(got, step(window)), (i, window)


def test_offsets_past_32_bits(saki_lib):
    """A pool of more than 2^32 bytes a layer, its last pages in use."""
    page, dim, heads = 64, 128, 8
    n_pages = (1 << 32) // (page * dim * heads * 2) + 64
    k = torch.zeros(1, n_pages, heads, page, dim, dtype=BF, device=DEV)
    v = torch.zeros_like(k)
    ids = torch.arange(n_pages - 4, n_pages, dtype=torch.int32, device=DEV)[None].contiguous()
    refs = torch.zeros(n_pages, dtype=torch.int32, device=DEV)
    refs[-4:] = 1
    one = torch.ones(1, dtype=torch.int32, device=DEV)
    c = saki_lib.PagedKV(k, v, ids, 200 * one, 4 * one, refs)
    g = torch.Generator(device=DEV).manual_seed(1)
    kb, vb = (torch.randn(201, heads, dim, generator=g, device=DEV).to(BF) for _ in range(2))
    pos = torch.arange(200, device=DEV)
    for x, y in ((k, kb), (v, vb)):
        x[0, ids[0, pos // page].long(), :, pos % page] = y[:200]
    q = torch.randn(1, 2 * heads, dim, generator=g, device=DEV).to(BF)
    c.append(0, kb[200:], vb[200:], n_new=1)
    out = c.attention(0, q, n_new=1)
    t = ocache.Table(1, 4, 1, page)
    t.length[0] = 200
    check(out, None, q, [0, 1], [(kb, vb)], t, dim**-0.5, 0, 0)


@pytest.mark.parametrize("dim,n", [(128, 64), (128, 63), (64, 64)])
def test_many_sequences_of_half_a_tile(saki_lib, dim, n):
    """36 to 64 rows a sequence and key head, where enough sequences change the kernel."""
    rng = np.random.default_rng(n + dim)
    args = make(saki_lib, BF, rng.integers(0, 90, n), [9] * n, 4, 8, dim, 16, dim + n)
    run(saki_lib, *args, uniform=9, rows=2)
    new = rng.integers(0, 33, n)
    args = make(saki_lib, BF, rng.integers(0, 90, n), new + (new.sum() < 9 * n), 4, 8, dim, 8, dim + n)
    run(saki_lib, *args, window=50, rows=2)
