"""Pages of the key-value cache on the GPU against the sequential oracle: every table array, status and
copied slot, exactly."""
import numpy as np
import pytest
import torch

from oracle import cache as ocache
from tests.kv_cases import filled, same_table, to_cache, token_major

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def i32(x):
    return torch.as_tensor(np.asarray(x, dtype=np.int32), device=DEV)


def pool_for(t, layers=2, heads=3, dim=16, dtype=torch.bfloat16, order="heads"):
    g = torch.Generator(device=DEV).manual_seed(t.refs.size)
    shape = (layers, t.refs.size, heads, t.page_size, dim)
    k, v = (token_major(*shape, dtype, DEV) if order == "tokens" else torch.empty(shape, dtype=dtype, device=DEV)
            for _ in range(2))
    for x in (k, v):
        x.copy_(torch.randn(shape, generator=g, device=DEV))
    return k, v


def expect_copies(x, moves, slots_of=None):
    y = x.clone()
    for m in moves:
        n = m[2] if len(m) > 2 else x.shape[3]
        y[:, m[1], :, :n] = x[:, m[0], :, :n]
    return y


@pytest.mark.parametrize("seed,n,page,order", [(0, 1, 8, "heads"), (1, 5, 16, "tokens"), (2, 70, 8, "heads"),
                                               (3, 1030, 32, "heads"), (4, 2100, 8, "tokens")])
def test_waves_forks_and_compaction(saki_lib, seed, n, page, order):
    rng = np.random.default_rng(seed)
    width, n_pages = 9, 4 * n + 30
    t = ocache.Table(n, width, n_pages, page)
    k, v = pool_for(t, order=order, dim=8 if n > 500 else 16)
    c = to_cache(saki_lib, t, k, v)
    for step in range(12 if n < 500 else 5):
        print(f"pages: seed {seed} step {step}", flush=True)
        most = 3 * page if step % 3 else page // 2
        want = rng.integers(-1 if step % 4 == 3 else 0, most, n)
        status, copies = t.reserve(want)
        wk, wv = expect_copies(k, copies), expect_copies(v, copies)
        got = c.reserve(i32(want))
        np.testing.assert_array_equal(got.cpu().numpy(), status)
        same_table(c, t)
        assert torch.equal(k, wk) and torch.equal(v, wv)
        delta = np.where(np.array(status) == 0, rng.integers(-2, most, n), rng.integers(-5, 5, n))
        done = (rng.random(n) < 0.1).astype(np.uint8)
        status = t.commit(delta, done)
        np.testing.assert_array_equal(c.commit(i32(delta), done=torch.as_tensor(done, device=DEV)).cpu().numpy(), status)
        same_table(c, t)
        m = int(rng.integers(1, n + 1))
        src, dst = rng.integers(-1, n + 1, m), rng.integers(-1, n + 1, m)
        status = t.fork(src, dst)
        np.testing.assert_array_equal(c.fork(i32(src), i32(dst)).cpu().numpy(), status)
        same_table(c, t)
        if step % 3 == 2:
            n_live, moves = t.compact()
            wk, wv = expect_copies(k, moves), expect_copies(v, moves)
            assert int(c.compact()) == n_live
            same_table(c, t)
            assert torch.equal(k, wk) and torch.equal(v, wv)


def test_fork_then_write_copies_the_shared_page(saki_lib):
    """4 prompts x 5 responses: every response gets its own last page, one of them the original."""
    t = filled([5, 16, 30, 1] + [0] * 16, 16, 60, 4, np.random.default_rng(1))
    k, v = pool_for(t, dtype=torch.float32)
    c = to_cache(saki_lib, t, k, v)
    src, dst = np.repeat(np.arange(4), 4), np.arange(4, 20)
    assert t.fork(src, dst) == c.fork(i32(src), i32(dst)).cpu().tolist() == [0] * 16
    status, copies = t.reserve([3] * 20)
    assert len(copies) == 4 * 3  # the prompt of 16 tokens ends with its page
    wk = expect_copies(k, copies)
    assert c.reserve(3).cpu().tolist() == status == [0] * 20
    same_table(c, t)
    assert torch.equal(k, wk)


def test_a_pool_too_small_changes_nothing(saki_lib):
    t = filled([7, 8, 3, 0, 20], 8, 9, 4, np.random.default_rng(2))
    k, v = pool_for(t)
    c = to_cache(saki_lib, t, k, v)
    before = k.clone()
    want = [2, 9, 0, 1, 50]  # 1 + 2 + 0 + 1 pages of 2 free ones; the last would need more than 4
    status, copies = t.reserve(want)
    assert status == [1, 1, 0, 1, 2] and not copies
    assert c.reserve(i32(want)).cpu().tolist() == status
    same_table(c, t)
    assert torch.equal(k, before)
    # exactly what is free
    want = [2, 1, 5, 0, 0]
    status, _ = t.reserve(want)
    assert c.reserve(i32(want)).cpu().tolist() == status == [0] * 5
    same_table(c, t)


def test_a_damaged_table_is_reported_and_stays_in_bounds(saki_lib):
    t = filled([5, 9, 12, 4, 6, 7], 8, 40, 4, np.random.default_rng(3))
    t.length[1], t.held[2], t.length[3] = 99, 7, -3
    t.pages[4, 0] = 1000
    k, v = pool_for(t)
    c = to_cache(saki_lib, t, k, v)
    assert c.reserve(2).cpu().tolist() == t.reserve([2] * 6)[0] == [0, 3, 3, 3, 3, 0]
    same_table(c, t)
    assert c.commit(i32([1] * 6)).cpu().tolist() == [0, 3, 3, 3, 0, 0]


def test_long_sequences_and_many_pages(saki_lib):
    """A prompt's pages at once, in order, from a pool of 200,000 with every seventh page taken."""
    n_pages, page = 200000, 8
    t = ocache.Table(3, 30000, n_pages, page)
    t.refs[::7] = 1
    k = torch.zeros(1, n_pages, 1, page, 8, dtype=torch.bfloat16, device=DEV)
    c = to_cache(saki_lib, t, k, k.clone())
    want = [100001, 5, 77777]
    status, _ = t.reserve(want)
    assert c.reserve(i32(want)).cpu().tolist() == status == [0, 0, 0]
    same_table(c, t)
    for b in range(3):
        t.length[b] = want[b]
    assert c.commit(i32(want)).cpu().tolist() == [0, 0, 0]
    same_table(c, t)
    n_live, moves = t.compact()
    assert int(c.compact()) == n_live and len(moves) > 0
    same_table(c, t)
    assert c.commit(done=torch.ones(3, dtype=torch.uint8, device=DEV)).cpu().tolist() == [0, 0, 0]
    t.commit(None, [1, 1, 1])
    same_table(c, t)


@pytest.mark.parametrize("n_pages", [524287, 524288, 600001])
def test_pools_around_half_a_million_pages(saki_lib, n_pages):
    """The free pages of larger pools are searched for in another way; refs need not lie on 16 bytes."""
    rng = np.random.default_rng(n_pages)
    t = ocache.Table(4, 60000, n_pages, 8)
    t.refs[:] = rng.random(n_pages) < 0.8
    k = torch.zeros(1, n_pages, 1, 8, 8, dtype=torch.bfloat16, device=DEV)
    c = to_cache(saki_lib, t, k, k.clone())
    refs = torch.zeros(n_pages + 1, dtype=torch.int32, device=DEV)[1:]
    refs.copy_(c.refs)
    c = saki_lib.PagedKV(c.k, c.v, c.pages, c.length, c.held, refs)
    for want in ([3, 0, 100, 9], [5, 40000 * 8, 1, 1], [0, 0, 0, 10**5 * 8]):
        status, _ = t.reserve(want)
        assert c.reserve(i32(want)).cpu().tolist() == status
        same_table(c, t)
    n_live, moves = t.compact()
    assert int(c.compact()) == n_live
    same_table(c, t)


def test_captured_wave_replays(saki_lib):
    """reserve and commit in a graph, replayed with eager work between: each replay as the oracle."""
    t = filled([5, 30, 17, 0], 8, 40, 12, np.random.default_rng(5))
    t.fork([1], [3])
    k, v = pool_for(t)
    c = to_cache(saki_lib, t, k, v)
    delta = i32([0, 0, 0, 0])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        c.reserve(0)
        c.commit(delta)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            status = c.reserve(6)
            after = c.commit(delta)
    torch.cuda.synchronize()
    rng = np.random.default_rng(6)
    for _ in range(4):
        d = rng.integers(-4, 7, 4)
        delta.copy_(i32(d))
        st, copies = t.reserve([6] * 4)
        wk = expect_copies(k, copies)
        st2 = t.commit(d)
        g.replay()
        torch.cuda.synchronize()
        assert status.cpu().tolist() == st and after.cpu().tolist() == st2
        same_table(c, t)
        assert torch.equal(k, wk)
        c.commit(i32([1, 0, 0, 0]))
        t.commit([1, 0, 0, 0])


def test_other_stream_and_no_sequences(saki_lib):
    t = filled([5, 9], 8, 20, 4, np.random.default_rng(7))
    k, v = pool_for(t)
    c = to_cache(saki_lib, t, k, v)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    st = c.reserve(10, stream=s)
    delta = i32([4, 10])
    s.wait_stream(torch.cuda.current_stream())
    c.commit(delta, stream=s)
    s.synchronize()
    assert st.cpu().tolist() == t.reserve([10, 10])[0]
    t.commit([4, 10])
    same_table(c, t)
    none = saki_lib.PagedKV.alloc(0, 4, 8, 1, 1, 8, 8, device=DEV)
    assert none.reserve(3).numel() == 0 and int(none.compact()) == 0
