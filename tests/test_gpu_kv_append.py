"""Rotary append on the GPU against the oracle in 64 bits.

Bound of an element: the angle is reduced in 64 bits and rounded to a fraction of a turn (2^-26 of a
turn: 9.4e-8 rad); cosine and sine are within 2 steps, their product with the amplitude and the two
products and their sum round 4 times more: in all less than 2^-20 amplitude (|a| + |b|).  Then the
rounding to the stored type, half a step."""
import numpy as np
import pytest
import torch

from oracle import cache as ocache
from tests.kv_cases import filled, to_cache, token_major

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HALF = {torch.bfloat16: 2.0**-8, torch.float32: 2.0**-24}


def make(saki, dtype, lengths, new, hq, hk, dim, page, seed, order="heads", ragged=True, shift=0, spare=0):
    rng = np.random.default_rng(seed)
    t = filled(lengths, page, sum(-(-(L + max(new) + shift) // page) for L in lengths) + 3, 40000 // page, rng,
               extra=max(new) + shift)
    shape = (2, t.refs.size, hk, page, dim)
    k, v = (token_major(*shape, dtype, DEV) if order == "tokens" else torch.empty(shape, dtype=dtype, device=DEV)
            for _ in range(2))
    g = torch.Generator(device=DEV).manual_seed(seed)
    for x in (k, v):
        x.copy_(torch.randn(shape, generator=g, device=DEV))
    offsets = np.concatenate([[0], np.cumsum(new)])
    x = torch.randn(offsets[-1] + spare, hq + 2 * hk, dim, generator=g, device=DEV).to(dtype)
    return t, to_cache(saki, t, k, v), x, offsets


def check(c, t, x, offsets, q_out, before, hq, layer, rope, shift=0):
    hk, dt = c.n_kv_heads, c.dtype
    f = None if rope is None else rope["freq"].cpu().numpy()
    r = 0 if rope is None else rope["rotary_dim"]
    amp = 1.0 if rope is None else rope["amplitude"]
    inter = rope is not None and rope["interleaved"]
    xs = x.double().cpu().numpy()
    wk, wv = before[0].clone(), before[1].clone()
    worst = 0.0
    for b in range(len(offsets) - 1):
        for j in range(offsets[b + 1] - offsets[b]):
            pos, row = int(t.length[b]) + shift + j, offsets[b] + j
            page, slot = int(t.pages[b, pos // t.page_size]), pos % t.page_size
            for h in range(hq + hk):
                src = xs[row, h]
                want = ocache.rope(src, pos, f, r, inter, amp)
                got = (q_out[row, h] if h < hq else c.k[layer, page, h - hq, slot]).double().cpu().numpy()
                size = np.abs(src).copy()
                for i in range(r // 2):
                    a, z = (2 * i, 2 * i + 1) if inter else (i, i + r // 2)
                    size[a] = size[z] = amp * (abs(src[a]) + abs(src[z]))
                tol = 2.0**-20 * size * (np.arange(len(src)) < r) + HALF[dt] * (np.abs(want) + 2.0**-20 * size)
                assert (np.abs(got - want) <= tol).all(), (b, j, h, np.abs(got - want).max())
                if h >= hq:
                    wk[layer, page, h - hq, slot] = c.k[layer, page, h - hq, slot]
            wv[layer, page, :, slot] = x[row, hq + hk:]
    # nothing else changed
    assert torch.equal(c.k, wk) and torch.equal(c.v, wv)


CASES = [  # dtype, dim, rotary, interleaved, page, order
    (torch.bfloat16, 128, 128, False, 16, "heads"), (torch.bfloat16, 128, 64, True, 16, "tokens"),
    (torch.float32, 64, 64, False, 8, "tokens"), (torch.float32, 96, 72, True, 32, "heads"),
    (torch.bfloat16, 80, 20, False, 8, "heads"), (torch.bfloat16, 72, 6, True, 16, "heads"),
    (torch.float32, 8, 2, False, 8, "heads"), (torch.bfloat16, 256, 256, False, 64, "tokens"),
    (torch.float32, 40, 34, False, 8, "heads"), (torch.bfloat16, 16, 0, False, 8, "heads")]


@pytest.mark.parametrize("dtype,dim,rot,inter,page,order", CASES)
def test_ragged_rows(saki_lib, dtype, dim, rot, inter, page, order):
    hq, hk = 6, 2
    new = [1, 0, 5, 2]
    t, c, x, off = make(saki_lib, dtype, [0, 7, page, 3 * page - 1], new, hq, hk, dim, page, rot + dim, order, spare=3)
    rope = saki_lib.rope(rot, interleaved=inter, scaling="ramp", factor=4.0, device=DEV) if rot else None
    before = c.k.clone(), c.v.clone()
    q_out = torch.full((x.shape[0], hq, dim), 7.0, dtype=dtype, device=DEV)
    out = c.append(1, x[:, hq:hq + hk], x[:, hq + hk:], q=x[:, :hq], q_out=q_out, rope=rope,
                   offsets=torch.as_tensor(off, dtype=torch.int32, device=DEV))
    assert out is q_out
    check(c, t, x, off, q_out, before, hq, 1, rope)
    assert (q_out[off[-1]:] == 7.0).all()  # rows behind the last sequence


@pytest.mark.parametrize("rot,inter", [(64, False), (64, True), (12, False)])
def test_uniform_rows_in_place_with_a_shift(saki_lib, rot, inter):
    hq, hk, dim, page = 4, 2, 64, 16
    t, c, x, off = make(saki_lib, torch.bfloat16, [3, 20, 11], [2, 2, 2], hq, hk, dim, page, 5, shift=3)
    rope = saki_lib.rope(rot, interleaved=inter, device=DEV)
    before, x0 = (c.k.clone(), c.v.clone()), x.clone()
    q = x[:, :hq]
    c.append(0, x[:, hq:hq + hk], x[:, hq + hk:], q=q, q_out=q, rope=rope, n_new=2, shift=3)
    check(c, t, x0, off, q, before, hq, 0, rope, shift=3)
    assert torch.equal(x[:, hq:], x0[:, hq:])


def test_far_positions(saki_lib):
    """Positions near 2^20 and 2^29: the angle needs 64 bits.  (The pages before the last are one page.)"""
    page, dim = 1024, 32
    for pos in (2**20 + 12345, 2**29 + 77):
        n = pos // page + 1
        pages = torch.zeros(1, n, dtype=torch.int32, device=DEV)
        k = torch.zeros(1, 2, 1, page, dim, device=DEV)
        c = saki_lib.PagedKV(k, k.clone(), pages, torch.tensor([pos], dtype=torch.int32, device=DEV),
                             torch.tensor([n], dtype=torch.int32, device=DEV), torch.ones(2, dtype=torch.int32, device=DEV))
        x = torch.randn(1, 3, dim, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV)
        rope = saki_lib.rope(dim, device=DEV)
        q = c.append(0, x[:, 1:2], x[:, 2:], q=x[:, :1], rope=rope, n_new=1)
        xs, f = x.double().cpu().numpy(), rope["freq"].cpu().numpy()
        for got, src in ((q[0, 0], xs[0, 0]), (c.k[0, 0, 0, pos % page], xs[0, 1])):
            want = ocache.rope(src, pos, f, dim, False, 1.0)
            size = np.tile(np.abs(src[:dim // 2]) + np.abs(src[dim // 2:]), 2)
            # (the frequency itself is rounded in 64 bits: 2^29 * 0.16 * 2^-53 of a turn, nothing)
            assert (np.abs(got.double().cpu().numpy() - want) <= 2.0**-20 * size + 2.0**-24 * np.abs(want)).all()


def test_rotation_is_undone_by_its_inverse(saki_lib):
    """A rotation by the negative frequencies is the transpose of the rotation: the gradient of a rotated
    query with respect to the query."""
    dim, page = 64, 16
    t, c, x, off = make(saki_lib, torch.float32, [100, 31], [3, 3], 4, 1, dim, page, 8)
    r = saki_lib.rope(48, device=DEV)
    kw = dict(n_new=3)
    q = c.append(0, x[:, 4:5], x[:, 5:], q=x[:, :4], rope=r, **kw)
    w = torch.randn(q.shape, generator=torch.Generator(device=DEV).manual_seed(2), device=DEV)
    back = c.append(0, x[:, 4:5], x[:, 5:], q=w, rope=dict(r, freq=-r["freq"]), **kw)
    # differences: sum(w * rot(q + h e)) - sum(w * rot(q)) = h <back, e>, rot being linear
    e = torch.randn(q.shape, generator=torch.Generator(device=DEV).manual_seed(3), device=DEV)
    moved = c.append(0, x[:, 4:5], x[:, 5:], q=x[:, :4] + e, rope=r, **kw)
    lhs = (w.double() * (moved.double() - q.double())).sum()
    rhs = (back.double() * e.double()).sum()
    scale = (w.double().abs() * (q.double().abs() + moved.double().abs())).sum()
    assert abs(float(lhs - rhs)) <= 2.0**-18 * float(scale)
    # there and back: each way moves an element by at most 2^-20 of its pair's size
    again = c.append(0, x[:, 4:5], x[:, 5:], q=q, rope=dict(r, freq=-r["freq"]), **kw)
    assert (again - x[:, :4]).abs().max() <= 2.0**-17 * x.abs().max()


def test_tokens_without_pages_are_not_written(saki_lib):
    hq, hk, dim, page = 2, 1, 16, 8
    t, c, x, off = make(saki_lib, torch.bfloat16, [6, 8, 3], [4, 4, 4], hq, hk, dim, page, 9)
    c.held[1] = 1     # the tokens behind its 8 have no page
    c.length[2] = -5  # damaged
    c.pages[0, 0] = 10**6
    before = c.k.clone(), c.v.clone()
    q = c.append(0, x[:, hq:hq + hk], x[:, hq + hk:], q=x[:, :hq], n_new=4)
    # sequence 0: positions 6, 7 lie on the page that is none, 8 and 9 on a good one
    bad = torch.tensor([1, 1, 0, 0, 1, 1, 1, 1, 1, 1, 1, 1], dtype=torch.bool, device=DEV)
    assert torch.equal(torch.isnan(q.float()).all(-1).all(-1), bad) and not torch.isnan(q[~bad]).any()
    changed = (c.k != before[0]).any(-1).any(-1).any(2)[0].nonzero()[:, 0].tolist()
    assert changed == [int(t.pages[0, 1])]
    # ranges out of order are empty
    before = c.k.clone()
    for o in ([0, 5, 3, 12], [-1, 2, 2, 2], [0, 0, 99, 99]):
        q.fill_(3.0)
        c.append(0, x[:, hq:hq + hk], x[:, hq + hk:], q=x[:, :hq], q_out=q,
                 offsets=torch.tensor(o, dtype=torch.int32, device=DEV))
        torch.cuda.synchronize()


def test_shared_pages_are_not_written(saki_lib):
    """After a fork both sequences hold the last page: neither may write to it before a reserve."""
    t, c, x, off = make(saki_lib, torch.float32, [11, 0], [2, 0], 2, 1, 16, 8, 4)
    pair = torch.tensor([0], dtype=torch.int32, device=DEV), torch.tensor([1], dtype=torch.int32, device=DEV)
    c.commit(done=torch.tensor([0, 1], dtype=torch.uint8, device=DEV))
    assert c.fork(*pair).tolist() == [0]
    before = c.k.clone()
    x = torch.cat([x, x + 1])
    q = c.append(0, x[:, 2:3], x[:, 3:], q=x[:, :2], n_new=2)
    assert torch.isnan(q).all() and torch.equal(c.k, before)
    assert c.reserve(2).tolist() == [0, 0]
    q = c.append(0, x[:, 2:3], x[:, 3:], q=x[:, :2], n_new=2)
    assert torch.equal(q, x[:, :2])
    for b in range(2):
        page = int(c.pages[b, 1])
        assert torch.equal(c.k[0, page, 0, 3:5], x[2 * b:2 * b + 2, 2])
        assert torch.equal(c.k[:, page, :, :3], before[:, int(t.pages[0, 1]), :, :3])  # the 3 slots they share


def test_many_sequences(saki_lib):
    """Ragged rows of 70,000 sequences (most without any): every row finds its own."""
    n = 70000
    rng = np.random.default_rng(11)
    new = (rng.random(n) < 0.02).astype(np.int64) * rng.integers(1, 4, n)
    off = np.concatenate([[0], np.cumsum(new)])
    page, dim = 8, 8
    k = torch.zeros(1, n, 1, page, dim, device=DEV)
    c = saki_lib.PagedKV(k, k.clone(), torch.arange(n, dtype=torch.int32, device=DEV)[:, None].contiguous(),
                         torch.zeros(n, dtype=torch.int32, device=DEV), torch.ones(n, dtype=torch.int32, device=DEV),
                         torch.ones(n, dtype=torch.int32, device=DEV))
    x = torch.randn(int(off[-1]), 1, dim, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV)
    c.append(0, x, x, offsets=torch.as_tensor(off, dtype=torch.int32, device=DEV))
    seq = torch.as_tensor(np.repeat(np.arange(n), new), device=DEV)
    slot = torch.as_tensor(np.arange(off[-1]) - np.repeat(off[:-1], new), device=DEV)
    want = torch.zeros_like(k)
    want[0, seq, :, slot] = x
    assert torch.equal(c.k, want) and torch.equal(c.v, want)
