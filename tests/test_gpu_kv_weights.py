"""The weights of the bf16 attention hold 2^-17 (two bf16 numbers, far less than the output's rounding) for up to 32 rows
(tokens times query heads of a key head) a sequence, and for heads past 128 elements.

Queries are small here, so that the scores' own errors (derived in test_gpu_kv_attention.py: e) are below 2^-17, and the bound of
an element is (2 e + 2^-21 + (n + 16) 2^-24 + 2^-17) sum w |v| and the output's half step, 2^-8 |o|: one value of a
thousand taken from another token is beyond it."""
import numpy as np
import pytest
import torch

from oracle import cache as ocache
from tests.test_gpu_kv_attention import make, put

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32
INF = float("inf")


@pytest.mark.parametrize("dim,group,hk,page,lengths,new,window,order", [
    (128, 2, 2, 16, [0, 31, 130, 517], 1, 0, "heads"), (128, 4, 2, 32, [40, 700], 7, 0, "tokens"),
    (64, 1, 2, 8, [33, 900], 1, 0, "tokens"), (64, 4, 1, 16, [300, 90], 8, 0, "heads"), (64, 8, 1, 16, [300, 90], 4, 100, "heads"),
    (80, 7, 1, 32, [517, 3], 2, 0, "heads"), (256, 4, 1, 64, [300, 65], 5, 0, "tokens"), (136, 3, 2, 16, [200], 30, 0, "heads"),
    (128, 4, 1, 16, [9001], 2, 0, "heads"), (64, 1, 1, 64, [20011], 1, 3000, "heads"), (8, 3, 2, 8, [150, 7], 3, 0, "heads")])
def test_weights(saki_lib, dim, group, hk, page, lengths, new, window, order):
    print(f"weights: dim {dim} group {group} {lengths} new {new}", flush=True)
    t, c, q, off, dense = make(saki_lib, BF, lengths, [new] * len(lengths), group, hk, dim, page, dim + new, order, scale_q=2.0**-7)
    scale = dim ** -0.5
    out = c.attention(1, q, n_new=new, window=window, sinks=3)
    for b, (kb, vb) in enumerate(x for x in dense):
        kb, vb = kb.double().cpu().numpy(), vb.double().cpu().numpy()
        qb = q[off[b]:off[b + 1]].double().cpu().numpy()
        pos = lengths[b] + np.arange(new)
        want, _ = ocache.attention(qb, kb, vb, pos, scale, window, 3)
        size, _ = ocache.attention(qb, kb, np.abs(vb), pos, scale, window, 3)
        e = scale * (dim + 8) * 2.0**-24 * np.einsum("ihd,d->ih", np.abs(qb), np.abs(kb).max((0, 1)))
        rel = 2 * e + 2.0**-21 + (kb.shape[0] + 16) * 2.0**-24 + 2.0**-17
        err = np.abs(out[off[b]:off[b + 1]].double().cpu().numpy() - want)
        tol = rel[..., None] * size + 2.0**-8 * np.abs(want)
        assert (err <= tol).all(), (b, (err / tol).max())


@pytest.mark.parametrize("dtype,dim,lengths,new", [(BF, 128, [200, 40], 1), (BF, 64, [200, 40], 7), (F32, 64, [200, 40], 2),
                                                   (BF, 256, [100, 64], 2), (BF, 128, [300, 0], 150), (BF, 128, [9000], 2)])
def test_infinite_values_that_are_seen(saki_lib, dtype, dim, lengths, new):
    """An element over one infinity is that infinity, over two of them NaN, also in blocks that are seen whole."""
    t, c, q, off, dense = make(saki_lib, dtype, lengths, [new] * len(lengths), 2, 2, dim, 16, dim + new, scale_q=0.25)
    before = c.attention(1, q, n_new=new)
    for b, (kb, vb) in enumerate(dense):
        vb[0, :, 1], vb[0, :, 2] = INF, -INF
        if vb.shape[0] > 20:
            vb[17, :, 3], vb[3, :, 4], vb[19, :, 4] = -INF, INF, -INF
        put(t, b, c.k, c.v, kb, vb)
    out = c.attention(1, q, n_new=new)
    for b, L in enumerate(lengths):
        o, rest = out[off[b]:off[b + 1]], before[off[b]:off[b + 1]]
        pos = L + torch.arange(new, device=DEV)
        assert (o[:, :, 1] == INF).all() and (o[:, :, 2] == -INF).all()
        assert ((o[:, :, 3] == -INF) == (pos >= 17)[:, None]).all()
        assert (torch.isnan(o[:, :, 4]) == (pos >= 19)[:, None]).all()
        assert ((o[:, :, 4] == INF) == ((pos >= 3) & (pos < 19))[:, None]).all()
        assert torch.equal(o[:, :, 5:], rest[:, :, 5:]) and torch.equal(o[:, :, 0], rest[:, :, 0])
