"""Attention over the paged cache where the scores are at the ends of their range."""
import pytest
import torch

from tests.test_gpu_kv_attention import make, put, run

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32
INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("dtype,dim,lengths,new", [
    (BF, 128, [200, 40, 0], 1), (F32, 64, [200, 40, 0], 1), (BF, 64, [9000, 33], 5), (F32, 128, [3000, 33], 3),
    (BF, 256, [5000, 64], 2), (BF, 128, [0, 300, 64], 150), (BF, 64, [4000], 100), (BF, 96, [0, 64], 140)])
def test_no_score_above_minus_infinity_over_values_of_any_kind(saki_lib, dtype, dim, lengths, new):
    """out = 0, lse = -infinity, in blocks that are seen whole and in split ones, also where the values are infinite or NaN."""
    print(f"no score: {dtype} dim {dim} {lengths} new {new}", flush=True)
    t, c, q, off, dense = make(saki_lib, dtype, lengths, [new] * len(lengths), 2, 2, dim, 16, dim + new)
    q.abs_().add_(0.125)
    for b, (kb, vb) in enumerate(dense):
        kb.fill_(-INF)
        for i, x in enumerate((INF, -INF, NAN)):
            vb[i::7] = x
        put(t, b, c.k, c.v, kb, vb)
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device=DEV)
    c.attention(1, q, out=out, lse=lse, n_new=new)
    assert bool((out == 0).all()) and bool((lse == -INF).all())
