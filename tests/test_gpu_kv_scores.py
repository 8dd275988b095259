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


@pytest.mark.parametrize("dtype,dim,lengths,new", [(BF, 128, [70, 5, 200], 2), (F32, 64, [70, 5, 200], 2),
                                                   (BF, 64, [3, 100], 140), (BF, 128, [0, 65], 130), (BF, 256, [40, 9], 3),
                                                   (F32, 256, [40, 9], 20)])
@pytest.mark.parametrize("power", [0, 61, 64])
def test_a_scale_of_zero_weighs_all_alike(saki_lib, dtype, dim, lengths, new, power):
    """Whatever the size of the products (2^power for each factor: past 2^127 together), in 64 bits or not."""
    t, c, q, off, dense = make(saki_lib, dtype, lengths, [new] * len(lengths), 2, 2, dim, 16, dim + new, scale_q=2.0**power)
    for b, (kb, vb) in enumerate(dense):
        kb.mul_(2.0**power)
        put(t, b, c.k, c.v, kb, vb)
    print(f"scale 0: {dtype} dim {dim} power {power}", flush=True)
    run(saki_lib, t, c, q, off, dense, scale=0.0, uniform=new, rows=5)
    run(saki_lib, t, c, q, off, dense, scale=-0.0, uniform=new, window=21, sinks=2, rows=5)
    q[1, 0, 3], q[2, 1, 0] = INF, NAN  # 0 times these is not 0
    dense[0][0][2, 0, 5] = INF
    put(t, 0, c.k, c.v, *dense[0])
    run(saki_lib, t, c, q, off, dense, scale=0.0, uniform=new, rows=5)


@pytest.mark.parametrize("dtype,new", [(BF, 2), (F32, 2), (BF, 140)])
@pytest.mark.parametrize("scale", [2.0**-128, -(2.0**-131), 2.0**-126])
def test_scales_of_the_lowest_size(saki_lib, dtype, new, scale):
    """Scales below 2^-126 on products near 2^126."""
    t, c, q, off, dense = make(saki_lib, dtype, [70, 5], [new] * 2, 2, 2, 64, 16, 5, scale_q=2.0**61)
    for b, (kb, vb) in enumerate(dense):
        kb.mul_(2.0**61)
        put(t, b, c.k, c.v, kb, vb)
    run(saki_lib, t, c, q, off, dense, scale=scale, uniform=new, rows=9)


@pytest.mark.parametrize("dtype,new", [(BF, 2), (F32, 2), (BF, 140)])
def test_the_largest_scale(saki_lib, dtype, new):
    """2^127 on products of -2^-124 .. 2^-124 (none below 2^-126), some of them 0."""
    t, c, q, off, dense = make(saki_lib, dtype, [70, 5], [new] * 2, 2, 2, 64, 16, 6)
    q.copy_(torch.where(q > 0, 2.0**-64, -(2.0**-64)) * torch.where(q.abs() > 0.7, 1.0, 0.5))
    for b, (kb, vb) in enumerate(dense):
        one = torch.nn.functional.one_hot(torch.arange(kb.shape[0], device=DEV) * 7 % 64, 64)[:, None]
        kb.copy_(torch.where(kb > 0, 2.0**-60, -(2.0**-60)) * one)
        kb[::5] = 0
        put(t, b, c.k, c.v, kb, vb)
    run(saki_lib, t, c, q, off, dense, scale=2.0**127, uniform=new, rows=9)
