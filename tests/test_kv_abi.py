"""Refusals of the paged key-value cache, found on the host before a device is touched."""
import ctypes
import os
import re

import pytest
import torch

import paper_2609_36601_amd as saki
from paper_2609_36601_amd import binding as b


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(b.LIB_PATH):
        from paper_2609_36601_amd import build
        build.build()
    return saki.load()


def test_header_and_exports_agree(lib):
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "saki_kv.h")).read()
    names = set(re.findall(r"^saki_status\s+(saki_\w+)\s*\(", text, re.M))
    assert names == set(b.EXPORTED_KV) and all(hasattr(lib, n) for n in names)


def table(**kw):
    t = dict(n_seq=4, max_pages=10, n_pages=100, page_size=16, reserved=0, pages=64, length=64, held=64, refs=64)
    t.update(kw)
    return ctypes.byref(b.SakiKVTable(**t))


def pool(**kw):
    p = dict(k=64, v=64, dtype=b.SAKI_BF16, n_kv_heads=2, head_dim=64, reserved=0, n_layers=3, token_stride=64,
             head_stride=64 * 16, page_stride=2 * 64 * 16, layer_stride=100 * 2 * 64 * 16)
    p.update(kw)
    return ctypes.byref(b.SakiKVPool(**p))


def tokens(**kw):
    t = dict(offsets=None, n_tokens=4, n_new=1, shift=0)
    t.update(kw)
    return ctypes.byref(b.SakiKVTokens(**t))


def heads(data=64, token_stride=256, head_stride=64):
    return ctypes.byref(b.SakiKVHeads(data, token_stride, head_stride))


BAD_TABLES = [(dict(reserved=1), 3), (dict(n_seq=-1), 2), (dict(n_seq=2**24 + 1), 2), (dict(n_pages=0), 2),
              (dict(n_pages=2**30 + 1), 2), (dict(page_size=4), 2), (dict(page_size=24), 2), (dict(page_size=2048), 2),
              (dict(page_size=0), 2), (dict(page_size=-16), 2), (dict(max_pages=0), 2), (dict(max_pages=2**26 + 1), 2),
              (dict(pages=0), 1), (dict(length=0), 1), (dict(held=0), 1), (dict(refs=0), 1), (dict(refs=66), 5)]
BAD_POOLS = [(dict(dtype=2), 4), (dict(reserved=3), 3), (dict(n_kv_heads=0), 2), (dict(n_kv_heads=1025), 2),
             (dict(head_dim=60), 2), (dict(head_dim=0), 2), (dict(head_dim=264), 2), (dict(n_layers=0), 2),
             (dict(n_layers=65537), 2), (dict(k=0), 1), (dict(v=0), 1), (dict(v=72), 5), (dict(token_stride=60), 5),
             (dict(token_stride=56), 2), (dict(head_stride=64 * 15), 2), (dict(page_stride=64 * 16), 2),
             (dict(layer_stride=64), 2), (dict(layer_stride=-64), 5), (dict(page_stride=2**62), 5),
             (dict(token_stride=2**26, head_stride=64, page_stride=128, layer_stride=2**31), 2),  # a page beyond 2^31 bytes
             # keys head-major and tokens inside, but pages closer than their tokens
             (dict(token_stride=128, head_stride=64, page_stride=1024), 2)]


def all_calls(lib, t, p):
    n = tokens()
    yield "reserve", lib.saki_kv_reserve(t, p, None, 1, None, 64, 1 << 30, None)
    yield "compact", lib.saki_kv_compact(t, p, None, 64, 1 << 30, None)
    yield "append", lib.saki_kv_append(t, p, 0, n, None, 0, None, None, heads(), heads(), None)
    yield "attention", lib.saki_kv_attention(t, p, 0, n, 2, heads(), heads(), None, 1.0, 0, 0, 64, 1 << 30, None)


@pytest.mark.parametrize("kw,code", BAD_TABLES)
def test_bad_tables(lib, kw, code):
    for name, st in all_calls(lib, table(**kw), pool()):
        assert st == code, name
    assert lib.saki_kv_commit(table(**kw), 64, None, None, None) == code
    assert lib.saki_kv_fork(table(**kw), 1, 64, 64, None, None) == code
    assert lib.saki_last_error()


@pytest.mark.parametrize("kw,code", BAD_POOLS)
def test_bad_pools(lib, kw, code):
    for name, st in all_calls(lib, table(), pool(**kw)):
        assert st == code, (name, lib.saki_last_error())


def test_null_descriptors(lib):
    assert [st for _, st in all_calls(lib, None, pool())] == [1] * 4
    assert [st for _, st in all_calls(lib, table(), None)] == [1] * 4


def test_reserve_commit_fork_compact(lib):
    t, p = table(), pool()
    need = lib.saki_workspace_bytes(b.SAKI_OP_KV_RESERVE, 4, 100)
    assert need >= 4 * 28 + 3 * 400
    assert lib.saki_kv_reserve(t, p, None, -1, None, 64, need, None) == 3
    assert lib.saki_kv_reserve(t, p, 66, 0, None, 64, need, None) == 5
    assert lib.saki_kv_reserve(t, p, None, 1, None, None, need, None) == 6
    assert lib.saki_kv_reserve(t, p, None, 1, None, 64, need - 1, None) == 6
    assert lib.saki_kv_reserve(t, p, None, 1, None, 72, need, None) == 5
    assert lib.saki_kv_commit(t, None, None, None, None) == 1
    assert lib.saki_kv_commit(t, 66, None, None, None) == 5
    assert lib.saki_kv_fork(t, -1, 64, 64, None, None) == 2
    assert lib.saki_kv_fork(t, 5, 64, 64, None, None) == 2
    assert lib.saki_kv_fork(t, 2, None, 64, None, None) == 1
    assert lib.saki_kv_fork(t, 2, 64, 65, None, None) == 5
    need = lib.saki_workspace_bytes(b.SAKI_OP_KV_COMPACT, 4, 100)
    assert lib.saki_kv_compact(t, p, 66, 64, need, None) == 5
    assert lib.saki_kv_compact(t, p, None, None, need, None) == 6
    assert lib.saki_kv_compact(t, p, None, 64, need - 1, None) == 6
    # nothing to do: no device is needed
    empty = dict(n_seq=0, pages=0, length=0, held=0, refs=0)
    assert lib.saki_kv_reserve(table(**empty), p, None, 1, None, None, 0, None) == 0
    assert lib.saki_kv_commit(table(**empty), 64, None, None, None) == 0
    assert lib.saki_kv_fork(t, 0, None, None, None, None) == 0
    assert lib.saki_kv_compact(table(**empty), p, None, None, 0, None) == 0
    assert lib.saki_last_error() == b""


def test_tokens_and_rows(lib):
    t, p, h = table(), pool(), heads()

    def append(n=None, layer=0, rope=None, hq=2, q=h, qo=h, k=h, v=h):
        return lib.saki_kv_append(t, p, layer, n or tokens(), rope, hq, q, qo, k, v, None)

    def attend(n=None, layer=0, hq=2, q=h, out=h, lse=None, scale=1.0, window=0, sinks=0, ws=64, ws_bytes=1 << 30):
        return lib.saki_kv_attention(t, p, layer, n or tokens(), hq, q, out, lse, scale, window, sinks, ws, ws_bytes, None)

    for f in (append, attend):
        assert f(layer=-1) == 2 and f(layer=3) == 2
        assert f(n=tokens(n_tokens=-1)) == 2 and f(n=tokens(n_tokens=2**31)) == 2
        assert f(n=tokens(n_tokens=5)) == 2 and f(n=tokens(n_new=-1, n_tokens=-4)) == 2
        assert f(n=tokens(shift=-1)) == 3 and f(n=tokens(shift=2**30 + 1)) == 3
        assert f(n=tokens(offsets=66)) == 5
        assert f(hq=-2) == 2 and f(hq=65538) == 2
        assert f(q=heads(data=0)) == 1 and f(q=heads(data=72)) == 5
        assert f(q=heads(token_stride=100)) == 5 and f(q=heads(head_stride=-64)) == 5
    assert lib.saki_kv_append(t, p, 0, None, None, 2, h, h, h, h, None) == 1
    assert append(qo=None) == 1 and append(q=None, qo=h) == 1 and append(hq=0) == 1 and append(q=None, qo=None) == 1
    assert append(n=tokens(n_tokens=0, n_new=0), hq=0, q=None, qo=None) == 0
    assert append(k=None) == 1 and append(v=heads(data=0)) == 1 and append(k=heads(data=65)) == 5
    assert append(qo=heads(token_stride=64)) == 2                       # rows of the output overlap
    assert append(qo=heads(token_stride=0)) == 2
    r = dict(freq=64, rotary_dim=64, interleaved=0, amplitude=1.0)

    def rope(**kw):
        return append(rope=ctypes.byref(b.SakiKVRope(**dict(r, **kw))))

    assert rope(rotary_dim=66) == 2 and rope(rotary_dim=31) == 2 and rope(rotary_dim=-2) == 2
    assert rope(interleaved=2) == 3 and rope(amplitude=float("nan")) == 3 and rope(amplitude=float("inf")) == 3
    assert rope(freq=0) == 1 and rope(freq=68) == 5
    assert attend(hq=3) == 2 and attend(hq=0) == 2
    assert attend(scale=float("nan")) == 3 and attend(scale=float("inf")) == 3
    assert attend(window=-1) == 3 and attend(sinks=-1) == 3 and attend(lse=66) == 5
    assert attend(n=tokens(n_tokens=2**31 - 4, n_new=2**29 - 1)) == 2
    assert attend(out=None) == 1 and attend(out=heads(head_stride=32)) == 2
    assert attend(ws=None) == 6 and attend(ws_bytes=100) == 6 and attend(ws=72) == 5
    assert attend(n=tokens(n_tokens=0, n_new=0), ws=None) == 0
    assert lib.saki_workspace_bytes(b.SAKI_OP_KV_ATTENTION, 8, 64) < lib.saki_workspace_bytes(
        b.SAKI_OP_KV_ATTENTION, 800, 128) < 1 << 28


def test_handle_refuses_what_does_not_fit():
    """PagedKV's own checks (tensors of the wrong shape, type or layout), on the CPU."""
    def cache(**kw):
        a = dict(n_seq=3, max_pages=4, n_pages=8, n_layers=2, n_kv_heads=2, page_size=8, head_dim=16, device="cpu")
        return saki.PagedKV.alloc(**dict(a, **kw))

    c = cache()
    k = torch.zeros(3, 2, 16, dtype=torch.bfloat16)
    q = torch.zeros(3, 4, 16, dtype=torch.bfloat16)
    i32 = torch.zeros(3, dtype=torch.int32)
    bad = [lambda: c.reserve(i32.long()), lambda: c.reserve(i32[:2]), lambda: c.commit(i32, done=i32),
           lambda: c.fork(i32, i32[:2]), lambda: c.append(0, k[:2], k, n_new=1), lambda: c.append(0, k, k),
           lambda: c.append(0, k, k, n_new=2), lambda: c.append(0, k, k, n_new=1, offsets=i32),
           lambda: c.append(0, k, k, offsets=i32), lambda: c.append(0, k.float(), k, n_new=1),
           lambda: c.append(0, k, k, n_new=1, shift=-1), lambda: c.append(0, k[:, :1], k, n_new=1),
           lambda: c.append(0, k, k, n_new=1, rope=dict(freq=torch.zeros(3), rotary_dim=6, interleaved=False,
                                                        amplitude=1.0)),
           lambda: c.attention(0, q.float(), n_new=1), lambda: c.attention(0, q[:, :, :8], n_new=1),
           lambda: c.attention(0, q, n_new=1, lse=torch.zeros(3, 2)),
           lambda: saki.PagedKV(c.k, c.v[:1], c.pages, c.length, c.held, c.refs),
           lambda: saki.PagedKV(c.k, c.v, c.pages, c.length, c.held, c.refs[:4]),
           lambda: saki.PagedKV(c.k, c.v, c.pages.t(), c.length, c.held, c.refs),
           lambda: cache(dtype=torch.float16)]
    for i, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            pytest.fail(str(i))
    for kw in (dict(rotary_dim=5), dict(rotary_dim=-2), dict(base=0.0), dict(scaling="half"), dict(factor=-1.0),
               dict(scaling="ramp", fast=1.0, slow=2.0)):
        with pytest.raises(ValueError):
            saki.rope(**dict(dict(rotary_dim=8, device="cpu"), **kw))


def test_streams_of_other_devices_are_refused():
    from types import SimpleNamespace
    c = saki.PagedKV.alloc(2, 4, 8, 1, 1, 8, 64, device="cpu")
    with pytest.raises(ValueError, match="a stream of cuda:1"):
        c.reserve(1, stream=SimpleNamespace(device=torch.device("cuda:1")))


def test_rope_scalings():
    f = saki.rope(64, device="cpu")
    assert f["freq"].shape == (32,) and f["amplitude"] == 1.0
    assert abs(float(f["freq"][0]) - 0.15915494309189535) < 1e-16
    lin = saki.rope(64, scaling="linear", factor=8.0, device="cpu")
    assert torch.equal(lin["freq"], f["freq"] / 8)
    ramp = saki.rope(64, scaling="ramp", factor=8.0, length=4096, device="cpu")
    turns = 4096 * f["freq"]
    assert torch.equal(ramp["freq"][turns >= 32], f["freq"][turns >= 32])
    assert torch.allclose(ramp["freq"][turns <= 1], f["freq"][turns <= 1] / 8, rtol=1e-15)
    between = (turns > 1) & (turns < 32)
    assert between.any() and (ramp["freq"][between] < f["freq"][between]).all()
    assert (ramp["freq"][between] > f["freq"][between] / 8).all()
    assert saki.rope(0, device="cpu")["freq"].numel() == 0


def test_more_rows_than_a_launch_takes(lib):
    t, p, h = table(), pool(), heads()
    for n in (2**22, 2**29 - 1):
        rows = tokens(n_tokens=4 * n, n_new=n)
        assert lib.saki_kv_append(t, p, 0, rows, None, 2, h, h, h, h, None) == 2
    assert lib.saki_kv_fork(table(n_seq=2**24), 2**20 + 1, 64, 64, None, None) == 2  # pairs are compared with each other
    rows = tokens(n_tokens=2**30, n_new=2**28)
    assert lib.saki_kv_attention(t, p, 0, rows, 2, h, h, None, 1.0, 0, 0, 64, 1 << 30, None) == 2


def test_raw_calls_refuse_strided_arrays(lib):
    import torch
    every_other = torch.zeros(8, dtype=torch.int32)[::2]
    t, p = b.SakiKVTable(4), b.SakiKVPool()
    with pytest.raises(ValueError, match="contiguous"):
        b.saki_kv_commit(t, every_other)
    with pytest.raises(ValueError, match="contiguous"):
        b.saki_kv_reserve(t, p, every_other)
    with pytest.raises(ValueError, match="contiguous"):
        b.saki_kv_fork(t, every_other, every_other)
