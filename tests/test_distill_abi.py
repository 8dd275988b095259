"""Refusals of the distillation operators, found on the host before a device is touched."""
import ctypes
import os
import re

import pytest
import torch

import paper_2609_36601_amd as saki
from paper_2609_36601_amd import binding as b

OK, NULLPTR, SHAPE, VALUE, DTYPE, ALIGN, WORKSPACE = 0, 1, 2, 3, 4, 5, 6


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(b.LIB_PATH):
        from paper_2609_36601_amd import build
        build.build()
    return saki.load()


def test_header_and_exports_agree(lib):
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "saki_distill.h")).read()
    names = set(re.findall(r"^(?:saki_status|size_t)\s+(saki_\w+)\s*\(", text, re.M))
    assert names == set(b.EXPORTED_DISTILL) and all(hasattr(lib, n) for n in names)


def top(lib, **kw):
    a = dict(logits=256, dtype=b.SAKI_BF16, n=4, V=1000, stride=1000, k=8, tau=1.0, top_logit=256, top_token=256, top_stride=8,
             rest=None, status=None, ws=None, ws_bytes=0)
    a.update(kw)
    return lib.saki_top_logits(*a.values(), None)


@pytest.mark.parametrize("code,kw", [
    (DTYPE, dict(dtype=2)), (DTYPE, dict(dtype=-1)), (SHAPE, dict(n=-1)), (SHAPE, dict(n=2**31)), (SHAPE, dict(V=0)),
    (SHAPE, dict(V=b.SAKI_MAX_VOCAB + 1, stride=2**22)), (SHAPE, dict(stride=999)), (SHAPE, dict(k=0)), (SHAPE, dict(k=257)),
    (SHAPE, dict(k=8, V=7)), (SHAPE, dict(top_stride=7)), (VALUE, dict(tau=0.0)), (VALUE, dict(tau=-1.0)),
    (VALUE, dict(tau=float("nan"))), (VALUE, dict(tau=float("inf"))), (VALUE, dict(tau=2.0**-65)), (NULLPTR, dict(logits=None)),
    (NULLPTR, dict(top_logit=None)), (NULLPTR, dict(top_token=None)), (ALIGN, dict(logits=264)), (ALIGN, dict(stride=1004)),
    (ALIGN, dict(top_logit=258)), (ALIGN, dict(rest=258)), (WORKSPACE, dict(V=120000, stride=120000)),
    (WORKSPACE, dict(V=120000, stride=120000, ws=256, ws_bytes=100)), (ALIGN, dict(V=120000, stride=120000, ws=264, ws_bytes=1 << 30)),
    (OK, dict(n=0, logits=None, top_logit=None, top_token=None))])
def test_top_logits(lib, code, kw):
    assert top(lib, **kw) == code


def distill(lib, list_kw={}, **kw):
    rows = dict(token=256, logit=256, rest_logit=256, stride=8, k=8, reserved=0)
    rows.update(list_kw)
    a = dict(student=256, dtype=b.SAKI_BF16, n=4, V=1000, stride=1000, list=ctypes.byref(b.SakiTopList(**rows)), tau=1.0,
             direction=0, valid=None, scale=1.0, row_loss=256, loss_sum=256, grad=256, grad_dtype=0, grad_stride=1000, status=None,
             ws=256, ws_bytes=1 << 20)
    a.update(kw)
    return lib.saki_distill_top(*a.values(), None)


@pytest.mark.parametrize("code,kw", [
    (DTYPE, dict(dtype=7)), (SHAPE, dict(n=-3)), (SHAPE, dict(n=2**31)), (SHAPE, dict(V=0)), (SHAPE, dict(stride=992)),
    (NULLPTR, dict(list=None)), (VALUE, dict(list_kw=dict(reserved=1))), (SHAPE, dict(list_kw=dict(k=0))),
    (SHAPE, dict(list_kw=dict(k=257, stride=300))), (SHAPE, dict(list_kw=dict(stride=7))), (VALUE, dict(direction=2)),
    (VALUE, dict(scale=float("inf"))), (VALUE, dict(tau=0.0)), (DTYPE, dict(grad_dtype=5)), (SHAPE, dict(grad_stride=999)),
    (ALIGN, dict(grad=260)), (ALIGN, dict(grad_stride=1001)), (ALIGN, dict(student=250)), (NULLPTR, dict(student=None)),
    (VALUE, dict(grad=256, grad_dtype=0, student=256)), (VALUE, dict(grad_dtype=1, grad_stride=1008)),
    (NULLPTR, dict(grad=1024, list_kw=dict(token=None))), (NULLPTR, dict(grad=1024, list_kw=dict(logit=None))),
    (NULLPTR, dict(grad=1024, direction=1, list_kw=dict(rest_logit=None))), (ALIGN, dict(grad=1024, list_kw=dict(token=257))),
    (ALIGN, dict(grad=1024, row_loss=257)), (ALIGN, dict(grad=1024, loss_sum=260)), (WORKSPACE, dict(grad=1024, ws=None)),
    (WORKSPACE, dict(grad=1024, ws_bytes=511)), (ALIGN, dict(grad=1024, ws=260)), (OK, dict(n=0, student=None, loss_sum=None))])
def test_distill_top(lib, code, kw):
    assert distill(lib, **kw) == code


def ce(lib, head_kw={}, args_kw={}, ws=256, ws_bytes=1 << 40):
    head = dict(hidden=256, weight=256, hidden_stride=64, weight_stride=64, n_rows=4, vocab=1000, hidden_size=64,
                dtype=b.SAKI_BF16, reserved=0)
    head.update(head_kw)
    args = dict(token=256, row_weight=None, valid_mask=None, grad_scale=1.0, reserved=0, row_loss=256, logp_token=256, loss_sum=256,
                row_status=None, grad_hidden=256, grad_weight=256, grad_hidden_stride=64, grad_weight_stride=64)
    args.update(args_kw)
    return lib.saki_linear_ce(ctypes.byref(b.SakiHead(**head)), ctypes.byref(b.SakiCEArgs(**args)), ws, ws_bytes, None)


@pytest.mark.parametrize("code,head,args", [
    (DTYPE, dict(dtype=3), {}), (VALUE, dict(reserved=1), {}), (SHAPE, dict(n_rows=-1), {}), (SHAPE, dict(n_rows=2**23), {}),
    (SHAPE, dict(vocab=0), {}), (SHAPE, dict(vocab=b.SAKI_MAX_VOCAB + 1), {}), (SHAPE, dict(hidden_size=0), {}),
    (SHAPE, dict(hidden_size=60), {}), (SHAPE, dict(hidden_size=b.SAKI_MAX_HIDDEN + 8, hidden_stride=2**20, weight_stride=2**20), {}),
    (SHAPE, dict(hidden_stride=56), {}), (SHAPE, dict(weight_stride=56), {}), (SHAPE, dict(weight_stride=2**22), {}),
    (VALUE, {}, dict(reserved=1)), (VALUE, {}, dict(grad_scale=float("nan"))), (SHAPE, {}, dict(grad_hidden_stride=56)),
    (SHAPE, {}, dict(grad_weight_stride=2**22)), (NULLPTR, dict(hidden=None), {}), (NULLPTR, dict(weight=None), {}),
    (NULLPTR, {}, dict(token=None)), (ALIGN, dict(hidden=264), {}), (ALIGN, dict(weight=264), {}), (ALIGN, dict(hidden_stride=68), {}),
    (ALIGN, {}, dict(grad_hidden=264)), (ALIGN, {}, dict(grad_weight=264)), (ALIGN, {}, dict(grad_weight_stride=68)),
    (ALIGN, {}, dict(token=258)), (ALIGN, {}, dict(row_loss=258)), (ALIGN, {}, dict(loss_sum=260)),
    (OK, dict(n_rows=0, hidden=None, weight=None), dict(token=None, grad_weight=None, loss_sum=None))])
def test_linear_ce(lib, code, head, args):
    assert ce(lib, head, args) == code


def test_linear_ce_workspace(lib):
    head = dict(hidden_stride=64, weight_stride=64, n_rows=4, vocab=1000, hidden_size=64, dtype=b.SAKI_BF16)
    size = lambda grads, **kw: lib.saki_linear_ce_workspace_bytes(ctypes.byref(b.SakiHead(**dict(head, **kw))), grads)  # noqa: E731
    sizes = [size(g) for g in range(4)]
    assert 0 < sizes[0] < sizes[2] < sizes[3] and sizes[1] == sizes[3]
    assert size(4) == size(-1) == size(3, n_rows=0) == size(3, hidden_size=63) == 0
    assert ce(lib, ws_bytes=sizes[3] - 1) == WORKSPACE and ce(lib, ws=None) == WORKSPACE and ce(lib, ws=128) == ALIGN
    # the logits of the largest calls are never there as a whole
    big = dict(n_rows=2**23 - 1, vocab=151936, hidden_size=4096, hidden_stride=4096, weight_stride=4096)
    assert 0 < size(3, **big) < 2**23 * 151936 * 2 // 4


def test_binding_refuses():
    f, i = torch.zeros(4, 16), torch.zeros(4, dtype=torch.int32)
    for call in (lambda: saki.top_logits(f, 2), lambda: saki.distill_top(f, i.view(4, 1), f[:, :1]), lambda: saki.linear_ce(f, f, i)):
        with pytest.raises(ValueError, match="on cpu"):
            call()
    with pytest.raises(ValueError, match="requires a gradient"):
        saki.top_logits(f.clone().requires_grad_(), 2)
    with pytest.raises(ValueError, match="requires a gradient"):
        saki.linear_ce(f, f.clone().requires_grad_(), i)
    with pytest.raises(ValueError, match="one dtype"):
        saki.linear_ce(f, f.to(torch.bfloat16), i)
