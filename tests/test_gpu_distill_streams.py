"""Calls on another stream than the current one: their inputs may be freed as soon as they return."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _inputs(saki):
    g = torch.Generator(device=DEV)
    g.manual_seed(5)
    n, V, D = 300, 20001, 256
    logits = saki.alloc_rows(n, V, torch.bfloat16, DEV)
    logits.copy_(3 * torch.randn(n, V, generator=g, device=DEV))
    x, w = torch.randn(n, D, generator=g, device=DEV).bfloat16(), (torch.randn(V, D, generator=g, device=DEV) / 16).bfloat16()
    token = torch.randint(0, V, (n,), generator=g, dtype=torch.int32, device=DEV)
    valid = (torch.rand(n, generator=g, device=DEV) < 0.7).to(torch.uint8)
    weight = torch.randn(n, generator=g, device=DEV)
    top = saki.top_logits(logits, 20)
    torch.cuda.synchronize()
    return dict(top=[logits], distill=[logits, top["top_token"], top["top_logit"], top["rest_logit"], valid],
                ce=[x, w, token, weight, valid])


def _copy(t):
    """The same rows in memory of its own (logit rows with their pitch)."""
    if t.is_contiguous():
        return t.clone()
    c = torch.empty_strided(t.shape, t.stride(), dtype=t.dtype, device=t.device)
    return c.copy_(t)


@pytest.mark.parametrize("form", ["allocating", "preallocated"])
@pytest.mark.parametrize("name", ["top", "distill", "ce"])
def test_inputs_freed_after_the_call(saki_lib, name, form):
    saki = saki_lib
    held = _inputs(saki)[name]
    f32 = dict(dtype=torch.float32, device=DEV)
    n = held[0].shape[0]
    if form == "allocating":
        call = {"top": lambda a, s: saki.top_logits(a[0], 20, stream=s),
                "distill": lambda a, s: saki.distill_top(*a[:4], valid_mask=a[4], grad_dtype=torch.bfloat16, stream=s),
                "ce": lambda a, s: saki.linear_ce(*a, stream=s)}[name]
    else:  # outputs are kept, inputs and workspace are not
        outs = {"top": lambda: dict(top_logit=torch.zeros(n, 20, **f32), top_token=torch.zeros(n, 20, dtype=torch.int32, device=DEV)),
                "distill": lambda: dict(row_loss=torch.zeros(n, **f32)), "ce": lambda: dict(row_loss=torch.zeros(n, **f32))}[name]
        ws = {"top": lambda a: saki.workspace_bytes(saki.SAKI_OP_TOP_LOGITS, n, a[0].shape[1]),
              "distill": lambda a: saki.workspace_bytes(saki.SAKI_OP_DISTILL_TOP, n, a[0].shape[1]),
              "ce": lambda a: saki.linear_ce_workspace_bytes(a[0], a[1], train=False)}[name]

        def call(a, s):
            out = outs()
            if s is not None:
                s.wait_stream(torch.cuda.current_stream())
            space = torch.empty(max(ws(a), 8), dtype=torch.uint8, device=DEV)
            kw = dict(out, workspace=space, stream=s)
            if name == "top":
                saki.saki_top_logits(a[0], 20, **kw)
            elif name == "distill":
                saki.saki_distill_top(*a[:4], valid_mask=a[4], **kw)
            else:
                saki.saki_linear_ce(*a, **kw)
            return out

    want = call(held, None)
    side = torch.cuda.Stream()
    work = torch.randn(8192, 8192, **f32)
    torch.cuda.synchronize()
    for _ in range(3):
        mine = [_copy(t) for t in held]
        torch.cuda.synchronize()
        with torch.cuda.stream(side):  # keeps the stream busy for some ten milliseconds
            for _ in range(4):
                torch.mm(work, work)
        side.wait_stream(torch.cuda.current_stream())
        got = call(mine, side)
        sizes = [t.untyped_storage().nbytes() for t in mine]
        del mine
        # what takes the inputs' place
        fill = [torch.zeros(s, dtype=torch.uint8, device=DEV) for s in sizes for _ in range(2)]
        torch.cuda.synchronize()
        for key in want:
            a, b = want[key], got[key]
            assert torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8)), key
        del fill, got
