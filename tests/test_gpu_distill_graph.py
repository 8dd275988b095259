"""A run of the distillation operators together, captured and replayed; two calls at once on two streams."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _calls(saki, seed, n=96, V=5003, D=136, k=24):
    """A teacher's and a student's head on hidden states: the teacher's top logits, the student's divergence from them
    and the cross entropy of the teacher's first choices; (step, outputs, everything it writes)."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    bf = dict(dtype=torch.bfloat16, device=DEV)
    rand = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    x, w = rand(n, D).to(torch.bfloat16), (rand(V, D) / 6).to(torch.bfloat16)
    s, t = saki.alloc_rows(n, V, torch.bfloat16, DEV), saki.alloc_rows(n, V, torch.bfloat16, DEV)
    s.copy_(rand(n, V) * 2)
    t.copy_(rand(n, V) * 2)
    valid = (torch.rand(n, generator=g, device=DEV) < 0.7).to(torch.uint8)
    f32 = dict(dtype=torch.float32, device=DEV)
    top = dict(top_logit=torch.empty(n, k, **f32), top_token=torch.empty(n, k, dtype=torch.int32, device=DEV),
               rest_logit=torch.empty(n, **f32))
    token = torch.empty(n, dtype=torch.int32, device=DEV)
    one = lambda: dict(row_loss=torch.empty(n, **f32), loss_sum=torch.empty(1, dtype=torch.float64, device=DEV))  # noqa: E731
    kl = dict(one(), grad=torch.empty(n, (V + 7) // 8 * 8, **bf)[:, :V])
    ce = dict(one(), logp_token=torch.empty(n, **f32), grad_hidden=torch.empty_like(x), grad_weight=torch.empty_like(w))
    ws = [torch.empty(b, dtype=torch.uint8, device=DEV) for b in
          (saki.workspace_bytes(saki.SAKI_OP_TOP_LOGITS, n, V), saki.workspace_bytes(saki.SAKI_OP_DISTILL_TOP, n, V),
           saki.linear_ce_workspace_bytes(x, w))]

    def step():
        saki.saki_top_logits(t, k, workspace=ws[0], **top)
        saki.saki_distill_top(s, top["top_token"], top["top_logit"], top["rest_logit"], valid_mask=valid, grad_scale=1.0 / n,
                              workspace=ws[1], **kl)
        token.copy_(top["top_token"][:, 0])
        saki.saki_linear_ce(x, w, token, valid_mask=valid, grad_scale=1.0 / n, workspace=ws[2], **ce)

    outs = list(top.values()) + list(kl.values()) + list(ce.values())
    return step, outs, outs + ws + [token]


def _same(got, want):
    return all(np.array_equal(a.cpu().contiguous().view(torch.uint8).numpy(), b.cpu().contiguous().view(torch.uint8).numpy())
               for a, b in zip(got, want))


def test_replays_equal_the_eager_calls(saki_lib):
    step, outs, written = _calls(saki_lib, 1)
    step()
    torch.cuda.synchronize()
    want = [o.clone() for o in outs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert _same(outs, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for rep in range(4):
        for t in written:
            t.fill_(0x5A if t.dtype == torch.uint8 else 77)
        if rep == 2:
            step()  # eager work between replays
            torch.cuda.synchronize()
            assert _same(outs, want)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert _same(outs, want), rep


def test_two_calls_at_once(saki_lib):
    a, b = _calls(saki_lib, 2), _calls(saki_lib, 3, n=200, V=3001, D=64)
    want = []
    for step, outs, _ in (a, b):
        step()
        torch.cuda.synchronize()
        want.append([o.clone() for o in outs])
    sides = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(5):
        for side, (step, _, _) in zip(sides, (a, b)):
            with torch.cuda.stream(side):
                step()
    torch.cuda.synchronize()
    assert _same(a[1], want[0]) and _same(b[1], want[1])


def test_calls_on_another_stream(saki_lib):
    """Outputs and workspaces of a call belong to its stream: allocations of the current one do not touch them while it runs."""
    torch.manual_seed(3)
    n, V, D = 300, 20001, 256
    logits = saki_lib.alloc_rows(n, V, torch.bfloat16, DEV)
    logits.copy_(3 * torch.randn(n, V, device=DEV))
    x, w = torch.randn(n, D, device=DEV).bfloat16(), (torch.randn(V, D, device=DEV) / 16).bfloat16()
    token = torch.randint(0, V, (n,), dtype=torch.int32, device=DEV)
    top = saki_lib.top_logits(logits, 20)
    calls = [lambda **k: saki_lib.top_logits(logits, 20, **k), lambda **k: saki_lib.top_logits(logits[:3], 20, **k),
             lambda **k: saki_lib.distill_top(logits, top["top_token"], top["top_logit"], top["rest_logit"], **k),
             lambda **k: saki_lib.linear_ce(x, w, token, **k)]
    want = [c() for c in calls]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(4):
        got = []
        for c in calls:
            got.append(c(stream=side))
            [torch.full((size,), 255, dtype=torch.uint8, device=DEV) for size in (1 << 12, 1 << 20, 1 << 24, 1 << 27)]
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            for key in a:
                assert torch.equal(a[key].view(torch.uint8), b[key].view(torch.uint8)) if a[key].is_contiguous() else torch.equal(a[key], b[key]), key
