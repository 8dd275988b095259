"""Performance cases of distillation from a teacher's top logits and of cross entropy from hidden states.

Each case is one pass as a training or scoring step makes it.  A case is a dict of plain values:

  kind      top      the k largest logits of every row with their tokens, and the log-sum-exp of the others:
                     what a teacher's pass leaves for the student
            distill  divergence between the student's row and a teacher's k top logits (with `rest`: and one
                     bucket for all other tokens), and its gradient with respect to the student's logits
            ce       cross entropy of softmax(hidden @ weight^T), without the logits in memory; `train`: with the
                     gradients of hidden and weight
  rows      positions
  V         vocabulary
  k         listed tokens a row
  D         elements of a hidden state
  dtype     bf16 | f32: of the logits (top, distill), of hidden, weight and their gradients (ce)
  grad      bf16 | f32: of the gradient (distill)
  tau       temperature of both sides
  reverse   KL(student || teacher) instead of KL(teacher || student)
  ragged    rows that list fewer than k tokens (-1 behind the last)
  masked    a padded batch: about a third of the rows take no part
  weighted  a weight of its own for every row, of either sign (ce)
"""
import math

import torch

own = False

DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
F64 = torch.float64
INF = float("inf")
MOST_TOP = 4096 * 151936  # entries of the largest listed case of each kind
MOST_DISTILL = 8192 * 151936
MOST_CE = 8192 * 4096 * 151936


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------
def listed():
    return [
        # a serving step that records its teacher's top logits: a few rows, latency
        dict(name="top_step_16", kind="top", rows=16, V=151936, k=20, dtype="bf16", tau=1.0),
        # a teacher's pass over a training batch
        dict(name="top_batch_4096", kind="top", rows=4096, V=151936, k=64, dtype="bf16", tau=1.0),
        # odd sizes, 32 bits, long lists
        dict(name="top_ragged_f32", kind="top", rows=777, V=49999, k=200, dtype="f32", tau=2.0),
        # a unit-sized training batch: launches
        dict(name="distill_tiny_f32", kind="distill", rows=256, V=4096, k=8, dtype="f32", grad="f32", tau=1.0, rest=False,
             reverse=False, ragged=False, masked=False),
        # the training step at the full vocabulary
        dict(name="distill_train_8192", kind="distill", rows=8192, V=151936, k=64, dtype="bf16", grad="bf16", tau=1.0,
             rest=True, reverse=False, ragged=False, masked=False),
        # a padded on-policy batch: reverse divergence, odd vocabulary, short lists, gradient in 32 bits
        dict(name="distill_reverse_ragged", kind="distill", rows=3001, V=49999, k=33, dtype="bf16", grad="f32", tau=1.0,
             rest=True, reverse=True, ragged=True, masked=True),
        # the log-probabilities of one decoded batch: the head's weight is read once
        dict(name="ce_score_8", kind="ce", rows=8, V=32000, D=2048, dtype="bf16", train=False, masked=False,
             weighted=False),
        # scoring a batch of responses
        dict(name="ce_score_4096", kind="ce", rows=4096, V=151936, D=2048, dtype="bf16", train=False, masked=False,
             weighted=False),
        # a short training batch: few rows against the whole head
        dict(name="ce_train_200", kind="ce", rows=200, V=32000, D=1024, dtype="bf16", train=True, masked=False,
             weighted=False),
        # a padded batch with weights of either sign (the routed objective's), odd sizes
        dict(name="ce_train_masked", kind="ce", rows=3001, V=49999, D=2056, dtype="bf16", train=True, masked=True,
             weighted=True),
        # 32 bits
        dict(name="ce_train_f32", kind="ce", rows=1024, V=32000, D=1024, dtype="f32", train=True, masked=False,
             weighted=False),
        # a large training batch at the full vocabulary
        dict(name="ce_train_8192", kind="ce", rows=8192, V=151936, D=4096, dtype="bf16", train=True, masked=False,
             weighted=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["top", "distill", "distill", "ce", "ce", "ce"])
    V = _log_int(rng, 500, 151936)
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind == "ce":
        c = dict(kind=kind, V=V, D=8 * _log_int(rng, 8, 512), dtype=dtype, train=rng.random() < 0.7,
                 masked=rng.random() < 0.4, weighted=rng.random() < 0.4)
        most = MOST_CE // (V * c["D"])
        c["rows"] = max(1, min(_log_int(rng, 1, 8192), most if dtype == "bf16" else most // 10))
        return c
    c = dict(kind=kind, V=V, k=_log_int(rng, 1, 256), dtype=dtype, tau=rng.choice([1.0, 1.0, rng.uniform(0.5, 4.0)]))
    if kind == "top":
        c["rows"] = max(1, min(_log_int(rng, 1, 4096), MOST_TOP // V // (1 if dtype == "bf16" else 2)))
        return c
    c.update(grad=rng.choice(["bf16", "f32"]), rest=rng.random() < 0.7, ragged=rng.random() < 0.4,
             masked=rng.random() < 0.4)
    c["reverse"] = c["rest"] and rng.random() < 0.5
    size = (2 if dtype == "bf16" else 4) + (2 if c["grad"] == "bf16" else 4)
    c["rows"] = max(1, min(_log_int(rng, 1, 8192), MOST_DISTILL * 4 // size // V))
    return c


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _gen(seed, salt=0):
    g = torch.Generator(device=DEV)
    g.manual_seed((seed * 1000003 + salt * 7919 + 977) % (1 << 62))
    return g


def _rows(n, V, dtype):
    """[n, V] with a row pitch of whole 16 bytes, as logits lie in memory."""
    per = 16 // torch.empty(0, dtype=dtype).element_size()
    return torch.empty(n, (V + per - 1) // per * per, dtype=dtype, device=DEV)[:, :V]


def _slices(n, V, most=1 << 28):
    step = max(1, most // V)
    return [(a, min(n, a + step)) for a in range(0, n, step)]


def _logits(n, V, dtype, g):
    """Rows of normal logits whose spread differs from row to row: flat ones to peaked ones."""
    x = _rows(n, V, dtype)
    for a, z in _slices(n, V):
        spread = torch.rand(z - a, 1, generator=g, device=DEV) * 3 + 1.5
        x[a:z] = torch.randn(z - a, V, generator=g, device=DEV) * spread
    return x


def _valid(case, g):
    if not case["masked"]:
        return None
    v = torch.rand(case["rows"], generator=g, device=DEV) < 0.67
    v[-1] = True
    return v.to(torch.uint8)


def prepare(case, seed):
    g = _gen(seed)
    kind, n, V = case["kind"], case["rows"], case["V"]
    dt = DTYPES[case["dtype"]]
    st = dict(kind=kind)
    if kind == "top":
        k = case["k"]
        st.update(logits=_logits(n, V, dt, g), k=k, tau=case["tau"])
        st["out"] = dict(top_logit=torch.empty(n, k, dtype=torch.float32, device=DEV),
                         top_token=torch.empty(n, k, dtype=torch.int32, device=DEV),
                         rest_logit=torch.empty(n, dtype=torch.float32, device=DEV))
    elif kind == "distill":
        k, tau = case["k"], case["tau"]
        s = _logits(n, V, dt, g)
        token = torch.empty(n, k, dtype=torch.int32, device=DEV)
        logit = torch.empty(n, k, dtype=torch.float32, device=DEV)
        rest = torch.empty(n, dtype=torch.float32, device=DEV)
        for a, z in _slices(n, V):
            # a teacher that agrees with the student to a degree of each row's own
            rho = torch.rand(z - a, 1, generator=g, device=DEV) * 0.65 + 0.3
            t = rho * s[a:z].float() + (1 - rho * rho).sqrt() * 3 * torch.randn(z - a, V, generator=g, device=DEV)
            val, at = t.topk(k, dim=1)
            if case["ragged"]:
                held = torch.randint(0 if a else 1, k + 1, (z - a, 1), generator=g, device=DEV)
                short = torch.arange(k, device=DEV)[None, :] >= held
            else:
                short = torch.zeros(z - a, k, dtype=torch.bool, device=DEV)
            t.scatter_(1, at, torch.where(short, val, -INF))
            rest[a:z] = torch.logsumexp(t.double() / tau, 1).mul(tau).float() if V <= 65536 else torch.logsumexp(t / tau, 1) * tau
            token[a:z] = torch.where(short, -1, at).to(torch.int32)
            logit[a:z] = torch.where(short, 0.0, val)
        st.update(student=s, top_token=token, top_logit=logit, rest_logit=rest if case["rest"] else None, tau=tau,
                  reverse=case["reverse"], valid=_valid(case, g), scale=1.0 / n,
                  out=dict(row_loss=torch.empty(n, dtype=torch.float32, device=DEV), grad=_rows(n, V, DTYPES[case["grad"]])))
    else:
        D = case["D"]
        w = torch.empty(V, D, dtype=dt, device=DEV)
        for a, z in _slices(V, D):
            w[a:z] = torch.randn(z - a, D, generator=g, device=DEV) * (2.5 / math.sqrt(D))
        y = torch.randint(0, V, (n,), generator=g, device=DEV)
        lean = torch.rand(n, 1, generator=g, device=DEV) * 8
        x = (torch.randn(n, D, generator=g, device=DEV) + lean * w[y].float() * (1 / 2.5)).to(dt)
        f32 = dict(dtype=torch.float32, device=DEV)
        out = dict(row_loss=torch.empty(n, **f32), logp_token=torch.empty(n, **f32))
        if case["train"]:
            out.update(grad_hidden=torch.empty_like(x), grad_weight=torch.empty_like(w))
        st.update(hidden=x, weight=w, token=y.to(torch.int32), valid=_valid(case, g), scale=1.0 / n,
                  row_weight=torch.randn(n, generator=g, **f32) if case["weighted"] else None, out=out)
    return st


# ---------------------------------------------------------------------------
# a pass
# ---------------------------------------------------------------------------
def run(st):
    return _run_own(st) if own else _run_plain(st)


def _run_own(st):
    import paper_2609_36601_amd as saki

    kind, out = st["kind"], st["out"]
    if kind == "top":
        n, V = st["logits"].shape
        if "ws" not in st:
            st["ws"] = torch.empty(saki.workspace_bytes(saki.SAKI_OP_TOP_LOGITS, n, V), dtype=torch.uint8, device=DEV)
        saki.saki_top_logits(st["logits"], st["k"], temperature=st["tau"], workspace=st["ws"], **out)
    elif kind == "distill":
        n, V = st["student"].shape
        if "ws" not in st:
            st["ws"] = torch.empty(saki.workspace_bytes(saki.SAKI_OP_DISTILL_TOP, n, V), dtype=torch.uint8, device=DEV)
        saki.saki_distill_top(st["student"], st["top_token"], st["top_logit"], st["rest_logit"], temperature=st["tau"],
                              direction=saki.SAKI_KL_REVERSE if st["reverse"] else saki.SAKI_KL_FORWARD,
                              valid_mask=st["valid"], grad_scale=st["scale"], workspace=st["ws"], **out)
    else:
        if "ws" not in st:
            st["ws"] = torch.empty(saki.linear_ce_workspace_bytes(st["hidden"], st["weight"], train="grad_hidden" in out),
                                   dtype=torch.uint8, device=DEV)
        saki.saki_linear_ce(st["hidden"], st["weight"], st["token"], row_weight=st["row_weight"], valid_mask=st["valid"],
                            grad_scale=st["scale"], workspace=st["ws"], **out)
    return out


def _lse(x):
    m = x.amax(1, keepdim=True).clamp(min=torch.finfo(x.dtype).min)
    return (m + (x - m).exp().sum(1, keepdim=True).log())[:, 0]


def _run_plain(st):
    kind = st["kind"]
    if kind == "top":
        return _top(st["logits"].float(), st["k"], st["tau"])
    if kind == "distill":
        loss, grad = _distill(st["student"].float(), st["top_token"].long(), st["top_logit"], st["rest_logit"], st["tau"],
                              st["reverse"], st["valid"], st["scale"])
        return dict(row_loss=loss, grad=grad.to(st["out"]["grad"].dtype))
    x, w = st["hidden"].float(), st["weight"].float()
    y, n = st["token"].long(), st["hidden"].shape[0]
    part = torch.ones(n, device=DEV) if st["row_weight"] is None else st["row_weight"]
    if st["valid"] is not None:
        part = torch.where(st["valid"] != 0, part, 0.0)
        x = torch.where((st["valid"] != 0)[:, None], x, 0.0)
    logits = x @ w.t()
    at = torch.arange(n, device=DEV)
    lse = _lse(logits)
    logp = logits[at, y] - lse
    if st["valid"] is not None:
        logp = torch.where(st["valid"] != 0, logp, 0.0)
    out = dict(row_loss=-part * logp, logp_token=logp)
    if "grad_hidden" in st["out"]:
        d = (logits - lse[:, None]).exp_()
        d[at, y] -= 1.0
        d *= (part * st["scale"])[:, None]
        out.update(grad_hidden=(d @ w).to(st["hidden"].dtype), grad_weight=(d.t() @ x).to(st["weight"].dtype))
    return out


def _top(x, k, tau):
    val, at = x.sort(dim=1, descending=True, stable=True)
    rest = _lse(val[:, k:] / tau) * tau if k < x.shape[1] else torch.full_like(val[:, 0], -INF)
    return dict(top_logit=val[:, :k].contiguous(), top_token=at[:, :k].to(torch.int32), rest_logit=rest)


def _distill(s, token, logit, rest, tau, reverse, valid, scale):
    """Loss and gradient; at the listed tokens p and t themselves, the others as one bucket with the student's shares
    in it.  Exponentials of the row in 32 bits, their sum and what goes by the list in 64: a divergence near 0 is a
    difference of large logarithms."""
    n, V = s.shape
    held = token >= 0
    at = token.clamp(min=0)
    top = torch.where(held, s.gather(1, at).to(F64) / tau, -INF)
    # (a row shorter than the list writes its missing entries behind the vocabulary)
    out = torch.cat([s, s.new_zeros(n, 1)], 1).scatter_(1, torch.where(held, at, V), -INF)[:, :V]
    m = out.amax(1, keepdim=True).clamp(min=torch.finfo(s.dtype).min)
    out = out.sub_(m).div_(tau).exp_()
    mass = out.sum(1, keepdim=True, dtype=F64)
    logp = torch.cat([top, m.to(F64) / tau + mass.log()], 1)
    logp = logp - _lse(logp)[:, None]
    teach = torch.cat([torch.where(held, logit.to(F64), -INF),
                       torch.full_like(top[:, :1], -INF) if rest is None else rest[:, None].to(F64)], 1) / tau
    some = teach.amax(1) > -INF
    logt = torch.where(some[:, None], teach - _lse(teach)[:, None], -INF)
    p, t = logp.exp(), logt.exp()
    if reverse:
        ratio = torch.where(p > 0, logp - logt, 0.0)
        loss = (p * ratio).sum(1)
        g = p * (ratio - loss[:, None])
    else:
        loss = torch.where(t > 0, t * (logt - logp), 0.0).sum(1)
        g = p - t
    take = some if valid is None else some & (valid != 0)
    loss = torch.where(take, loss, 0.0)
    g = torch.where(take[:, None], g, 0.0) * (scale / tau)
    grad = out * torch.where(mass > 0, g[:, -1:] / mass, 0.0).float()
    grad = torch.cat([grad, grad.new_zeros(n, 1)], 1).scatter_(1, torch.where(held, at, V), g[:, :-1].float())[:, :V]
    return loss.float(), grad


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    n, V = case["rows"], case["V"]
    size = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "top":
        return dict(bytes=n * (V * size + case["k"] * 8 + 4), flops=3 * n * V)
    if case["kind"] == "distill":
        g = 2 if case["grad"] == "bf16" else 4
        return dict(bytes=n * (V * (size + g) + case["k"] * 8 + 8), flops=6 * n * V)
    D = case["D"]
    bytes_ = (n + V) * D * size + 12 * n
    flops = 2 * n * V * D
    if case["train"]:
        bytes_ += (n + V) * D * size
        flops *= 3
    return dict(bytes=bytes_, flops=flops)


# ---------------------------------------------------------------------------
# the definitions in 64 bits, a block of rows at a time
# ---------------------------------------------------------------------------
def exact(case, seed):
    st = prepare(case, seed)
    kind, n, V = case["kind"], case["rows"], case["V"]
    if kind == "top":
        logit, token, rest = [], [], []
        for a, z in _slices(n, V, 1 << 27):
            x = st["logits"][a:z].to(F64)
            val, at = x.sort(dim=1, descending=True, stable=True)
            logit.append(val[:, :case["k"]].clone())
            token.append(at[:, :case["k"]].to(torch.int32))
            rest.append(torch.logsumexp(val[:, case["k"]:] / case["tau"], 1) * case["tau"])
        return dict(top_logit=torch.cat(logit), top_token=torch.cat(token), rest_logit=torch.cat(rest))
    if kind == "distill":
        loss, grad = torch.empty(n, dtype=F64, device=DEV), torch.empty(n, V, dtype=F64, device=DEV)
        for a, z in _slices(n, V, 1 << 27):
            _exact_distill(st, a, z, loss, grad)
        return dict(row_loss=loss, grad=grad)
    D = case["D"]
    w = st["weight"].to(F64)
    loss, logp = torch.empty(n, dtype=F64, device=DEV), torch.empty(n, dtype=F64, device=DEV)
    dx, dw = (torch.zeros_like(st["hidden"], dtype=F64), torch.zeros_like(w)) if case["train"] else (None, None)
    for a, z in _slices(n, V, 1 << 29):
        x, y = st["hidden"][a:z].to(F64), st["token"][a:z].long()[:, None]
        share = torch.ones(z - a, 1, dtype=F64, device=DEV)
        if st["row_weight"] is not None:
            share = st["row_weight"][a:z, None].to(F64)
        keep = torch.ones_like(share, dtype=torch.bool) if st["valid"] is None else st["valid"][a:z, None] != 0
        lp = torch.log_softmax(x @ w.t(), 1)
        here = torch.where(keep, lp.gather(1, y), 0.0)
        logp[a:z], loss[a:z] = here[:, 0], -(share * here)[:, 0]
        if case["train"]:
            d = lp.exp_()
            d.scatter_add_(1, y, torch.full_like(share, -1.0))
            d *= torch.where(keep, share, 0.0) * st["scale"]
            dx[a:z] = d @ w
            dw += d.t() @ torch.where(keep, x, 0.0)
    out = dict(row_loss=loss, logp_token=logp)
    if case["train"]:
        out.update(grad_hidden=dx, grad_weight=dw)
    return out


def _exact_distill(st, a, z, loss, grad):
    """Probabilities over the buckets of rows a .. z: p_b the student's, t_b the teacher's, and the chain rule through
    p_b: d p_b / d s_j = p_j ([j in b] - p_b) / tau."""
    s, tau = st["student"][a:z].to(F64), st["tau"]
    token, V = st["top_token"][a:z].long(), s.shape[1]
    k = token.shape[1]
    held = token >= 0
    bucket = torch.full((z - a, V + 1), k, dtype=torch.int64, device=DEV)  # the bucket of each token
    bucket.scatter_(1, torch.where(held, token, V), torch.arange(k, device=DEV).expand(z - a, k))
    bucket = bucket[:, :V]
    p = torch.softmax(s / tau, 1)
    pb = torch.cat([torch.where(held, p.gather(1, token.clamp(min=0)), 0.0),
                    torch.where(bucket == k, p, 0.0).sum(1, keepdim=True)], 1)
    teach = torch.cat([torch.where(held, st["top_logit"][a:z].to(F64), -INF),
                       torch.full((z - a, 1), -INF, dtype=F64, device=DEV) if st["rest_logit"] is None
                       else st["rest_logit"][a:z, None].to(F64)], 1)
    take = teach.amax(1, keepdim=True) > -INF
    if st["valid"] is not None:
        take = take & (st["valid"][a:z, None] != 0)
    t = torch.softmax(torch.where(take, teach, 0.0) / tau, 1)
    here = torch.where(pb > 0, pb, 1.0)
    there = torch.where(t > 0, t, 1.0)
    if st["reverse"]:
        each = torch.where(pb > 0, here.log() - there.log(), 0.0)
        value, slope = pb * each, torch.where(pb > 0, each + 1.0, 0.0)  # of the sum by p_b
    else:
        value, slope = torch.where(t > 0, t * (there.log() - here.log()), 0.0), -t / here
    loss[a:z] = torch.where(take, value.sum(1, keepdim=True), 0.0)[:, 0]
    mean = (slope * pb).sum(1, keepdim=True)
    grad[a:z] = torch.where(take, p * (slope.gather(1, bucket) - mean) * (st["scale"] / tau), 0.0)
