"""Performance cases of the paged key-value cache: its pages, what writes them and what reads them.

Each case is one pass as a speculative rollout makes it.  A case is a dict of plain values:

  kind    wave     a wave's bookkeeping: pages for k more tokens of every sequence, then the commit
                   of the accepted ones (the rest rolled back, finished sequences freed)
          fork     every prompt's sequence forked into its responses, then room for k tokens of
                   each of them, with copies of the shared last pages
          compact  the pages that live move to the lowest ids
          append   rotary positions on q and k of new tokens, k and v into their pages
          attend   attention of new tokens over the cache
  seqs    sequences (fork: prompts, each with `responses` responses)
  length  tokens a sequence holds at most (spread over the upper three quarters)
  page    tokens per page
  new     new tokens per sequence (ragged: spread over 1 up to so many)
  layers, heads (of keys and values), group (query heads per key head), dim (of a head)
"""
import math

import torch

own = False

DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
F64 = torch.float64
MOST_BYTES = 512 * 4480 * 8 * 128 * 2 * 2  # keys and values of the largest listed case
MOST_FLOPS = 4 * 16 * 128 * 16 * 2500 * 1250.0  # products of the longest listed prompts


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------
def listed():
    return [
        # a wave of a rollout batch, 64 prompts x 8 responses of up to 7,168 tokens: launches and one table
        dict(name="wave_512_sequences", kind="wave", seqs=512, length=7168, page=32, new=8),
        # a batch of prompts forked into 8 responses each and their shared last pages copied, 4 layers
        dict(name="fork_64_prompts_8_responses", kind="fork", seqs=64, responses=8, length=1000, page=32, new=8,
             layers=4, heads=8, dim=128, dtype="bf16"),
        # the cache compacted after most sequences ended, before its memory is given to the update
        dict(name="compact_after_rollout", kind="compact", seqs=256, length=2000, page=32, layers=4, heads=8, dim=128,
             dtype="bf16"),
        # one draft position of a small batch: the launch is what counts
        dict(name="append_draft_16", kind="append", seqs=16, length=2048, page=16, new=1, ragged=False, heads=8, group=2,
             dim=128, rot=128, interleaved=False, scaled=False, dtype="bf16"),
        # ragged prompts into the cache; interleaved pairs, half of the head rotated, positions scaled
        dict(name="append_ragged_prompts", kind="append", seqs=32, length=500, page=64, new=2047, ragged=True, heads=8,
             group=4, dim=128, rot=64, interleaved=True, scaled=True, dtype="bf16"),
        # a verification of 8 drafts far into long sequences, 32 bits
        dict(name="append_far_f32", kind="append", seqs=8, length=131072, page=128, new=8, ragged=False, heads=4,
             group=7, dim=96, rot=96, interleaved=False, scaled=False, dtype="f32"),
        # one draft position of a small batch
        dict(name="attend_draft_16", kind="attend", seqs=16, length=2048, page=16, new=1, ragged=False, heads=8, group=2,
             dim=128, window=0, sinks=0, dtype="bf16"),
        # one draft position of the whole rollout batch
        dict(name="attend_draft_512", kind="attend", seqs=512, length=7168, page=32, new=1, ragged=False, heads=8,
             group=2, dim=128, window=0, sinks=0, dtype="bf16"),
        # the teacher's verification of 8 drafts a sequence
        dict(name="attend_verify_128", kind="attend", seqs=128, length=7168, page=32, new=8, ragged=False, heads=8,
             group=4, dim=128, window=0, sinks=0, dtype="bf16"),
        # one token of one long sequence: the work has to be split over its length
        dict(name="attend_long_1", kind="attend", seqs=1, length=131072, page=64, new=1, ragged=False, heads=4, group=8,
             dim=128, window=0, sinks=0, dtype="bf16"),
        # the prompts of a batch, ragged
        dict(name="attend_prompts", kind="attend", seqs=16, length=0, page=32, new=2500, ragged=True, heads=8, group=2,
             dim=128, window=0, sinks=0, dtype="bf16"),
        # continued prompts with a sliding window and 4 first tokens that stay visible, 32 bits
        dict(name="attend_window_sinks_f32", kind="attend", seqs=5, length=3000, page=16, new=777, ragged=True, heads=2,
             group=5, dim=80, window=500, sinks=4, dtype="f32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _page(rng):
    return rng.choice([8, 16, 32, 64, 128])


def draw(rng):
    kind = rng.choice(["wave", "fork", "compact", "append", "append", "attend", "attend", "attend", "attend"])
    page = _page(rng)
    if kind == "wave":
        return dict(kind=kind, seqs=_log_int(rng, 1, 512), length=_log_int(rng, page, 7168), page=page,
                    new=rng.randint(1, 16))
    c = dict(kind=kind, page=page, heads=rng.choice([1, 2, 4, 5, 8]), dim=8 * rng.randint(8, 16),
             dtype=rng.choice(["bf16", "bf16", "f32"]))
    row = c["heads"] * c["dim"] * 2 * (2 if c["dtype"] == "bf16" else 4)  # bytes of a token's key and value
    if kind in ("fork", "compact"):
        c.update(layers=rng.randint(1, 4), length=_log_int(rng, 20, 4000))
        most = MOST_BYTES // 16 // (row * c["layers"])
        if kind == "fork":
            c.update(responses=rng.randint(2, 8), new=rng.randint(1, 8))
            c["seqs"] = max(1, min(_log_int(rng, 1, 64), most // (c["length"] + 16 * page)))
        else:
            c["seqs"] = max(1, min(_log_int(rng, 2, 256), most // (c["length"] + page)))
        return c
    c["group"] = rng.randint(1, 8)
    long = rng.random() < 0.3
    c["length"] = _log_int(rng, 1, 131072 if long else 8192)
    c["new"] = _log_int(rng, 64, 2500) if rng.random() < 0.25 else rng.choice([1, 1, rng.randint(2, 16)])
    c["ragged"] = c["new"] > 1 and rng.random() < 0.5
    tokens = c["length"] + c["new"] + page
    most = MOST_BYTES // (row * tokens)
    if kind == "append":
        c.update(rot=2 * rng.randint(1, c["dim"] // 2) if rng.random() < 0.5 else c["dim"],
                 interleaved=rng.random() < 0.5, scaled=rng.random() < 0.5)
        most = min(most, 60000 // c["new"])
    else:
        if rng.random() < 0.4:
            c.update(window=_log_int(rng, 1, 4096), sinks=rng.choice([0, 1, 4, rng.randint(0, 64)]))
        else:
            c.update(window=0, sinks=0)
        # (the plain form holds every score)
        scores = c["heads"] * c["group"] * c["new"] * tokens
        flops = MOST_FLOPS * (1 if c["dtype"] == "bf16" else 0.1)
        most = min(most, int(flops / (4 * c["dim"] * scores)), int(2e9 / scores))
        if not most:
            c["new"], most = 1, MOST_BYTES // (row * tokens)
            c["ragged"] = False
    c["seqs"] = max(1, min(_log_int(rng, 1, 512), most))
    return c


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _gen(seed, salt=0):
    g = torch.Generator(device=DEV)
    g.manual_seed((seed * 1000003 + salt * 7919 + 4711) % (1 << 62))
    return g


def _ints(g, lo, hi, n):
    return torch.randint(lo, hi + 1, (n,), generator=g, device=DEV, dtype=torch.int64)


def _spread(g, lo, hi, n):
    """n whole numbers spread evenly over lo .. hi, in any order: their sum, and with it every shape, is the case's."""
    return torch.linspace(lo if n > 1 else hi, hi, n, dtype=F64).round().long().to(DEV)[torch.randperm(n, generator=g, device=DEV)]


def _randn(shape, dtype, g):
    """Normal values, made a slice at a time (a pool in 32 bits beside itself would be large)."""
    x = torch.empty(shape, dtype=dtype, device=DEV)
    flat = x.view(-1)
    step = 1 << 27
    for a in range(0, flat.numel(), step):
        z = min(flat.numel(), a + step)
        flat[a:z] = torch.randn(z - a, generator=g, device=DEV)
    return x


def _table(case, lengths, extra, spare, g):
    """A table whose sequences hold room for lengths + extra tokens on scattered pages; `spare` more pages and
    table columns are free."""
    page, new = case["page"], case.get("new", 0)
    held = (lengths + extra + page - 1) // page
    n, live = lengths.numel(), int(held.sum())
    n_pages = int(((lengths + new + page - 1) // page).sum()) + spare
    width = (int(lengths.max()) + new) // page + 9
    ids = torch.randperm(n_pages, generator=g, device=DEV)[:live]
    j = torch.arange(width, device=DEV)
    filled = j[None, :] < held[:, None]
    pages = torch.full((n, width), -1, dtype=torch.int32, device=DEV)
    pages[filled] = ids.to(torch.int32)
    refs = torch.zeros(n_pages, dtype=torch.int32, device=DEV)
    refs[ids] = 1
    return dict(pages=pages, length=lengths.to(torch.int32), held=held.to(torch.int32), refs=refs)


def _lengths(case, g):
    return _spread(g, case["length"] - case["length"] * 3 // 4, case["length"], case["seqs"])


def _pool(case, n_pages, g):
    shape = (case.get("layers", 1), n_pages, case["heads"], case["page"], case["dim"])
    return _randn(shape, DTYPES[case["dtype"]], g), _randn(shape, DTYPES[case["dtype"]], g)


def _frequencies(case):
    """Turns (angle / 2 pi) a position advances each pair, in 64 bits: base 10,000; scaled: the slow pairs (fewer
    than one turn in 4,096 positions) four times slower, those of more than 32 turns as they are, a ramp between."""
    r = case["rot"]
    f = 10000.0 ** (-torch.arange(0, r, 2, dtype=F64, device=DEV) / r) / (2 * math.pi)
    if case["scaled"]:
        turns = 4096 * f
        ramp = ((turns - 1) / 31).clamp(0, 1)
        f = f * (ramp + (1 - ramp) / 4)
    return f


def _amplitude(case):
    return 0.1 * math.log(4.0) + 1.0 if case["scaled"] else 1.0


def prepare(case, seed):
    g = _gen(seed)
    kind = case["kind"]
    st = dict(kind=kind, page=case["page"])
    if kind == "wave":
        lengths = _lengths(case, g)
        t = _table(case, lengths, 0, 64, g)
        pools = torch.zeros(2, 1, t["refs"].numel(), 1, case["page"], 8, dtype=torch.bfloat16, device=DEV)
        st.update(table=t, k=pools[0], v=pools[1], n_new=torch.full_like(t["length"], case["new"]),
                  accepted=_ints(g, 0, case["new"], case["seqs"]).to(torch.int32),
                  done=(torch.rand(case["seqs"], generator=g, device=DEV) < 0.03).to(torch.uint8))
    elif kind == "fork":
        n, r = case["seqs"], case["responses"]
        lengths = _lengths(case, g)
        most = (case["length"] + case["new"]) // case["page"] + 2
        t = _table(case, lengths, 0, n * r * (case["new"] // case["page"] + 2), g)
        # prompts are sequences 0, r, 2 r, ...: the others of a group hold nothing yet
        wide = dict(pages=torch.full((n * r, most), -1, dtype=torch.int32, device=DEV),
                    length=torch.zeros(n * r, dtype=torch.int32, device=DEV),
                    held=torch.zeros(n * r, dtype=torch.int32, device=DEV), refs=t["refs"])
        w = min(most, t["pages"].shape[1])
        wide["pages"][::r, :w] = t["pages"][:, :w]
        wide["length"][::r], wide["held"][::r] = t["length"], t["held"]
        all_ = torch.arange(n * r, device=DEV, dtype=torch.int32)
        k, v = _pool(case, t["refs"].numel(), g)
        st.update(table=wide, k=k, v=v, dst=all_[all_ % r != 0], src=(all_ - all_ % r)[all_ % r != 0],
                  n_new=torch.full_like(wide["length"], case["new"]))
    elif kind == "compact":
        t = _table(case, _lengths(case, g), 0, 16, g)
        # three of four sequences have ended and given back their pages
        gone = torch.rand(case["seqs"], generator=g, device=DEV) < 0.75
        dropped = t["pages"][gone]
        t["refs"][dropped[dropped >= 0].long()] = 0
        t["pages"][gone] = -1
        t["length"][gone] = 0
        t["held"][gone] = 0
        k, v = _pool(case, t["refs"].numel(), g)
        st.update(table=t, k=k, v=v)
    else:
        n, dt = case["seqs"], DTYPES[case["dtype"]]
        lengths = _lengths(case, g)
        new = _spread(g, 1, case["new"], n) if case["ragged"] else torch.full((n,), case["new"], device=DEV)
        t = _table(case, lengths, new, 1, g)
        k, v = _pool(case, t["refs"].numel(), g)
        offsets = torch.zeros(n + 1, dtype=torch.int64, device=DEV)
        offsets[1:] = new.cumsum(0)
        tokens = int(offsets[-1])
        st.update(table=t, k=k, v=v, new=case["new"], ragged=case["ragged"], offsets=offsets.to(torch.int32))
        hq = case["heads"] * case["group"]
        if kind == "append":
            # one projection's output: q, k and v of a token side by side
            x = _randn((tokens, hq + 2 * case["heads"], case["dim"]), dt, g)
            st.update(q=x[:, :hq], new_k=x[:, hq:hq + case["heads"]], new_v=x[:, hq + case["heads"]:],
                      q_out=torch.empty(tokens, hq, case["dim"], dtype=dt, device=DEV),
                      rope=dict(freq=_frequencies(case), rotary_dim=case["rot"], interleaved=case["interleaved"],
                                amplitude=_amplitude(case)))
        else:
            # the first tokens draw attention: their keys lean towards every query
            lean = torch.randn(case["dim"], generator=g, device=DEV)
            first = t["pages"][:, 0].long()
            k[0, first, :, :4] += lean.to(dt)
            q = torch.randn(tokens, hq, case["dim"], generator=g, device=DEV) * 1.5 + 0.3 * lean
            st.update(q=q.to(dt), out=torch.empty(tokens, hq, case["dim"], dtype=dt, device=DEV),
                      lse=torch.empty(tokens, hq, dtype=torch.float32, device=DEV), scale=case["dim"] ** -0.5,
                      window=case["window"], sinks=case["sinks"])
    if kind in ("wave", "fork", "compact"):
        # the bookkeeping changes the table: a pass starts from the state as it is before the step
        flat = torch.cat([st["table"][f].reshape(-1) for f in FIELDS])
        work = torch.empty_like(flat)
        at, t = 0, {}
        for f in FIELDS:
            m = st["table"][f].numel()
            t[f] = work[at:at + m].view(st["table"][f].shape)
            at += m
        st.update(before=flat, now=work, table=t)
    if own:
        import paper_2609_36601_amd as saki

        st["cache"] = saki.PagedKV(k=st["k"], v=st["v"], **st["table"])
    return st


FIELDS = ("pages", "length", "held", "refs")


# ---------------------------------------------------------------------------
# a pass
# ---------------------------------------------------------------------------
def run(st):
    kind = st["kind"]
    if kind in ("wave", "fork", "compact"):
        st["now"].copy_(st["before"])
    return _run_own(st) if own else _run_plain(st)


def _run_own(st):
    kind, cache = st["kind"], st["cache"]
    if kind == "wave":
        status = cache.reserve(st["n_new"])
        cache.commit(st["accepted"], done=st["done"])
        return dict(st["table"], status=status)
    if kind == "fork":
        status = cache.fork(st["src"], st["dst"])
        return dict(st["table"], forked=status, status=cache.reserve(st["n_new"]), k=st["k"], v=st["v"])
    if kind == "compact":
        n_live = cache.compact()
        return dict(st["table"], n_live=n_live, k=st["k"], v=st["v"])
    tokens = dict(offsets=st["offsets"]) if st["ragged"] else dict(n_new=st["new"])
    if kind == "append":
        cache.append(0, st["new_k"], st["new_v"], q=st["q"], q_out=st["q_out"], rope=st["rope"], **tokens)
        return dict(q=st["q_out"], k=st["k"], v=st["v"])
    cache.attention(0, st["q"], out=st["out"], lse=st["lse"], scale=st["scale"], window=st["window"], sinks=st["sinks"],
                    **tokens)
    return dict(out=st["out"], lse=st["lse"])


def _reserve_plain(t, n_new, page, k, v):
    L, H, n, refs = t["length"].long(), t["held"].long(), n_new.long(), t["refs"]
    width, b = t["pages"].shape[1], torch.arange(L.numel(), device=DEV)
    slot = (L // page).clamp(max=width - 1)
    cur = t["pages"].gather(1, slot[:, None])[:, 0].clamp(min=0).long()
    shared = (n > 0) & (L % page != 0) & (refs[cur] > 1)
    # a shared page stays with its last writer if all that hold it write now
    writers = torch.zeros_like(refs).scatter_add(0, cur, shared.to(torch.int32))
    last = torch.full_like(refs, -1).scatter_reduce(0, cur, torch.where(shared, b, -1).to(torch.int32), "amax")
    copy = shared & ~((writers[cur] == refs[cur]) & (last[cur] == b))
    need = (L + n + page - 1) // page
    new = torch.where(n > 0, (need - H).clamp(min=0), 0)
    take = new + copy
    base = take.cumsum(0) - take
    total = take.sum()
    order = (refs != 0).to(torch.int8).argsort(stable=True)  # free pages first, the lowest first
    bad = (total > (refs == 0).sum()) & (n > 0)
    j = torch.arange(width, device=DEV)
    fresh = (j >= H[:, None]) & (j < (H + new)[:, None])
    at = base[:, None] + copy[:, None] + (j - H[:, None])
    is_copy = copy[:, None] & (j == slot[:, None])
    at = torch.where(is_copy, base[:, None], at)
    taken = order[at.clamp(0, refs.numel() - 1)].to(torch.int32)
    t["pages"].copy_(torch.where(fresh | is_copy, taken, t["pages"]))
    used = (torch.arange(refs.numel(), device=DEV) < total).to(torch.int32)
    refs.add_(torch.zeros_like(refs).scatter(0, order, used))
    refs.sub_(torch.zeros_like(refs).scatter_add(0, cur, copy.to(torch.int32)))
    t["held"].copy_(H + new)
    # the tokens of the copied pages, in every layer
    at = copy.nonzero()[:, 0]
    src, dst = cur[at], t["pages"][at, slot[at]].long()
    filled = (torch.arange(page, device=DEV) < (L % page)[at, None])[None, :, None, :, None]
    for x in (k, v):
        x[:, dst] = torch.where(filled, x[:, src], x[:, dst])
    return bad.to(torch.uint8)


def _rotate_plain(x, cos, sin, rope):
    """x [n, heads, dim] in 32 bits, rotated by cos, sin [n, 1, pairs] in 64."""
    r, x = rope["rotary_dim"], x.to(F64)
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if rope["interleaved"] else (x[..., :r // 2], x[..., r // 2:r])
    y, z = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([y, z], -1).flatten(-2) if rope["interleaved"] else torch.cat([y, z], -1)
    return torch.cat([turned, x[..., r:]], -1)


def _rows_plain(st):
    """Sequence and position of every new token."""
    n = st["offsets"].numel() - 1
    rows = torch.arange(st["q"].shape[0], device=DEV)
    seq = torch.searchsorted(st["offsets"][1:].long(), rows, right=True)
    return n, rows, seq, st["table"]["length"].long()[seq] + rows - st["offsets"].long()[seq]


def _run_plain(st):
    kind, t, page = st["kind"], st["table"], st["page"]
    if kind == "wave":
        status = _reserve_plain(t, st["n_new"], page, st["k"], st["v"])
        L = torch.where(st["done"] != 0, 0, t["length"] + st["accepted"])
        held = (L + page - 1) // page
        j = torch.arange(t["pages"].shape[1], device=DEV)
        drop = (j >= held[:, None]) & (j < t["held"][:, None])
        at = torch.where(drop, t["pages"], 0).long().reshape(-1)
        t["refs"].sub_(torch.zeros_like(t["refs"]).scatter_add(0, at, drop.reshape(-1).to(torch.int32)))
        t["pages"].copy_(torch.where(drop, -1, t["pages"]))
        t["length"].copy_(L)
        t["held"].copy_(held)
        return dict(t, status=status)
    if kind == "fork":
        src, dst = st["src"].long(), st["dst"].long()
        L = t["length"][src]
        held = (L + page - 1) // page
        j = torch.arange(t["pages"].shape[1], device=DEV)
        share = j < held[:, None]
        t["pages"][dst] = torch.where(share, t["pages"][src], -1)
        at = torch.where(share, t["pages"][src], 0).long().reshape(-1)
        t["refs"].add_(torch.zeros_like(t["refs"]).scatter_add(0, at, share.reshape(-1).to(torch.int32)))
        t["length"][dst], t["held"][dst] = L, held
        forked = torch.zeros(dst.numel(), dtype=torch.uint8, device=DEV)
        return dict(t, forked=forked, status=_reserve_plain(t, st["n_new"], page, st["k"], st["v"]), k=st["k"], v=st["v"])
    if kind == "compact":
        refs = t["refs"]
        ids = torch.arange(refs.numel(), device=DEV)
        live = refs > 0
        n = live.sum()
        src = (live & (ids >= n)).nonzero()[:, 0]
        dst = (~live & (ids < n)).nonzero()[:, 0]
        to = ids.scatter(0, src, dst)
        for x in (st["k"], st["v"]):
            x[:, dst] = x[:, src]
        refs[dst] = refs[src]
        refs[src] = 0
        t["pages"].copy_(torch.where(t["pages"] >= 0, to[t["pages"].clamp(min=0).long()].to(torch.int32), -1))
        return dict(t, n_live=n.to(torch.int32).reshape(1), k=st["k"], v=st["v"])
    n, rows, seq, pos = _rows_plain(st)
    if kind == "append":
        rope = st["rope"]
        turns = pos.to(F64)[:, None, None] * rope["freq"]  # a far position's angle needs 64 bits
        angle = (turns - turns.round()) * (2 * math.pi)
        cos, sin = rope["amplitude"] * angle.cos(), rope["amplitude"] * angle.sin()
        st["q_out"].copy_(_rotate_plain(st["q"].float(), cos, sin, rope))
        id_ = t["pages"][seq, pos // page].long()
        st["k"][0, id_, :, pos % page] = _rotate_plain(st["new_k"].float(), cos, sin, rope).to(st["k"].dtype)
        st["v"][0, id_, :, pos % page] = st["new_v"]
        return dict(q=st["q_out"], k=st["k"], v=st["v"])
    # attention: every sequence padded to the longest, every score held
    new, L, q = st["new"], t["length"].long(), st["q"]
    count = st["offsets"].long().diff()
    heads, dim = st["k"].shape[2], q.shape[2]
    group = q.shape[1] // heads
    width = t["pages"].shape[1] - 8  # the table's columns in use
    total = width * page
    ids = t["pages"][:, :width].clamp(min=0).long()

    def gathered(x):
        return x[0][ids].permute(0, 2, 1, 3, 4).reshape(n, heads, total, dim).float()

    padded = torch.zeros(n, new, heads, group, dim, device=DEV)
    padded[seq, rows - st["offsets"].long()[seq]] = q.float().view(-1, heads, group, dim)
    padded = padded.permute(0, 2, 3, 1, 4).reshape(n, heads, group * new, dim)
    s = torch.matmul(padded, gathered(st["k"]).transpose(2, 3).contiguous()).mul_(st["scale"])
    i = L[:, None] + torch.arange(new, device=DEV)
    j = torch.arange(total, device=DEV)
    seen = j <= i[:, :, None]
    if st["window"]:
        seen &= (j > i[:, :, None] - st["window"]) | (j < st["sinks"])
    seen &= (torch.arange(new, device=DEV) < count[:, None])[:, :, None]
    s = s.view(n, heads, group, new, total).masked_fill_(~seen[:, None, None], -math.inf)
    top = s.amax(-1, keepdim=True).clamp(min=-3e38)
    p = s.sub_(top).exp_()
    total_p = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(n, heads, group * new, total), gathered(st["v"])).view(n, heads, group, new, dim) / total_p
    lse = (top + total_p.log())[..., 0]
    back = (seq, slice(None), slice(None), rows - st["offsets"].long()[seq])
    st["out"].copy_(o[back].reshape(-1, heads * group, dim))
    st["lse"].copy_(lse[back].reshape(-1, heads * group))
    return dict(out=st["out"], lse=st["lse"])


# ---------------------------------------------------------------------------
# the definition in 64 bits
# ---------------------------------------------------------------------------
def exact(case, seed):
    """Sequence by sequence, token by token, in 64 bits; whole numbers have no such value."""
    global own
    kind, page, was = case["kind"], case["page"], own
    if kind in ("wave", "fork", "compact"):
        return None  # whole numbers, and copies of rounded values
    own = False
    st = prepare(case, seed)
    own = was
    t = {f: st["table"][f].cpu() for f in FIELDS}
    offsets = st["offsets"].cpu().tolist()
    if kind == "append":
        rope, r, tokens = st["rope"], case["rot"], st["q"].shape[0]
        where = [(b, i) for b in range(case["seqs"]) for i in range(offsets[b + 1] - offsets[b])]
        b = torch.tensor([w[0] for w in where])
        pos = t["length"].long()[b] + torch.tensor([w[1] for w in where])
        angle = 2 * math.pi * torch.remainder(pos.to(F64)[:, None] * rope["freq"].cpu(), 1.0)
        # the rotation as one complex factor a pair
        turn = torch.polar(torch.full_like(angle, rope["amplitude"]), angle).to(DEV)[:, None]

        def rotated(x):
            x = x.to(F64)
            y = x.clone()
            first, second = (slice(0, r, 2), slice(1, r, 2)) if rope["interleaved"] else (slice(0, r // 2), slice(r // 2, r))
            w = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * turn
            y[..., first], y[..., second] = w.real, w.imag
            return y

        kk, vv = st["k"].to(F64), st["v"].to(F64)
        id_, off = t["pages"][b, pos // page].long().to(DEV), (pos % page).to(DEV)
        kk[0][id_, :, off] = rotated(st["new_k"])
        vv[0][id_, :, off] = st["new_v"].to(F64)
        assert tokens == len(where)
        return dict(q=rotated(st["q"]), k=kk, v=vv)
    heads = st["k"].shape[2]
    out, lse = torch.empty(st["out"].shape, dtype=F64, device=DEV), torch.empty(st["lse"].shape, dtype=F64, device=DEV)
    group = st["q"].shape[1] // heads
    for b in range(case["seqs"]):
        a, z = offsets[b], offsets[b + 1]
        n0 = int(t["length"][b])
        m = n0 + z - a
        ids = t["pages"][b, :-(-m // page)].long().to(DEV)
        i = torch.arange(n0, m, device=DEV)[:, None]
        j = torch.arange(m, device=DEV)[None, :]
        hidden = (j > i) if not case["window"] else (j > i) | ((j <= i - case["window"]) & (j >= case["sinks"]))
        for h in range(heads):
            kh = st["k"][0, ids, h].reshape(-1, case["dim"])[:m].to(F64)
            vh = st["v"][0, ids, h].reshape(-1, case["dim"])[:m].to(F64)
            for q0 in range(0, group, max(1, (1 << 26) // ((z - a) * m))):
                hs = slice(h * group + q0, min(h * group + group, h * group + q0 + max(1, (1 << 26) // ((z - a) * m))))
                s = torch.matmul(st["q"][a:z, hs].to(F64).transpose(0, 1), kh.t().contiguous()) * case["dim"] ** -0.5
                s = s.masked_fill(hidden, -math.inf)
                lse[a:z, hs] = torch.logsumexp(s, -1).t()
                out[a:z, hs] = torch.matmul(torch.softmax(s, -1), vh).transpose(0, 1)
    return dict(out=out, lse=lse)


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    kind, page = case["kind"], case["page"]
    n, mean = case["seqs"], case["length"] * 5 / 8
    if kind in ("wave", "fork", "compact"):
        pages = n * (mean / page + 0.5)
        if kind == "wave":  # reference counts, lengths and pages held in and out, steps, status, new entries
            return dict(bytes=2 * 4 * pages + n * (4 * 4 + 4 + 4 + 2) + 8 * n * case["new"] / page, flops=0)
        row = 2 * case["heads"] * case["dim"] * (2 if case["dtype"] == "bf16" else 4) * case["layers"]
        if kind == "fork":  # the prompts' entries to their responses, and all but one copy of each last page
            r = case["responses"]
            return dict(bytes=2 * 4 * pages + 4 * pages * r + 24 * n * r + 2 * row * n * (r - 1) * (page - 1) / 2, flops=0)
        return dict(bytes=16 * pages + 2 * row * 0.75 * 0.25 * pages * page, flops=0)
    new = (case["new"] + 1) / 2 if case["ragged"] else case["new"]
    e = 2 if case["dtype"] == "bf16" else 4
    tokens, hq = n * new, case["heads"] * case["group"]
    if kind == "append":
        return dict(bytes=2 * e * tokens * (hq + 2 * case["heads"]) * case["dim"] + 4 * tokens / page,
                    flops=3 * tokens * (hq + case["heads"]) * case["rot"])
    # visible pairs, from the mean length (a window's sum is over the positions of a mean sequence)
    i = torch.arange(int(round(new)), dtype=F64) + mean + 1
    if case["window"]:
        first = (i - case["window"]).clamp(min=0)
        seen = i - first + torch.minimum(first, torch.tensor(float(case["sinks"]), dtype=F64))
        keys = min(mean + new, case["window"] + new + case["sinks"])
    else:
        seen, keys = i, mean + new
    return dict(bytes=e * (2 * n * keys * case["heads"] * case["dim"] + 2 * tokens * hq * case["dim"]) + 4 * tokens * hq,
                flops=4 * case["dim"] * hq * n * float(seen.sum()))
