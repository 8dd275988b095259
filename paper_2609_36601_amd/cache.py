"""Paged key-value caches of a rollout's student and teacher (include/saki_kv.h).

PagedKV holds a pool of pages and a table of which pages each sequence holds; its
methods are the library's calls with their outputs and workspaces allocated.  Every step runs
on the device without a host synchronisation, in the order of the calls on a stream, and may be
captured into a graph.  speculative.rollout drives the caches of a model that has some.
"""
import contextlib
import math

import torch

from . import binding as _b


def rope(rotary_dim, base=10000.0, interleaved=False, scaling=None, factor=1.0, length=4096, fast=32.0, slow=1.0,
         device="cuda"):
    """Rotary positions for PagedKV.append: pair i turns base^(-2 i / rotary_dim) radians a position.

    scaling: None; "linear": every pair `factor` times slower; "ramp": pairs that turn fewer than
    `slow` times in `length` positions are `factor` times slower, those that turn more than `fast` times
    are as they are, with a linear ramp in the number of turns between, and cosines and sines are
    multiplied by 1 + 0.1 ln(factor).
    """
    if rotary_dim < 0 or rotary_dim % 2:
        raise ValueError("rotary_dim must be even, >= 0")
    if not base > 0 or not factor > 0:
        raise ValueError("base and factor must be positive")
    f = base ** (-torch.arange(0, rotary_dim, 2, dtype=torch.float64) / max(rotary_dim, 1)) / (2 * math.pi)
    amplitude = 1.0
    if scaling == "linear":
        f = f / factor
    elif scaling == "ramp":
        if not fast > slow:
            raise ValueError("fast must be more than slow")
        ramp = ((length * f - slow) / (fast - slow)).clamp(0, 1)
        f = f * (ramp + (1 - ramp) / factor)
        amplitude = 1.0 + 0.1 * math.log(factor)
    elif scaling is not None:
        raise ValueError("scaling must be None, 'linear' or 'ramp'")
    return dict(freq=f.to(device), rotary_dim=rotary_dim, interleaved=interleaved, amplitude=amplitude)


_HERE = contextlib.nullcontext()


class PagedKV:
    """A cache: tensors k, v [n_layers, n_pages, n_kv_heads, page_size, head_dim] (any order of the
    first four axes in memory), pages [n_seq, max_pages], length [n_seq], held [n_seq], refs [n_pages]
    (int32; the table, see saki_kv_table).  The tensors are the caller's; PagedKV.alloc makes empty ones.
    A cache takes no part in autograd: tensors that record their history are refused (torch.no_grad())."""

    def __init__(self, k, v, pages, length, held, refs):
        if refs.device != k.device or pages.device != k.device:
            raise ValueError("the table and the pool must be on one device")
        if k.shape[1] != refs.numel():
            raise ValueError("refs must have an entry for every page of the pool")
        self.k, self.v, self.pages, self.length, self.held, self.refs = k, v, pages, length, held, refs
        self.device, self.dtype = k.device, k.dtype
        self._sizes = {}  # workspace bytes of the calls made so far
        self.n_layers, self.n_pages, self.n_kv_heads, self.page_size, self.head_dim = k.shape
        self.n_seq = pages.shape[0]
        self.pool = _b.kv_pool(k, v)
        self.table = _b.kv_table(pages, length, held, refs, self.page_size)

    @classmethod
    def alloc(cls, n_seq, max_pages, n_pages, n_layers, n_kv_heads, page_size, head_dim, dtype=torch.bfloat16,
              device="cuda"):
        """An empty cache.  Its pages are not cleared: what a token does not see has no influence."""
        k, v = (torch.empty(n_layers, n_pages, n_kv_heads, page_size, head_dim, dtype=dtype, device=device)
                for _ in range(2))
        ints = dict(dtype=torch.int32, device=device)
        return cls(k, v, torch.full((n_seq, max_pages), -1, **ints), torch.zeros(n_seq, **ints),
                   torch.zeros(n_seq, **ints), torch.zeros(n_pages, **ints))

    # -- helpers ---------------------------------------------------------------
    def _on(self, stream):
        """The cache's device and the call's stream current: outputs and workspaces are allocated for it."""
        if stream is None and torch.cuda.current_device() == self.device.index:
            return _HERE
        if stream is not None and stream.device != self.device:
            raise ValueError(f"a stream of {stream.device} for a cache on {self.device}")
        return self._elsewhere(stream)

    @contextlib.contextmanager
    def _elsewhere(self, stream):
        with torch.cuda.device(self.device), torch.cuda.stream(stream):  # (no change where stream is None)
            yield

    def _new(self, dtype, *shape):
        return torch.empty(shape, dtype=dtype, device=self.device)

    def _workspace(self, op, n, m):
        size = self._sizes.get((op, n))
        if size is None:
            if len(self._sizes) > 1000:
                self._sizes.clear()
            size = self._sizes[op, n] = max(_b.workspace_bytes(op, n, m), 16)
        return self._new(torch.uint8, size)

    def _ints(self, name, t, n=None):
        _b._want(name, t, torch.int32, (self.n_seq if n is None else n,), self.device)

    def _tokens(self, n_tokens, n_new, offsets, shift):
        if (n_new is None) == (offsets is None):
            raise ValueError("give either n_new or offsets")
        if offsets is not None:
            self._ints("offsets", offsets, self.n_seq + 1)
        elif n_tokens != self.n_seq * n_new:
            raise ValueError(f"{n_tokens} token rows for {self.n_seq} sequences of {n_new}")
        if not 0 <= shift <= 2**30:
            raise ValueError("shift outside [0, 2^30]")
        return _b.SakiKVTokens(_b._ptr(offsets), n_tokens, n_new or 0, shift)

    def _rows(self, name, t, n_tokens, heads):
        if t.shape != (n_tokens, heads, self.head_dim):
            raise ValueError(f"{name} must be [{n_tokens}, {heads}, {self.head_dim}]: got {tuple(t.shape)}")
        if t.dtype != self.dtype or t.device != self.device:
            raise ValueError(f"{name} must be {self.dtype} on {self.device}")
        if t.requires_grad and torch.is_grad_enabled():
            raise ValueError(f"{name} requires a gradient, and a cache passes none on: call under torch.no_grad()")

    # -- pages -----------------------------------------------------------------
    def reserve(self, n_new, stream=None):
        """Room for n_new more tokens (int32 tensor [n_seq], or one number) of every sequence, shared pages
        that they would be written to copied.  Returns the status [n_seq] (KV_*)."""
        if isinstance(n_new, torch.Tensor):
            self._ints("n_new", n_new)
        with self._on(stream):
            status = self._new(torch.uint8, self.n_seq)
            ws = self._workspace(_b.SAKI_OP_KV_RESERVE, self.n_seq, self.n_pages)
            _b.saki_kv_reserve(self.table, self.pool, n_new, status, ws)
        return status

    def commit(self, delta=None, done=None, stream=None):
        """length += delta (int32 [n_seq]; negative: tokens dropped), 0 where done (uint8 [n_seq]) is non-zero; pages
        behind the length are given back.  Returns the status [n_seq]."""
        if delta is not None:
            self._ints("delta", delta)
        if done is not None:
            _b._want("done", done, torch.uint8, (self.n_seq,), self.device)
        with self._on(stream):
            status = self._new(torch.uint8, self.n_seq)
            _b.saki_kv_commit(self.table, delta, done, status)
        return status

    def fork(self, src, dst, stream=None):
        """Sequences dst (which hold nothing) share the pages of sequences src (int32 tensors).  Returns the
        status of each pair."""
        self._ints("src", src, src.numel())
        self._ints("dst", dst, src.numel())
        with self._on(stream):
            status = self._new(torch.uint8, src.numel())
            _b.saki_kv_fork(self.table, src, dst, status)
        return status

    def compact(self, stream=None):
        """Moves the live pages to ids 0 .. n_live - 1.  Returns n_live (int32 tensor [1])."""
        with self._on(stream):
            if self.n_seq == 0:
                return torch.zeros(1, dtype=torch.int32, device=self.device)
            n_live = self._new(torch.int32, 1)
            ws = self._workspace(_b.SAKI_OP_KV_COMPACT, self.n_seq, self.n_pages)
            _b.saki_kv_compact(self.table, self.pool, n_live, ws)
        return n_live

    # -- tokens ----------------------------------------------------------------
    def append(self, layer, k, v, q=None, q_out=None, rope=None, n_new=None, offsets=None, shift=0, stream=None):
        """Writes k and v [n_tokens, n_kv_heads, head_dim] to the pages of their positions, k rotated, and q
        [n_tokens, heads, head_dim] rotated to q_out (allocated if None; may be q).  The j-th row of
        sequence b (rows b * n_new + j, or offsets[b] + j) is the token at position length[b] + shift + j.
        rope: what rope() returns, or None.  Returns q_out."""
        n = k.shape[0]
        self._rows("k", k, n, self.n_kv_heads)
        self._rows("v", v, n, self.n_kv_heads)
        if q is not None:
            self._rows("q", q, n, q.shape[1])
        tokens = self._tokens(n, n_new, offsets, shift)
        turn = None
        if rope is not None:
            f = rope["freq"]
            _b._want("rope freq", f, torch.float64, (rope["rotary_dim"] // 2,), self.device)
            turn = _b.SakiKVRope(_b._ptr(f), rope["rotary_dim"], int(rope["interleaved"]), rope["amplitude"])
        with self._on(stream):
            if q is not None:
                q_out = self._new(self.dtype, *q.shape) if q_out is None else q_out
                self._rows("q_out", q_out, n, q.shape[1])
            _b.saki_kv_append(self.table, self.pool, layer, tokens, k, v, q, q_out, turn)
        return q_out

    def attention(self, layer, q, out=None, lse=None, scale=None, window=0, sinks=0, n_new=None, offsets=None, shift=0,
                  stream=None):
        """Attention of the tokens' queries q [n_tokens, heads, head_dim] over their sequences' pages (rows as
        in append, which comes first): causal, with window > 0 over the last `window` positions and the first
        `sinks`.  scale: head_dim^-1/2 if None.  lse: float32 [n_tokens, heads] to fill, or None.  Returns out."""
        n, heads = q.shape[0], q.shape[1]
        self._rows("q", q, n, heads)
        tokens = self._tokens(n, n_new, offsets, shift)
        if lse is not None:
            _b._want("lse", lse, torch.float32, (n, heads), self.device)
        with self._on(stream):
            out = self._new(self.dtype, *q.shape) if out is None else out
            self._rows("out", out, n, heads)
            ws = self._workspace(_b.SAKI_OP_KV_ATTENTION, n * heads, self.head_dim)
            _b.saki_kv_attention(self.table, self.pool, layer, tokens, q, out, lse,
                                 self.head_dim ** -0.5 if scale is None else scale, window, sinks, ws)
        return out
