"""Random caches for the tests of the paged key-value cache: the library's tensors and the oracle's table
with the same contents."""
import numpy as np
import torch

from oracle import cache as ocache


def filled(lengths, page_size, n_pages, max_pages, rng, extra=0):
    """An oracle table whose sequences hold `lengths` tokens and room for `extra` more, on scattered pages."""
    t = ocache.Table(len(lengths), max_pages, n_pages, page_size)
    ids = list(rng.permutation(n_pages))
    for b, L in enumerate(lengths):
        for i in range(-(-(L + extra) // page_size)):
            t.pages[b, i] = ids.pop()
            t.refs[t.pages[b, i]] = 1
            t.held[b] += 1
        t.length[b] = L
    return t


def to_cache(saki, t, k, v):
    """The library's cache of the oracle's table t on the device of k and v."""
    ints = {f: torch.as_tensor(getattr(t, f).astype(np.int32), device=k.device) for f in
            ("pages", "length", "held", "refs")}
    return saki.PagedKV(k, v, **ints)


def same_table(cache, t):
    for f in ("pages", "length", "held", "refs"):
        np.testing.assert_array_equal(getattr(cache, f).cpu().numpy(), getattr(t, f), err_msg=f)


def token_major(n_layers, n_pages, heads, page, dim, dtype, device):
    """A pool tensor whose memory order is [page, layer, token, head]: the same view, other strides."""
    return torch.empty(n_pages, n_layers, page, heads, dim, dtype=dtype, device=device).permute(1, 0, 3, 2, 4)
