"""A reserve that copies a shared page for more than 2^23 sequences at once."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_more_than_2_to_the_23_copies(saki_lib):
    """All sequences hold page 0 and its one token; all but the last write: each gets the next page, with a copy."""
    n, page, dim = 2**23 + 2, 8, 8
    i32 = dict(dtype=torch.int32, device=DEV)
    k, v = (torch.zeros(1, n, 1, page, dim, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    first = torch.arange(1, dim + 1, device=DEV)
    k[0, 0, 0, 0], v[0, 0, 0, 0] = first, -first
    k[0, 0, 0, 1:] = 9.0  # behind the token: not copied
    refs = torch.zeros(n, **i32)
    refs[0] = n
    c = saki_lib.PagedKV(k, v, torch.zeros(n, 1, **i32), torch.ones(n, **i32), torch.ones(n, **i32), refs)
    new = torch.ones(n, **i32)
    new[-1] = 0
    print(f"{n - 1} copies", flush=True)
    assert int(c.reserve(new).max()) == saki_lib.KV_OK
    assert torch.equal(c.pages[:-1, 0], torch.arange(1, n, **i32)) and int(c.pages[-1, 0]) == 0
    assert bool((refs == 1).all()) and bool((c.held == 1).all()) and bool((c.length == 1).all())
    assert bool((k[0, :, 0, 0] == first).all()) and bool((v[0, :, 0, 0] == -first).all())
    assert bool((k[0, 1:, 0, 1:] == 0).all()) and bool((k[0, 0, 0, 1:] == 9.0).all())
