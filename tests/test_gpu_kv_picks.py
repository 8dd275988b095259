"""Which keys and values the bf16 attention reads, token by token: every query is the key of one token, so that its output is
that token's value.

Keys are random rows of +-1, and a query's score with its own key is `gap` above that with any other (asserted), so that
all others together weigh less than 2^-20.  The output is then the picked value, rounded once as a weight over
its sum (2^-8: the weight is rounded, the sum is not) and once as an output (2^-8)."""
import numpy as np
import pytest
import torch

from tests.test_gpu_kv_attention import make, put

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF = torch.bfloat16


@pytest.mark.parametrize("dim,page,order,lengths,new,group,window,sinks", [
    # the kernel for prompts: split keys, pages shorter and longer than a block of 64, tails, windows
    (128, 8, "heads", [2500, 0], [70, 200], 3, 0, 0), (128, 16, "tokens", [0, 3000], [65, 130], 3, 0, 0),
    (64, 8, "heads", [3001], [100], 3, 0, 0), (64, 32, "tokens", [0, 37, 300], [300, 129, 1], 2, 0, 0),
    (128, 256, "heads", [1, 257], [128, 255], 2, 0, 0), (96, 32, "heads", [90, 700], [130, 67], 2, 0, 0),
    (40, 16, "heads", [700, 30, 0], [90, 0, 129], 3, 0, 0), (128, 32, "heads", [1500], [300], 2, 333, 70),
    (64, 16, "tokens", [40, 900], [200, 150], 1, 100, 5), (128, 1024, "heads", [1025], [140], 1, 0, 0),
    # single tokens and verifications, of every number of row tiles; wide heads
    (128, 16, "heads", [0, 517, 9001], [1, 1, 1], 2, 0, 0), (128, 32, "tokens", [700, 41], [8, 8], 4, 0, 0),
    (64, 8, "heads", [900, 33], [9, 3], 7, 0, 0), (64, 64, "tokens", [2000], [1], 8, 500, 4), (256, 16, "heads", [300, 65], [9, 30], 2, 0, 0),
    (136, 64, "tokens", [800], [3], 5, 0, 0)])
def test_every_token_is_read_where_it_lies(saki_lib, dim, page, order, lengths, new, group, window, sinks):
    print(f"picks: dim {dim} page {page} {order} {lengths} {new} group {group} window {window}", flush=True)
    hk, scale = 2, 192 / dim
    t, c, q, off, dense = make(saki_lib, BF, lengths, new, group, hk, dim, page, dim + page, order)
    offsets = torch.as_tensor(off, dtype=torch.int32, device=DEV)
    for b, (kb, vb) in enumerate(dense):
        kb.copy_(torch.where(kb > 0, 1.0, -1.0))
        if kb.shape[0] > 1:
            like = torch.matmul(kb.float().transpose(0, 1), kb.float().permute(1, 2, 0).contiguous())
            like.diagonal(dim1=1, dim2=2).zero_()
            gap = scale * (dim - float(like.max()))
            assert kb.shape[0] * np.exp(-gap) < 2.0**-20
        put(t, b, c.k, c.v, kb, vb)
    # rows of a key head and the tokens that each sees
    read = [torch.zeros(kb.shape[0], hk, dtype=torch.bool, device=DEV) for kb, _ in dense]
    rng = np.random.default_rng(dim)
    for call in range(60):
        picked = []
        for b, (kb, vb) in enumerate(dense):
            rows = []
            for j in range(new[b]):
                pos = lengths[b] + j
                first = max(0, pos - window + 1) if window else 0
                seen = np.concatenate([np.arange(min(sinks, first)), np.arange(first, pos + 1)])
                # by turns through all that the sequence sees, and back from the row's own token
                at = (call // 2 * new[b] + j) * group + np.arange(group) if call % 2 else -1 - call // 2 * group - np.arange(group)
                rows.append(seen[at % len(seen)] if call < 50 else rng.choice(seen, group))
            if not rows:
                continue
            pick = torch.as_tensor(np.stack(rows), device=DEV)  # [new, group]
            picked.append((b, pick))
            for h in range(hk):
                q[off[b]:off[b + 1], h * group:(h + 1) * group] = kb[pick, h]
                read[b][pick.reshape(-1), h] = True
        out = c.attention(1, q, scale=scale, window=window, sinks=sinks, offsets=offsets)
        for b, pick in picked:
            for h in range(hk):
                want = dense[b][1][pick, h].float()
                got = out[off[b]:off[b + 1], h * group:(h + 1) * group].float()
                bad = (got - want).abs() > (2.0**-8 + 2.0**-8) * want.abs() + 2.0**-18
                assert not bad.any(), (call, b, h, pick.reshape(-1)[bad.reshape(-1, dim).any(1)][:8].tolist())
        if all(bool(r.all()) for r in read):
            break
    # every token has been read, where the calls have rows enough for it
    for b, L in enumerate(lengths):
        if not window and new[b] * group * 25 >= L + new[b]:
            assert bool(read[b].all()), (b, int((~read[b]).sum()))
