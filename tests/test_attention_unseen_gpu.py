"""GPU: attention of rows that see no key: empty slots and tokens ahead of
their sequence's first place, in blocks of many rows; every such row is 0 and
its log-sum-exp -inf, the others are as the definition says."""
import numpy as np
import pytest

from serving_inputs import Case
from test_attention_gpu import _check, _run

pytestmark = pytest.mark.gpu

# heads, new, own, page; no prefix.  More than 32 rows a key head of a sequence: 256 at a time.
WIDE = {
    # a key head for 64 query heads: an empty slot is a row block without a tile, beside others with some
    "slots-128": ((64, 1, 128), [1] * 64, [0, 1, 0, 40] * 16, 16),
    "slots-64": ((64, 1, 64), [1] * 64, [0, 1, 0, 40] * 16, 16),
    "slots-alone": ((64, 1, 128), [1] * 40, [0] * 39 + [1], 32),
    # fewer own tokens than new ones: whole row blocks before the first place, others across it
    "ahead-128": ((16, 2, 128), [80] * 20, [20, 5, 0, 80] * 5, 16),
    "ahead-64": ((4, 4, 64), [700] * 12, [30, 0, 300] * 4, 64),
    "odd": ((10, 2, 128), [77] * 30, [1, 0, 70] * 10, 16),
}


@pytest.mark.parametrize("name", WIDE)
def test_row_blocks_that_see_nothing(sdq, name):
    import torch
    heads, new, own, page = WIDE[name]
    c = Case(heads, new, own, 0, page, seed=len(name))
    out, lse = _run(sdq, torch, c)
    _check(c, out, lse)
    unseen = np.concatenate([np.arange(n) < n - m for n, m in zip(new, own)])
    assert unseen.any() and np.all(out[torch.from_numpy(unseen).cuda()].view(torch.int16).cpu().numpy() & 0x7FFF == 0)
    for _ in range(20):
        again, _ = _run(sdq, torch, c)
        assert torch.equal(again, out)


# heads, new, page: no sequence has a key, and some bring more rows than the kernel for few rows takes otherwise
NO_KEYS = {
    "one": ((64, 8, 128), [1], 16),
    "group-8": ((64, 8, 128), [1025], 16),
    "group-8-many": ((64, 8, 128), [3, 1, 0, 1500, 1, 1025, 40], 16),
    "group-16": ((16, 1, 64), [300, 5], 32),
    "group-5": ((10, 2, 64), [700, 3, 650], 64),
    "group-1": ((1, 1, 64), [65540, 1], 16),
    "group-4096": ((4096, 1, 64), [2, 1], 128),
    "many": ((12, 12, 64), [1, 0, 2] * 200, 16),
}


def _no_keys(sdq, torch, heads, new, page):
    i = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
    cache = sdq.KVCache(sdq.CacheDesc(heads[1], heads[2], page, 2))
    start = np.concatenate([[0], np.cumsum(new)]).tolist()
    return cache, sdq.Batch(i(start), i([0] * len(new)), i([[0]] * len(new)), start[-1], max(new), 0)


@pytest.mark.parametrize("name", NO_KEYS)
def test_calls_without_any_keys(sdq, name):
    """Every row is 0 and -inf, and nothing behind the last one is written."""
    import torch
    heads, new, page = NO_KEYS[name]
    cache, batch = _no_keys(sdq, torch, heads, new, page)
    shape = (batch.n_tokens, heads[0], heads[2])
    rows, guard = shape[0] * shape[1], 4096
    q = torch.randn(shape, device="cuda").to(torch.bfloat16)
    for with_lse in (True, False):
        out = torch.full((rows + guard, heads[2]), 7.0, dtype=torch.bfloat16, device="cuda")
        lse = torch.full((rows + guard,), 7.0, device="cuda")
        ws = cache.alloc_workspace(batch, heads[0])
        ws.random_(0, 256)
        sdq.sdq_attention(cache.handle, batch, heads[0], q, heads[0] * heads[2], 0.1, out, lse if with_lse else None, ws)
        assert sdq.sdq_attention_status(ws) == 0
        assert not out[:rows].any() and (out[rows:] == 7).all()
        assert torch.isneginf(lse[:rows]).all() if with_lse else (lse == 7).all()
        assert (lse[rows:] == 7).all()


@pytest.mark.parametrize("name", NO_KEYS)
def test_workspace_of_calls_without_any_keys(sdq, name):
    """Tickets, and no room for partial results (fp32 rows of them would take gigabytes)."""
    import torch
    heads, new, page = NO_KEYS[name]
    cache, batch = _no_keys(sdq, torch, heads, new, page)
    size = sdq.sdq_attention_workspace_bytes(cache.handle, batch, heads[0])
    assert 0 < size <= 8 * len(new) * heads[1] + 4096
