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
