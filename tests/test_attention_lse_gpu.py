"""GPU: the log-sum-exp of rows whose scores are all NaN is NaN, as their
output is, on every route (-inf means that a row sees nothing, and a caller
that joins further parts would drop the NaN)."""
import pytest

from serving_inputs import Case, to_bf16
from test_attention_gpu import H7, H70, H125, ODD, _run

pytestmark = pytest.mark.gpu

CASES = {
    # the kernel for few rows: whole from registers, pieces of a thread block's warps, of several thread blocks
    "whole": (H125, [1] * 300, [1 + i % 9 for i in range(300)], 0, 16),
    "pieces": (H7, [1, 2], [120, 40], 0, 16),
    "pieces-far": (H70, [3], [5003], 0, 64),
    "prefix-few": (H125, [1] * 4, [0] * 4, 300, 16),
    # the one for many: rows of the output, shares of the keys, behind a prefix in one line
    "wide": (H70, [70, 1, 37] * 12, [70, 50, 200] * 12, 0, 32),
    "wide-64": ((4, 4, 64), [300, 260], [300, 700], 0, 32),
    "wide-shares": (H70, [40, 1], [3000, 1], 0, 16),
    "wide-behind": ((4, 4, 64), [300, 260], [300, 700], 257, 32),
    "prefix-many": (H70, [1] * 33, [0] * 33, 5003, 16),
    # two parts joined
    "both-few": (H125, [1] * 3, [5, 0, 40], 100, 16),
    "both": (H70, [1] * 9, [1, 7, 16, 30, 0, 65, 128, 3, 200], 301, 16),
    "both-wide": (ODD, [9] + [1] * 6, [900] + [0] * 6, 1800, 32),
}


@pytest.mark.parametrize("name", CASES)
def test_lse_of_a_query_that_is_nan(sdq, name):
    import torch
    heads, new, own, prefix, page = CASES[name]
    c = Case(heads, new, own, prefix, page, seed=len(name))
    want, want_lse = _run(sdq, torch, c)
    t = sum(new[:-1])   # the last sequence's first new token, and head 1 of it
    c.q[t, 1, 5] = float("nan")
    out, lse = _run(sdq, torch, c)
    assert torch.isnan(out[t, 1]).all() and torch.isnan(lse[t, 1])
    rest = torch.ones(lse.shape, dtype=torch.bool, device="cuda")
    rest[t, 1] = False
    assert torch.equal(out[rest], want[rest]) and torch.equal(lse[rest], want_lse[rest])


@pytest.mark.parametrize("name", ["pieces", "pieces-far", "wide", "wide-shares", "both"])
def test_lse_of_keys_that_are_all_nan(sdq, name):
    import torch
    heads, new, own, prefix, page = CASES[name]
    c = Case(heads, new, own, prefix, page, seed=len(name))
    cache, batch, q = c.cache(sdq, torch), c.batch(sdq, torch), to_bf16(torch, c.q)
    cache.k_pages[:, 0] = float("nan")
    lse = torch.zeros((c.tokens, c.q_heads), device="cuda")
    out = cache.attend(batch, q, lse=lse)
    group = c.q_heads // c.kv_heads
    assert torch.isnan(out[:, :group]).all() and torch.isnan(lse[:, :group]).all()
    assert torch.isfinite(out[:, group:].float()).all() and torch.isfinite(lse[:, group:]).all()
