"""GPU: attention whose row blocks' keys are shared by several thread blocks,
joined with the other part or alone: lines of fewer tiles than there are shares,
sequences without keys beside long ones, and values that are not finite."""
import numpy as np
import pytest

from serving_inputs import Case, to_bf16
from test_attention_gpu import H7, H70, H125, ODD, _check, _run

pytestmark = pytest.mark.gpu

CASES = {
    # a prompt's few row blocks over long lines, no prefix: shares of their own keys alone
    "own": (H70, [40, 1, 0], [3000, 1, 0], 0, 16),
    "own-64": (H125, [50], [2500], 0, 32),
    "own-uneven": (H70, [40, 33, 40], [2200, 33, 300], 0, 64),
    "own-and-empty-slots": (H7, [36, 1, 2], [1500, 0, 1], 0, 128),
    # both parts on the tensor cores, each in shares
    "both": (H70, [20] + [1] * 9, [1200] + [5] * 9, 2900, 16),
    "both-64": (ODD, [9] + [1] * 6, [900] + [0] * 6, 1800, 32),
    # a prefix in shares: alone, with short and long own parts beside it
    "prefix": (H70, [1] * 33, [0] * 33, 5003, 16),
    "prefix-mha": (H7, [1] * 21, [1 + 37 * i for i in range(21)], 2051, 64),
    "prefix-long-own": (H70, [1] * 9, [3000, 1, 0, 700, 16, 2, 2999, 128, 5], 1500, 16),
    # long chains of parts of one sequence in the kernel for few rows
    "narrow-parts": (H70, [2, 1], [9001, 40], 0, 16),
    "narrow-parts-64": (H125, [4], [7000], 0, 16),
}


@pytest.mark.parametrize("name", CASES)
def test_shares_match_the_definition(sdq, name):
    import torch
    heads, new, own, prefix, page = CASES[name]
    c = Case(heads, new, own, prefix, page, seed=100 + len(name))
    out, lse = _run(sdq, torch, c)
    _check(c, out, lse)
    again, lse2 = _run(sdq, torch, c)   # (the workspace filled with other leftovers)
    assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("name", ["own", "both", "prefix-mha", "narrow-parts"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_value_that_is_not_finite_reaches_those_that_see_it(sdq, name, bad):
    """One key head's value of one token of sequence 0: its rows of that head, and nothing else."""
    import torch
    heads, new, own, prefix, page = CASES[name]
    c = Case(heads, new, own, prefix, page, seed=7)
    want, want_lse = _run(sdq, torch, c)
    at = max(0, own[0] - new[0] - 1) if own[0] > new[0] else 0   # seen by all of its new tokens
    cache, batch, q = c.cache(sdq, torch), c.batch(sdq, torch), to_bf16(torch, c.q)
    cache.v_pages[c.pages[0, at // page], 0, at % page, 3] = bad
    out = cache.attend(batch, q)
    group = c.q_heads // c.kv_heads
    hit = torch.zeros(out.shape, dtype=torch.bool, device="cuda")
    hit[:new[0], :group, 3] = True
    assert not torch.isfinite(out[hit]).any()
    assert torch.equal(out[~hit], want[~hit])
    # and a key: the whole row of that head is lost, its log-sum-exp too
    cache = c.cache(sdq, torch)
    cache.k_pages[c.pages[0, at // page], 0, at % page, 3] = float("nan")
    lse = torch.zeros_like(want_lse)
    out = cache.attend(batch, q, lse=lse)
    hit = torch.zeros(out.shape, dtype=torch.bool, device="cuda")
    hit[:new[0], :group] = True
    assert torch.isnan(out[hit]).all() and torch.isnan(lse[:new[0], :group]).all()
    assert torch.equal(out[~hit], want[~hit])
