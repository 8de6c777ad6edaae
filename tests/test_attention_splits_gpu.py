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


MASKED = {
    "draft": (H70, [3, 2, 4], [30, 130, 67], 0, 16, 1),
    "draft-whole": (H70, [4, 1], [3, 9], 0, 16, 2),          # (a slot whose first new token has no place)
    "draft-odd": (ODD, [5, 3], [205, 140], 60, 64, 3),
    "draft-64": (H125, [30, 1], [30, 20], 0, 32, 11),
    "prompt": (H70, [70, 1, 37], [70, 50, 200], 0, 32, 40),
    "prompt-last": (H7, [300], [420], 0, 16, 299),
    "prompt-64": (H125, [260, 5], [300, 5], 0, 16, 131),
    "prompt-behind": ((4, 4, 64), [300, 260], [300, 700], 257, 32, 200),
    "shares": (H70, [40, 1, 0], [3000, 1, 0], 0, 16, 25),
    "both": (H70, [20] + [1] * 9, [1200] + [5] * 9, 2900, 16, 12),
}


@pytest.mark.parametrize("name", MASKED)
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_tokens_do_not_meet_later_ones(sdq, name, bad):
    """Key and value of new token j of sequence 0, one head: the tokens before it are as without it."""
    import torch
    heads, new, own, prefix, page, j = MASKED[name]
    c = Case(heads, new, own, prefix, page, seed=len(name))
    want, _ = _run(sdq, torch, c)
    batch, q = c.batch(sdq, torch), to_bf16(torch, c.q)
    at, group = own[0] - new[0] + j, c.q_heads // c.kv_heads
    spot = int(c.pages[0, at // page]), c.kv_heads - 1, at % page
    for key in (False, True):
        cache = c.cache(sdq, torch)
        cache.v_pages[spot][7] = bad
        cache.v_pages[spot][c.dim - 2] = bad
        if key:
            cache.k_pages[spot][1] = bad
        out = cache.attend(batch, q)
        hit = torch.zeros(out.shape, dtype=torch.bool, device="cuda")
        rows = hit[j:new[0], (c.kv_heads - 1) * group:]
        if key:
            rows[:] = True   # (a score that is not finite: what is left of the row is not looked at)
        else:
            rows[..., 7] = rows[..., c.dim - 2] = True
            assert not torch.isfinite(out[hit]).any()
        assert torch.equal(out[~hit], want[~hit])
