"""GPU: rows that no sequence has stay as they were under a window, whatever it covers and
whichever route that takes."""
import numpy as np
import pytest

from serving_inputs import Case, to_bf16
from test_attention_window_gpu import _check

pytestmark = pytest.mark.gpu

H70, H7 = (16, 2, 128), (4, 4, 128)
ROWS = {
    # heads, new tokens, own tokens, prefix, page
    "prefix-narrow": (H7, [1, 1], [0, 0], 70, 16),
    "prefix-narrow-64": ((3, 3, 64), [1], [0], 130, 32),
    "prefix-wide": (H70, [1, 1, 2], [0, 0, 0], 77, 16),
    "prefix-wide-64": ((4, 2, 64), [40], [0], 200, 64),
    "prefix-shares": ((2, 1, 128), [1, 1, 40], [0, 0, 0], 3000, 128),
    "both-narrow": (H7, [1, 1], [40, 5], 70, 16),
    "both": (H70, [1, 2, 1], [40, 5, 0], 130, 16),
    "own-wide": (H70, [9, 1, 1], [40, 5, 0], 130, 32),
    "own-wide-shares": (H70, [9, 1], [3000, 5], 1200, 64),
    "one-line": (H70, [100, 60], [100, 90], 150, 16),
    "own-narrow": (H70, [1, 3], [900, 5], 0, 16),
    "own-alone": (H7, [150], [300], 0, 16),
    "own-shares": ((2, 1, 128), [20], [3000], 0, 64),
    "nothing": (H7, [2, 1], [0, 0], 0, 16),
}


@pytest.mark.parametrize("cover", ["window", "largest", "sinks", "no"])
@pytest.mark.parametrize("name", ROWS)
def test_rows_of_nobody_stay(sdq, name, cover):
    import torch
    heads, new, own, prefix, page = ROWS[name]
    c = Case(heads, new, own, prefix, page, seed=len(name))
    top = max(1, prefix + max(own))
    window, sinks = {"window": (top, 0), "largest": ((1 << 30) - 1, 3), "sinks": (1, top), "no": (max(1, top - 1), 0)}[cover]
    i = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()
    n, extra = c.tokens, 5
    cache = c.cache(sdq, torch)
    batch = sdq.Batch(i(c.start), i(own), i(c.pages), n + extra, max(new), max(own), i(c.prefix_pages), prefix)
    q = torch.cat([to_bf16(torch, c.q), torch.ones((extra, c.q_heads, c.dim), dtype=torch.bfloat16, device="cuda")])
    ws = cache.alloc_workspace(batch, c.q_heads, window=window, sinks=sinks)
    ws.random_(0, 256)
    out = torch.full((n + extra, c.q_heads, c.dim), 3.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((n + extra, c.q_heads), 3.0, device="cuda")
    sdq.sdq_attention_window(cache.handle, batch, c.q_heads, q, c.q_heads * c.dim, c.dim ** -0.5, window, sinks, out, lse, ws)
    assert sdq.sdq_attention_status(ws) == 0
    assert torch.all(out[n:] == 3.0) and torch.all(lse[n:] == 3.0)
    _check(c, out[:n], lse[:n], window, sinks)
