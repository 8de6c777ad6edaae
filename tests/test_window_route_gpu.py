"""GPU: which windowed calls read a shared prefix once for all sequences, and that the rule
goes both ways on the same batches."""
import pytest

from serving_inputs import Case
from test_attention_window_gpu import APART, _check, _run

pytestmark = pytest.mark.gpu


def _reads_apart(sdq, torch, c, window, sinks):
    """A call that reads the prefix apart keeps both parts' sums, fp32 for every row.  The rest of the workspace is the
    narrow kernel's, of the same size for every window; with a window of one position nothing of the prefix is worth it."""
    cache, batch = c.cache(sdq, torch), c.batch(sdq, torch)
    size = lambda w, s: sdq.sdq_attention_window_workspace_bytes(cache.handle, batch, c.q_heads, w, s)
    more = size(window, sinks) - size(1, 0)
    assert more == 0 or more >= 8 * c.tokens * c.q_heads * c.dim
    return more > 0


@pytest.mark.parametrize("name", APART)
def test_which_calls_read_a_shared_prefix_apart(sdq, name):
    import torch
    heads, new, own, prefix, page, window, sinks = APART[name]
    c = Case(heads, new, own, prefix, page, seed=len(name))
    assert _reads_apart(sdq, torch, c, window, sinks)
    for few in ((1, 0), (16, 4), (1, 16)):                 # the same batch, which now sees next to nothing of it
        assert not _reads_apart(sdq, torch, c, *few)
    out, lse = _run(sdq, torch, c, 16, 4)
    _check(c, out, lse, 16, 4)
