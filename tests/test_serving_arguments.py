"""CPU: what the attention call of the binding checks of its tensors before a
pointer of theirs reaches a kernel, with stand-ins for tensors on the GPU."""
import pytest
import torch


class _Cuda:
    """A tensor that says it is on the GPU."""

    def __init__(self, t):
        self.t = t

    is_cuda = True
    device = "cuda"

    def __getattr__(self, name):
        return getattr(self.t, name)


class _Reached(Exception):
    pass


@pytest.fixture
def call(sdq, monkeypatch):
    cache = sdq.KVCache.__new__(sdq.KVCache)
    cache.handle, cache.desc = None, sdq.CacheDesc(2, 64, 16, 4)
    i = lambda a: _Cuda(torch.tensor(a, dtype=torch.int32))
    batch = sdq.Batch(i([0, 3]), i([3]), i([[0, 1]]), 3, 3, 3)
    monkeypatch.setattr(sdq, "_empty", lambda shape, dtype, device, stream: torch.empty(shape, dtype=dtype))

    def reached(*a):
        raise _Reached

    monkeypatch.setattr(sdq, "sdq_attention", reached)
    q = _Cuda(torch.zeros((3, 4, 64), dtype=torch.bfloat16))
    return lambda ws: cache.attend(batch, q, ws=ws)


def test_workspace_of_attention(call):
    wide = torch.empty((64, 512), dtype=torch.uint8)
    with pytest.raises(_Reached):
        call(_Cuda(wide))
    for bad in (wide, _Cuda(wide[:, ::2]), _Cuda(wide.t()), _Cuda(wide[:, :256])):   # on the host; not one piece of memory
        with pytest.raises(ValueError):
            call(bad)
