"""CPU: serving calls refuse tensors on other devices than the cache's, or than
the current one, before a pointer of theirs reaches a kernel; with stand-ins
for tensors on several GPUs."""
import pytest
import torch


class _On:
    """A tensor that says which GPU it is on."""

    is_cuda = True

    def __init__(self, t, index):
        self.t, self.device = t, torch.device("cuda", index)

    def get_device(self):
        return self.device.index

    def __getattr__(self, name):
        return getattr(self.t, name)


class _Reached(Exception):
    pass


NAMES = ("k_pages", "v_pages", "token_start", "own_len", "pages", "prefix_pages", "cos", "sin", "q", "k", "v", "weight", "lse", "ws")


def _run(sdq, op, home, away=(), current=0):
    """The call with everything on device `home`, what `away` names on another one."""
    on = lambda name, t: _On(t, 1 - home if name in away else home)
    ints = lambda name, a: on(name, torch.tensor(a, dtype=torch.int32))
    pages = torch.zeros((4, 2, 16, 64), dtype=torch.bfloat16)
    cache = sdq.KVCache(sdq.CacheDesc(2, 64, 16, 4), on("k_pages", pages), on("v_pages", pages.clone()))
    batch = sdq.Batch(ints("token_start", [0, 3]), ints("own_len", [3]), ints("pages", [[0, 1]]), 3, 3, 3, ints("prefix_pages", [2]), 5)
    if op == "append":
        rope = sdq.Rope(on("cos", torch.zeros((8, 32))), on("sin", torch.zeros((8, 32))))
        q, k, v = (on(n, torch.zeros((3, h * 64))) for n, h in (("q", 4), ("k", 2), ("v", 2)))
        return cache.append(batch, q, k, v, rope, norm=sdq.HeadNorm(on("weight", torch.ones(64))))
    q = on("q", torch.zeros((3, 4, 64), dtype=torch.bfloat16))
    window = dict(window=3) if op == "window" else {}
    return cache.attend(batch, q, ws=on("ws", torch.zeros(1 << 12, dtype=torch.uint8)), lse=on("lse", torch.zeros((3, 4))), **window)


@pytest.fixture
def fakes(sdq, monkeypatch):
    def reached(*a, **k):
        raise _Reached
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(sdq, "sdq_cache_create", lambda *a: None)
    monkeypatch.setattr(sdq, "_empty", reached)
    return sdq


@pytest.mark.parametrize("op", ["append", "attend", "window"])
def test_cache_calls_need_everything_on_the_caches_device(fakes, op):
    with pytest.raises(_Reached):
        _run(fakes, op, 0)
    used = set(NAMES) - ({"lse", "ws"} if op == "append" else {"cos", "sin", "k", "v", "weight"})
    for name in sorted(used):
        with pytest.raises(ValueError):
            _run(fakes, op, 0, {name})
    with pytest.raises(ValueError):                       # all of it together, but not the current device
        _run(fakes, op, 1)


def test_sample_needs_everything_on_the_current_device(fakes):
    z, f, i = torch.zeros((2, 10)), torch.ones(2), torch.ones(2, dtype=torch.int32)
    args = lambda at: [_On(z, at[0]), _On(f, at[1]), _On(f, at[2]), _On(i, at[3]), _On(f, at[4]), _On(f, at[5])]
    with pytest.raises(_Reached):
        fakes.sample(*args([0] * 6))
    for away in range(6):
        with pytest.raises(ValueError):
            fakes.sample(*args([int(n == away) for n in range(6)]))
    with pytest.raises(ValueError):
        fakes.sample(*args([1] * 6))
