"""GPU: appends without norms of more tokens than the device has places for their
thread blocks give, bit by bit, what appends of few tokens give."""
import numpy as np
import pytest

from serving_inputs import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads", [(64, 8, 128), (12, 12, 64), (8, 1, 128), (5, 1, 64)])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rot,interleaved", [("all", False), ("half", True), ("quarter", False), ("none", False)])
def test_many_tokens_are_those_of_small_calls(sdq, heads, kind, rot, interleaved):
    """Several sequences, an empty slot, a page outside the cache, padded rows; and the same rows a hundred at a time."""
    import torch
    hq, hk, dim = heads
    places = 2 * torch.cuda.get_device_properties(0).multi_processor_count
    new = [places - 60, 1, 37, 25]                          # three tokens more than the places
    own = [new[0] + 5, 0, 37, 140]
    c = Case(heads, new, own, 11, 16, seed=hq)
    c.pages[2, 1] = -1
    g = torch.Generator("cuda").manual_seed(hq)
    dtype = torch.float32 if kind == "f32" else torch.bfloat16
    x = [torch.randn((c.tokens, h * dim + 8), device="cuda", generator=g).to(dtype)[:, :h * dim] for h in (hq, hk, hk)]
    n_rot = {"all": dim, "half": dim // 2, "quarter": dim // 4}.get(rot, 0)
    rope = sdq.Rope.table(11 + max(own) + 1, n_rot, interleaved=interleaved) if n_rot else sdq.Rope()
    a, b = c.cache(sdq, torch), c.cache(sdq, torch)
    got = a.append(c.batch(sdq, torch), *x, rope)
    want = torch.empty_like(got)
    i = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    for s, n in enumerate(new):
        for t in range(0, n, 100):
            m = min(100, n - t)
            rows = slice(int(c.start[s]) + t, int(c.start[s]) + t + m)
            last = own[s] - n + t + m if own[s] else 0
            batch = sdq.Batch(i([0, m]), i([last]), i(c.pages[s:s + 1].tolist()), m, m, max(own), i(c.prefix_pages.tolist()), 11)
            want[rows] = b.append(batch, *(v[rows] for v in x), rope)
    assert torch.equal(got.view(torch.int16), want.view(torch.int16))
    for u, v in ((a.k_pages, b.k_pages), (a.v_pages, b.v_pages)):
        assert torch.equal(u.view(torch.int16), v.view(torch.int16))


def test_rows_of_nobody_and_the_line_between_the_two(sdq):
    """One token fewer and one more than the places; rows behind the last sequence leave the cache as it was."""
    import torch
    places = 2 * torch.cuda.get_device_properties(0).multi_processor_count
    for tokens in (places - 1, places, places + 1):
        c = Case((4, 2, 64), [tokens - 3], [tokens - 3], 0, 16, seed=1)
        i = lambda v: torch.from_numpy(np.ascontiguousarray(v, np.int32)).cuda()
        x = [torch.randn((tokens, h * 64), device="cuda", generator=torch.Generator("cuda").manual_seed(h)) for h in (4, 2, 2)]
        rope, (a, b) = sdq.Rope.table(tokens, 64), (c.cache(sdq, torch) for _ in range(2))
        batch = sdq.Batch(i(c.start), i(c.own), i(c.pages), tokens, tokens, tokens - 3)
        got = a.append(batch, *x, rope)
        want = b.append(sdq.Batch(i([0, 1]), i([1]), i(c.pages), 1, 1, 1), *(v[:1] for v in x), rope)
        assert torch.equal(got[0], want[0])
        flat = a.v_pages.transpose(1, 2).reshape(-1, 2, 64)
        places_of = i((c.pages[0][np.arange(tokens - 3) // 16] * 16 + np.arange(tokens - 3) % 16)).long()
        assert torch.equal(flat[places_of].reshape(tokens - 3, -1), x[2][:tokens - 3].to(torch.bfloat16))
        rest = torch.ones(flat.shape[0], dtype=torch.bool, device="cuda")
        rest[places_of] = False
        assert flat[rest].isnan().all()
