"""GPU: appending keys and values to the paged cache with the position
rotation, against the fp64 definition, and what it refuses."""
import ctypes

import numpy as np
import pytest

import oracle as O
from serving_inputs import Case, bf16, to_bf16

pytestmark = pytest.mark.gpu


def _rows(torch, x, kind, pad):
    """x (tokens, heads, dim) as rows of `kind` whose stride is `pad` elements longer than they are."""
    t = torch.from_numpy(np.ascontiguousarray(x.reshape(len(x), -1), np.float32)).cuda()
    wide = torch.full((t.shape[0], t.shape[1] + pad), float("nan"), device="cuda")
    wide[:, :t.shape[1]] = t
    return wide.to(torch.float32 if kind == "f32" else torch.bfloat16)[:, :t.shape[1]]


SHAPES = [
    # heads (q, kv, dim), new tokens, own tokens, prefix, page
    ((8, 1, 128), [1], [1], 0, 16),
    ((64, 8, 128), [1], [1037], 0, 16),
    ((12, 12, 64), [1] * 9, [1, 16, 17, 32, 33, 5, 31, 0, 64], 13, 32),
    ((10, 2, 64), [3, 0, 7, 1, 130], [3, 5, 40, 0, 200], 70, 64),
    ((4, 4, 128), [1, 300], [128, 301], 0, 128),
]


@pytest.mark.parametrize("heads,new,own,prefix,page", SHAPES)
@pytest.mark.parametrize("kind,pad", [("f32", 0), ("f32", 24), ("bf16", 8)])
@pytest.mark.parametrize("rot,interleaved", [("all", False), ("all", True), ("part", False), ("part", True), (0, False), (8, False)])
def test_append_matches_the_definition(sdq, heads, new, own, prefix, page, kind, pad, rot, interleaved):
    import torch
    c = Case(heads, new, own, prefix, page, seed=len(new))
    rot = {"all": c.dim, "part": c.dim // 4}.get(rot, rot)
    rng = np.random.default_rng(5)
    x = [rng.standard_normal((c.tokens, h, c.dim)).astype(np.float32) for h in (c.q_heads, c.kv_heads, c.kv_heads)]
    if kind == "bf16":
        x = [bf16(a) for a in x]
    n_pos = prefix + max(own) + 1
    cos, sin = sdq.sdq_rope_table(n_pos, rot) if rot else (np.zeros((n_pos, 0), np.float32),) * 2
    rope = sdq.Rope(torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda(), interleaved) if rot else sdq.Rope()
    cache = c.cache(sdq, torch)
    before = [cache.k_pages.clone(), cache.v_pages.clone()]
    q = cache.append(c.batch(sdq, torch), *(_rows(torch, a, kind, pad) for a in x), rope)
    ref = O.serving.append(*x, c.k, c.v, c.start, own, c.pages, prefix, cos, sin, interleaved)
    # one rounding to bf16 (2^-8 of the result), three fp32 operations on terms no larger than the pair's
    half = rot // 2
    for got, want, src in zip((q, cache.k_pages, cache.v_pages), ref, x):
        got = got.float().cpu().numpy().astype(np.float64)
        bound = 2.0 ** -8 * np.abs(want) + 2.0 ** -22 * 2 * np.abs(src).max()
        ok = np.abs(got - want) <= bound
        assert np.all(ok | (np.isnan(want) & np.isnan(got)))
    # everything else in the cache kept its bits
    written = np.zeros(c.k.shape[:1] + c.k.shape[2:3], bool)
    for s, m in enumerate(own):
        for j in range(max(0, m - new[s]), m):
            written[c.pages[s, j // page], j % page] = True
    keep = torch.from_numpy(~written).cuda()[:, None, :, None]
    for a, b in zip(before, (cache.k_pages, cache.v_pages)):
        assert torch.equal(a.view(torch.int16) * keep, b.view(torch.int16) * keep)
    if half == 0:
        assert torch.equal(q, to_bf16(torch, x[0]))


def test_pages_outside_the_cache_and_tokens_beyond_the_bounds_are_left_out(sdq):
    import torch
    c = Case((4, 2, 64), [2, 3], [40, 20], 0, 16, seed=3)
    c.pages[0, 2] = c.n_pages          # the page of sequence 0's new tokens
    c.pages[1, 1] = -1
    cache = c.cache(sdq, torch)
    before = cache.k_pages.clone()
    x = [torch.randn((5, h * 64), device="cuda") for h in (4, 2, 2)]
    q = cache.append(c.batch(sdq, torch), *x, sdq.Rope())
    assert torch.equal(cache.k_pages.view(torch.int16), before.view(torch.int16))
    assert torch.equal(q.reshape(5, -1), x[0].to(torch.bfloat16))
    c = Case((4, 2, 64), [4], [20], 0, 16, seed=4)
    cache = c.cache(sdq, torch)
    before = cache.k_pages.clone()
    x = [torch.randn((4, h * 64), device="cuda") for h in (4, 2, 2)]
    cache.append(c.batch(sdq, torch, max_new=1, max_own=16), *x, sdq.Rope.table(16, 64))   # as 1 new token of 16
    changed = (cache.k_pages.view(torch.int16) != before.view(torch.int16)).any(3).any(1).nonzero().tolist()
    assert changed == [[int(c.pages[0, 0]), 15]]


def test_positions_far_out(sdq):
    """The table is read at the position itself, also behind a prefix of more than 2^20 tokens (nothing of the
    prefix is read here)."""
    import torch
    c = Case((2, 1, 64), [2], [5], 0, 16, seed=6)
    n_pos = (1 << 20) + 40
    cos, sin = (torch.rand((n_pos, 4), device="cuda") for _ in range(2))
    cache = c.cache(sdq, torch)
    b = c.batch(sdq, torch)
    b._c.prefix_len, b._c.prefix_pages = (1 << 20) + 3, b._c.pages
    x = [torch.randn((2, h * 64), device="cuda") for h in (2, 1, 1)]
    out = torch.empty((2, 2, 64), dtype=torch.bfloat16, device="cuda")
    sdq.sdq_cache_append(cache.handle, b, 2, *x, sdq.Rope(cos, sin), out)
    for i in range(2):
        p = (1 << 20) + 3 + 3 + i
        want = O.serving.rotate(x[0][i].reshape(2, 64).cpu().numpy().astype(np.float64), 0, cos[p:p + 1].cpu().numpy(),
                                sin[p:p + 1].cpu().numpy(), False)
        assert np.abs(out[i].float().cpu().numpy() - want).max() <= 2.0 ** -8 * np.abs(want).max() + 2.0 ** -20


def test_append_on_another_stream_and_in_a_graph(sdq):
    import torch
    c = Case((4, 2, 64), [1, 1], [17, 3], 0, 16, seed=7)
    cache, batch = c.cache(sdq, torch), c.batch(sdq, torch, max_own=32)
    x = [torch.randn((2, h * 64), device="cuda") for h in (4, 2, 2)]
    want = cache.append(batch, *x, sdq.Rope.table(64, 64))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = cache.append(batch, *x, sdq.Rope.table(64, 64))
    side.synchronize()
    assert torch.equal(got, want)
    rope, out = sdq.Rope.table(64, 64), torch.empty_like(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sdq.sdq_cache_append(cache.handle, batch, 4, *x, rope, out)
    batch.tensors[1].copy_(torch.tensor([18, 4], dtype=torch.int32))     # the next step: one more token each
    graph.replay()
    torch.cuda.synchronize()
    for s, own in enumerate((18, 4)):
        page, slot = int(c.pages[s, (own - 1) // 16]), (own - 1) % 16
        assert torch.equal(cache.v_pages[page, :, slot].reshape(-1), x[2][s].to(torch.bfloat16))


def test_append_refusals(sdq):
    import torch
    c = Case((4, 2, 64), [1, 2], [17, 3], 5, 16, seed=8)
    cache, batch, rope = c.cache(sdq, torch), c.batch(sdq, torch), sdq.Rope.table(64, 64)
    x = [torch.randn((3, h * 64), device="cuda") for h in (4, 2, 2)]
    out = torch.empty((3, 4, 64), dtype=torch.bfloat16, device="cuda")

    def refused(batch=batch, q_heads=4, q=x[0], k=x[1], v=x[2], rope=rope, out=out, **fields):
        saved = {n: getattr(batch._c, n) for n in fields}
        for n, val in fields.items():
            setattr(batch._c, n, val)
        try:
            with pytest.raises(sdq.SdqError) as e:
                sdq.sdq_cache_append(cache.handle, batch, q_heads, q, k, v, rope, out)
            assert e.value.status == -1
        finally:
            for n, val in saved.items():
                setattr(batch._c, n, val)

    for fields in (dict(n_seqs=0), dict(n_tokens=0), dict(max_new=0), dict(max_new=4), dict(max_own=-1), dict(max_own=33),
                   dict(prefix_len=-1), dict(token_start=None), dict(own_len=None), dict(pages=None),
                   dict(prefix_pages=None), dict(prefix_len=1 << 30)):
        refused(**fields)
    refused(q_heads=3)
    refused(q_heads=0)
    refused(q_heads=6)                                        # wider than q's rows
    refused(q=x[0].double())
    refused(k=x[1].half())
    refused(k=x[1].to(torch.bfloat16))                        # two types in one call
    refused(rope=sdq.Rope.table(21, 64))                      # 5 + 17 positions
    refused(rope=sdq.Rope.table(64, 128))
    refused(rope=sdq.Rope.table(64, 12))
    odd = torch.randn(3 * 258 + 2, device="cuda")
    refused(q=odd[:3 * 258].reshape(3, 258)[:, :256])         # a row stride of 258 x 4 bytes
    refused(q=odd[1:1 + 3 * 256].reshape(3, 256))
    refused(out=torch.empty(3 * 256 + 4, dtype=torch.bfloat16, device="cuda")[4:])
    for bad in (lambda: cache.append(batch, x[0][:2], x[1], x[2], rope), lambda: cache.append(batch, x[0], x[1][:, :64], x[2], rope),
                lambda: cache.append(batch, x[0][:, :200], x[1], x[2], rope), lambda: cache.append(batch, x[0], x[1], x[2].cpu(), rope),
                lambda: sdq.Rope(torch.zeros((4, 4), device="cuda")), lambda: sdq.KVCache(c.desc(sdq), cache.k_pages),
                lambda: sdq.KVCache(c.desc(sdq), cache.k_pages, cache.v_pages.float()),
                lambda: sdq.Batch(batch.tensors[0].long(), *batch.tensors[1:3], 3, 2, 17),
                lambda: sdq.Batch(batch.tensors[0][:2], *batch.tensors[1:3], 3, 2, 17)):
        with pytest.raises(ValueError):
            bad()
    for desc in (sdq.CacheDesc(0, 64, 16, 4), sdq.CacheDesc(2, 96, 16, 4), sdq.CacheDesc(2, 64, 24, 4), sdq.CacheDesc(2, 64, 16, 0),
                 sdq.CacheDesc(1024, 64, 128, 1 << 14)):
        assert sdq.sdq_cache_bytes(desc) == 0
        h = ctypes.c_void_p()
        assert sdq.lib().sdq_cache_create(ctypes.byref(desc.c()), cache.k_pages.data_ptr(), cache.v_pages.data_ptr(), ctypes.byref(h)) == -1
    torch.cuda.synchronize()
