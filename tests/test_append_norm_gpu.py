"""GPU: appending with every head of q and k normalised ahead of the rotation,
against the fp64 definition, and what it refuses."""
import numpy as np
import pytest

import oracle as O
from serving_inputs import Case, bf16

pytestmark = pytest.mark.gpu


def _rows(torch, x, kind, pad):
    t = torch.from_numpy(np.ascontiguousarray(x.reshape(len(x), -1), np.float32)).cuda()
    wide = torch.full((t.shape[0], t.shape[1] + pad), float("nan"), device="cuda")
    wide[:, :t.shape[1]] = t
    return wide.to(torch.float32 if kind == "f32" else torch.bfloat16)[:, :t.shape[1]]


SHAPES = [
    # heads (q, kv, dim), new tokens, own tokens, prefix, page
    ((8, 1, 128), [1], [1], 0, 16),
    ((64, 8, 128), [1], [1037], 0, 16),
    ((12, 12, 64), [1] * 9, [1, 16, 17, 32, 33, 5, 31, 0, 64], 13, 32),
    ((3, 1, 64), [3, 0, 7, 1, 130], [3, 5, 40, 0, 200], 70, 64),       # 5 heads of 8 threads: no whole warps
    ((4, 4, 128), [1, 300], [128, 301], 0, 128),
]


@pytest.mark.parametrize("heads,new,own,prefix,page", SHAPES)
@pytest.mark.parametrize("kind,pad", [("f32", 0), ("f32", 24), ("bf16", 8)])
@pytest.mark.parametrize("rot,interleaved", [("all", False), ("part", True), (0, False), (8, False)])
@pytest.mark.parametrize("weights", ["both", "each", "q", "k-each", "none"])
def test_append_norm_matches_the_definition(sdq, heads, new, own, prefix, page, kind, pad, rot, interleaved, weights):
    import torch
    c = Case(heads, new, own, prefix, page, seed=len(new))
    rot = {"all": c.dim, "part": c.dim // 4}.get(rot, rot)
    rng = np.random.default_rng(5)
    x = [(10.0 ** rng.uniform(-3, 2, (c.tokens, h, 1)) * rng.standard_normal((c.tokens, h, c.dim))).astype(np.float32)
         for h in (c.q_heads, c.kv_heads, c.kv_heads)]
    x[0][0, 0] = 0                                            # a head of zeros stays one
    if kind == "bf16":
        x = [bf16(a) for a in x]
    qw = rng.standard_normal((c.q_heads, c.dim) if weights == "each" else c.dim).astype(np.float32) if weights in ("both", "each", "q") else None
    kw = rng.standard_normal(c.dim if weights == "both" else (c.kv_heads, c.dim)).astype(np.float32) if weights in ("both", "each", "k-each") else None
    dev = lambda a: None if a is None else torch.from_numpy(a).cuda()
    eps = 1e-5
    n_pos = prefix + max(own) + 1
    cos, sin = sdq.sdq_rope_table(n_pos, rot) if rot else (np.zeros((n_pos, 0), np.float32),) * 2
    rope = sdq.Rope(dev(cos), dev(sin), interleaved) if rot else sdq.Rope()
    cache = c.cache(sdq, torch)
    before = [cache.k_pages.clone(), cache.v_pages.clone()]
    q = cache.append(c.batch(sdq, torch), *(_rows(torch, a, kind, pad) for a in x), rope, norm=sdq.HeadNorm(dev(qw), dev(kw), eps))
    normed = [O.serving.head_norm(x[0], qw, eps), O.serving.head_norm(x[1], kw, eps), x[2].astype(np.float64)]
    ref = O.serving.append(*normed, c.k, c.v, c.start, own, c.pages, prefix, cos, sin, interleaved)
    # One rounding to bf16 (2^-8 of the result).  Ahead of it in fp32: the sum of squares (dim + 1 roundings, half of
    # their relative error after the root), the root (2^-22), two products; then three operations on a pair.  So
    # 2^-24 ((dim + 1) / 2 + 4 + 2 + 3) < 2^-17 of the pair's terms, twice a head's largest.
    for got, want, src in zip((q, cache.k_pages, cache.v_pages), ref, normed):
        got = got.float().cpu().numpy().astype(np.float64)
        top = np.abs(src).max() if want.shape != src.shape else np.abs(src).max(-1, keepdims=True)
        bound = 2.0 ** -8 * np.abs(want) + 2.0 ** -16 * top
        ok = np.abs(got - want) <= bound
        assert np.all(ok | (np.isnan(want) & np.isnan(got)))
    written = np.zeros(c.k.shape[:1] + c.k.shape[2:3], bool)
    for s, m in enumerate(own):
        for j in range(max(0, m - new[s]), m):
            written[c.pages[s, j // page], j % page] = True
    keep = torch.from_numpy(~written).cuda()[:, None, :, None]
    for a, b in zip(before, (cache.k_pages, cache.v_pages)):
        assert torch.equal(a.view(torch.int16) * keep, b.view(torch.int16) * keep)


@pytest.mark.parametrize("heads", [(64, 8, 128), (12, 12, 64), (20, 1, 128), (5, 1, 64)])
@pytest.mark.parametrize("kind,norm", [("f32", True), ("bf16", True), ("bf16", False)])
def test_many_tokens_are_those_of_small_calls(sdq, heads, kind, norm):
    """The calls of many tokens (pieces streamed through shared memory) give what the calls of few give, bit by bit:
    several sequences, an empty slot, tokens of nobody between and behind them, a page outside the cache."""
    import torch
    hq, hk, dim = heads
    rng = np.random.default_rng(9)
    total = -(-26000 // (hq + 2 * hk))
    cuts = np.sort(rng.choice(np.arange(1, total), 9, replace=False))
    new = np.diff(np.concatenate([[0], cuts, [total]])).tolist()
    own = [n + int(rng.integers(0, 40)) for n in new]
    own[3] = 0
    c = Case((hq, hk, dim), new, own, 11, 16, seed=2)
    c.pages[1, 0] = -1
    x = [torch.from_numpy((10.0 ** rng.uniform(-2, 1, (total, 1)) * rng.standard_normal((total, h * dim))).astype(np.float32)).cuda()
         for h in (hq, hk, hk)]
    x = [t if kind == "f32" else t.to(torch.bfloat16) for t in x]
    weights = sdq.HeadNorm(torch.randn((hq, dim), device="cuda"), torch.randn(dim, device="cuda")) if norm else None
    rope = sdq.Rope.table(11 + max(own) + 1, dim // 2, interleaved=dim == 64)
    a, b = c.cache(sdq, torch), c.cache(sdq, torch)
    got = a.append(c.batch(sdq, torch, max_new=max(new) - 1), *x, rope, norm=weights)
    i = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    want = torch.empty_like(got)
    for s, n in enumerate(new):                               # (the bound cuts a sequence's last token off)
        rows = slice(int(c.start[s]), int(c.start[s + 1]))
        few = max(1, 20000 // (hq + 2 * hk))
        for t in range(0, n, few):
            m = min(few, n - t)
            part = slice(rows.start + t, rows.start + t + m)
            kept = min(n, max(new) - 1)
            # the same places: own tokens up to the part's last one
            last = own[s] - kept + t + m if own[s] else 0
            start, keep = [0, m], m
            if t + m > kept:
                keep, last = kept - t, own[s]
                start = [0, keep]
            batch = sdq.Batch(i(start), i([last]), i(c.pages[s:s + 1].tolist()), m, max(1, keep), max(own), i(c.prefix_pages.tolist()), 11)
            want[part] = b.append(batch, *(v[part] for v in x), rope, norm=weights)
    assert torch.equal(a.k_pages.view(torch.int16), b.k_pages.view(torch.int16))
    assert torch.equal(a.v_pages.view(torch.int16), b.v_pages.view(torch.int16))
    assert torch.equal(got.view(torch.int16), want.view(torch.int16))


def test_without_weights_nothing_changes(sdq):
    import torch
    c = Case((4, 2, 64), [3, 20], [40, 20], 7, 16, seed=3)
    x = [torch.randn((23, h * 64), device="cuda") for h in (4, 2, 2)]
    a, b = c.cache(sdq, torch), c.cache(sdq, torch)
    rope = sdq.Rope.table(64, 64)
    assert torch.equal(a.append(c.batch(sdq, torch), *x, rope), b.append(c.batch(sdq, torch), *x, rope, norm=sdq.HeadNorm()))
    assert torch.equal(a.k_pages.view(torch.int16), b.k_pages.view(torch.int16))


def test_values_that_are_not_finite_stay_in_their_head(sdq):
    import torch
    c = Case((4, 2, 64), [2], [2], 0, 16, seed=4)
    x = [torch.randn((2, h * 64), device="cuda") for h in (4, 2, 2)]
    w = torch.ones(64, device="cuda")
    rope, norm = sdq.Rope.table(64, 64), sdq.HeadNorm(w, w)
    want = c.cache(sdq, torch).append(c.batch(sdq, torch), *x, rope, norm=norm)
    x[0][0, 70], x[0][1, 3] = float("nan"), float("inf")
    got = c.cache(sdq, torch).append(c.batch(sdq, torch), *x, rope, norm=norm)
    assert got[0, 1].isnan().all() and got[1, 0].isnan().any()
    for t, h in ((0, 0), (0, 2), (0, 3), (1, 1), (1, 2), (1, 3)):
        assert torch.equal(got[t, h], want[t, h])


def test_append_norm_in_a_graph_and_on_another_stream(sdq):
    import torch
    c = Case((4, 2, 64), [1, 1], [17, 3], 0, 16, seed=7)
    cache, batch = c.cache(sdq, torch), c.batch(sdq, torch, max_own=32)
    x = [torch.randn((2, h * 64), device="cuda") for h in (4, 2, 2)]
    norm = sdq.HeadNorm(torch.rand(64, device="cuda"), torch.rand((2, 64), device="cuda"))
    rope = sdq.Rope.table(64, 64)
    want = cache.append(batch, *x, rope, norm=norm)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = cache.append(batch, *x, rope, side, norm)
    side.synchronize()
    assert torch.equal(got, want)
    out, graph = torch.empty_like(want), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sdq.sdq_cache_append_norm(cache.handle, batch, 4, *x, rope, norm, out)
    for t in x:
        t.mul_(-3.0)                                          # the same heads, turned round
    graph.replay()
    torch.cuda.synchronize()
    assert (out.float() + want.float()).abs().max() <= 2.0 ** -7 * want.float().abs().max()


def test_append_norm_refusals(sdq):
    import torch
    c = Case((4, 2, 64), [1, 2], [17, 3], 5, 16, seed=8)
    cache, batch, rope = c.cache(sdq, torch), c.batch(sdq, torch), sdq.Rope.table(64, 64)
    x = [torch.randn((3, h * 64), device="cuda") for h in (4, 2, 2)]
    out = torch.empty((3, 4, 64), dtype=torch.bfloat16, device="cuda")
    w = torch.ones(64, device="cuda")
    for bad in (lambda: sdq.HeadNorm(w.double()), lambda: sdq.HeadNorm(w.cpu()), lambda: sdq.HeadNorm(w, torch.ones((2, 128), device="cuda")[:, ::2]),
                lambda: sdq.HeadNorm(w, w, 0.0), lambda: sdq.HeadNorm(w, w, float("nan")), lambda: sdq.HeadNorm(w[None, None]),
                lambda: cache.append(batch, *x, rope, norm=sdq.HeadNorm(w[:32].clone())),
                lambda: cache.append(batch, *x, rope, norm=sdq.HeadNorm(None, w.expand(4, 64).contiguous()))):
        with pytest.raises(ValueError):
            bad()
    for field, value in (("eps", 0.0), ("eps", float("inf")), ("q_per_head", 2), ("k_per_head", -1), ("q", w.data_ptr() + 4)):
        norm = sdq.HeadNorm(w, w)
        setattr(norm._c, field, value)
        with pytest.raises(sdq.SdqError) as e:
            sdq.sdq_cache_append_norm(cache.handle, batch, 4, *x, rope, norm, out)
        assert e.value.status == -1
    torch.cuda.synchronize()
