"""GPU: attention over the paged cache against the fp64 definition, where it
can go wrong: lengths around pages and tiles, one token and many, empty slots,
prefixes that end inside a page, leftovers in free places, extreme scores; and
what it refuses."""
import numpy as np
import pytest

import oracle as O
from serving_inputs import Case, bf16, to_bf16

pytestmark = pytest.mark.gpu


def _run(sdq, torch, c, scale=None, lse=True, **bounds):
    cache, batch = c.cache(sdq, torch), c.batch(sdq, torch, **bounds)
    q = to_bf16(torch, c.q)
    ws = cache.alloc_workspace(batch, c.q_heads)
    ws.random_(0, 256)                       # a workspace needs no initialization
    out_lse = torch.full((c.tokens, c.q_heads), 7.0, device="cuda") if lse else None
    out = cache.attend(batch, q, scale, ws=ws, lse=out_lse)
    assert sdq.sdq_attention_status(ws) == 0
    return out, out_lse


def _check(c, out, lse, scale=None):
    scale = c.dim ** -0.5 if scale is None else scale
    want, want_lse, mag = O.serving.attend(c.q, c.k, c.v, c.start, c.own, c.pages, c.prefix_pages, c.prefix, scale)
    got = out.float().cpu().numpy().astype(np.float64)
    # Scores: fp32 sums of `dim` products, |q||k| scale (dim + 8) 2^-24 in all, as a relative error of each weight
    # (of numerator and denominator); weights rounded to bf16 (2^-8, half its spacing), by ex2.approx (2^-22) and up
    # to 2^-10 in all for fp32 sums of them; the output rounded once (2^-8 of it).
    norm = np.linalg.norm(c.q, axis=-1).max() * np.linalg.norm(np.nan_to_num(c.k), axis=-1).max()
    score = norm * scale * (c.dim + 8) * 2.0 ** -24
    bound = mag * (2 * score + 2.0 ** -8 + 2.0 ** -10) + 2.0 ** -8 * np.abs(want) + 1e-30
    assert np.all(np.isfinite(got))
    assert np.all(np.abs(got - want) <= bound), float((np.abs(got - want) / bound).max())
    if lse is not None:
        got_lse = lse.cpu().numpy().astype(np.float64)
        empty = np.isinf(want_lse)
        assert np.array_equal(np.isinf(got_lse), empty) and np.all(got_lse[empty] < 0)
        fine = ~empty
        assert np.all(np.abs(got_lse - want_lse)[fine] <= (score + 2.0 ** -10 + 2.0 ** -20 * np.abs(want_lse))[fine])


H70, H7, H125, ODD = (16, 2, 128), (4, 4, 128), (3, 3, 64), (10, 2, 64)

CASES = {
    # one token over contexts that end before, at and after the edges of pages and tiles
    "edges": (H70, [1] * 13, [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 191, 257], 0, 16),
    "edges-64": (H125, [1] * 9, [1, 31, 32, 33, 127, 128, 129, 255, 400], 0, 32),
    "one": (H70, [1], [1], 0, 16),
    "one-mha": (H7, [1], [700], 0, 128),
    "long": (H70, [1], [5003], 0, 64),
    # empty slots, sequences without new tokens, both ends
    "empty": (H70, [1, 1, 0, 1, 0], [0, 40, 33, 0, 0], 0, 16),
    "all-empty": (H125, [1, 1], [0, 0], 0, 16),
    # drafted tokens: causal rows in one tile, some sequences shorter than their own draft allows
    "draft": (H70, [3, 2, 1, 4], [3, 130, 64, 67], 0, 16),
    "draft-odd": (ODD, [5, 3], [5, 140], 0, 64),
    # prompts: more rows than one block holds
    "prompt": (H70, [70, 1, 37], [70, 50, 200], 0, 32),
    "prompt-mha": (H7, [150], [300], 0, 16),
    "prompt-long": (H7, [500, 3], [700, 300], 0, 16),
    "prompt-behind": ((4, 4, 64), [300, 260], [300, 700], 257, 32),
    "prompt-short-behind": (H70, [9, 20, 5, 1], [9, 400, 5, 1], 140, 16),
    "prompt-odd": (ODD, [33, 129], [40, 129], 0, 16),
    # prefixes: alone, ending inside a page and a tile, with everything behind them
    "prefix-only": (H70, [1, 1, 1], [0, 0, 0], 77, 16),
    "prefix-1": (H7, [1, 1], [5, 0], 1, 16),
    "prefix": (H70, [1] * 9, [1, 7, 16, 30, 0, 65, 128, 3, 200], 301, 16),
    "prefix-mha": (H7, [1] * 20, list(range(1, 21)), 128, 64),
    "prefix-draft": (ODD, [3, 1, 5], [3, 90, 5], 515, 128),
    "prefix-prompt": (H70, [100, 1, 20], [100, 30, 25], 150, 16),
    "prefix-many": (H70, [1] * 40, [(7 * i) % 50 for i in range(40)], 270, 32),
    "prefix-split": (H70, [1] * 33, [(3 * i) % 20 for i in range(33)], 2900, 64),
    "prefix-64": (H125, [1] * 140, [1 + i % 9 for i in range(140)], 200, 16),
    "many": (H125, [1] * 70, [(5 * i) % 97 for i in range(70)], 0, 16),
}


@pytest.mark.parametrize("name", CASES)
def test_attention_matches_the_definition(sdq, name):
    import torch
    heads, new, own, prefix, page = CASES[name]
    c = Case(heads, new, own, prefix, page, seed=len(name))
    _check(c, *_run(sdq, torch, c))


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("heads", [H70, H125])
@pytest.mark.parametrize("new", [1, 3, 40])
@pytest.mark.parametrize("prefix", [0, 130])
def test_pages_of_every_size(sdq, page, heads, new, prefix):
    import torch
    c = Case(heads, [new, 1, new], [new, 150, new + 129], prefix, page, seed=page + new)
    _check(c, *_run(sdq, torch, c, lse=False))


@pytest.mark.parametrize("spread,scale", [(30.0, None), (1.0, 1e-6), (1.0, 20.0), (1e-3, 1.0)])
@pytest.mark.parametrize("heads,new", [(H70, 1), (H125, 70)])
def test_scores_of_every_size(sdq, spread, scale, heads, new):
    """From weights that are all alike to one key that takes everything."""
    import torch
    c = Case(heads, [new, new], [new + 100, new], 140, 16, seed=11, spread=spread)
    out, lse = _run(sdq, torch, c, scale)
    want, _, mag = O.serving.attend(c.q, c.k, c.v, c.start, c.own, c.pages, c.prefix_pages, c.prefix,
                                    c.dim ** -0.5 if scale is None else scale)
    if spread * (scale or 0.1) < 1.5:
        _check(c, out, lse, scale)
    else:
        # scores of hundreds: an error of 2^-24 of them in every score (see _check), at least a weight's error of 1 %
        s = np.linalg.norm(c.q, axis=-1).max() * np.linalg.norm(np.nan_to_num(c.k), axis=-1).max() * (scale or c.dim ** -0.5)
        err = np.abs(out.float().cpu().numpy() - want)
        assert np.all(err <= mag * (2 * s * (c.dim + 8) * 2.0 ** -24 + 2.0 ** -8 + 2.0 ** -10) + 2.0 ** -8 * np.abs(want))


def test_keys_increasing_and_decreasing(sdq):
    """The running maximum changes at every tile, or never after the first."""
    import torch
    for order in (1, -1):
        for heads, new in ((H70, 1), (H7, 40)):
            c = Case(heads, [new], [900], 0, 16, seed=13)
            ramp = np.linspace(0, 3, 900)[::order]
            for j in range(900):
                c.k[c.pages[0, j // 16], :, j % 16] = bf16(ramp[j])
            c.q[:] = bf16(np.abs(c.q) * 0.3)
            _check(c, *_run(sdq, torch, c))


def test_strided_queries_streams_and_workspaces(sdq):
    import torch
    c = Case(H70, [1, 2, 30], [20, 30, 40], 33, 16, seed=17)
    cache, batch = c.cache(sdq, torch), c.batch(sdq, torch)
    q = to_bf16(torch, c.q)
    want = cache.attend(batch, q)
    torch.cuda.synchronize()
    wide = torch.full((c.tokens, c.q_heads + 4, c.dim), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, 2:2 + c.q_heads] = q
    assert torch.equal(cache.attend(batch, wide[:, 2:2 + c.q_heads]), want)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = cache.attend(batch, q)
    side.synchronize()
    assert torch.equal(got, want)
    # one workspace for other batches in between; the same bits every time
    ws = torch.empty(1 << 26, dtype=torch.uint8, device="cuda")
    other = Case(H70, [1] * 30, [100] * 30, 0, 16, seed=18)
    oc, ob, oq = other.cache(sdq, torch), other.batch(sdq, torch), to_bf16(torch, other.q)
    for _ in range(5):
        oc.attend(ob, oq, ws=ws)
        assert torch.equal(cache.attend(batch, q, ws=ws), want)


@pytest.mark.parametrize("new,prefix", [(1, 0), (1, 200), (30, 200)])
def test_in_a_graph_with_growing_lengths(sdq, new, prefix):
    """A captured call follows the device arrays: the sequences grow by tokens appended between replays."""
    import torch
    c = Case(H70, [new, new], [new + 90, new + 60], prefix, 16, seed=19)
    cache, batch = c.cache(sdq, torch), c.batch(sdq, torch)
    q, ws = to_bf16(torch, c.q), cache.alloc_workspace(batch, c.q_heads)
    out = torch.empty_like(q)
    call = lambda: sdq.sdq_attention(cache.handle, batch, c.q_heads, q, c.q_heads * c.dim, c.dim ** -0.5, out, None, ws)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for own in ([new, new + 60], [new + 89, new], [new + 90, new + 1]):
        batch.tensors[1].copy_(torch.tensor(own, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        c.own = own
        _check(c, out, None)


def test_inputs_from_the_kernel_before(sdq):
    """Append and attention back to back, with nothing between them."""
    import torch
    c = Case(H70, [1, 1, 1], [17, 200, 64], 40, 16, seed=23)
    rng = np.random.default_rng(1)
    x = [bf16(rng.standard_normal((3, h, c.dim))) for h in (c.q_heads, c.kv_heads, c.kv_heads)]
    cos, sin = sdq.sdq_rope_table(300, c.dim)
    cache, batch = c.cache(sdq, torch), c.batch(sdq, torch)
    rope = sdq.Rope(torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda())
    rows = [torch.from_numpy(a.reshape(3, -1)).cuda() for a in x]
    for _ in range(20):
        cache.k_pages.copy_(to_bf16(torch, c.k))
        q = cache.append(batch, *rows, rope)
        out = cache.attend(batch, q)
    qr, kr, vr = O.serving.append(*x, c.k, c.v, c.start, c.own, c.pages, c.prefix, cos, sin, False)
    c.q, c.k, c.v = bf16(qr), bf16(kr), bf16(vr)
    assert torch.equal(q, to_bf16(torch, c.q))
    _check(c, out, None)


def test_pages_outside_the_cache_read_as_zeros(sdq):
    import torch
    c = Case(H70, [1, 1], [40, 20], 0, 16, seed=29)
    c.pages[0, 1], c.pages[1, 0] = c.n_pages + 5, -3
    zero = Case(H70, [1, 1], [40, 20], 0, 16, seed=29)
    for table, i in ((zero.pages[0], 1), (zero.pages[1], 0)):
        zero.k[table[i]] = zero.v[table[i]] = 0
    zero.q = c.q
    out, lse = _run(sdq, torch, c)
    _check(zero, out, lse)


@pytest.mark.parametrize("new,prefix", [(1, 0), (1, 200), (1, 3000), (2, 40), (40, 0), (40, 200)])
@pytest.mark.parametrize("where", ["own", "prefix", "query"])
def test_nan_reaches_the_rows_that_see_it(sdq, new, prefix, where):
    """A NaN key reaches the tokens that see it, all of its sequence's for the oldest own key, every one's for a
    prefix's; a NaN query its own head; other rows keep their values."""
    import torch
    if where == "prefix" and prefix == 0:
        pytest.skip("no prefix")
    for dim_heads in (H70, H125):
        c = Case(dim_heads, [new, new, new], [new + 70, new + 33, 700 + new], prefix, 16, seed=41)
        clean = Case(dim_heads, [new, new, new], [new + 70, new + 33, 700 + new], prefix, 16, seed=41)
        bad = np.zeros((c.tokens, c.q_heads), bool)
        group = c.q_heads // c.kv_heads
        if where == "own":
            c.k[c.pages[1, 0], 0, 0] = np.nan
            bad[new:2 * new, :group] = True
        elif where == "prefix":
            c.k[c.prefix_pages[0], 1, 3] = np.nan
            bad[:, group:2 * group] = True
        else:
            c.q[new, 1] = np.nan
            bad[new, 1] = True
        out, _ = _run(sdq, torch, c)
        want, _ = _run(sdq, torch, clean)
        nan = torch.isnan(out).any(-1).cpu().numpy()
        assert np.array_equal(nan, bad)
        good = torch.from_numpy(~bad).cuda()
        assert torch.equal(out[good], want[good])


def test_lengths_beyond_the_bounds_are_cut(sdq):
    import torch
    c = Case(H70, [1], [90], 0, 16, seed=31)
    out, lse = _run(sdq, torch, c, max_own=50)
    c.own = [50]
    _check(c, out, lse)


def test_attention_refusals(sdq):
    import torch
    c = Case(H70, [1, 2], [20, 30], 33, 16, seed=37)
    cache, batch = c.cache(sdq, torch), c.batch(sdq, torch)
    q = to_bf16(torch, c.q)
    out, ws = torch.empty_like(q), cache.alloc_workspace(batch, c.q_heads)
    lse = torch.empty((3, c.q_heads), device="cuda")

    def refused(status=-1, handle=cache.handle, batch=batch, heads=c.q_heads, q=q, ldq=c.q_heads * c.dim, scale=0.1, out=out,
                lse=lse, ws=ws, **fields):
        saved = {n: getattr(batch._c, n) for n in fields}
        for n, val in fields.items():
            setattr(batch._c, n, val)
        try:
            with pytest.raises(sdq.SdqError) as e:
                sdq.sdq_attention(handle, batch, heads, q, ldq, scale, out, lse, ws)
            assert e.value.status == status
        finally:
            for n, val in saved.items():
                setattr(batch._c, n, val)

    for scale in (0.0, -1.0, float("nan"), float("inf")):
        refused(scale=scale)
    refused(heads=3)
    refused(heads=0)
    refused(ldq=c.q_heads * c.dim - 8)
    refused(ldq=c.q_heads * c.dim + 4)
    refused(handle=None)
    refused(ws=ws[:-1], status=-3)
    refused(ws=torch.empty(ws.numel() + 64, dtype=torch.uint8, device="cuda")[64:])
    refused(q=torch.empty(4 * q.numel(), dtype=torch.bfloat16, device="cuda")[4:])
    refused(out=torch.empty(4 * q.numel(), dtype=torch.bfloat16, device="cuda")[4:])
    for fields in (dict(n_seqs=0), dict(n_tokens=0), dict(max_new=0), dict(max_new=4), dict(max_own=-1), dict(max_own=33),
                   dict(prefix_len=-1), dict(token_start=None), dict(own_len=None), dict(pages=None), dict(prefix_pages=None)):
        refused(**fields)
    for bad in (lambda: cache.attend(batch, q[:2]), lambda: cache.attend(batch, q.float()), lambda: cache.attend(batch, q[..., :64]),
                lambda: cache.attend(batch, q.transpose(0, 1).contiguous().transpose(0, 1)),
                lambda: cache.attend(batch, q, lse=lse[:2]), lambda: cache.attend(batch, q, lse=lse.double())):
        with pytest.raises(ValueError):
            bad()
    assert sdq.lib().sdq_attention_status(None, None) == -1
    torch.cuda.synchronize()
