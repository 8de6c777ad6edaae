"""GPU: attention with a window of positions and first tokens that stay visible
against the fp64 definition, where it can go wrong: windows that end inside a
tile, a page or the prefix, first tokens inside the window or behind the
prefix, rows that see different keys of one tile, values that are not finite
where some rows see them and others do not; and what it refuses."""
import numpy as np
import pytest

import oracle as O
from serving_inputs import Case, bf16, to_bf16

pytestmark = pytest.mark.gpu


def _run(sdq, torch, c, window, sinks, scale=None, lse=True, **bounds):
    cache, batch = c.cache(sdq, torch), c.batch(sdq, torch, **bounds)
    q = to_bf16(torch, c.q)
    ws = cache.alloc_workspace(batch, c.q_heads, window=window, sinks=sinks)
    ws.random_(0, 256)                       # a workspace needs no initialization
    out_lse = torch.full((c.tokens, c.q_heads), 7.0, device="cuda") if lse else None
    out = cache.attend(batch, q, scale, ws=ws, lse=out_lse, window=window, sinks=sinks)
    assert sdq.sdq_attention_status(ws) == 0
    return out, out_lse


def _check(c, out, lse, window, sinks, rows=slice(None)):
    scale = c.dim ** -0.5
    want, want_lse, mag = O.serving.attend(c.q, c.k, c.v, c.start, c.own, c.pages, c.prefix_pages, c.prefix, scale, window, sinks)
    got = out.float().cpu().numpy().astype(np.float64)
    # Scores: fp32 sums of `dim` products, |q||k| scale (dim + 8) 2^-24 in all, as a relative error of each weight
    # (of numerator and denominator); weights rounded to bf16 (2^-8, half its spacing), by ex2.approx (2^-22) and up
    # to 2^-10 in all for fp32 sums of them; the output rounded once (2^-8 of it).
    norm = np.linalg.norm(c.q, axis=-1).max() * np.nanmax(np.linalg.norm(np.nan_to_num(c.k, posinf=0, neginf=0), axis=-1))
    score = norm * scale * (c.dim + 8) * 2.0 ** -24
    bound = mag * (2 * score + 2.0 ** -8 + 2.0 ** -10) + 2.0 ** -8 * np.abs(want) + 1e-30
    got, want, bound = got[rows], want[rows], bound[rows]
    assert np.all(np.isfinite(got))
    assert np.all(np.abs(got - want) <= bound), float((np.abs(got - want) / bound).max())
    if lse is not None:
        got_lse, want_lse = lse.cpu().numpy().astype(np.float64)[rows], want_lse[rows]
        empty = np.isinf(want_lse)
        assert np.array_equal(np.isinf(got_lse), empty) and np.all(got_lse[empty] < 0)
        fine = ~empty
        assert np.all(np.abs(got_lse[fine] - want_lse[fine]) <= score + 2.0 ** -10 + 2.0 ** -20 * np.abs(want_lse[fine]))


H70, H7, H125, ODD = (16, 2, 128), (4, 4, 128), (3, 3, 64), (10, 2, 64)

CASES = {
    "edges": (H70, [1] * 13, [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 191, 257], 0, 16),
    "edges-64": (H125, [1] * 9, [1, 31, 32, 33, 127, 128, 129, 255, 400], 0, 32),
    "one": (H70, [1], [1], 0, 16),
    "one-mha": (H7, [1], [700], 0, 128),
    "long": (H70, [1], [5003], 0, 64),
    "empty": (H70, [1, 1, 0, 1, 0], [0, 40, 33, 0, 0], 0, 16),
    "all-empty": (H125, [1, 1], [0, 0], 0, 16),
    "draft": (H70, [3, 2, 1, 4], [3, 130, 64, 67], 0, 16),
    "draft-odd": (ODD, [5, 3], [5, 140], 0, 64),
    "draft-short": (ODD, [5, 3, 2], [2, 140, 0], 21, 64),           # more new tokens than places
    "prompt": (H70, [70, 1, 37], [70, 50, 200], 0, 32),
    "prompt-short": (H70, [70, 50], [30, 0], 20, 32),
    "prompt-mha": (H7, [150], [300], 0, 16),
    "prompt-long": (H7, [500, 3], [700, 300], 0, 16),
    "prompt-behind": ((4, 4, 64), [300, 260], [300, 700], 257, 32),
    "prompt-odd": (ODD, [33, 129], [40, 129], 0, 16),
    "prefix-only": (H70, [1, 1, 1], [0, 0, 0], 77, 16),
    "prefix-1": (H7, [1, 1], [5, 0], 1, 16),
    "prefix": (H70, [1] * 9, [1, 7, 16, 30, 0, 65, 128, 3, 200], 301, 16),
    "prefix-mha": (H7, [1] * 20, list(range(1, 21)), 128, 64),
    "prefix-draft": (ODD, [3, 1, 5], [3, 90, 5], 515, 128),
    "prefix-prompt": (H70, [100, 1, 20], [100, 30, 25], 150, 16),
    "many": (H125, [1] * 70, [(5 * i) % 97 for i in range(70)], 0, 16),
}


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (7, 3), (16, 16), (33, 0), (64, 100), (129, 4), (400, 130)])
@pytest.mark.parametrize("name", CASES)
def test_window_matches_the_definition(sdq, name, window, sinks):
    import torch
    heads, new, own, prefix, page = CASES[name]
    c = Case(heads, new, own, prefix, page, seed=len(name))
    out, lse = _run(sdq, torch, c, window, sinks)
    _check(c, out, lse, window, sinks)


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("heads", [H70, H125])
@pytest.mark.parametrize("new", [1, 3, 40])
@pytest.mark.parametrize("prefix", [0, 130])
def test_pages_of_every_size(sdq, page, heads, new, prefix):
    import torch
    c = Case(heads, [new, 1, new], [new, 150, new + 129], prefix, page, seed=page + new)
    out, _ = _run(sdq, torch, c, 50, 5, lse=False)
    _check(c, out, None, 50, 5)


def _mark(c, s, j, value, keys=False):
    """Sets elements of the value (or key) at position j of sequence s."""
    table, at = (c.prefix_pages, j) if j < c.prefix else (c.pages[s], j - c.prefix)
    (c.k if keys else c.v)[table[at // c.page], :, at % c.page, 3::7] = value


SPREAD = {
    "decode": (H70, [1], [300], 0, 16),
    "draft": (ODD, [4], [300], 37, 16),
    "draft-64": (H125, [5], [300], 0, 32),
    "wide": (H70, [60], [300], 37, 16),
    "wide-64": ((4, 4, 64), [290], [300], 20, 64),
    "wide-split": ((2, 1, 128), [20], [3000], 0, 64),
}


@pytest.mark.parametrize("name", SPREAD)
@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("window,sinks", [(40, 0), (100, 5), (1000, 3)])
def test_values_reach_the_rows_that_see_them_and_no_others(sdq, name, bad, window, sinks):
    import torch
    heads, new, own, prefix, page = SPREAD[name]
    c = Case(heads, new, own, prefix, page, seed=len(name))
    n, total = new[0], prefix + own[0]
    first = total - n
    marks = sorted({0, 4, 5, first, total - 1, max(0, first - window), max(0, first - window + 1), max(0, total - 1 - window),
                    max(0, total - 2 - window // 2)})
    for at in marks:
        c2 = Case(heads, new, own, prefix, page, seed=len(name))
        _mark(c2, 0, at, bad)
        out, lse = _run(sdq, torch, c2, window, sinks)
        pos = first + np.arange(n)
        sees = (at <= pos) & ((at > pos - window) | (at < sinks))
        got = out.float().cpu().numpy()
        hit = got[sees][..., 3::7]
        assert np.all(np.isnan(hit) if np.isnan(bad) else hit == bad)
        rest = np.delete(got[sees], np.s_[3::7], axis=-1)
        assert np.all(np.isfinite(rest))
        _check(c, torch.from_numpy(got).nan_to_num(0, 0, 0) if not sees.all() else torch.zeros(got.shape), None, window, sinks, ~sees) \
            if (~sees).any() else None


@pytest.mark.parametrize("name", SPREAD)
@pytest.mark.parametrize("bad", [np.nan, np.inf])
def test_keys_that_nobody_sees_may_hold_anything(sdq, name, bad):
    """Keys and values of positions that no token's window has, in tiles that are read for their neighbours."""
    import torch
    heads, new, own, prefix, page = SPREAD[name]
    c = Case(heads, new, own, prefix, page, seed=1)
    window, sinks = 45, 3
    first = prefix + own[0] - new[0]
    for at in range(sinks, first - window + 1):
        _mark(c, 0, at, bad)
        _mark(c, 0, at, bad, keys=True)
    out, lse = _run(sdq, torch, c, window, sinks)
    _check(c, out, lse, window, sinks)


@pytest.mark.parametrize("name", ["edges", "draft-odd", "prompt", "prompt-behind", "prefix", "prefix-draft"])
def test_windows_over_everything_leave_attention_as_it_is(sdq, name):
    import torch
    heads, new, own, prefix, page = CASES[name]
    c = Case(heads, new, own, prefix, page, seed=2)
    cache, batch, q = c.cache(sdq, torch), c.batch(sdq, torch), to_bf16(torch, c.q)
    want = cache.attend(batch, q)
    top = prefix + max(own)
    for window, sinks in ((top, 0), ((1 << 30) - 1, 4), (1, top)):
        assert torch.equal(cache.attend(batch, q, window=window, sinks=sinks), want)
    _check(c, *_run(sdq, torch, c, top - 1, 0), top - 1, 0)
    _check(c, *_run(sdq, torch, c, 1, top - 1), 1, top - 1)


def test_long_windows_in_shares(sdq):
    """Few row blocks over long windows: thread blocks that share a line, in both kernels."""
    import torch
    for heads, new, own, window, sinks in (((2, 1, 128), [17], [6000], 4100, 70), ((2, 1, 128), [16], [6000], 4100, 70),
                                           ((4, 1, 64), [40, 9], [5000, 100], 3900, 1), (H70, [1, 1], [9000, 40], 7000, 33)):
        c = Case(heads, new, own, 100, 64, seed=5)
        _check(c, *_run(sdq, torch, c, window, sinks), window, sinks)


def test_extreme_scores(sdq):
    """The largest score outside the window, and rows whose window's scores are all far below those of the first tokens."""
    import torch
    for heads, new in ((H70, 1), (H7, 40)):
        c = Case(heads, [new], [900], 0, 16, seed=13)
        ramp = np.linspace(3, 0, 900)
        for j in range(900):
            c.k[c.pages[0, j // 16], :, j % 16] = bf16(ramp[j])
        c.q[:] = bf16(np.abs(c.q) * 0.3)
        for sinks in (0, 2):
            _check(c, *_run(sdq, torch, c, 100, sinks), 100, sinks)


def test_bounds_larger_than_the_lengths_and_graphs(sdq):
    """A captured step follows the lengths as they move on, through a page's end and out of the prefix."""
    import torch
    own = [14, 40, 1, 63]
    c = Case(H70, [1] * 4, [m + 12 for m in own], 30, 16, seed=21)
    cache, q = c.cache(sdq, torch), to_bf16(torch, c.q)
    batch = c.batch(sdq, torch, max_own=80)
    assert batch.tensors[2].shape[1] * 16 >= 80
    lens = batch.tensors[1]
    lens.copy_(torch.tensor(own, dtype=torch.int32))
    ws = cache.alloc_workspace(batch, 16, window=20, sinks=2)
    out, graph = torch.empty((4, 16, 128), dtype=torch.bfloat16, device="cuda"), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        sdq.sdq_attention_window(cache.handle, batch, 16, q, 16 * 128, 128 ** -0.5, 20, 2, out, None, ws)
    for i in range(12):
        graph.replay()
        torch.cuda.synchronize()
        now = Case(H70, [1] * 4, [m + 12 for m in own], 30, 16, seed=21)
        now.own = [m + i for m in own]
        _check(now, out, None, 20, 2)
        lens.add_(1)


def test_streams_strides_and_repeats(sdq):
    import torch
    c = Case(H70, [1, 2, 30], [20, 30, 40], 33, 16, seed=17)
    cache, batch, q = c.cache(sdq, torch), c.batch(sdq, torch), to_bf16(torch, c.q)
    want = cache.attend(batch, q, window=25, sinks=3)
    torch.cuda.synchronize()
    wide = torch.full((c.tokens, c.q_heads + 4, c.dim), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, 2:2 + c.q_heads] = q
    assert torch.equal(cache.attend(batch, wide[:, 2:2 + c.q_heads], window=25, sinks=3), want)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = [cache.attend(batch, q, window=25, sinks=3, stream=side) for _ in range(5)]
    side.synchronize()
    assert all(torch.equal(g, want) for g in got)


def test_rows_behind_the_last_sequence_stay(sdq):
    import torch
    c = Case(H70, [1, 1], [40, 60], 0, 16, seed=19)
    cache = c.cache(sdq, torch)
    i = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()
    batch = sdq.Batch(i(c.start), i(c.own), i(c.pages), 5, 1, 60)            # 5 rows, 2 of them sequences'
    q = torch.randn((5, 16, 128), device="cuda").to(torch.bfloat16)
    ws = cache.alloc_workspace(batch, 16, window=9)
    out = torch.full((5, 16, 128), 3.0, dtype=torch.bfloat16, device="cuda")
    sdq.sdq_attention_window(cache.handle, batch, 16, q, 16 * 128, 128 ** -0.5, 9, 0, out, None, ws)
    torch.cuda.synchronize()
    assert torch.all(out[2:] == 3.0) and torch.all(out[:2] != 3.0)


def test_window_refusals(sdq):
    import torch
    c = Case(H70, [1, 2], [20, 30], 5, 16, seed=23)
    cache, batch, q = c.cache(sdq, torch), c.batch(sdq, torch), to_bf16(torch, c.q)
    for window, sinks in ((0, 0), (-1, 0), (1 << 30, 0), (4, -1), (4, 1 << 30)):
        with pytest.raises(sdq.SdqError) as e:
            cache.attend(batch, q, window=window, sinks=sinks)
        assert e.value.status == -1
        ws, out = torch.empty(1 << 20, dtype=torch.uint8, device="cuda"), torch.empty_like(q)
        with pytest.raises(sdq.SdqError) as e:
            sdq.sdq_attention_window(cache.handle, batch, 16, q, 16 * 128, 0.1, window, sinks, out, None, ws)
        assert e.value.status == -1
    with pytest.raises(ValueError):
        cache.attend(batch, q, sinks=4)
    small = cache.alloc_workspace(batch, 16, window=9)[:256]
    with pytest.raises(sdq.SdqError) as e:
        cache.attend(batch, q, ws=small, window=9)
    assert e.value.status not in (0, -1)
    torch.cuda.synchronize()


@pytest.mark.parametrize("prefix", [0, 70])
@pytest.mark.parametrize("bad", [None, np.nan, np.inf])
def test_many_row_blocks_one_after_another(sdq, prefix, bad):
    """More row blocks than thread blocks, of all kinds in turn: short and long, one half and two, an odd number of
    pieces, without a key; a value that is not finite stays in the rows of its sequence that see it."""
    import torch
    rng = np.random.default_rng(prefix)
    new = [int(n) for n in rng.choice([33, 40, 64, 128, 129, 150], 64)]
    own = [0 if s % 13 == 5 else int(n + rng.choice([0, 0, 1, 30, 200, 400])) for s, n in enumerate(new)]
    c = Case((8, 8, 64), new, own, prefix, 16, seed=31)
    assert sum(-(-n // 256) for n in new) * 8 > 3 * 152
    window, sinks = 90, 3
    marked = [s for s in range(64) if own[s] > 250][:3] if bad is not None else []
    seen = np.zeros(c.tokens, bool)
    for s in marked:
        at = prefix + own[s] - new[s] // 2
        _mark(c, s, at, bad)
        pos = prefix + own[s] - new[s] + np.arange(new[s])
        seen[c.start[s]:c.start[s + 1]] = (pos >= at) & (pos - window < at)
    out, lse = _run(sdq, torch, c, window, sinks)
    if bad is None:
        _check(c, out, lse, window, sinks)
        return
    assert len(marked) == 3 and seen.any()
    got = out.float()
    hit = got[torch.from_numpy(seen).cuda()][..., 3::7]
    assert torch.all(hit.isnan() if np.isnan(bad) else hit == bad)
    clean = Case((8, 8, 64), new, own, prefix, 16, seed=31)
    assert np.all(np.isfinite(np.delete(got.cpu().numpy(), np.s_[3::7], axis=-1)))
    _check(clean, got.nan_to_num(0, 0, 0), lse, window, sinks, ~seen)


def test_outputs_off_32_bytes_and_shares_of_few_row_blocks(sdq):
    import torch
    for heads, new, own in ((H7, [40], [3000]), ((4, 4, 64), [300], [301])):
        c = Case(heads, new, own, 0, 16, seed=33)
        cache, batch, q = c.cache(sdq, torch), c.batch(sdq, torch), to_bf16(torch, c.q)
        want = cache.attend(batch, q, window=70, sinks=1)
        flat = torch.full((q.numel() + 16,), 5.0, dtype=torch.bfloat16, device="cuda")
        out = flat[8:8 + q.numel()].reshape(q.shape)                         # 16 bytes behind a boundary
        ws = cache.alloc_workspace(batch, c.q_heads, window=70, sinks=1)
        sdq.sdq_attention_window(cache.handle, batch, c.q_heads, q, c.q_heads * c.dim, c.dim ** -0.5, 70, 1, out, None, ws)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.all(flat[:8] == 5.0) and torch.all(flat[8 + q.numel():] == 5.0)


# A prefix that is long against the own lengths, and many sequences: what they see of it is read once for all of
# them and joined with each sequence's own part.
APART = {
    # heads, new tokens, own tokens, prefix, page, window, sinks
    "decode": (H7, [1] * 100, [(7 * i) % 90 for i in range(100)], 1900, 64, 1500, 5),
    "decode-70b": (H70, [1] * 128, [1 + (5 * i) % 60 for i in range(128)], 3001, 16, 2900, 0),
    "window-over-the-prefix": (H7, [1] * 90, [1 + (37 * i) % 900 for i in range(90)], 1200, 32, 2000, 3),
    "sinks-over-the-prefix": (H7, [1] * 90, [1 + (11 * i) % 300 for i in range(90)], 1300, 16, 200, 1350),
    "draft": (ODD, [1 + i % 4 for i in range(128)], [4 + (13 * i) % 70 for i in range(128)], 2500, 128, 2300, 9),
    "draft-short": (ODD, [1 + i % 4 for i in range(128)], [(3 * i) % 5 for i in range(128)], 2500, 16, 2300, 0),
    "64": ((12, 12, 64), [1] * 70, [(5 * i) % 97 for i in range(70)], 1501, 16, 1400, 1),
    "shares": ((8, 1, 128), [1] * 128, [1 + i % 50 for i in range(128)], 16000, 128, 15000, 20),
}


def _apart(sdq, torch, c, window, sinks):
    """Does the call keep two parts' sums (fp32, for a row each)?"""
    cache, batch = c.cache(sdq, torch), c.batch(sdq, torch)
    return sdq.sdq_attention_window_workspace_bytes(cache.handle, batch, c.q_heads, window, sinks) >= 8 * c.tokens * c.q_heads * c.dim


@pytest.mark.parametrize("name", APART)
def test_a_prefix_shared_by_many_sequences(sdq, name):
    import torch
    heads, new, own, prefix, page, window, sinks = APART[name]
    c = Case(heads, new, own, prefix, page, seed=len(name))
    assert _apart(sdq, torch, c, window, sinks)
    out, lse = _run(sdq, torch, c, window, sinks)
    _check(c, out, lse, window, sinks)
    again, lse2 = _run(sdq, torch, c, window, sinks)
    assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("bad", [np.nan, np.inf])
@pytest.mark.parametrize("name", ["decode", "draft", "64"])
def test_values_of_a_shared_prefix_reach_the_rows_that_see_them(sdq, name, bad):
    import torch
    heads, new, own, prefix, page, window, sinks = APART[name]
    c = Case(heads, new, own, prefix, page, seed=1)
    marked = Case(heads, new, own, prefix, page, seed=1)
    at = prefix - window + 45
    _mark(marked, 0, at, bad)
    for j in range(sinks, prefix - window):                  # and what no row sees may hold anything
        _mark(marked, 0, j, np.nan)
        _mark(marked, 0, j, np.nan, keys=True)
    out, lse = _run(sdq, torch, marked, window, sinks)
    pos = np.concatenate([prefix + np.maximum(-1, m - n + np.arange(n)) for n, m in zip(new, own)])
    sees = at > pos - window
    assert sees.any() and not sees.all()
    got = out.float()
    hit = got[torch.from_numpy(sees).cuda()][..., 3::7]
    assert torch.all(hit.isnan() if np.isnan(bad) else hit == bad)
    assert np.all(np.isfinite(np.delete(got.cpu().numpy(), np.s_[3::7], axis=-1)))
    _check(c, got.nan_to_num(0, 0, 0), lse, window, sinks, ~sees)


def test_rows_of_nobody_stay_beside_a_shared_prefix(sdq):
    import torch
    heads, new, own, prefix, page, window, sinks = APART["decode"]
    c = Case(heads, new, own, prefix, page, seed=3)
    cache = c.cache(sdq, torch)
    i = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()
    batch = sdq.Batch(i(c.start), i(c.own), i(c.pages), 107, 1, max(own), i(c.prefix_pages), prefix)
    q = torch.randn((107, 4, 128), device="cuda").to(torch.bfloat16)
    c.q = q[:100].float().cpu().numpy()
    ws = cache.alloc_workspace(batch, 4, window=window, sinks=sinks)
    out = torch.full((107, 4, 128), 3.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((107, 4), 3.0, device="cuda")
    sdq.sdq_attention_window(cache.handle, batch, 4, q, 512, 128 ** -0.5, window, sinks, out, lse, ws)
    assert sdq.sdq_attention_status(ws) == 0
    assert torch.all(out[100:] == 3.0) and torch.all(lse[100:] == 3.0)
    _check(c, out[:100], lse[:100], window, sinks)


def test_a_shared_prefix_in_a_graph(sdq):
    """Lengths move on under a captured call, rows that saw much of the prefix see less."""
    import torch
    own = [(7 * i) % 90 for i in range(100)]
    c = Case(H7, [1] * 100, [m + 40 for m in own], 1900, 64, seed=4)
    cache, q = c.cache(sdq, torch), to_bf16(torch, c.q)
    batch = c.batch(sdq, torch)
    ws = cache.alloc_workspace(batch, 4, window=1500, sinks=2)
    out, graph = torch.empty((100, 4, 128), dtype=torch.bfloat16, device="cuda"), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        sdq.sdq_attention_window(cache.handle, batch, 4, q, 512, 128 ** -0.5, 1500, 2, out, None, ws)
    for step in (0, 1, 40):
        now = Case(H7, [1] * 100, [m + 40 for m in own], 1900, 64, seed=4)
        now.own = [m + step for m in own]
        batch.tensors[1].copy_(torch.tensor(now.own, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        _check(now, out, None, 1500, 2)


@pytest.mark.parametrize("name", ["draft", "wide", "64", "apart"])
def test_scores_that_are_not_a_number_stay_in_their_rows(sdq, name):
    """A key that is NaN: NaN, and a log-sum-exp that is NaN, for the rows that see it alone."""
    import torch
    heads, new, own, prefix, page, window, sinks = {"draft": (ODD, [4], [300], 37, 16, 100, 5), "wide": (H70, [60], [300], 37, 16, 100, 5),
                                                    "64": ((4, 4, 64), [290], [300], 20, 64, 40, 0), "apart": APART["decode"]}[name]
    c, marked = (Case(heads, new, own, prefix, page, seed=6) for _ in range(2))
    at = prefix - window + 60 if name == "apart" else prefix + own[0] - new[0] // 2 - window // 2
    _mark(marked, 0, at, np.nan, keys=True)
    out, lse = _run(sdq, torch, marked, window, sinks)
    pos = np.concatenate([prefix + np.maximum(-1, m - n + np.arange(n)) for n, m in zip(new, own)])
    sees = (at <= pos) & ((at > pos - window) | (at < sinks))
    assert sees.any() and sees.all() == (name in ("draft", "wide"))
    hit = torch.from_numpy(sees).cuda()
    assert out[hit].isnan().all() and lse[hit].isnan().all()
    if not sees.all():
        _check(c, out.nan_to_num(0), lse.nan_to_num(0), window, sinks, ~sees)


def test_scores_that_grow_and_shrink_along_the_window(sdq):
    """Maxima that rise by a little at every tile, by much at some, and fall: references that are raised late."""
    import torch
    for heads, new in ((H70, 1), (H70, 3), (ODD, 5), (H7, 40)):
        for shape in (np.linspace(-6, 6, 900), np.linspace(6, -6, 900), 8 * np.sin(np.arange(900) / 40.0), np.where(np.arange(900) % 300 == 299, 12.0, -12.0)):
            c = Case(heads, [new], [900], 0, 16, seed=15)
            for j in range(900):
                c.k[c.pages[0, j // 16], :, j % 16] = bf16(shape[j] + 0.05 * c.k[c.pages[0, j // 16], :, j % 16])
            c.q[:] = bf16(np.abs(c.q) * 0.25)
            _check(c, *_run(sdq, torch, c, 700, 3), 700, 3)
