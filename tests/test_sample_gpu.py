"""GPU: one token per row of logits against the fp64 definition, where it can
go wrong: equal logits, rows of one value, cuts inside a crowd, masks of -inf
and of the type's lowest value, infinities and NaN, vocabularies of every size;
and what it refuses.

A row counts where the definition's decision is clear: u and top_p further than
MARGIN, as shares of the mass, from the next token's interval.  fp32 weights
(quotient x rounded to |x| 2^-23, exp to 2^-23) are off by (|x| + 2) 2^-23 each,
|x| < 8 on the average of any of these rows: 1.2e-6 of the mass."""
import numpy as np
import pytest

import oracle as O
from paper_2510_03275_gb300 import workloads as W
from serving_inputs import bf16

pytestmark = pytest.mark.gpu

MARGIN = 2e-6


def _device(torch, z, kind="f32", pad=0):
    rows, v = z.shape
    wide = torch.full((rows, v + pad), float("nan"), device="cuda")
    wide[:, :v] = torch.from_numpy(np.asarray(z, np.float32)).cuda()
    return (wide if kind == "f32" else wide.to(torch.bfloat16))[:, :v]


def _check(sdq, z, u, t, k, p, m, kind="f32", pad=0, clear=0.9):
    import torch
    rows = len(z)
    col = lambda x, d: np.broadcast_to(np.asarray(x, d), rows).copy()
    t, k, p, m, u = col(t, np.float32), col(k, np.int32), col(p, np.float32), col(m, np.float32), col(u, np.float32)
    dev = lambda a: torch.from_numpy(a).cuda()
    got = sdq.sample(_device(torch, z, kind, pad), dev(u), dev(t), dev(k), dev(p), dev(m)).cpu().numpy()
    want, margin = O.serving.sample(z, u, t, k, p, m)
    sure = margin > MARGIN
    assert sure.mean() >= clear
    assert np.array_equal(got[sure], want[sure])
    return got


def _rows(rng, rows, v, sharp=1.0):
    z = 1.5 * sharp * rng.standard_normal((rows, v))
    for i in range(rows):
        few = rng.integers(0, v, size=min(v, 30))
        z[i, few] += sharp * (2 + 3 * np.abs(rng.standard_normal(len(few))))
    return z.astype(np.float32)


SETTINGS = [(1.0, 0, 1.0, 0.0), (0.0, 5, 0.5, 0.1), (0.7, 40, 1.0, 0.0), (1.0, 0, 0.9, 0.0), (1.0, 0, 1.0, 0.05),
            (1.3, 50, 0.8, 0.01), (0.5, 1, 1.0, 0.0), (1.0, 3, 0.2, 0.0), (1.0, 1 << 30, 0.0, 0.0), (1.0, -4, 1.5, 2.0)]


@pytest.mark.parametrize("vocab", [1, 2, 31, 33, 1000, 2048, 2049, 4096, 5001, 32000, 50272, 128255])
@pytest.mark.parametrize("kind,pad", [("f32", 0), ("f32", 5), ("bf16", 0), ("bf16", 3)])
def test_sample_matches_the_definition(sdq, vocab, kind, pad):
    rng = np.random.default_rng(vocab + pad)
    rows = 40
    z = _rows(rng, rows, vocab)
    if kind == "bf16":
        z = bf16(z)
    s = np.array([SETTINGS[i % len(SETTINGS)] for i in range(rows)])
    # (clear: the definition alone decides how many rows count; a tenth have top_p 0, and more tokens crowd the edges
    # of the largest vocabulary's unfiltered rows)
    got = _check(sdq, z, rng.random(rows), s[:, 0], s[:, 1], s[:, 2], s[:, 3], kind, pad, clear=0.8 if vocab < 100000 else 0.6)
    assert got.min() >= 0 and got.max() < vocab


def test_the_largest_vocabulary(sdq):
    rng = np.random.default_rng(1)
    z = _rows(rng, 3, 393216)
    _check(sdq, z, rng.random(3), 0.8, [0, 40, 0], [0.9, 1, 0.5], 0, clear=0.3)


def test_equal_logits_are_taken_by_index(sdq):
    rng = np.random.default_rng(2)
    for vocab in (7, 3000, 40000):
        z = np.full((6, vocab), 1.25, np.float32)
        # one value: the first k, or the first p of them, each as likely
        _check(sdq, z, [0, 0.2, 0.4, 0.6, 0.8, 0.999], 1.0, [5, 6, 7, 700, 2999, 20000], 1.0, 0.0, clear=0.5)
        _check(sdq, z, [0.1, 0.2, 0.4, 0.6, 0.8, 0.999], 1.0, 0, [0.1, 0.3, 0.5, 0.7, 0.9, 0.0], 0.0, clear=0.0)
        # two values, the cut among the lower ones; the same behind a few larger ones
        z[:, rng.permutation(vocab)[:vocab // 3]] = 2.5
        z[3:, rng.permutation(vocab)[:3]] = 9.0
        k = vocab // 3 + np.array([1, 2, vocab // 2, 3, 4, vocab // 3])
        got = _check(sdq, z, rng.random(6), 0.9, k, 1.0, 0.0, clear=0.0)
        assert np.all((got >= 0) & (got < vocab))
    # the last one kept: top_k of equal logits and u at the end
    z = np.zeros((1, 40000), np.float32)
    for k in (1, 2, 513, 30001, 39999):
        assert _check(sdq, z, 0.9999999, 1.0, k, 1.0, 0.0, clear=0.0)[0] in (k - 1, k - 2)


def test_a_crowd_in_one_bucket(sdq):
    """More logits than are gathered at once, a few thousandths apart; also across 0, where equal steps of the
    logits' bits are most unequal, and with most of the row far below."""
    rng = np.random.default_rng(3)
    for vocab in (5000, 60000):
        rows = 12
        z = (0.02 * rng.random((rows, vocab))).astype(np.float32)
        z[4:8] -= 0.01
        z[8:] = np.where(rng.random((4, vocab)) < 0.5, z[8:], -50.0 * rng.random((4, vocab)).astype(np.float32))
        for k in (700, vocab // 3):
            _check(sdq, z, rng.random(rows), 1.0, k, 1.0, 0.0, clear=0.1)
        # the cut by mass, seen through the largest u: the kept set itself
        want = [np.sort(np.argsort(-r.astype(np.float64), kind="stable")[:k])[-1] for r in z]
        got = _check(sdq, z, 1.0, 1.0, k, 1.0, 0.0, clear=0.0)
        assert np.array_equal(got, want)
        _check(sdq, z, rng.random(rows), 1.0, 0, 0.4, 0.0, clear=0.0)


def test_a_flat_tail_below_the_histogram(sdq):
    """One token far above 50000 alike: the cut by count falls among logits 20 nats down."""
    rng = np.random.default_rng(4)
    z = rng.standard_normal((8, 50000)).astype(np.float32) * 0.1
    z[:, 777] = 20.0
    want = [np.sort(np.argsort(-r.astype(np.float64), kind="stable")[:300])[-1] for r in z]
    got = _check(sdq, z, 1.0, 1.0, 300, 1.0, 0.0, clear=0.0)
    assert np.array_equal(got, want)
    _check(sdq, z, rng.random(8), 1.0, 300, 0.99, 0.0)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_masks_infinities_and_nan(sdq, kind):
    rng = np.random.default_rng(5)
    z = bf16(_rows(rng, 12, 9001))
    low = np.float32(-3.3895314e38)          # bf16's lowest value
    z[0] = -np.inf
    z[1] = np.nan
    z[2], z[2, 8999] = -np.inf, -7.0
    z[3], z[3, 5], z[3, 6] = low, 1.0, 1.0
    z[4, ::2] = np.nan
    z[5, 100:] = -np.inf
    z[6, 200:] = low
    z[7, 300], z[7, 4000] = np.inf, np.inf
    z[8] = low
    z[9, :] = np.where(rng.random(9001) < 0.9, -np.inf, z[9])
    z[10, :4500], z[10, 4500] = -np.inf, np.nan
    u = rng.random(12)
    for t, k, p, m in [(1.0, 0, 1.0, 0.0), (0.8, 50, 0.9, 0.0), (0.0, 0, 1.0, 0.0), (1.0, 2, 1.0, 0.0), (1.0, 0, 0.5, 0.3)]:
        got = _check(sdq, z, u, t, k, p, m, kind, clear=0.6)
        assert got[0] == got[1] == -1 and got[2] == 8999 and got[3] in (5, 6) and got[7] in (300, 4000)


def test_settings_at_their_ends(sdq):
    import torch
    rng = np.random.default_rng(6)
    z = _rows(rng, 4, 3001)
    best = z.argmax(1)
    for t, k, p, m in [(1.0, 1, 1.0, 0.0), (1.0, 0, 0.0, 0.0), (1.0, 0, -1.0, 0.0), (1.0, 0, 1.0, 1.0), (1.0, 0, 1.0, 7.0),
                       (1e-30, 0, 1.0, 0.0), (-1.0, 0, 1.0, 0.0), (float("nan"), 0, 1.0, 0.0), (1e-4, 0, 1.0, 0.0)]:
        assert np.array_equal(_check(sdq, z, 0.37, t, k, p, m, clear=0.0), best)
    # no settings at all; the ends of u; an infinite temperature makes all alike
    dz, u = _device(torch, z), torch.tensor([0.0, 0.25, 0.5, 0.99], device="cuda")
    want, margin = O.serving.sample(z, u.cpu().numpy(), [1.0] * 4, [0] * 4, [1.0] * 4, [0.0] * 4)
    got = sdq.sample(dz, u).cpu().numpy()
    assert np.array_equal(got[margin > MARGIN], want[margin > MARGIN])
    hot = torch.full((4,), float("inf"), device="cuda")
    assert sdq.sample(dz, u, hot).tolist() == [0, 750, 1500, 2970]
    assert sdq.sample(dz, torch.tensor([-1.0, 1.0, 2.0, float("nan")], device="cuda"), hot).tolist() == [0, 3000, 3000, 0]


def test_frequencies_follow_the_weights(sdq):
    """u at the midpoints of 20000 equal steps: every kept token as often as its weight says, to one step."""
    import torch
    rng = np.random.default_rng(7)
    z = _rows(rng, 1, 700, 0.5)
    n = 20000
    u = torch.from_numpy(((np.arange(n) + 0.5) / n).astype(np.float32)).cuda()
    got = sdq.sample(_device(torch, z).expand(n, 700).contiguous(), u, torch.full((n,), 0.9, device="cuda"),
                     torch.full((n,), 60, dtype=torch.int32, device="cuda")).cpu().numpy()
    order = np.argsort(-z[0], kind="stable")[:60]
    w = np.zeros(700)
    w[order] = np.exp((z[0, order].astype(np.float64) - z.max()) / np.float32(0.9))
    assert np.abs(np.bincount(got, minlength=700) - n * w / w.sum()).max() <= 1.01


def test_sample_streams_graphs_and_repeats(sdq):
    import torch
    rng = np.random.default_rng(8)
    z = _rows(rng, 9, 20011)
    dz, u = _device(torch, z), torch.rand(9, device="cuda")
    t, k, p = (torch.full((9,), v, device="cuda") for v in (0.8, 30, 0.9))
    k = k.int()
    want = sdq.sample(dz, u, t, k, p)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = sdq.sample(dz, u, t, k, p)
    side.synchronize()
    assert torch.equal(got, want)
    tokens = torch.empty(9, dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sdq.sdq_sample(dz, u, t, k, p, None, tokens)
    for _ in range(20):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(tokens, want)


def test_sample_refusals(sdq):
    import torch
    z, u = torch.zeros((2, 100), device="cuda"), torch.zeros(2, device="cuda")
    out = torch.empty(2, dtype=torch.int32, device="cuda")
    L = sdq.lib()
    args = lambda **kw: [{**dict(z=z.data_ptr(), kind=0, rows=2, vocab=100, ld=100, u=u.data_ptr(), t=None, k=None, p=None, m=None,
                                 out=out.data_ptr(), st=None), **kw}[n] for n in
                         ("z", "kind", "rows", "vocab", "ld", "u", "t", "k", "p", "m", "out", "st")]
    for kw in (dict(z=None), dict(u=None), dict(out=None), dict(kind=2), dict(rows=0), dict(rows=65536), dict(vocab=0), dict(ld=99),
               dict(vocab=393217, ld=393217), dict(z=z.data_ptr() + 2)):
        assert L.sdq_sample(*args(**kw)) == -1, kw
    for bad in (lambda: sdq.sample(z[0], u), lambda: sdq.sample(z.t(), u), lambda: sdq.sample(z, u.double()), lambda: sdq.sample(z, u[:1]),
                lambda: sdq.sample(z, u, top_k=u), lambda: sdq.sample(z, u, u.cpu())):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(sdq.SdqError):
        sdq.sample(z.half(), u)
    torch.cuda.synchronize()
