"""GPU: a step's operators as they run together: several calls at once on two
streams, captured and replayed beside eager ones, each with what it alone has."""
import pytest

from serving_inputs import Case, to_bf16

pytestmark = pytest.mark.gpu


def _calls(sdq, torch, seed):
    """Calls of every kernel of the step, on tensors of their own; each returns what it wrote."""
    g = torch.Generator("cuda").manual_seed(seed)
    calls = []
    for heads, new, own, prefix, window in (((16, 2, 128), [1] * 9, [200 + 7 * i for i in range(9)], 33, 90),       # few rows
                                            ((4, 4, 64), [150, 40], [300, 60], 20, 77),                              # prompts
                                            ((4, 4, 128), [1] * 100, [(7 * i) % 90 for i in range(100)], 1900, 1500)):   # a shared prefix
        c = Case(heads, new, own, prefix, 16, seed=seed)
        cache, batch, q = c.cache(sdq, torch), c.batch(sdq, torch), to_bf16(torch, c.q)
        ws = cache.alloc_workspace(batch, c.q_heads, window=window, sinks=2)
        calls.append(lambda s, cache=cache, batch=batch, q=q, ws=ws, window=window: cache.attend(batch, q, ws=ws, stream=s, window=window, sinks=2))
    for tokens in (5, 700):
        c = Case((32, 4, 64), [tokens], [tokens + 3], 0, 16, seed=seed)
        cache, batch = c.cache(sdq, torch), c.batch(sdq, torch)
        x = [torch.randn((tokens, h * 64), device="cuda", generator=g) for h in (32, 4, 4)]
        norm, rope = sdq.HeadNorm(torch.rand(64, device="cuda", generator=g), torch.rand((4, 64), device="cuda", generator=g)), sdq.Rope.table(800, 64)
        calls.append(lambda s, cache=cache, batch=batch, x=x, norm=norm, rope=rope: cache.append(batch, *x, rope, s, norm))
        calls.append(lambda s, cache=cache, batch=batch, x=x, norm=norm, rope=rope: (cache.append(batch, *x, rope, s, norm), cache.k_pages)[1])
    for rows, vocab in ((1, 5000), (40, 130001)):
        z = torch.randn((rows, vocab), device="cuda", generator=g)
        h = torch.randint(0, vocab, (rows, 3000), device="cuda", generator=g, dtype=torch.int32)
        ids = torch.randint(0, vocab, (rows, 40), device="cuda", generator=g, dtype=torch.int32)
        b, r = torch.randn((rows, 40), device="cuda", generator=g), torch.full((rows,), 1.3, device="cuda")
        calls.append(lambda s, z=z, h=h, ids=ids, b=b, r=r: sdq.adjust_logits(z, h, repetition=r, frequency=r, bias_ids=ids, bias=b, stream=s))
    for n, tokens in ((70, 1), (5, 3000)):
        own = torch.randint(0, 50, (n,), device="cuda", generator=g, dtype=torch.int32)
        new, tables = torch.full((n,), tokens, dtype=torch.int32, device="cuda"), torch.zeros((n, 200), dtype=torch.int32, device="cuda")
        pool = sdq.PagePool(16, n_pages=2000)
        calls.append(lambda s, pool=pool, own=own, new=new, tables=tables, n=n, t=tokens: pool.step(own, new, tables, n * t, in_place=False, stream=s).slots)
    return calls


def test_calls_at_once_on_two_streams(sdq):
    import torch
    a, b = _calls(sdq, torch, 1), _calls(sdq, torch, 2)
    want = [[f(None).clone() for f in calls] for calls in (a, b)]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], [[], []]
    for _ in range(5):
        for i in range(len(a)):
            for k, calls in enumerate((a, b)):
                with torch.cuda.stream(streams[k]):
                    got[k].append(calls[i](None))
    torch.cuda.synchronize()
    for k in range(2):
        for i, out in enumerate(got[k]):
            assert torch.equal(out.nan_to_num(0) if out.is_floating_point() else out,
                               want[k][i % len(a)].nan_to_num(0) if out.is_floating_point() else want[k][i % len(a)]), (k, i)


def test_captured_calls_beside_eager_ones(sdq):
    import torch
    a, b = _calls(sdq, torch, 3), _calls(sdq, torch, 4)
    want = [[f(None).clone() for f in calls] for calls in (a, b)]
    torch.cuda.synchronize()
    graph, outs = torch.cuda.CUDAGraph(), []
    with torch.cuda.graph(graph):
        for f in a:
            outs.append(f(None))
    side = torch.cuda.Stream()
    same = lambda x, y: torch.equal(x.nan_to_num(0), y.nan_to_num(0)) if x.is_floating_point() else torch.equal(x, y)
    for _ in range(4):
        graph.replay()
        with torch.cuda.stream(side):
            eager = [f(None) for f in b]
        torch.cuda.synchronize()
        assert all(same(x, y) for x, y in zip(outs, want[0])) and all(same(x, y) for x, y in zip(eager, want[1]))
