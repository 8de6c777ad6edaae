"""GPU: what `serve.generate` does to the decoder's pool of pages: a call that
raises gives back what it took, a pool that others use too is looked at before
and after, and no call answers from rows that a request did not get."""
import pytest

pytestmark = pytest.mark.gpu

PREFIX, PROMPTS, NEW = list(range(5, 25)), [[1], [2, 3, 4], [5] * 17, [9, 8] * 20], 4


def _decoder(n_pages=24):
    from paper_2510_03275_gb300 import serve
    shape = serve.Shape(hidden=128, ffn=128, layers=1, q_heads=2, kv_heads=2, head_dim=64, vocab=100)
    return serve.Decoder(shape, serve.random_weights(shape), n_pages=n_pages, n_pos=128)


def _answer(dec, u, graph=True, **more):
    from paper_2510_03275_gb300 import serve
    return serve.generate(dec, PREFIX, PROMPTS, NEW, u, graph=graph, **more)


def _whole(dec, n_pages=24):
    return int(dec.pool.n_free) == n_pages and sorted(dec.pool.free.tolist()) == list(range(n_pages))


@pytest.mark.parametrize("graph", [True, False])
def test_a_call_that_raises_leaves_nothing_behind(sdq, graph):
    import torch
    u = torch.rand((NEW, 4), device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    want = _answer(_decoder(), u)
    dec, one = _decoder(), torch.ones(4, device="cuda")
    for error, rows, more in ((IndexError, u[:1], {}), (IndexError, u[:2], {}), (IndexError, u[:NEW - 1], {}),
                              (ValueError, u, dict(temperature=one.double())), (ValueError, u, dict(repetition=one[:3])),
                              (ValueError, u.double(), {})):
        with pytest.raises(error):
            _answer(dec, rows, graph, **more)
        assert _whole(dec)
    assert torch.equal(_answer(dec, u, graph), want)
    assert _whole(dec)


def test_a_pool_that_others_use(sdq):
    """Pages that somebody else holds stay theirs; with too few left the call is refused before it takes one."""
    import torch
    from paper_2510_03275_gb300 import serve
    dev = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
    u = torch.rand((NEW, 4), device="cuda", generator=torch.Generator("cuda").manual_seed(2))
    want = _answer(_decoder(), u)
    dec, own, table = _decoder(), dev([0]), torch.full((1, 24), -1, dtype=torch.int32, device="cuda")
    dec.pool.step(own, dev([16 * 14]), table, 16 * 14)              # 10 left: 2 of the prefix, 1 + 1 + 2 + 3 of the requests
    held = table.clone()
    assert torch.equal(_answer(dec, u), want)
    assert int(dec.pool.n_free) == 10 and torch.equal(table, held)
    assert sorted(dec.pool.free[:10].tolist() + held[0, :14].tolist()) == list(range(24))
    dec.pool.step(own, dev([32]), table, 32)                        # 8 left, and 9 needed
    before = dec.pool.free[:8].clone()
    with pytest.raises(ValueError):
        _answer(dec, u)
    with pytest.raises(ValueError):
        serve.generate(dec, [], [[1]] * 9, NEW, torch.rand((NEW, 9), device="cuda"))
    assert int(dec.pool.n_free) == 8 and torch.equal(dec.pool.free[:8], before)


@pytest.mark.parametrize("at,graph", [(0, True), (1, True), (2, False), (3, True)])
def test_pages_that_run_out_on_the_way_are_an_error(sdq, at, graph):
    """Somebody empties the pool ahead of the call's at-th step: the prefix's, the prompts', a token's."""
    import torch
    dec, calls = _decoder(), []
    step = dec.pool.step

    def emptied(*a, **more):
        if len(calls) == at:
            dec.pool.n_free.zero_()
        calls.append(1)
        return step(*a, **more)

    dec.pool.step = emptied
    # (15 + 1 tokens fill a page: the second token of the answer needs another)
    from paper_2510_03275_gb300 import serve
    with pytest.raises(RuntimeError):
        serve.generate(dec, PREFIX, [[1] * 16, [2, 3], [4] * 15], NEW, torch.rand((NEW, 3), device="cuda"), graph=graph)
