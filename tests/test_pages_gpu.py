"""GPU: a step's block tables against the definition, page by page on the
host: pools that run out, sequences that end, tables that are too short, rows
that nobody has, pages that end with a token."""
import numpy as np
import pytest

import oracle as O

pytestmark = pytest.mark.gpu


class Pool:
    """Sequences with own[s] tokens on pages of a pool that has `spare` more, in random order."""

    def __init__(self, page, own, new, done=None, columns=None, spare=1000, seed=0):
        rng = np.random.default_rng(seed)
        self.page, self.own, self.new = page, np.array(own, np.int32), np.array(new, np.int32)
        self.done = np.zeros(len(own), np.int32) if done is None else np.array(done, np.int32)
        have = -(-np.maximum(self.own, 0) // page)
        need = -(-(np.maximum(self.own, 0).astype(np.int64) + np.maximum(self.new, 0)) // page)
        columns = int(max(1, have.max(), min(need.max(), 4096))) if columns is None else columns
        self.n_pages = int(have.sum()) + spare
        order = rng.permutation(self.n_pages).astype(np.int32)
        self.tables = np.full((len(own), columns), -5, np.int32)
        at = 0
        for s, n in enumerate(have):
            self.tables[s, :n] = order[at:at + n]
            at += n
        self.free = order[at:]

    def run(self, sdq, torch, n_tokens, prefix=0, stride=None, in_place=False):
        dev = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()
        free = np.full(self.n_pages, -9, np.int32)
        free[:len(self.free)] = self.free
        pool = sdq.PagePool(self.page, dev(free), dev([len(self.free)]))
        columns = self.tables.shape[1]
        wide = torch.full((len(self.own), stride or columns), -77, dtype=torch.int32, device="cuda")
        tables = wide[:, :columns]
        tables.copy_(dev(self.tables))
        own, new, done = dev(self.own), dev(self.new), dev(self.done)
        step = pool.step(own, new, tables, n_tokens, done if self.done.any() else None, prefix, in_place)
        want = O.serving.pages_step(self.page, self.n_pages, self.free.tolist(), self.own.tolist(), self.new.tolist(), self.done.tolist(),
                                    self.tables.tolist(), n_tokens, prefix)
        start, lens, left, slots, positions, want_tables = want
        assert step.token_start.tolist() == start
        assert step.own_len.tolist() == lens
        assert step.n_free.tolist() == [len(left)]
        assert pool.free[:len(left)].tolist() == left
        assert step.slots.tolist() == slots and step.positions.tolist() == positions
        assert tables.tolist() == want_tables
        assert torch.all(wide[:, columns:] == -77)
        assert torch.equal(new, dev(self.new)) and torch.equal(done, dev(self.done))
        assert (own.tolist() == lens and pool.n_free.tolist() == [len(left)]) if in_place else \
               (torch.equal(own, dev(self.own)) and pool.n_free.tolist() == [len(self.free)])
        return step


CASES = {
    "one": ([0], [1], None),
    "edges": ([0, 15, 16, 17, 31, 32, 1, 127], [1] * 8, None),
    "nothing-new": ([5, 0, 40], [0, 0, 0], None),
    "prompts": ([0, 16, 3, 0, 200], [1, 300, 16, 77, 1], None),
    "done": ([5, 16, 17, 0, 64, 33], [0, 0, 0, 0, 0, 1], [1, 1, 0, 1, 1, 0]),
    "done-and-again": ([5, 16, 170, 0, 64, 33], [40, 1, 16, 2, 0, 1], [1, 1, 1, 0, -3, 0]),
    "all-done": ([50, 16, 170], [0, 0, 0], [1, 1, 1]),
    "negative": ([-4, 20, 7], [3, -2, 1], [0, 0, 1]),
}


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("name", CASES)
def test_pages_match_the_definition(sdq, name, page, in_place):
    import torch
    own, new, done = CASES[name]
    total = sum(max(0, n) for n in new)
    p = Pool(page, own, new, done, seed=len(name))
    p.run(sdq, torch, max(1, total), in_place=in_place)
    p.run(sdq, torch, total + 9, prefix=33, stride=p.tables.shape[1] + 3, in_place=in_place)


@pytest.mark.parametrize("n", [1, 2, 31, 33, 1000, 1024, 1025, 3000, 65535])
@pytest.mark.parametrize("kind", ["decode", "mixed"])
def test_many_sequences(sdq, n, kind):
    import torch
    rng = np.random.default_rng(n)
    own = rng.integers(0, 60, n)
    new = np.ones(n, int) if kind == "decode" else rng.choice([0, 1, 1, 5, 17], n)
    done = np.zeros(n, int) if kind == "decode" else (rng.random(n) < 0.2).astype(int)
    Pool(16, own, new, done, spare=2 * n + 10, seed=n).run(sdq, torch, int(new.sum()) + 3, prefix=7)


@pytest.mark.parametrize("spare", [0, 1, 2, 5, 20, 21, 22])
def test_pools_that_run_out(sdq, spare):
    """In the order of the sequences; one that needs no page is served behind one that gets none."""
    import torch
    Pool(16, [16, 3, 32, 0, 15, 48], [1, 2, 20, 300, 1, 1], spare=spare).run(sdq, torch, 325)
    Pool(16, [16, 3, 32, 0, 15, 48], [1, 2, 20, 300, 1, 1], [0, 0, 0, 0, 0, 1], spare=spare).run(sdq, torch, 325)


@pytest.mark.parametrize("n_tokens", [1, 4, 23, 24, 100, 347, 348])
def test_steps_with_too_few_rows(sdq, n_tokens):
    import torch
    Pool(16, [16, 3, 32, 0, 15, 48], [1, 2, 20, 300, 1, 24]).run(sdq, torch, n_tokens)


def test_tables_that_are_too_short(sdq):
    import torch
    Pool(16, [16, 3, 32, 0, 15, 48], [1, 2, 20, 60, 1, 17], columns=4).run(sdq, torch, 101)
    Pool(16, [0, 3], [2 ** 31 - 1, 5]).run(sdq, torch, 10)


def test_long_prompts(sdq):
    import torch
    Pool(64, [0, 5, 100], [70000, 30000, 1], spare=4000).run(sdq, torch, 100001)
    Pool(16, [70000, 5, 30000], [0, 3, 0], [1, 0, 1], spare=7).run(sdq, torch, 3)


def test_entries_outside_the_pool(sdq):
    """A page that the pool does not have gives no slot; more pages than the pool has do not come back."""
    import torch
    p = Pool(16, [20, 8], [1, 1])
    p.tables[0, 1], p.tables[1, 0] = p.n_pages, -1
    p.run(sdq, torch, 2)
    p = Pool(16, [64, 64], [0, 0], [1, 1], spare=0)
    p.free = np.arange(5, dtype=np.int32)                    # five of the eight are in the pool already
    p.run(sdq, torch, 1)


def test_steps_in_a_graph(sdq):
    """Decoding with the lengths, the pool and the tables on the GPU: a captured step replayed, sequences that end
    and begin again between the replays, against the same steps one by one."""
    import torch
    dev = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
    pool = sdq.PagePool(16, n_pages=40)
    own, new, done, tables = dev([0] * 4), dev([30, 15, 1, 7]), dev([0] * 4), torch.full((4, 8), -1, dtype=torch.int32, device="cuda")
    state = list(range(39, -1, -1)), [0] * 4, [[-1] * 8] * 4
    first = pool.step(own, new, tables, 53, done)
    n = 4
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step = pool.step(own, new, tables, n, done)
    assert own.tolist() == [30, 15, 1, 7] and first.slots.tolist()[:16] == list(range(16))
    s, o, free, _, _, t = O.serving.pages_step(16, 40, state[0], state[1], [30, 15, 1, 7], [0] * 4, state[2], 53)
    for i in range(40):
        ask, end = ([1, 1, 1, 1], [0, 0, i % 13 == 12, i % 20 == 5])
        if end[2]:
            ask[2] = 2 if i % 2 else 1
        new.copy_(dev(ask))
        done.copy_(dev([int(e) for e in end]))
        graph.replay()
        s, o, free, slots, pos, t = O.serving.pages_step(16, 40, free, o, ask, end, t, n)
        torch.cuda.synchronize()
        assert step.token_start.tolist() == s and own.tolist() == o and tables.tolist() == t
        assert step.slots.tolist() == slots and step.positions.tolist() == pos
        assert pool.n_free.tolist() == [len(free)] and pool.free[:len(free)].tolist() == free


def test_a_batch_on_the_pools_tables(sdq):
    """Sequences appended through the pool's tables: every token's value stands in the slot that the step named."""
    import torch
    dev = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
    pool = sdq.PagePool(16, n_pages=12)
    cache = sdq.KVCache(sdq.CacheDesc(1, 64, 16, 12))
    own, tables = dev([0, 0, 0]), torch.full((3, 4), -1, dtype=torch.int32, device="cuda")
    for new in ([20, 0, 3], [1, 17, 1], [12, 1, 0]):
        n = sum(new)
        step = pool.step(own, dev(new), tables, n)
        batch = sdq.Batch(step.token_start, step.own_len, tables, n, max(new), 64)
        x = [torch.randn((n, h * 64), device="cuda") for h in (2, 1, 1)]
        cache.append(batch, *x, sdq.Rope())
        flat = cache.v_pages.reshape(12 * 16, 64)
        assert torch.equal(flat[step.slots.long()], x[2].to(torch.bfloat16))
    assert sorted(set(tables.flatten().tolist()) - {-1}) == sorted(pool.free[int(pool.n_free):].tolist())


def test_pages_on_another_stream(sdq):
    import torch
    dev = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
    pool = sdq.PagePool(16, n_pages=30)
    own, new, tables = dev([5, 0]), dev([20, 40]), torch.zeros((2, 5), dtype=torch.int32, device="cuda")
    want = pool.step(own, new, tables, 60, in_place=False)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = pool.step(own, new, tables, 60, in_place=False, stream=side)
    side.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_pages_refusals(sdq):
    import torch
    i = torch.zeros(4, dtype=torch.int32, device="cuda")
    t = torch.zeros((4, 3), dtype=torch.int32, device="cuda")
    pool = sdq.PagePool(16, n_pages=8)
    for bad in (lambda: sdq.PagePool(16), lambda: sdq.PagePool(16, i.long()), lambda: sdq.PagePool(16, i.cpu()),
                lambda: sdq.PagePool(16, i, i), lambda: sdq.PagePool(16, n_pages=0), lambda: pool.step(i.long(), i, t, 4),
                lambda: pool.step(i, i[:3], t, 4), lambda: pool.step(i, i, t[:3], 4), lambda: pool.step(i, i, t.t(), 4),
                lambda: pool.step(i, i, t.cpu(), 4), lambda: pool.step(i, i.clone(), t, 4, done=i[:2]), lambda: pool.step(i, i.clone(), t, 4, done=i),
                lambda: pool.step(i, i, t, 4)):
        with pytest.raises(ValueError):
            bad()
    j = i.clone()
    for bad in (lambda: pool.step(i, j, t, 0), lambda: pool.step(i, j, t, (1 << 20) + 1), lambda: pool.step(i, j, t, 4, prefix_len=-1),
                lambda: pool.step(i[:0], j[:0], t[:0], 4), lambda: pool.step(i, j, t[:, :0], 4),
                lambda: sdq.PagePool(24, n_pages=8).step(i, j, t, 4)):
        with pytest.raises(sdq.SdqError) as e:
            bad()
        assert e.value.status == -1
    torch.cuda.synchronize()
