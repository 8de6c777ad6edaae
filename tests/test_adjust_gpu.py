"""GPU: penalties, biases and allowed tokens on logits against the fp64
definition, where they can go wrong: rows off 16-byte boundaries, tokens named
twice, empty histories and sets, values that are not finite, in place."""
import numpy as np
import pytest

import oracle as O
from serving_inputs import bf16

pytestmark = pytest.mark.gpu


class Rows:
    """Rows of logits with what is done to them, on the host."""

    def __init__(self, rows, vocab, history=0, biases=0, allowed=None, kind="f32", seed=0):
        rng = np.random.default_rng(seed)
        self.kind, self.rows, self.vocab = kind, rows, vocab
        self.z = (3 * rng.standard_normal((rows, vocab))).astype(np.float32)
        if kind == "bf16":
            self.z = bf16(self.z)
        self.history = self.bias_ids = self.bias = self.allowed = self.allowed_row = None
        if history:
            self.history = (rng.random((rows, history)) ** 3 * vocab).astype(np.int32)
            self.history_len = rng.integers(0, history + 1, rows).astype(np.int32)
            self.history_len[0] = history
            self.prompt_len = (self.history_len * rng.random(rows)).astype(np.int32)
        self.repetition = rng.choice([0.9, 1.0, 1.2], rows).astype(np.float32)
        self.frequency, self.presence = (rng.choice([-0.3, 0.0, 0.25], rows).astype(np.float32) for _ in range(2))
        if biases:
            self.bias_ids = rng.integers(-1, vocab, (rows, biases)).astype(np.int32)
            self.bias_ids[:, -1] = self.bias_ids[:, 0]
            self.bias = (4 * rng.standard_normal((rows, biases))).astype(np.float32)
            self.bias[rng.random((rows, biases)) < 0.05] = -np.inf
        if allowed is not None:
            sets = max(1, rows // 2)
            bits = rng.random((sets, -(-vocab // 32) * 32)) < allowed
            self.allowed = np.packbits(bits, axis=1, bitorder="little").view(np.int32)
            self.bits = bits
            self.allowed_row = rng.integers(-1, sets, rows).astype(np.int32)

    def arguments(self, torch):
        dev = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()
        a = dict(repetition=dev(self.repetition), frequency=dev(self.frequency), presence=dev(self.presence), bias_ids=dev(self.bias_ids),
                 bias=dev(self.bias), allowed=dev(self.allowed), allowed_row=dev(self.allowed_row))
        if self.history is not None:
            a.update(history=dev(self.history), history_len=dev(self.history_len), prompt_len=dev(self.prompt_len))
        return a

    def logits(self, torch, lead=0, pad=0):
        """Rows that begin `lead` elements behind a boundary, `pad` elements apart."""
        dtype = torch.bfloat16 if self.kind == "bf16" else torch.float32
        flat = torch.full((lead + self.rows * (self.vocab + pad),), float("nan"), dtype=dtype, device="cuda")
        z = flat[lead:].reshape(self.rows, self.vocab + pad)[:, :self.vocab]
        z.copy_(torch.from_numpy(self.z))
        return z

    def check(self, got):
        got = got.float().cpu().numpy().astype(np.float64)
        for i in range(self.rows):
            history = [] if self.history is None else self.history[i, :max(0, self.history_len[i])].tolist()
            bias = [] if self.bias is None else list(zip(self.bias_ids[i].tolist(), self.bias[i].astype(np.float64).tolist()))
            allowed = None
            if self.allowed is not None and 0 <= self.allowed_row[i] < len(self.allowed):
                allowed = set(np.flatnonzero(self.bits[self.allowed_row[i]]).tolist())
            n0 = 0 if self.history is None else max(0, int(self.prompt_len[i]))
            r, f, p = (float(a[i]) for a in (self.repetition, self.frequency, self.presence))
            want = O.serving.adjust_row(self.z[i], history, n0, r, f, p, bias, allowed)
            # fp32: the quotient or product, frequency c + presence (2), the difference, the biases' sum (one each),
            # the sum with it; every one 2^-24 of no more than the magnitudes added up; bf16 rounds once more
            count = len(history)
            size = np.abs(self.z[i]) * max(r, 1 / r) + abs(f) * count + abs(p) + sum(abs(b) for _, b in bias if np.isfinite(b))
            bound = 2.0 ** -24 * (5 + len(bias)) * size + (2.0 ** -8 * np.abs(want) if self.kind == "bf16" else 0)
            same = (got[i] == want) | (np.isnan(got[i]) & np.isnan(want))
            with np.errstate(invalid="ignore"):
                assert np.all(same | (np.abs(got[i] - want) <= bound)), i
            touched = set(history) | {t for t, _ in bias}
            rest = np.array([t for t in range(self.vocab) if t not in touched and (allowed is None or t in allowed)], int)
            assert np.array_equal(got[i, rest], self.z[i, rest].astype(np.float64), equal_nan=True)


CASES = {
    "one": dict(rows=1, vocab=1),
    "few": dict(rows=3, vocab=5, history=7, biases=3, allowed=0.5),
    "penalties": dict(rows=4, vocab=2001, history=700),
    "long-history": dict(rows=2, vocab=999, history=20000),
    "biases": dict(rows=3, vocab=4099, biases=70),
    "many-biases": dict(rows=2, vocab=300, biases=4096, history=10),
    "grammar": dict(rows=5, vocab=10007, allowed=0.1),
    "grammar-32": dict(rows=3, vocab=64, allowed=0.5, history=40),
    "all": dict(rows=7, vocab=30011, history=900, biases=33, allowed=0.6),
    "chunks": dict(rows=2, vocab=70001, history=3000, biases=200, allowed=0.9),
    "tokens-of-nobody": dict(rows=2, vocab=33000, history=1),
}


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("name", CASES)
def test_adjust_matches_the_definition(sdq, name, kind):
    import torch
    r = Rows(**CASES[name], kind=kind, seed=len(name))
    z = r.logits(torch)
    r.check(sdq.adjust_logits(z, **r.arguments(torch)))
    assert torch.equal(z, torch.from_numpy(r.z).to(z.dtype).cuda())      # the logits stay
    assert sdq.adjust_logits(z, **r.arguments(torch), out=z) is z
    r.check(z)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("lead,pad", [(1, 0), (3, 5), (0, 8), (7, 16)])
@pytest.mark.parametrize("out_lead,out_pad", [(0, 0), (1, 0), (3, 5)])
def test_rows_off_boundaries(sdq, kind, lead, pad, out_lead, out_pad):
    import torch
    r = Rows(5, 8209, 300, 9, 0.7, kind, seed=lead + pad)
    z, out = r.logits(torch, lead, pad), r.logits(torch, out_lead, out_pad)
    around = out.untyped_storage()
    whole = torch.empty(0, dtype=out.dtype, device="cuda").set_(around)
    whole.fill_(-7.0)
    sdq.adjust_logits(z, **r.arguments(torch), out=out)
    r.check(out)
    inside = torch.zeros_like(whole, dtype=torch.bool)
    inside[out_lead:].reshape(5, -1)[:, :8209] = True
    assert torch.all(whole[~inside] == -7.0)                              # nothing between the rows is written
    sdq.adjust_logits(z, **r.arguments(torch), out=z)
    r.check(z)


@pytest.mark.parametrize("in_place", [False, True])
def test_values_that_are_not_finite(sdq, in_place):
    import torch
    r = Rows(2, 5000, 2000, 30, 0.8, seed=3)
    r.bias[r.bias == -np.inf] = 0.5
    r.z[:, ::7], r.z[:, 1::7], r.z[:, 2::7], r.z[:, 3::7] = np.nan, np.inf, -np.inf, -np.finfo(np.float32).max
    r.repetition[:], r.frequency[:], r.presence[:] = 0.9, 0.25, -0.25
    z = r.logits(torch)
    with np.errstate(invalid="ignore"):
        r.check(sdq.adjust_logits(z, **r.arguments(torch), out=z if in_place else None))


def test_lengths_and_tokens_out_of_range(sdq):
    """Lengths are cut to the bounds; tokens that the vocabulary does not have, and sets that there are not, mean nothing."""
    import torch
    r = Rows(6, 700, 50, 8, 0.5, seed=4)
    r.history[:, 3::5], r.history[:, 4::5] = 700, -3
    r.bias_ids[:, 2], r.bias_ids[:, 5] = 700, -(1 << 31)
    a = r.arguments(torch)
    a["history_len"] = torch.tensor([1000, -5, 50, 0, 1 << 30, 20], dtype=torch.int32, device="cuda")
    a["prompt_len"] = torch.tensor([-4, 3, 1000, 0, 10, 20], dtype=torch.int32, device="cuda")
    a["allowed_row"] = torch.tensor([3, -1, 1 << 30, 0, 1, -(1 << 31)], dtype=torch.int32, device="cuda")
    r.history_len, r.prompt_len, r.allowed_row = np.array([50, 0, 50, 0, 50, 20]), np.array([0, 0, 50, 0, 10, 20]), a["allowed_row"].cpu().numpy()
    r.check(sdq.adjust_logits(r.logits(torch), **a))


def test_parts_that_are_left_out(sdq):
    import torch
    z = torch.randn((3, 1000), device="cuda")
    assert torch.equal(sdq.adjust_logits(z), z)
    h = torch.full((3, 4), 9, dtype=torch.int32, device="cuda")
    assert torch.equal(sdq.adjust_logits(z, h), z)
    got = sdq.adjust_logits(z, h, presence=torch.ones(3, device="cuda"))     # all of the history is the answer's
    assert torch.equal(got[:, 9], z[:, 9] - 1) and torch.equal(got[:, 10:], z[:, 10:])
    words = torch.zeros((3, 32), dtype=torch.int32, device="cuda")
    words[0, 0], words[1, 31] = -(1 << 31), 1 << 7                           # tokens 31 and 999; row 2: none
    got = sdq.adjust_logits(z, allowed=words)
    assert got.isfinite().nonzero().tolist() == [[0, 31], [1, 999]]
    assert torch.equal(sdq.adjust_logits(z, bias_ids=h[:, :0], bias=z[:, :0]), z)


def test_shared_rows_and_equal_ids(sdq):
    """One list for all rows (stride 0); biases of one token are added up in their order."""
    import torch
    z = torch.zeros((4, 300), device="cuda")
    big = torch.tensor([[1e8, 1.0, -1e8, 0.5]], device="cuda").expand(4, 4)
    ids = torch.tensor([[7, 7, 7, 7]], dtype=torch.int32, device="cuda").expand(4, 4)
    got = sdq.adjust_logits(z, bias_ids=ids, bias=big)
    assert got[:, 7].tolist() == [0.5] * 4                                   # (1e8 + 1 rounds to 1e8)
    many = torch.tensor([[7] * 40 + [8] * 40 + [7] * 40], dtype=torch.int32, device="cuda").expand(4, 120)
    got = sdq.adjust_logits(z, bias_ids=many, bias=torch.ones((4, 120), device="cuda"))
    assert got[:, 7].tolist() == [80.0] * 4 and got[:, 8].tolist() == [40.0] * 4 and got.sum() == 480


def test_adjust_streams_graphs_and_repeats(sdq):
    import torch
    r = Rows(9, 20011, 5000, 40, 0.7, seed=5)
    z, a = r.logits(torch), r.arguments(torch)
    want = sdq.adjust_logits(z, **a)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = sdq.adjust_logits(z, **a, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    out, graph = torch.empty_like(z), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sdq.adjust_logits(z, **a, out=out)
    for _ in range(10):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    a["history_len"].zero_()
    graph.replay()
    torch.cuda.synchronize()
    r.history_len[:] = 0
    r.check(out)


def test_adjust_refusals(sdq):
    import torch
    z = torch.zeros((2, 100), device="cuda")
    i = torch.zeros((2, 4), dtype=torch.int32, device="cuda")
    f = torch.zeros((2, 4), device="cuda")
    one = torch.ones(2, device="cuda")
    for bad in (lambda: sdq.adjust_logits(z[0]), lambda: sdq.adjust_logits(z.t()), lambda: sdq.adjust_logits(z.cpu()),
                lambda: sdq.adjust_logits(z, i.long()), lambda: sdq.adjust_logits(z, i[:1]), lambda: sdq.adjust_logits(z, i, one),
                lambda: sdq.adjust_logits(z, i, repetition=one.double()), lambda: sdq.adjust_logits(z, i, repetition=one[:1]),
                lambda: sdq.adjust_logits(z, bias_ids=i), lambda: sdq.adjust_logits(z, bias_ids=i, bias=f[:, :3]),
                lambda: sdq.adjust_logits(z, allowed=i[:, :3]), lambda: sdq.adjust_logits(z, allowed_row=i[:, 0].contiguous()),
                lambda: sdq.adjust_logits(z, history_len=i[:, 0].contiguous()), lambda: sdq.adjust_logits(z, out=z[:1]),
                lambda: sdq.adjust_logits(z, out=z.half()), lambda: sdq.adjust_logits(z, i.t().contiguous().t())):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: sdq.adjust_logits(z.half()), lambda: sdq.adjust_logits(z, allowed=i[:1]),
                lambda: sdq.adjust_logits(z, bias_ids=torch.zeros((2, 4097), dtype=torch.int32, device="cuda"),
                                          bias=torch.zeros((2, 4097), device="cuda")),
                lambda: sdq.adjust_logits(torch.zeros((1, 393217), device="cuda"))):
        with pytest.raises(sdq.SdqError) as e:
            bad()
        assert e.value.status == -1
    flat = torch.zeros(300, device="cuda")                                   # out over the logits, but not in their place
    with pytest.raises(sdq.SdqError):
        sdq.adjust_logits(flat[:200].reshape(2, 100), out=flat[4:204].reshape(2, 100))
    torch.cuda.synchronize()
