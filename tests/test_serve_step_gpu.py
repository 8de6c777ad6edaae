"""GPU: a decoder with norms of queries and keys, windowed attention, pages
from the pool and penalties (`serve`) against the same decoder in fp64 on the
host: every request's whole sequence at once, no cache, no pages."""
import numpy as np
import pytest

import oracle as O
from paper_2510_03275_gb300 import workloads as W

pytestmark = pytest.mark.gpu


def _norm(x):
    return x / np.sqrt(np.square(x).mean(-1, keepdims=True) + 1e-5)


def _host_logits(shape, w, emb, seq):
    """fp64 logits after every token of one sequence."""
    n, d, group = len(seq), shape.head_dim, shape.q_heads // shape.kv_heads
    angle = np.arange(n)[:, None] * 10000.0 ** (-np.arange(d // 2) / (d // 2))
    cos, sin = np.cos(angle), np.sin(angle)
    turn = lambda x: np.stack([O.serving.rotate(x[t], t, cos, sin, False) for t in range(n)])
    p, j = np.arange(n)[:, None], np.arange(n)[None]
    hidden = j > p
    if shape.window:
        hidden |= (j <= p - shape.window) & (j >= shape.sinks)
    h = emb[seq]
    for i in range(shape.layers):
        qkv = _norm(h) @ w[f"{i}.qkv"].T
        q, k, v = np.split(qkv, [shape.q_heads * d, (shape.q_heads + shape.kv_heads) * d], axis=1)
        q, k, v = q.reshape(n, -1, d), k.reshape(n, -1, d), v.reshape(n, -1, d)
        if shape.qk_norm:
            q, k = O.serving.head_norm(q, w[f"{i}.q_norm"], 1e-5), O.serving.head_norm(k, w[f"{i}.k_norm"], 1e-5)
        q, k = turn(q), turn(k)
        a = np.empty_like(q)
        for hd in range(shape.q_heads):
            s = q[:, hd] @ k[:, hd // group].T * d ** -0.5
            s[hidden] = -np.inf
            e = np.exp(s - s.max(1, keepdims=True))
            a[:, hd] = e / e.sum(1, keepdims=True) @ v[:, hd // group]
        h = h + a.reshape(n, -1) @ w[f"{i}.o"].T
        gate, up = np.split(_norm(h) @ w[f"{i}.gate_up"].T, 2, axis=1)
        h = h + (gate / (1 + np.exp(-gate)) * up) @ w[f"{i}.down"].T
    return _norm(h) @ w["head"].T


def _decoder(serve, **more):
    shape = serve.Shape(hidden=256, ffn=384, layers=2, q_heads=4, kv_heads=2, vocab=500, **more)
    weights = serve.random_weights(shape, seed=shape.head_dim)
    signs = W.hadamard_signs(W.config(1).linears[0], shape.block)
    dec = serve.Decoder(shape, weights, n_pages=40, n_pos=256, signs=signs)
    w = {name: x.cpu().numpy().astype(np.float64) for name, x in weights.items()}
    for name, _, _ in shape.linears():
        codes, alpha = O.encode(weights[name].cpu().numpy(), shape.block, 2 * shape.block, O.TERNARY, O.ALPHA_MAXABS, signs)
        w[name] = O.reconstruct(codes, alpha, shape.block, 2 * shape.block, signs)
    return dec, w


@pytest.mark.parametrize("head_dim,prefix_len,window,sinks,graph", [(64, 37, 20, 3, True), (128, 0, 33, 0, True), (64, 16, 1, 2, False),
                                                                     (128, 9, 0, 0, True)])
def test_a_step_of_all_operators_matches_the_decoder_in_fp64(sdq, head_dim, prefix_len, window, sinks, graph):
    """The same roundings as without norms and windows (26 to bf16, 3 sqrt(26) 2^-9 = 3.0e-2 of the logits' rms; see
    the tests of `generate`); a penalty multiplies a logit, and its error, by 1.25 at most."""
    import torch
    from paper_2510_03275_gb300 import serve
    dec, w = _decoder(serve, head_dim=head_dim, qk_norm=True, window=window, sinks=sinks)
    shape, vocab = dec.shape, dec.shape.vocab
    rng = np.random.default_rng(prefix_len + 1)
    draw = lambda n: rng.integers(0, vocab, n).tolist()
    prefix, prompts, n_new, n = draw(prefix_len), [draw(1), draw(70), draw(16), draw(5)], 6, 4
    u = rng.random((n_new, n)).astype(np.float32)
    t, k, p, m = np.float32([0, 1, 0.8, 1.2]), np.int32([0, 40, 0, 0]), np.float32([1, 0.9, 0.8, 1]), np.float32([0, 0, 0, 0.02])
    rep, freq, pres = np.float32([1.25, 1, 0.8, 1.1]), np.float32([0.5, 0, 0.3, -0.2]), np.float32([0.1, 0.2, 0, 0])
    ids = np.stack([rng.permutation(vocab)[:9] for _ in range(n)]).astype(np.int32)
    bias = (2 * rng.standard_normal((n, 9))).astype(np.float32)
    bits = rng.random((2, -(-vocab // 32) * 32)) < 0.7
    words, row = np.packbits(bits, axis=1, bitorder="little").view(np.int32), np.int32([-1, 0, 1, -1])
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    got, logits = serve.generate(dec, prefix, prompts, n_new, dev(u), dev(t), dev(k), dev(p), dev(m), graph=graph, keep_logits=True,
                                 repetition=dev(rep), frequency=dev(freq), presence=dev(pres), bias_ids=dev(ids), bias=dev(bias),
                                 allowed=dev(words), allowed_row=dev(row))
    got, logits = got.cpu().numpy(), logits.cpu().numpy()
    for r, prompt in enumerate(prompts):
        history = prefix + prompt + got[:, r].tolist()
        raw = _host_logits(shape, w, w["embedding"], np.array(history[:-1]))[-n_new:]
        allowed = None if row[r] < 0 else set(np.flatnonzero(bits[row[r]]).tolist())
        for i in range(n_new):
            before = history[:len(prefix) + len(prompt) + i]
            want = O.serving.adjust_row(raw[i], before, len(prefix) + len(prompt), float(rep[r]), float(freq[r]), float(pres[r]),
                                        list(zip(ids[r].tolist(), bias[r].astype(float).tolist())), allowed)
            fine = np.isfinite(want)
            assert np.array_equal(np.isfinite(logits[i, r]), fine)
            err = (logits[i, r] - want)[fine]
            assert np.sqrt(np.square(err).mean()) <= 1.25 * 3.0e-2 * np.sqrt(np.square(raw[i]).mean())
    for i in range(n_new):   # the tokens, from the logits that the GPU had
        token, margin = O.serving.sample(logits[i], u[i], t, k, p, m)
        assert np.array_equal(got[i][margin > 2e-6], token[margin > 2e-6])
    # every page is back, and the next answers find them in another order
    assert int(dec.pool.n_free) == 40 and sorted(dec.pool.free.tolist()) == list(range(40))
    again = serve.generate(dec, prefix, prompts, n_new, dev(u), dev(t), dev(k), dev(p), dev(m), graph=not graph,
                           repetition=dev(rep), frequency=dev(freq), presence=dev(pres), bias_ids=dev(ids), bias=dev(bias),
                           allowed=dev(words), allowed_row=dev(row))
    assert np.array_equal(again.cpu().numpy(), got)
