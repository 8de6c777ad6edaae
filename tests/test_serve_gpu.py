"""GPU: the linears, the cache, attention and sampling together (`serve`)
against the same decoder in fp64 on the host: the codes' reconstructed weights,
every request's whole sequence at once, no cache and no shared prefix."""
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
    h = emb[seq]
    for i in range(shape.layers):
        qkv = _norm(h) @ w[f"{i}.qkv"].T
        q, k, v = np.split(qkv, [shape.q_heads * d, (shape.q_heads + shape.kv_heads) * d], axis=1)
        q, k, v = turn(q.reshape(n, -1, d)), turn(k.reshape(n, -1, d)), v.reshape(n, -1, d)
        a = np.empty_like(q)
        for hd in range(shape.q_heads):
            s = q[:, hd] @ k[:, hd // group].T * d ** -0.5
            s[np.triu_indices(n, 1)] = -np.inf
            p = np.exp(s - s.max(1, keepdims=True))
            a[:, hd] = p / p.sum(1, keepdims=True) @ v[:, hd // group]
        h = h + a.reshape(n, -1) @ w[f"{i}.o"].T
        gate, up = np.split(_norm(h) @ w[f"{i}.gate_up"].T, 2, axis=1)
        h = h + (gate / (1 + np.exp(-gate)) * up) @ w[f"{i}.down"].T
    return _norm(h) @ w["head"].T


@pytest.mark.parametrize("head_dim,prefix_len,graph", [(64, 37, True), (128, 0, True), (64, 16, False)])
def test_generate_matches_the_decoder_in_fp64(sdq, head_dim, prefix_len, graph):
    """Roundings to bf16 on a logit's path (relative 2^-9 rms at most each, about 2^-9 for a decode call's terms): a
    layer's 2 norms, q, k, v, p, a, the product of gate and up and x_tilde of its 4 linears, 12; 2 layers and the
    head's 2: 26 independent ones, sqrt(26) 2^-9 = 1.0e-2 of the logits' rms where a rounding reaches them
    undamped; the bar is 3 times that."""
    import torch
    from paper_2510_03275_gb300 import serve
    shape = serve.Shape(hidden=256, ffn=384, layers=2, q_heads=4, kv_heads=2, head_dim=head_dim, vocab=500)
    weights = serve.random_weights(shape, seed=head_dim)
    signs = W.hadamard_signs(W.config(1).linears[0], shape.block)
    dec = serve.Decoder(shape, weights, n_pages=40, n_pos=256, signs=signs)
    w = {}
    for name, _, _ in shape.linears():
        codes, alpha = O.encode(weights[name].cpu().numpy(), shape.block, 2 * shape.block, O.TERNARY, O.ALPHA_MAXABS, signs)
        w[name] = O.reconstruct(codes, alpha, shape.block, 2 * shape.block, signs)
    emb = weights["embedding"].cpu().numpy().astype(np.float64)
    rng = np.random.default_rng(prefix_len)
    draw = lambda n: rng.integers(0, shape.vocab, n).tolist()
    prefix, prompts, n_new = draw(prefix_len), [draw(1), draw(70), draw(16), draw(5)], 5
    u = rng.random((n_new, 4)).astype(np.float32)
    t, k, p, m = np.float32([0, 1, 0.8, 1.2]), np.int32([0, 40, 0, 0]), np.float32([1, 0.9, 0.8, 1]), np.float32([0, 0, 0, 0.02])
    dev = lambda a: torch.from_numpy(a).cuda()
    got, logits = serve.generate(dec, prefix, prompts, n_new, dev(u), dev(t), dev(k), dev(p), dev(m), graph=graph, keep_logits=True)
    got, logits = got.cpu().numpy(), logits.cpu().numpy()
    for r, prompt in enumerate(prompts):
        seq = np.array(prefix + prompt + got[:, r].tolist())
        want = _host_logits(shape, w, emb, seq[:-1])[-n_new:]
        assert np.sqrt(np.square(logits[:, r] - want).mean()) <= 3.0e-2 * np.sqrt(np.square(want).mean())
    for i in range(n_new):   # the tokens, from the logits that the GPU had (MARGIN of the sampling tests)
        token, margin = O.serving.sample(logits[i], u[i], t, k, p, m)
        assert np.array_equal(got[i][margin > 2e-6], token[margin > 2e-6])


def test_generate_refuses(sdq):
    import torch
    from paper_2510_03275_gb300 import serve
    shape = serve.Shape(hidden=128, ffn=128, layers=1, q_heads=2, kv_heads=2, head_dim=64, vocab=100)
    dec = serve.Decoder(shape, serve.random_weights(shape), n_pages=2, n_pos=64)
    u = torch.zeros((4, 2), device="cuda")
    for prefix, prompts in (([], [[1], []]), ([1], [[1], [2]])):   # an empty prompt; 3 pages
        with pytest.raises(ValueError):
            serve.generate(dec, prefix, prompts, 4, u)


def test_calls_on_another_stream(sdq):
    """What a call allocates belongs to the stream that it runs on: a busy stream's results do not depend on what
    the current one allocates meanwhile."""
    import torch
    from serving_inputs import Case
    case = Case((8, 2, 64), [1, 3, 40], [90, 3, 200], prefix=50, seed=5)
    cache, batch = case.cache(sdq, torch), case.batch(sdq, torch)
    q = torch.from_numpy(case.q).to(torch.bfloat16).cuda()
    z = torch.from_numpy(np.random.default_rng(0).standard_normal((5, 3000)).astype(np.float32)).cuda()
    u = torch.linspace(0, 0.9, 5, device="cuda")
    want, want_t = cache.attend(batch, q).clone(), sdq.sample(z, u).clone()
    torch.cuda.synchronize()
    side, big = torch.cuda.Stream(), torch.zeros(1 << 28, device="cuda")
    side.wait_stream(torch.cuda.current_stream())
    for stream in (side, side.cuda_stream):
        with torch.cuda.stream(side):
            big.add_(1)   # (keeps it busy for some hundred us)
        got = [(cache.attend(batch, q, stream=stream), sdq.sample(z, u, stream=stream)) for _ in range(3)]
        junk = [torch.full((1 << 16,), -1, dtype=torch.int32, device="cuda") for _ in range(8)]
        torch.cuda.synchronize()
        for a, t in got:
            assert torch.equal(a, want) and torch.equal(t, want_t)
        del junk
