"""Serving with the quantized layer: a decoder whose linears are Sigma-Delta
plans, a paged cache behind a prefix that all requests share, attention over
it, and sampling.

    python -m paper_2510_03275_gb300.serve --batch 32 --prefix 2000 --new 64

builds one of random weights, answers a batch of random requests and prints a
JSON line.  Decoding steps replay one CUDA graph: its batch's lengths and last
tokens live on the GPU and move on inside the graph.
"""
from __future__ import annotations

import argparse
import json
import time
from dataclasses import dataclass
from fractions import Fraction

from . import Batch, CacheDesc, KVCache, LayerDesc, Plan, Rope, sample, workloads as W


@dataclass(frozen=True)
class Shape:
    hidden: int = 2048
    ffn: int = 5632
    layers: int = 4
    q_heads: int = 16
    kv_heads: int = 4
    head_dim: int = 128
    vocab: int = 32000
    block: int = 128
    osr: Fraction = Fraction(2)

    def linears(self):
        """(name, n_out, k_in) of every linear; those that read the same input are one."""
        q, kv = self.q_heads * self.head_dim, self.kv_heads * self.head_dim
        for i in range(self.layers):
            yield f"{i}.qkv", q + 2 * kv, self.hidden
            yield f"{i}.o", self.hidden, q
            yield f"{i}.gate_up", 2 * self.ffn, self.hidden
            yield f"{i}.down", self.hidden, self.ffn
        yield "head", self.vocab, self.hidden


def random_weights(shape: Shape, seed=0, device="cuda"):
    """fp32 weights by name; outputs of unit variance for inputs of unit variance."""
    import torch
    g = torch.Generator(device).manual_seed(seed)
    w = {name: torch.randn((n, k), generator=g, device=device) * k ** -0.5 for name, n, k in shape.linears()}
    w["embedding"] = torch.randn((shape.vocab, shape.hidden), generator=g, device=device)
    return w


def _norm(x):
    """Rows of unit mean square, in bf16 (the linears' input type)."""
    import torch
    return (x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-5)).to(torch.bfloat16)


class Decoder:
    """The plans and codes of a decoder, and a cache per layer."""

    def __init__(self, shape: Shape, weights, n_pages: int, page_tokens=16, n_pos=8192, signs=None):
        self.shape, self.page_tokens, self.n_pages = shape, page_tokens, n_pages
        self.embedding = weights["embedding"]
        self.layers = {}
        for name, n, k in shape.linears():
            plan = Plan(LayerDesc(n, k, shape.block, shape.osr, W.TERNARY), signs)
            codes, alpha = plan.encode(weights[name])
            self.layers[name] = plan, plan.pack(codes), alpha
        desc = CacheDesc(shape.kv_heads, shape.head_dim, page_tokens, n_pages)
        self.caches = [KVCache(desc, device=self.embedding.device) for _ in range(shape.layers)]
        self.rope = Rope.table(n_pos, shape.head_dim, device=self.embedding.device)

    def linear(self, name, x):
        plan, codes, alpha = self.layers[name]
        return plan.forward(codes, alpha, x)

    def forward(self, tokens, batch: Batch, rows=None):
        """Append the batch's tokens to the caches; fp32 logits of the given rows (all of them: None)."""
        import torch
        s = self.shape
        q_width, kv_width = s.q_heads * s.head_dim, s.kv_heads * s.head_dim
        ws = self.caches[0].alloc_workspace(batch, s.q_heads)   # (the layers take turns on it)
        h = self.embedding[tokens.long()]
        for i, cache in enumerate(self.caches):
            q, k, v = self.linear(f"{i}.qkv", _norm(h)).split([q_width, kv_width, kv_width], dim=1)
            q = cache.append(batch, q, k, v, self.rope)
            a = cache.attend(batch, q, ws=ws)
            h = h + self.linear(f"{i}.o", a.flatten(1))
            gate, up = self.linear(f"{i}.gate_up", _norm(h)).chunk(2, dim=1)
            h = h + self.linear(f"{i}.down", (gate * torch.sigmoid(gate) * up).to(torch.bfloat16))
        return self.linear("head", _norm(h if rows is None else h[rows]))


def generate(dec: Decoder, prefix, prompts, n_new, u, temperature=None, top_k=None, top_p=None, min_p=None, graph=True,
             keep_logits=False):
    """Answer requests that all begin with the tokens `prefix` (a list, may be
    empty) and go on with their own `prompts` (lists of at least one token):
    n_new tokens each, from random numbers u (n_new x requests, on the GPU), as
    an int32 tensor (n_new x requests); with keep_logits also the logits that
    they were drawn from.  Settings as in `sample`."""
    import torch
    dev, page, n = dec.embedding.device, dec.page_tokens, len(prompts)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)
    lens = [len(p) for p in prompts]
    per = [-(-(m + n_new) // page) for m in lens]
    n_prefix = -(-len(prefix) // page)
    if min(lens) < 1 or n_prefix + sum(per) > dec.n_pages:
        raise ValueError("generate: an empty prompt, or more tokens than the cache has pages for")
    prefix_pages = list(range(n_prefix))
    at, table = n_prefix, []
    for m in per:
        table.append(list(range(at, at + m)) + [-1] * (max(per) - m))
        at += m
    shared = dict(prefix_pages=ints(prefix_pages) if prefix else None, prefix_len=len(prefix))
    if prefix:   # its keys and values, once for everybody
        dec.forward(ints(prefix), Batch(ints([0, len(prefix)]), ints([len(prefix)]), ints([prefix_pages]), len(prefix),
                                        len(prefix), len(prefix)), rows=slice(-1, None))
    ends = torch.tensor(lens).cumsum(0).tolist()
    pages = ints(table)
    prompt = Batch(ints([0] + ends), ints(lens), pages, ends[-1], max(lens), max(lens), **shared)
    own = ints(lens)
    step = Batch(torch.arange(n + 1, dtype=torch.int32, device=dev), own, pages, n, 1, max(lens) + n_new, **shared)
    last = ints([e - 1 for e in ends]).long()
    u_now, tokens, out, logits = u[0].clone(), torch.empty(n, dtype=torch.int32, device=dev), [], []

    def choose(z):
        tokens.copy_(sample(z, u_now, temperature, top_k, top_p, min_p))
        return z

    def decode():
        own.add_(1)
        return choose(dec.forward(tokens, step))

    z, replay = choose(dec.forward(ints([t for p in prompts for t in p]), prompt, rows=last)), None
    for i in range(n_new):
        if i > 0:
            u_now.copy_(u[i])
            if replay is not None:
                replay.replay()
            else:
                z = decode()
        out.append(tokens.clone())
        if keep_logits:
            logits.append(z.clone())
        if graph and i == 1 and n_new > 2:   # (after a step of the same sizes has run)
            replay = torch.cuda.CUDAGraph()
            with torch.cuda.graph(replay):
                z = decode()
    return (torch.stack(out), torch.stack(logits)) if keep_logits else torch.stack(out)


def main(argv=None):
    import torch
    ap = argparse.ArgumentParser(description="answer a batch of random requests with a decoder of random weights (JSON)")
    ap.add_argument("--batch", type=int, default=32)
    ap.add_argument("--prefix", type=int, default=2000, help="tokens that all requests share")
    ap.add_argument("--prompt", type=int, default=100, help="the longest prompt")
    ap.add_argument("--new", type=int, default=64, help="tokens to generate per request")
    ap.add_argument("--layers", type=int, default=4)
    a = ap.parse_args(argv)
    shape = Shape(layers=a.layers)
    g = torch.Generator().manual_seed(1)
    draw = lambda m: torch.randint(shape.vocab, (m,), generator=g).tolist()
    prefix = draw(a.prefix)
    prompts = [draw(int(torch.randint(1, a.prompt + 1, (1,), generator=g))) for _ in range(a.batch)]
    pages = -(-a.prefix // 16) + a.batch * -(-(a.prompt + a.new) // 16)
    dec = Decoder(shape, random_weights(shape), pages, n_pos=a.prefix + a.prompt + a.new)
    u = torch.rand((a.new, a.batch), generator=g).cuda()
    col = lambda x, dtype=torch.float32: torch.full((a.batch,), x, dtype=dtype, device="cuda")
    settings = dict(temperature=col(0.8), top_k=col(50, torch.int32), top_p=col(0.95))
    seconds = []
    for _ in range(2):   # (the first run also loads the kernels)
        torch.cuda.synchronize()
        t = time.perf_counter()
        tokens = generate(dec, prefix, prompts, a.new, u, **settings)
        torch.cuda.synchronize()
        seconds.append(time.perf_counter() - t)
    out = {"requests": a.batch, "prefix": a.prefix, "prompt_tokens": sum(map(len, prompts)), "new_tokens": tokens.numel(),
           "seconds": round(seconds[1], 4), "tokens_per_second": round(tokens.numel() / seconds[1], 1),
           "first_request": tokens[:, 0].tolist()[:16]}
    print(json.dumps(out))
    return out


if __name__ == "__main__":
    main()
