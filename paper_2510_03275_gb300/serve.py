"""Serving with the quantized layer: a decoder whose linears are Sigma-Delta
plans, a paged cache behind a prefix that all requests share, whose pages come
from a pool, attention over it (all of it, or a window and first tokens),
penalties and sampling.

    python -m paper_2510_03275_gb300.serve --batch 32 --prefix 2000 --new 64

builds one of random weights, answers a batch of random requests and prints a
JSON line.  Decoding steps replay one CUDA graph: its batch's lengths, block
tables, histories and last tokens live on the GPU and move on inside the graph.
"""
from __future__ import annotations

import argparse
import json
import time
from dataclasses import dataclass
from fractions import Fraction

from . import Batch, CacheDesc, HeadNorm, KVCache, LayerDesc, PagePool, Plan, Rope, adjust_logits, sample, workloads as W


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
    qk_norm: bool = False        # norms of the heads of queries and keys
    window: int = 0              # positions that a token sees (0: all), beside the first `sinks`
    sinks: int = 0

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
    if shape.qk_norm:
        for i in range(shape.layers):
            for name in ("q_norm", "k_norm"):
                w[f"{i}.{name}"] = 1 + 0.2 * torch.randn(shape.head_dim, generator=g, device=device)
    return w


def _norm(x):
    """Rows of unit mean square, in bf16 (the linears' input type)."""
    import torch
    return (x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-5)).to(torch.bfloat16)


class Decoder:
    """The plans and codes of a decoder, a cache per layer, and the pool of their pages."""

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
        self.pool = PagePool(page_tokens, n_pages=n_pages, device=self.embedding.device)
        self.rope = Rope.table(n_pos, shape.head_dim, device=self.embedding.device)
        self.norms = [HeadNorm(weights[f"{i}.q_norm"], weights[f"{i}.k_norm"], 1e-5) if shape.qk_norm else None
                      for i in range(shape.layers)]
        self.seen = dict(window=shape.window, sinks=shape.sinks) if shape.window else {}

    def linear(self, name, x):
        plan, codes, alpha = self.layers[name]
        return plan.forward(codes, alpha, x)

    def forward(self, tokens, batch: Batch, rows=None):
        """Append the batch's tokens to the caches; fp32 logits of the given rows (all of them: None)."""
        import torch
        s = self.shape
        q_width, kv_width = s.q_heads * s.head_dim, s.kv_heads * s.head_dim
        ws = self.caches[0].alloc_workspace(batch, s.q_heads, **self.seen)   # (the layers take turns on it)
        h = self.embedding[tokens.long()]
        for i, cache in enumerate(self.caches):
            q, k, v = self.linear(f"{i}.qkv", _norm(h)).split([q_width, kv_width, kv_width], dim=1)
            q = cache.append(batch, q, k, v, self.rope, norm=self.norms[i])
            a = cache.attend(batch, q, ws=ws, **self.seen)
            h = h + self.linear(f"{i}.o", a.flatten(1))
            gate, up = self.linear(f"{i}.gate_up", _norm(h)).chunk(2, dim=1)
            h = h + self.linear(f"{i}.down", (gate * torch.sigmoid(gate) * up).to(torch.bfloat16))
        return self.linear("head", _norm(h if rows is None else h[rows]))


def generate(dec: Decoder, prefix, prompts, n_new, u, temperature=None, top_k=None, top_p=None, min_p=None, graph=True,
             keep_logits=False, repetition=None, frequency=None, presence=None, **adjust):
    """Answer requests that all begin with the tokens `prefix` (a list, may be
    empty) and go on with their own `prompts` (lists of at least one token):
    n_new tokens each, from random numbers u (n_new x requests, on the GPU), as
    an int32 tensor (n_new x requests); with keep_logits also the logits that
    they were drawn from.  Settings as in `sample`; penalties for tokens that
    repeat, biases and allowed tokens (bias_ids, bias, allowed, allowed_row) as
    in `adjust_logits`.  The decoder's pool has as many free pages behind the
    call as ahead of it, also where it raises; ValueError where they are too few,
    RuntimeError where somebody else took them meanwhile."""
    import torch
    dev, page, n = dec.embedding.device, dec.page_tokens, len(prompts)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)
    lens = [len(p) for p in prompts]
    per = [-(-(m + n_new) // page) for m in lens]
    n_prefix = -(-len(prefix) // page)
    if min(lens) < 1 or n_new < 1 or n_prefix + sum(per) > min(dec.n_pages, int(dec.pool.n_free)):
        raise ValueError("generate: an empty prompt, no token to answer with, or more tokens than the cache has free pages for")
    own, front_own = ints([0] * n), ints([0])
    pages, front = (torch.full(size, -1, dtype=torch.int32, device=dev) for size in ((n, max(per)), (1, max(1, n_prefix))))
    shared = dict(prefix_pages=front[0] if prefix else None, prefix_len=len(prefix))
    ends, ones = torch.tensor(lens).cumsum(0).tolist(), ints([1] * n)
    adjust.update(repetition=repetition, frequency=frequency, presence=presence)
    if any(x is not None for x in (repetition, frequency, presence)):
        # each request's tokens so far, the answer's behind the prompt's
        width = len(prefix) + max(lens) + n_new
        adjust["history"] = ints([list(prefix) + p + [-1] * (width - len(prefix) - len(p)) for p in prompts])
        adjust["prompt_len"] = ints([len(prefix) + m for m in lens])
        adjust["history_len"] = adjust["prompt_len"].clone()

    def batch_of(new, tokens, max_new, max_own):
        at = dec.pool.step(own, new, pages, tokens, prefix_len=len(prefix))
        return Batch(at.token_start, own, pages, tokens, max_new, max_own, **shared)

    def choose(z):
        if any(x is not None for x in adjust.values()):
            adjust_logits(z, **adjust, out=z)
        tokens.copy_(sample(z, u_now, temperature, top_k, top_p, min_p))
        if "history" in adjust:
            adjust["history"].scatter_(1, adjust["history_len"].long()[:, None], tokens[:, None])
            adjust["history_len"].add_(1)
        return z

    def decode():
        return choose(dec.forward(tokens, batch_of(ones, n, 1, max(lens) + n_new)))

    try:
        if prefix:   # its keys and values, once for everybody
            at = dec.pool.step(front_own, ints([len(prefix)]), front, len(prefix))
            dec.forward(ints(prefix), Batch(at.token_start, at.own_len, front, len(prefix), len(prefix), len(prefix)),
                        rows=slice(-1, None))
        last = ints([e - 1 for e in ends]).long()
        u_now, tokens, out, logits = u[0].clone(), torch.empty(n, dtype=torch.int32, device=dev), [], []
        z = dec.forward(ints([t for p in prompts for t in p]), batch_of(ints(lens), ends[-1], max(lens), max(lens)), rows=last)
        z, replay = choose(z), None
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
        got, lengths = torch.stack(out), torch.cat([own, front_own])
        logits = torch.stack(logits) if keep_logits else None
    finally:   # the pages go back, whatever has become of the call
        dec.pool.step(own, ones - 1, pages, 1, done=ones)
        if prefix:
            dec.pool.step(front_own, ones[:1] - 1, front, 1, done=ones[:1])
    # (a step that does not get its pages leaves a request's tokens out, and shifts the rows of those behind it)
    if lengths.tolist() != [m + n_new - 1 for m in lens] + [len(prefix)]:
        raise RuntimeError("generate: the pool ran out of pages on the way (other calls take from it meanwhile)")
    return (got, logits) if keep_logits else got


def main(argv=None):
    import torch
    ap = argparse.ArgumentParser(description="answer a batch of random requests with a decoder of random weights (JSON)")
    ap.add_argument("--batch", type=int, default=32)
    ap.add_argument("--prefix", type=int, default=2000, help="tokens that all requests share")
    ap.add_argument("--prompt", type=int, default=100, help="the longest prompt")
    ap.add_argument("--new", type=int, default=64, help="tokens to generate per request")
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--qk-norm", action="store_true", help="norms of the heads of queries and keys")
    ap.add_argument("--window", type=int, default=0, help="positions that a token sees (0: all)")
    ap.add_argument("--sinks", type=int, default=0, help="first positions that stay visible beside a window")
    ap.add_argument("--repetition", type=float, default=None, help="penalty for tokens that repeat")
    a = ap.parse_args(argv)
    shape = Shape(layers=a.layers, qk_norm=a.qk_norm, window=a.window, sinks=a.sinks)
    g = torch.Generator().manual_seed(1)
    draw = lambda m: torch.randint(shape.vocab, (m,), generator=g).tolist()
    prefix = draw(a.prefix)
    prompts = [draw(int(torch.randint(1, a.prompt + 1, (1,), generator=g))) for _ in range(a.batch)]
    pages = -(-a.prefix // 16) + a.batch * -(-(a.prompt + a.new) // 16)
    dec = Decoder(shape, random_weights(shape), pages, n_pos=a.prefix + a.prompt + a.new)
    u = torch.rand((a.new, a.batch), generator=g).cuda()
    col = lambda x, dtype=torch.float32: torch.full((a.batch,), x, dtype=dtype, device="cuda")
    settings = dict(temperature=col(0.8), top_k=col(50, torch.int32), top_p=col(0.95))
    if a.repetition is not None:
        settings["repetition"] = col(a.repetition)
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
