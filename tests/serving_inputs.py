"""Batches, caches and tables of the attention tests, made on the host."""
import numpy as np

from paper_2510_03275_gb300 import workloads as W


def bf16(x):
    """The values of x rounded to bf16, as fp32."""
    return W.bf16_to_float(W.float_to_bf16(np.asarray(x, np.float32)))


def to_bf16(torch, x):
    return torch.from_numpy(W.float_to_bf16(np.asarray(x, np.float32)).view(np.int16)).view(torch.bfloat16).cuda()


class Case:
    """Sequences with new[s] tokens and own[s] own tokens, behind a prefix; pages in random order, all other
    places of the cache NaN (a free page holds anything)."""

    def __init__(self, heads, new, own, prefix=0, page=16, seed=0, spread=1.0):
        self.q_heads, self.kv_heads, self.dim = heads
        self.new, self.own, self.prefix, self.page = list(new), list(own), prefix, page
        rng = self.rng = np.random.default_rng(seed)
        self.start = np.concatenate([[0], np.cumsum(self.new)]).astype(np.int32)
        self.tokens = int(self.start[-1])
        need, n_prefix = [-(-m // page) for m in self.own], -(-prefix // page)
        self.n_pages = sum(need) + n_prefix + 2
        order = rng.permutation(self.n_pages).astype(np.int32)
        self.pages = np.full((len(self.own), max(1, max(need))), -7, np.int32)
        at = n_prefix
        for s, k in enumerate(need):
            self.pages[s, :k] = order[at:at + k]
            at += k
        self.prefix_pages = order[:n_prefix]
        self.k, self.v = (np.full((self.n_pages, self.kv_heads, page, self.dim), np.nan, np.float32) for _ in range(2))
        for table, count in [(self.prefix_pages, prefix)] + [(self.pages[s], m) for s, m in enumerate(self.own)]:
            for j in range(count):
                for a, sigma in ((self.k, spread), (self.v, 1.0)):
                    a[table[j // page], :, j % page] = bf16(sigma * rng.standard_normal((self.kv_heads, self.dim)))
        self.q = bf16(rng.standard_normal((self.tokens, self.q_heads, self.dim)))

    def desc(self, sdq):
        return sdq.CacheDesc(self.kv_heads, self.dim, self.page, self.n_pages)

    def cache(self, sdq, torch):
        return sdq.KVCache(self.desc(sdq), to_bf16(torch, self.k), to_bf16(torch, self.v))

    def batch(self, sdq, torch, **bounds):
        i = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()
        b = dict(n_tokens=self.tokens, max_new=max(1, max(self.new)), max_own=max(self.own))
        b.update(bounds)
        return sdq.Batch(i(self.start), i(self.own), i(self.pages), prefix_pages=i(self.prefix_pages),
                         prefix_len=self.prefix, **b)
