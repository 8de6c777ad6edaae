"""Operators around the quantized linears of a decoder layer, as a serving program calls them.

  append  new keys and values of a batch into a paged cache, the position rotation applied on the way, and
          the rotated queries in bf16
  attend  attention of the batch's new tokens over that cache: a prefix that all sequences share (computed
          once for all of them), then each sequence's own pages, causal over its newest tokens
  sample  one token per row of logits, with temperature, top-k, top-p and min-p, from given random numbers

A case is a dict of plain values. `q_heads`, `kv_heads`, `dim` are the attention's heads, `page` the tokens
per page; `seqs` sequences of which sequence i brings new[i] tokens and then has own[i] tokens of its own in
the cache, behind `prefix` shared ones. new and own are drawn from `mix`, `new_lo`..`new_hi` and
`own_lo`..`own_hi` (`lengths`); `pad` of the sequences are empty slots of a serving batch (one token, nothing
in the cache).

Ranges: 1 to 128 sequences of 0 to 131072 tokens, 1 to 4096 new tokens a sequence, prefixes of 0 to 16384,
heads of LLaMA and OPT layers and odd groups (1 to 8 query heads a key head, dimension 64 and 128), pages of
16 to 128 tokens; 1 to 128 rows of 1000 to 131072 logits in fp32 and bf16.
"""
from __future__ import annotations

import math
import random

import torch

own = False

FLOOR_GBS, FLOOR_TFLOPS = 6694.5, 1901.8     # rates that bound a drawn case by the largest listed one


def _attn(name, op, heads, page, seqs, new, own_len, prefix, mix, pad=0, **more):
    c = {"op": op, "q_heads": heads[0], "kv_heads": heads[1], "dim": heads[2], "page": page, "seqs": seqs,
         "new_lo": new[0], "new_hi": new[1], "own_lo": own_len[0], "own_hi": own_len[1], "prefix": prefix,
         "pad": pad, "mix": mix, **more}
    return {"name": name, **c} if name else c


def _sample(name, rows, vocab, bf16, mix):
    c = {"op": "sample", "rows": rows, "vocab": vocab, "bf16": bf16, "mix": mix}
    return {"name": name, **c} if name else c


LLAMA70B, LLAMA13B, LLAMA7B, OPT125M = (64, 8, 128), (40, 40, 128), (32, 32, 128), (12, 12, 64)


def listed():
    return [
        # one sequence decoding: the q, k and v of one token, as the q/k/v plan's fp32 row
        _attn("append-70b-1", "append", LLAMA70B, 16, 1, (1, 1), (1037, 1037), 0, 1,
              rot=128, interleaved=False, bf16=False),
        # a batch decoding on a small model, bf16 rows, half of each head rotated in neighbouring pairs
        _attn("append-125m-64", "append", OPT125M, 32, 64, (1, 1), (1, 1500), 515, 2,
              rot=32, interleaved=True, bf16=True),
        # prompts of odd lengths taken in at once: about 4000 tokens
        _attn("append-70b-prompts", "append", LLAMA70B, 16, 5, (300, 1500), (300, 1500), 0, 3,
              rot=128, interleaved=False, bf16=False),
        # one sequence decoding over a short context: latency
        _attn("attend-70b-1", "attend", LLAMA70B, 16, 1, (1, 1), (1037, 1037), 0, 4),
        # a ragged batch decoding, two of its slots empty, no prefix
        _attn("attend-70b-64", "attend", LLAMA70B, 16, 64, (1, 1), (1, 4096), 0, 5, pad=2),
        # the same behind a long prefix (a system prompt and its examples): what each user adds is short
        _attn("attend-70b-prefix-64", "attend", LLAMA70B, 16, 64, (1, 1), (1, 512), 8199, 6),
        # a head for every key head, pages of 64, a prefix that ends inside a tile
        _attn("attend-7b-prefix-16", "attend", LLAMA7B, 64, 16, (1, 1), (1, 300), 2051, 7),
        # long documents, three drafted tokens checked at once
        _attn("attend-70b-long-draft", "attend", LLAMA70B, 128, 2, (3, 3), (65537, 131072), 0, 8),
        # prompts taken in behind a prefix: causal attention, bound by the tensor cores
        _attn("attend-70b-prompts", "attend", LLAMA70B, 16, 4, (400, 2500), (400, 2500), 1021, 9),
        # one row of a LLaMA vocabulary
        _sample("sample-1", 1, 32000, False, 10),
        # a batch on OPT's vocabulary in bf16 (many equal logits)
        _sample("sample-32-bf16", 32, 50272, True, 11),
        # a large batch on a large vocabulary of odd size
        _sample("sample-96", 96, 128255, False, 12),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _floor(case):
    w = work(case)
    return max(w["bytes"] / FLOOR_GBS / 1e9, w["flops"] / FLOOR_TFLOPS / 1e12)


def draw(rng):
    op = rng.choice(["append", "attend", "attend", "attend", "sample"])
    top = max(_floor(c) for c in listed() if c["op"] == op)
    while True:
        mix = rng.randrange(1 << 30)
        if op == "sample":
            c = _sample(None, _log_int(rng, 1, 128), _log_int(rng, 1000, 131072), rng.random() < 0.4, mix)
        else:
            heads = rng.choice([LLAMA70B, LLAMA70B, LLAMA13B, LLAMA7B, OPT125M, (10, 2, 64), (24, 8, 128)])
            page = rng.choice([16, 16, 32, 64, 128])
            prefix = 0 if rng.random() < 0.4 else _log_int(rng, 16, 16384)
            kind = rng.choice(["decode", "decode", "draft", "prompt"])
            if kind == "prompt":
                seqs, hi = _log_int(rng, 1, 8), _log_int(rng, 8, 4096)
                new = (max(1, hi // rng.randint(1, 8)), hi)
            else:
                seqs = _log_int(rng, 1, 128)
                new = (1, 1) if kind == "decode" else (1, rng.randint(2, 6))
            top_own = _log_int(rng, max(new[1], 16), 131072 if seqs <= 4 else 8192)
            c = _attn(None, op, heads, page, seqs, new, (max(1, top_own // rng.choice([1, 4, 64])), top_own), prefix,
                      mix, pad=rng.randint(1, 3) if seqs > 8 and rng.random() < 0.3 else 0)
            if op == "append":
                rot = rng.choice([heads[2], heads[2], heads[2] // 2, heads[2] // 4])
                c.update(rot=rot, interleaved=rng.random() < 0.4, bf16=rng.random() < 0.4)
        if _floor(c) <= top and _elements(c) <= 2 ** 31:
            return c


def lengths(case):
    """(new tokens, own tokens) of each sequence: over the logarithm of the range; the empty slots last."""
    rng = random.Random(case["mix"])
    new, held = [], []
    for i in range(case["seqs"]):
        if i >= case["seqs"] - case["pad"]:
            new.append(1)
            held.append(0)
            continue
        n = _log_int(rng, case["new_lo"], case["new_hi"])
        new.append(n)
        held.append(max(n, _log_int(rng, case["own_lo"], case["own_hi"])))
    return new, held


def _elements(case):
    """Scores that the plain form holds at once."""
    if case["op"] != "attend":
        return 0
    new, held = lengths(case)
    return case["q_heads"] * max(sum(new) * case["prefix"], max(n * m for n, m in zip(new, held)))


# ----------------------------------------------------------------- inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * seed + 17)
    return g


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _batch(case, g):
    """The batch's tokens and its pages, scattered over the cache in random order."""
    new, held = lengths(case)
    page = case["page"]
    need = [-(-m // page) for m in held]
    n_prefix = -(-case["prefix"] // page)
    n_pages = sum(need) + n_prefix + 3
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    table = torch.zeros((case["seqs"], max(1, max(need))), dtype=torch.int32, device="cuda")
    at = n_prefix
    for i, k in enumerate(need):
        table[i, :k] = order[at:at + k]
        at += k
    start = [0]
    for n in new:
        start.append(start[-1] + n)
    return {"new": new, "held": held, "start": start, "n_pages": n_pages, "pages": table,
            "prefix_pages": order[:n_prefix].clone(), "token_start": _ints(start), "lens": _ints(held)}


def _cache(case, g, n_pages):
    """Keys with some channels larger than the others, as models have them; values; leftovers in free pages."""
    shape = (n_pages, case["kv_heads"], case["page"], case["dim"])
    lift = torch.exp(0.4 * torch.randn((1, case["kv_heads"], 1, case["dim"]), generator=g, device="cuda"))
    k = (torch.randn(shape, generator=g, device="cuda") * lift).to(torch.bfloat16)
    v = torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)
    return k, v


def _rope_table(n_pos, rot):
    f = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
    a = torch.arange(n_pos, dtype=torch.float64, device="cuda")[:, None] * f[None]
    return torch.cos(a).float(), torch.sin(a).float()


def _logits(case, g):
    """A few likely tokens above a broad floor, another temperature of the model on each row; some tokens are
    forbidden, and the vocabulary's padding holds the type's lowest value."""
    m, v = case["rows"], case["vocab"]
    z = 1.6 * torch.randn((m, v), generator=g, device="cuda")
    few = torch.randint(0, v, (m, 64), generator=g, device="cuda")
    z.scatter_add_(1, few, 3.0 + 3.5 * torch.randn((m, 64), generator=g, device="cuda").abs())
    z = z * (0.8 + 0.4 * torch.rand((m, 1), generator=g, device="cuda")) + 5.0
    z = torch.where(torch.rand((m, v), generator=g, device="cuda") < 0.02, -math.inf, z)
    dtype = torch.bfloat16 if case["bf16"] else torch.float32
    z = z.to(dtype)
    z[:, v - v // 500:] = torch.finfo(dtype).min
    return z


def prepare(case, seed):
    g = _gen(seed)
    state = {"case": case}
    if case["op"] == "sample":
        m, rng = case["rows"], random.Random(case["mix"])
        state["logits"] = _logits(case, g)
        # requests of several kinds: greedy, top-k, nucleus, min-p, and mixtures of them
        kinds = [rng.choice([(0.0, 0, 1.0, 0.0), (0.7, 40, 1.0, 0.0), (1.0, 50, 0.95, 0.0), (0.8, 0, 0.9, 0.0),
                             (1.0, 0, 1.0, 0.05), (0.9, 200, 0.92, 0.02), (0.6, 0, 0.95, 0.0)]) for _ in range(m)]
        state["temperature"] = torch.tensor([k[0] for k in kinds], device="cuda")
        state["top_k"] = _ints([k[1] for k in kinds])
        state["top_p"] = torch.tensor([k[2] for k in kinds], device="cuda")
        state["min_p"] = torch.tensor([k[3] for k in kinds], device="cuda")
        state["u"] = torch.rand(m, generator=g, device="cuda")
        return state
    b = _batch(case, g)
    k, v = _cache(case, g, b["n_pages"])
    state.update(batch=b, k=k, v=v)
    tokens = b["start"][-1]
    if case["op"] == "append":
        dtype = torch.bfloat16 if case["bf16"] else torch.float32
        width = (case["q_heads"] + 2 * case["kv_heads"]) * case["dim"]
        state["qkv"] = torch.randn((tokens, width), generator=g, device="cuda").to(dtype)
        state["cos"], state["sin"] = _rope_table(case["prefix"] + max(b["held"]) + 1, case["rot"])
    else:
        state["q"] = (1.2 * torch.randn((tokens, case["q_heads"], case["dim"]), generator=g,
                                        device="cuda")).to(torch.bfloat16)
        state["scale"] = case["dim"] ** -0.5
    if own:
        import paper_2510_03275_gb300 as P
        desc = P.CacheDesc(case["kv_heads"], case["dim"], case["page"], b["n_pages"])
        state["cache"] = P.KVCache(desc, k, v)
        state["own_batch"] = P.Batch(b["token_start"], b["lens"], b["pages"], tokens, max(b["new"]), max(b["held"]),
                                     b["prefix_pages"], case["prefix"])
        if case["op"] == "append":
            state["rope"] = P.Rope(state["cos"], state["sin"], interleaved=case["interleaved"])
        else:
            state["ws"] = state["cache"].alloc_workspace(state["own_batch"], case["q_heads"])
    return state


# -------------------------------------------------------------- one pass
def run(state):
    op = state["case"]["op"]
    if not own:
        return {"append": _plain_append, "attend": _plain_attend, "sample": _plain_sample}[op](state)
    if op == "sample":
        import paper_2510_03275_gb300 as P
        return P.sample(state["logits"], state["u"], state["temperature"], state["top_k"], state["top_p"],
                        state["min_p"])
    case, cache = state["case"], state["cache"]
    if op == "attend":
        return cache.attend(state["own_batch"], state["q"], state["scale"], ws=state["ws"])
    nq, nk = case["q_heads"] * case["dim"], case["kv_heads"] * case["dim"]
    qkv = state["qkv"]
    q = cache.append(state["own_batch"], qkv[:, :nq], qkv[:, nq:nq + nk], qkv[:, nq + nk:], state["rope"])
    return [q, state["k"], state["v"]]


# ------------------------------------------------------------ plain forms
def _plain_rotate(x, cos, sin, rot, interleaved):
    """x (tokens, heads, dim) in fp32; cos, sin (tokens, rot / 2)."""
    c, s = cos[:, None], sin[:, None]
    if interleaved:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack([a * c - b * s, b * c + a * s], dim=-1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat([a * c - b * s, b * c + a * s], dim=-1)
    return torch.cat([turned, x[..., rot:]], dim=-1)


def _plain_append(state):
    case, b = state["case"], state["batch"]
    hq, hk, d, page = case["q_heads"], case["kv_heads"], case["dim"], case["page"]
    start, lens = b["token_start"].long(), b["lens"].long()
    new = start[1:] - start[:-1]
    tokens = state["qkv"].shape[0]
    seq = torch.repeat_interleave(torch.arange(case["seqs"], device="cuda"), new, output_size=tokens)
    at = lens[seq] - new[seq] + torch.arange(tokens, device="cuda") - start[seq]      # place among the own tokens
    pos = (at + case["prefix"]).clamp_min(0)
    x = state["qkv"].float().reshape(tokens, hq + 2 * hk, d)
    cos, sin = state["cos"][pos], state["sin"][pos]
    turned = _plain_rotate(x[:, :hq + hk], cos, sin, case["rot"], case["interleaved"])
    live = (at >= 0).nonzero()[:, 0]                                                    # an empty slot keeps nothing
    page_of = b["pages"][seq[live], at[live] // page].long()
    state["k"][page_of, :, at[live] % page] = turned[live, hq:].to(torch.bfloat16)
    state["v"][page_of, :, at[live] % page] = x[live, hq + hk:].to(torch.bfloat16)
    return [turned[:, :hq].to(torch.bfloat16), state["k"], state["v"]]


def _gather(pages, table, count):
    """The first `count` tokens of the pages in `table`: (kv_heads, count, dim)."""
    heads, page, dim = pages.shape[1:]
    got = pages[table[:-(-count // page)].long()]
    return got.transpose(0, 1).reshape(heads, -1, dim)[:, :count]


def _plain_attend(state):
    case, b = state["case"], state["batch"]
    hq, hk, d, prefix = case["q_heads"], case["kv_heads"], case["dim"], case["prefix"]
    group, tokens = hq // hk, b["start"][-1]
    # (kv_heads, tokens * group, dim): a key head's queries, token by token
    q = (state["q"].float() * state["scale"]).reshape(tokens, hk, group, d).transpose(0, 1).reshape(hk, -1, d)
    out = torch.zeros((hk, tokens * group, d), device="cuda")
    if prefix:
        kp, vp = (_gather(t, b["prefix_pages"], prefix).float() for t in (state["k"], state["v"]))
        sp = q @ kp.transpose(1, 2)
        mp = sp.amax(-1, keepdim=True)
        sp = torch.exp(sp - mp)
        lp, op = sp.sum(-1, keepdim=True), sp @ vp
        del sp
    for i, (n, held) in enumerate(zip(b["new"], b["held"])):
        rows = slice(b["start"][i] * group, b["start"][i + 1] * group)
        if held:
            ko, vo = (_gather(t, b["pages"][i], held).float() for t in (state["k"], state["v"]))
            s = q[:, rows] @ ko.transpose(1, 2)
            if n > 1:
                last = held - n + torch.arange(n, device="cuda").repeat_interleave(group)
                s.masked_fill_(torch.arange(held, device="cuda")[None] > last[:, None], -math.inf)
            m = s.amax(-1, keepdim=True)
            s = torch.exp(s - m)
            total, o = s.sum(-1, keepdim=True), s @ vo
            if prefix:
                top = torch.maximum(m, mp[:, rows])
                wa, wb = torch.exp(m - top), torch.exp(mp[:, rows] - top)
                total, o = total * wa + lp[:, rows] * wb, o * wa + op[:, rows] * wb
            out[:, rows] = o / total
        elif prefix:
            out[:, rows] = op[:, rows] / lp[:, rows]
    return out.reshape(hk, tokens, group, d).transpose(0, 1).reshape(tokens, hq, d).to(torch.bfloat16)


def _plain_sample(state):
    z = state["logits"].float()
    top, temp = z.amax(1, keepdim=True), state["temperature"][:, None]
    zs, order = torch.sort(z, dim=1, descending=True, stable=True)                   # equal logits by index
    rank = torch.arange(z.shape[1], device="cuda")[None]
    w = torch.where(zs == top, 1.0, torch.exp((zs - top) / torch.where(temp > 0, temp, 1.0)))
    k = state["top_k"][:, None]
    w = torch.where((k > 0) & (rank >= k), 0.0, w)
    c = torch.cumsum(w, 1)
    p = state["top_p"][:, None]
    before = torch.cat([torch.zeros_like(c[:, :1]), c[:, :-1]], 1)
    keep = ((p >= 1) | (before < p * c[:, -1:])) & (w >= state["min_p"][:, None])
    w = torch.where(keep, w, 0.0)
    by_index = torch.zeros_like(w).scatter_(1, order, w)
    c = torch.cumsum(by_index, 1)
    hit = (c > state["u"][:, None] * c[:, -1:]) & (by_index > 0)
    return torch.where(temp[:, 0] > 0, hit.int().argmax(1), order[:, 0]).to(torch.int32)


# ------------------------------------------------- what a pass cannot do without
def work(case):
    if case["op"] == "sample":
        m, n = case["rows"], case["rows"] * case["vocab"]
        # per logit a comparison for the largest, a difference, a quotient, an exponential and a sum
        return {"bytes": n * (2 if case["bf16"] else 4) + 24 * m, "flops": 5 * n}
    new, held = lengths(case)
    hq, hk, d, tokens = case["q_heads"], case["kv_heads"], case["dim"], sum(new)
    if case["op"] == "append":
        live = sum(n for n, m in zip(new, held) if m)
        rows = tokens * (hq + 2 * hk) * d * (2 if case["bf16"] else 4)
        table = 4 * case["rot"] * len({m - n + i for n, m in zip(new, held) for i in range(n)})
        return {"bytes": rows + table + 2 * d * (tokens * hq + 2 * live * hk),
                "flops": 3 * tokens * (hq + hk) * case["rot"]}
    keys = sum(n * (m - n) + n * (n + 1) // 2 if m else 0 for n, m in zip(new, held)) + tokens * case["prefix"]
    return {"bytes": 4 * tokens * hq * d + 4 * hk * d * (sum(held) + case["prefix"]), "flops": 4 * hq * d * keys}


# ------------------------------------------------------------ in 64 bits
def _exact_sample(state):
    out = []
    for i in range(state["logits"].shape[0]):
        z = state["logits"][i].double()
        temp, k, p, least, u = (float(state[n][i]) for n in ("temperature", "top_k", "top_p", "min_p", "u"))
        best = int((z == z.max()).nonzero()[0, 0])
        if temp == 0:
            out.append(best)
            continue
        w = torch.exp((z - z.max()) / temp)
        order = torch.argsort(-z, stable=True)
        if k > 0:
            order = order[:int(k)]
        mass = w[order]
        if p < 1:
            done = torch.cumsum(mass, 0) - mass
            order = order[done < p * mass.sum()]
        order = order[w[order] >= least]
        kept = torch.sort(order).values                                                # by index
        c = torch.cumsum(w[kept], 0)
        out.append(int(kept[int((c <= u * c[-1]).sum().clamp_max(len(kept) - 1))]))
    return _ints(out)


def _exact_append(state):
    case, b = state["case"], state["batch"]
    hq, hk, d, rot, page = case["q_heads"], case["kv_heads"], case["dim"], case["rot"], case["page"]
    x = state["qkv"].double().reshape(-1, hq + 2 * hk, d)
    first = torch.arange(0, rot, 2, device="cuda") if case["interleaved"] else torch.arange(rot // 2, device="cuda")
    second = first + (1 if case["interleaved"] else rot // 2)
    keys, values = state["k"].double(), state["v"].double()
    q = x[:, :hq].clone()
    for i, (n, held) in enumerate(zip(b["new"], b["held"])):
        rows = torch.arange(b["start"][i], b["start"][i + 1], device="cuda")
        own_at = torch.arange(held - n, held, device="cuda")
        at = (own_at + case["prefix"]).clamp_min(0)
        turn = torch.complex(state["cos"][at].double(), state["sin"][at].double())[:, None]
        pair = torch.complex(x[rows][:, :hq + hk][..., first], x[rows][:, :hq + hk][..., second]) * turn
        y = x[rows][:, :hq + hk].clone()
        y[..., first], y[..., second] = pair.real, pair.imag
        q[rows] = y[:, :hq]
        if held:
            page_of, slot = b["pages"][i][own_at // page].long(), own_at % page
            keys[page_of, :, slot], values[page_of, :, slot] = y[:, hq:], x[rows][:, hq + hk:]
    return [q, keys, values]


def _exact_attend(state):
    case, b = state["case"], state["batch"]
    hq, hk, d, page, prefix = case["q_heads"], case["kv_heads"], case["dim"], case["page"], case["prefix"]
    group, q = hq // hk, state["q"].double()
    out = torch.zeros_like(q)
    front = torch.arange(prefix, device="cuda")
    for i, (n, held) in enumerate(zip(b["new"], b["held"])):
        if prefix + held == 0:
            continue
        at = torch.arange(held, device="cuda")
        page_of = torch.cat([b["prefix_pages"][front // page], b["pages"][i][at // page]]).long()
        slot = torch.cat([front, at]) % page
        for h in range(hk):
            k, v = state["k"][page_of, h, slot].double(), state["v"][page_of, h, slot].double()
            for t in range(0, n, 256):           # 256 tokens of the sequence at a time
                rows = slice(b["start"][i] + t, b["start"][i] + min(n, t + 256))
                heads = slice(h * group, (h + 1) * group)
                s = torch.einsum("tgd,kd->tgk", q[rows, heads], k) * state["scale"]
                seen = prefix + held - n + t + 1 + torch.arange(s.shape[0], device="cuda")
                if held:
                    s[(torch.arange(k.shape[0], device="cuda")[None] >= seen[:, None])[:, None].expand_as(s)] = -math.inf
                out[rows, heads] = torch.softmax(s, -1) @ v
    return out


def exact(case, seed):
    global own
    was, own = own, False
    try:
        state = prepare(case, seed)
    finally:
        own = was
    return {"append": _exact_append, "attend": _exact_attend, "sample": _exact_sample}[case["op"]](state)
