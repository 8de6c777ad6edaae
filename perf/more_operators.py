"""Operators of one decoding step around the quantized linears, as a serving program calls them.

  pages   block tables for a step: pages of finished sequences go back to the pool, the new tokens' are taken from
          it; each token's slot in the cache and its position
  append  new keys and values into a paged cache, every head of q and k normalised (root mean square, a weight per
          element) and rotated by its position on the way, and the queries in bf16
  window  attention of the new tokens over that cache where a token sees the last `window` positions up to its own
          and the first `sinks` ones, behind a prefix that all sequences share
  adjust  logits before the choice of a token: penalties for repeated tokens, biases, a grammar's allowed tokens

A case is a dict of plain values. Of attention cases `q_heads`, `kv_heads`, `dim` are the heads, `page` the tokens per
page; `seqs` sequences of which sequence i brings new[i] tokens and then has own[i] tokens of its own in the cache,
behind `prefix` shared ones. new and own are drawn from `mix`, `new_lo`..`new_hi` and `own_lo`..`own_hi` (`lengths`);
`pad` of the sequences are empty slots of a serving batch (one token, nothing in the cache).

Ranges: 1 to 4096 sequences of 0 to 131072 tokens (1 to 128 where there is attention), 1 to 8192 new tokens a sequence,
prefixes of 0 to 4096, windows of 16 to 32768 with 0 to 128 first tokens, heads of LLaMA and OPT layers and odd groups
(1 to 8 query heads a key head, dimension 64 and 128), pages of 16 to 128 tokens; 1 to 128 rows of 1000 to 131072 logits
in fp32 and bf16 after 0 to 32768 tokens, with 0 to 1024 biases.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

FLOOR_GBS, FLOOR_TFLOPS = 6790.0, 1859.2     # rates that bound a drawn case by the largest listed one


def _attn(name, op, heads, page, seqs, new, own_len, prefix, mix, pad=0, **more):
    c = {"op": op, "q_heads": heads[0], "kv_heads": heads[1], "dim": heads[2], "page": page, "seqs": seqs,
         "new_lo": new[0], "new_hi": new[1], "own_lo": own_len[0], "own_hi": own_len[1], "prefix": prefix,
         "pad": pad, "mix": mix, **more}
    return {"name": name, **c} if name else c


def _adjust(name, rows, vocab, bf16, history, biases, allowed, mix):
    c = {"op": "adjust", "rows": rows, "vocab": vocab, "bf16": bf16, "history_lo": history[0],
         "history_hi": history[1], "biases": biases, "allowed": allowed, "mix": mix}
    return {"name": name, **c} if name else c


def _pages(name, page, seqs, new, own_len, done, prefix, mix):
    c = {"op": "pages", "page": page, "seqs": seqs, "new_lo": new[0], "new_hi": new[1], "own_lo": own_len[0],
         "own_hi": own_len[1], "done": done, "prefix": prefix, "pad": 0, "mix": mix}
    return {"name": name, **c} if name else c


LLAMA70B, LLAMA13B, LLAMA7B, OPT125M = (64, 8, 128), (40, 40, 128), (32, 32, 128), (12, 12, 64)


def listed():
    return [
        # a batch decoding: a token for each of its sequences, a page for some, a few that have just ended
        _pages("pages-decode-256", 16, 256, (1, 1), (1, 4096), 12, 0, 21),
        # many prompts of odd lengths taken in at once
        _pages("pages-prompts-450", 16, 450, (1, 1000), (1, 1000), 30, 515, 22),
        # one sequence decoding: the q, k and v of one token, as the q/k/v plan's fp32 row
        _attn("append-norm-70b-1", "append", LLAMA70B, 16, 1, (1, 1), (1037, 1037), 0, 23,
              rot=128, interleaved=False, bf16=False, each=False),
        # a batch decoding on a small model, bf16 rows, half of each head rotated in neighbouring pairs, a weight for every head
        _attn("append-norm-125m-64", "append", OPT125M, 32, 64, (1, 1), (1, 1500), 515, 24,
              rot=32, interleaved=True, bf16=True, each=True),
        # prompts of odd lengths taken in at once
        _attn("append-norm-70b-prompts", "append", LLAMA70B, 16, 5, (300, 1500), (300, 1500), 0, 25,
              rot=128, interleaved=False, bf16=False, each=False),
        # a ragged batch decoding, some contexts shorter than the window and some far longer, two slots empty
        _attn("window-70b-64", "window", LLAMA70B, 16, 64, (1, 1), (1, 16384), 0, 26, pad=2, window=1024, sinks=4),
        # a head for every key head, windows that reach into a shared prefix, pages of 64: few keys, latency
        _attn("window-7b-prefix-16", "window", LLAMA7B, 64, 16, (1, 1), (1, 900), 2051, 27, window=515, sinks=4),
        # long documents, three drafted tokens checked at once, a wide window
        _attn("window-70b-long-draft", "window", LLAMA70B, 128, 2, (3, 3), (65537, 131072), 0, 28, window=32768, sinks=64),
        # prompts taken in behind a prefix, bound by the tensor cores
        _attn("window-70b-prompts", "window", LLAMA70B, 16, 4, (1500, 6000), (1500, 6000), 515, 29, window=1024, sinks=4),
        # one row of a LLaMA vocabulary after a short chat, penalties alone
        _adjust("adjust-1", 1, 32000, False, (700, 700), 0, "none", 30),
        # a batch on OPT's vocabulary in bf16, a grammar's allowed tokens for each row
        _adjust("adjust-32-bf16", 32, 50272, True, (10, 4000), 17, "all", 31),
        # a large batch on a large vocabulary of odd size, long contexts, many biases, a grammar for some rows
        _adjust("adjust-96", 96, 128255, False, (100, 32768), 300, "some", 32),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _floor(case):
    w = work(case)
    return max(w["bytes"] / FLOOR_GBS / 1e9, w["flops"] / FLOOR_TFLOPS / 1e12)


def draw(rng):
    op = rng.choice(["pages", "append", "window", "window", "window", "adjust", "adjust"])
    top = max(_floor(c) for c in listed() if c["op"] == op)
    while True:
        mix = rng.randrange(1 << 30)
        if op == "adjust":
            hi = _log_int(rng, 1, 32768)
            c = _adjust(None, _log_int(rng, 1, 128), _log_int(rng, 1000, 131072), rng.random() < 0.4,
                        (rng.choice([0, max(1, hi // 50), hi]), hi), rng.choice([0, _log_int(rng, 1, 1024)]),
                        rng.choice(["none", "all", "some"]), mix)
        elif op == "pages":
            seqs, page = _log_int(rng, 1, 4096), rng.choice([16, 16, 32, 64, 128])
            hi = 1 if rng.random() < 0.5 else _log_int(rng, 2, 8192)
            c = _pages(None, page, seqs, (1, hi), (1, _log_int(rng, max(hi, 16), 32768)),
                       rng.choice([0, rng.randint(0, seqs), seqs // 10]), rng.choice([0, _log_int(rng, 1, 4096)]), mix)
        else:
            heads = rng.choice([LLAMA70B, LLAMA70B, LLAMA13B, LLAMA7B, OPT125M, (10, 2, 64), (48, 8, 128)])
            page = rng.choice([16, 16, 32, 64, 128])
            prefix = 0 if rng.random() < 0.5 else _log_int(rng, 1, 4096)
            kind = rng.choice(["decode", "decode", "draft", "prompt"])
            if kind == "prompt":
                seqs, hi = _log_int(rng, 1, 8), _log_int(rng, 8, 8192)
                new = (max(1, hi // rng.randint(1, 8)), hi)
            else:
                seqs = _log_int(rng, 1, 128)
                new = (1, 1) if kind == "decode" else (1, rng.randint(2, 6))
            top_own = _log_int(rng, max(new[1], 16), 131072 if seqs <= 4 else 16384)
            c = _attn(None, op, heads, page, seqs, new, (max(1, top_own // rng.choice([1, 4, 64])), top_own), prefix,
                      mix, pad=rng.randint(1, 3) if seqs > 8 and rng.random() < 0.3 else 0)
            if op == "append":
                rot = rng.choice([heads[2], heads[2], heads[2] // 2, heads[2] // 4])
                c.update(rot=rot, interleaved=rng.random() < 0.4, bf16=rng.random() < 0.4, each=rng.random() < 0.4)
            else:
                c.update(window=_log_int(rng, 16, 32768), sinks=0 if rng.random() < 0.2 else _log_int(rng, 1, 128))
        if _floor(c) <= top and _tokens(c) <= 2 ** 17:
            return c


def lengths(case):
    """(new tokens, own tokens with them) of each sequence: over the logarithm of the range; the empty slots last."""
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


def _tokens(case):
    return 0 if case["op"] == "adjust" else sum(lengths(case)[0])


def _done(case):
    """The sequences that have ended, in no order."""
    return random.Random(case["mix"] + 1).sample(range(case["seqs"]), case["done"])


def _histories(case):
    """(tokens so far, of them the prompt's) of each row."""
    rng = random.Random(case["mix"])
    lo, hi = case["history_lo"], case["history_hi"]
    lens = [_log_int(rng, lo, hi) if lo else rng.choice([0, _log_int(rng, 1, hi)]) for _ in range(case["rows"])]
    return lens, [int(n * rng.choice([0.0, rng.random(), rng.random(), 1.0])) for n in lens]


def _grammars(case):
    """The allowed set of each row, -1 where it has none: a few sets, that rows share."""
    rng = random.Random(case["mix"] + 2)
    sets = max(1, case["rows"] // 2)
    return [rng.randrange(sets) if case["allowed"] == "all" or rng.random() < 0.5 else -1 for _ in range(case["rows"])], sets


# ----------------------------------------------------------------- inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * seed + 19)
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


def _prepare_pages(case, g, state):
    """Tables of sequences that hold what they had before the step, their pages and the free ones in random order."""
    new, held = lengths(case)
    page, done = case["page"], set(_done(case))
    new = [0 if i in done else n for i, n in enumerate(new)]
    before = [m if i in done else m - n for i, (n, m) in enumerate(zip(new, held))]
    have, end = [-(-m // page) for m in before], [-(-m // page) for m in held]
    n_pages = sum(end) + 5
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    table = torch.full((case["seqs"], max(end)), -1, dtype=torch.int32, device="cuda")
    used = torch.arange(max(end), device="cuda")[None] < torch.tensor(have, device="cuda")[:, None]
    table[used] = order[:sum(have)]
    free = torch.full((n_pages,), -1, dtype=torch.int32, device="cuda")
    free[:n_pages - sum(have)] = order[sum(have):]
    state.update(tokens=sum(new), own_len=_ints(before), new_len=_ints(new), pages=table, free=free,
                 n_free=_ints([n_pages - sum(have)]), done=_ints([int(i in done) for i in range(case["seqs"])]))
    if own:
        import paper_2510_03275_gb300 as P
        state["pool"] = P.PagePool(page, free, state["n_free"])


def _prepare_adjust(case, g, state):
    """Logits as a head writes them; histories in which common tokens come again and again; biases of requests, some
    of them bans, with a token named twice now and then; allowed sets from nearly nothing to nearly everything."""
    m, v = case["rows"], case["vocab"]
    z = 2.0 + 2.5 * torch.randn((m, v), generator=g, device="cuda")
    state["logits"] = z.to(torch.bfloat16) if case["bf16"] else z
    lens, prompts = _histories(case)
    width = max(1, max(lens))
    common = torch.rand((m, width), generator=g, device="cuda")
    ids = (common ** 3 * v).to(torch.int32).clamp_max(v - 1)
    state["history"] = torch.where(torch.arange(width, device="cuda")[None] < _ints(lens)[:, None], ids, -1)
    state["history_len"], state["prompt_len"] = _ints(lens), _ints(prompts)
    rng = random.Random(case["mix"] + 3)
    column = lambda values: torch.tensor([rng.choice(values) for _ in range(m)], device="cuda")
    state["repetition"] = column([1.0, 1.05, 1.1, 1.3, 0.9])
    state["frequency"] = column([0.0, 0.1, 0.5, -0.2])
    state["presence"] = column([0.0, 0.3, 1.0, -0.4])
    if case["biases"]:
        n = case["biases"]
        state["bias_ids"] = torch.randint(0, v, (m, n), generator=g, device="cuda", dtype=torch.int32)
        state["bias_ids"][:, n // 2] = state["bias_ids"][:, 0]
        state["bias_ids"][:, n - n // 8:] = -1                      # shorter lists end in places that are not used
        state["bias"] = 4.0 * torch.randn((m, n), generator=g, device="cuda")
        state["bias"][torch.rand((m, n), generator=g, device="cuda") < 0.1] = -math.inf
    if case["allowed"] != "none":
        rows, sets = _grammars(case)
        share = torch.rand((sets, 1), generator=g, device="cuda") ** 2
        words = -(-v // 32)
        bits = torch.rand((sets, 32 * words), generator=g, device="cuda") < share
        weight = torch.tensor([1 << i for i in range(31)] + [-(1 << 31)], dtype=torch.int64, device="cuda")
        state["allowed"] = (bits.reshape(sets, words, 32) * weight).sum(-1).to(torch.int32)
        state["allowed_row"] = _ints(rows)


def prepare(case, seed):
    g = _gen(seed)
    state = {"case": case}
    if case["op"] == "pages":
        _prepare_pages(case, g, state)
        return state
    if case["op"] == "adjust":
        _prepare_adjust(case, g, state)
        return state
    b = _batch(case, g)
    k, v = _cache(case, g, b["n_pages"])
    state.update(batch=b, k=k, v=v)
    tokens, hq, hk, d = b["start"][-1], case["q_heads"], case["kv_heads"], case["dim"]
    if case["op"] == "append":
        dtype = torch.bfloat16 if case["bf16"] else torch.float32
        # rows of another size each, as the linears write them
        size = torch.exp(0.5 * torch.randn((tokens, 1), generator=g, device="cuda"))
        state["qkv"] = (size * torch.randn((tokens, (hq + 2 * hk) * d), generator=g, device="cuda")).to(dtype)
        state["cos"], state["sin"] = _rope_table(case["prefix"] + max(b["held"]) + 1, case["rot"])
        for name, heads in (("q_weight", hq), ("k_weight", hk)):
            shape = (heads, d) if case["each"] else (d,)
            state[name] = 1.0 + 0.3 * torch.randn(shape, generator=g, device="cuda")
        state["eps"] = 1e-6
    else:
        state["q"] = (1.2 * torch.randn((tokens, hq, d), generator=g, device="cuda")).to(torch.bfloat16)
        state["scale"] = d ** -0.5
    if own:
        import paper_2510_03275_gb300 as P
        state["cache"] = P.KVCache(P.CacheDesc(hk, d, case["page"], b["n_pages"]), k, v)
        state["own_batch"] = P.Batch(b["token_start"], b["lens"], b["pages"], tokens, max(b["new"]), max(b["held"]),
                                     b["prefix_pages"], case["prefix"])
        if case["op"] == "append":
            state["rope"] = P.Rope(state["cos"], state["sin"], interleaved=case["interleaved"])
            state["norm"] = P.HeadNorm(state["q_weight"], state["k_weight"], state["eps"])
        else:
            state["ws"] = state["cache"].alloc_workspace(state["own_batch"], hq, window=case["window"], sinks=case["sinks"])
    return state


# -------------------------------------------------------------- one pass
def run(state):
    case = state["case"]
    if not own:
        return {"pages": _plain_pages, "append": _plain_append, "window": _plain_window, "adjust": _plain_adjust}[case["op"]](state)
    if case["op"] == "pages":
        s = state["pool"].step(state["own_len"], state["new_len"], state["pages"], state["tokens"], done=state["done"],
                               prefix_len=case["prefix"], in_place=False)
        return [s.token_start, s.own_len, s.n_free, s.slots, s.positions, state["pages"], state["free"]]
    if case["op"] == "adjust":
        import paper_2510_03275_gb300 as P
        return P.adjust_logits(state["logits"], state["history"], state["history_len"], state["prompt_len"],
                               state["repetition"], state["frequency"], state["presence"], state.get("bias_ids"),
                               state.get("bias"), state.get("allowed"), state.get("allowed_row"))
    cache = state["cache"]
    if case["op"] == "window":
        return cache.attend(state["own_batch"], state["q"], state["scale"], ws=state["ws"], window=case["window"],
                            sinks=case["sinks"])
    nq, nk = case["q_heads"] * case["dim"], case["kv_heads"] * case["dim"]
    qkv = state["qkv"]
    q = cache.append(state["own_batch"], qkv[:, :nq], qkv[:, nq:nq + nk], qkv[:, nq + nk:], state["rope"], norm=state["norm"])
    return [q, state["k"], state["v"]]


# ------------------------------------------------------------ plain forms
def _plain_pages(state):
    case, table, free = state["case"], state["pages"], state["free"]
    page, columns = case["page"], table.shape[1]
    before, new = state["own_len"].long(), state["new_len"].long()
    column = torch.arange(columns, device="cuda")[None]
    # pages that come back, sequence by sequence, go on top of the free ones
    back = torch.where(state["done"] != 0, (before + page - 1) // page, 0)
    given = table[column < back[:, None]]
    n1 = state["n_free"].long() + given.shape[0]
    free[state["n_free"].long() + torch.arange(given.shape[0], device="cuda")] = given
    at = torch.where(state["done"] != 0, 0, before)
    held, end = (at + page - 1) // page, (at + new + page - 1) // page
    fits = end <= columns
    new = torch.where(fits, new, 0)
    need = torch.where(fits, end - held, 0)
    taken = (new.cumsum(0) <= state["tokens"]) & ((need == 0) | (need.cumsum(0) <= n1))
    new, need = torch.where(taken, new, 0), torch.where(taken, need, 0)
    start = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), new.cumsum(0)])
    first = need.cumsum(0) - need
    fresh = (column >= held[:, None]) & (column < (held + need)[:, None])
    which = n1 - 1 - (first[:, None] + column - held[:, None])
    table.copy_(torch.where(fresh, free[which.clamp(0, free.shape[0] - 1)], table))
    t = torch.arange(state["tokens"], device="cuda")
    seq = torch.searchsorted(start, t, right=True).clamp_max(case["seqs"]) - 1
    place = at[seq] + t - start[seq]
    real = t < start[-1]
    slots = table[seq, (place // page).clamp_max(columns - 1)].long() * page + place % page
    slots, position = torch.where(real, slots, -1), torch.where(real, case["prefix"] + place, 0)
    return [start.to(torch.int32), (at + new).to(torch.int32), (n1 - need.sum()).to(torch.int32), slots.to(torch.int32),
            position.to(torch.int32), table, free]


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
    qk = x[:, :hq + hk]
    qk = qk * torch.rsqrt((qk * qk).mean(-1, keepdim=True) + state["eps"])
    weight = torch.cat([state["q_weight"].expand(hq, d), state["k_weight"].expand(hk, d)])
    turned = _plain_rotate(qk * weight, state["cos"][pos], state["sin"][pos], case["rot"], case["interleaved"])
    live = (at >= 0).nonzero()[:, 0]                                                    # an empty slot keeps nothing
    page_of = b["pages"][seq[live], at[live] // page].long()
    state["k"][page_of, :, at[live] % page] = turned[live, hq:].to(torch.bfloat16)
    state["v"][page_of, :, at[live] % page] = x[live, hq + hk:].to(torch.bfloat16)
    return [turned[:, :hq].to(torch.bfloat16), state["k"], state["v"]]


def _plain_window(state):
    """512 tokens of a sequence at a time, over the keys that one of them sees."""
    case, b = state["case"], state["batch"]
    hq, hk, d, page = case["q_heads"], case["kv_heads"], case["dim"], case["page"]
    prefix, window, sinks = case["prefix"], case["window"], case["sinks"]
    group, tokens = hq // hk, b["start"][-1]
    # (kv_heads, tokens * group, dim): a key head's queries, token by token
    q = (state["q"].float() * state["scale"]).reshape(tokens, hk, group, d).transpose(0, 1).reshape(hk, -1, d)
    out = torch.zeros((hk, tokens * group, d), device="cuda")
    front = torch.arange(-(-prefix // page) * page, device="cuda")[:prefix]
    for i, (n, held) in enumerate(zip(b["new"], b["held"])):
        at = torch.arange(held, device="cuda")
        page_of = torch.cat([b["prefix_pages"][front // page], b["pages"][i][at // page]]).long()
        slot = torch.cat([front, at]) % page
        for t in range(0, n, 512):
            m = min(512, n - t)
            first = prefix + max(-1, held - n + t)                     # position of the first of them
            end, low = min(prefix + held, first + m), max(0, first - window + 1)
            if end == 0:
                continue
            few = min(sinks, low, end)
            seen = torch.cat([torch.arange(few, device="cuda"), torch.arange(low, end, device="cuda")])
            k, v = (x[page_of[seen], :, slot[seen]].transpose(0, 1).float() for x in (state["k"], state["v"]))
            rows = slice((b["start"][i] + t) * group, (b["start"][i] + t + m) * group)
            s = q[:, rows] @ k.transpose(1, 2)
            pos = (first + torch.arange(m, device="cuda")).clamp_max(end - 1).repeat_interleave(group)[:, None]
            hidden = (seen[None] > pos) | ((seen[None] <= pos - window) & (seen[None] >= sinks))
            s.masked_fill_(hidden, -math.inf)
            s = torch.exp(s - s.amax(-1, keepdim=True))
            out[:, rows] = (s @ v) / s.sum(-1, keepdim=True)
    return out.reshape(hk, tokens, group, d).transpose(0, 1).reshape(tokens, hq, d).to(torch.bfloat16)


def _plain_adjust(state):
    case, z = state["case"], state["logits"].float()
    m, v = z.shape
    history, place = state["history"], torch.arange(state["history"].shape[1], device="cuda")[None]
    real = place < state["history_len"][:, None]
    answered = real & (place >= state["prompt_len"][:, None])
    ids = history.clamp(0, v - 1).long()
    count = torch.zeros((m, v), dtype=torch.int32, device="cuda").scatter_add_(1, ids, answered.int())
    seen = torch.zeros((m, v), dtype=torch.int32, device="cuda").scatter_add_(1, ids, real.int()) > 0
    r = state["repetition"][:, None]
    z = torch.where(seen, torch.where(z > 0, z / r, z * r), z)
    z = z - (state["frequency"][:, None] * count + state["presence"][:, None] * (count > 0))
    if "bias" in state:
        named = state["bias_ids"] >= 0
        z = z + torch.zeros_like(z).scatter_add_(1, state["bias_ids"].clamp_min(0).long(), torch.where(named, state["bias"], 0.0))
    if "allowed" in state:
        words = state["allowed"][state["allowed_row"].clamp_min(0).long()]
        bits = (words[:, :, None] >> torch.arange(32, device="cuda", dtype=torch.int32)) & 1
        forbidden = (bits.reshape(m, -1)[:, :v] == 0) & (state["allowed_row"][:, None] >= 0)
        z = torch.where(forbidden, -math.inf, z)
    return z.to(state["logits"].dtype)


# ------------------------------------------------- what a pass cannot do without
def work(case):
    if case["op"] == "adjust":
        n = case["rows"] * case["vocab"]
        masks = len({r for r in _grammars(case)[0] if r >= 0}) if case["allowed"] != "none" else 0
        used = case["biases"] - case["biases"] // 8
        return {"bytes": n * (4 if case["bf16"] else 8) + 4 * sum(_histories(case)[0]) + 8 * case["rows"] * used
                + 4 * masks * -(-case["vocab"] // 32), "flops": n}
    new, held = lengths(case)
    tokens = sum(new)
    if case["op"] == "pages":
        done, page = set(_done(case)), case["page"]
        tokens = sum(n for i, n in enumerate(new) if i not in done)
        moved = sum(-(-m // page) if i in done else -(-m // page) + (n - m) // page for i, (n, m) in enumerate(zip(new, held)))
        return {"bytes": 20 * case["seqs"] + 8 * moved + 8 * tokens, "flops": 4 * (case["seqs"] + tokens)}
    hq, hk, d, prefix = case["q_heads"], case["kv_heads"], case["dim"], case["prefix"]
    if case["op"] == "append":
        live = sum(n for n, m in zip(new, held) if m)
        rows = tokens * (hq + 2 * hk) * d * (2 if case["bf16"] else 4)
        table = 4 * case["rot"] * len({m - n + i for n, m in zip(new, held) for i in range(n)})
        return {"bytes": rows + table + 2 * d * (tokens * hq + 2 * live * hk),
                "flops": tokens * (hq + hk) * (3 * case["rot"] + 4 * d)}
    window, sinks = case["window"], case["sinks"]
    read, pairs, low_prefix = 0, 0, prefix
    for n, m in zip(new, held):
        p0 = prefix + max(-1, m - n)                                    # its first and last token's positions
        p1 = prefix + m - 1
        low = max(0, p0 - window + 1)
        low_prefix = min(low_prefix, low)
        read += m - min(m, max(0, low - prefix)) + min(max(0, sinks - prefix), max(0, low - prefix))
        # position p sees min(p + 1, window) keys in the window, and the first ones before it
        pairs += _sum_min(p0 + 1, p1 + 1, window) + _sum_min(max(0, p0 + 1 - window), max(0, p1 + 1 - window), sinks)
    read += prefix - low_prefix + min(sinks, low_prefix)
    return {"bytes": 4 * tokens * hq * d + 4 * hk * d * read, "flops": 4 * hq * d * pairs}


def _sum_min(a, b, cap):
    """The sum of min(x, cap) over x = a .. b."""
    low = max(0, min(b, cap) - a + 1)
    return low * (2 * a + low - 1) // 2 + cap * (b - a + 1 - low)


# ------------------------------------------------------------ in 64 bits
def _exact_pages(state):
    case, page = state["case"], state["case"]["page"]
    before, new, done = state["own_len"].tolist(), state["new_len"].tolist(), state["done"].tolist()
    table, free = state["pages"].tolist(), state["free"].tolist()
    stack = free[:int(state["n_free"])]
    for i, d in enumerate(done):
        if d:
            stack += table[i][:-(-before[i] // page)]
            before[i] = 0
    free[:len(stack)] = stack
    available, asked, room = len(stack), 0, state["tokens"]
    start, lens, slots, positions = [0], [], [], []
    for i, n in enumerate(new):
        held, end = -(-before[i] // page), -(-(before[i] + n) // page)
        if end > len(table[i]):
            n = 0
        else:
            asked, room = asked + end - held, room - n
            if room < 0 or (end > held and asked > available):
                n = 0
        for place in range(before[i], before[i] + n):
            if place % page == 0:
                table[i][place // page] = stack.pop()
            slots.append(table[i][place // page] * page + place % page)
            positions.append(case["prefix"] + place)
        start.append(start[-1] + n)
        lens.append(before[i] + n)
    rest = state["tokens"] - len(slots)
    return [_ints(x) for x in (start, lens, [len(stack)], slots + [-1] * rest, positions + [0] * rest, table, free)]


def _exact_append(state):
    case, b = state["case"], state["batch"]
    hq, hk, d, rot, page = case["q_heads"], case["kv_heads"], case["dim"], case["rot"], case["page"]
    x = state["qkv"].double().reshape(-1, hq + 2 * hk, d)
    for heads, name in ((slice(0, hq), "q_weight"), (slice(hq, hq + hk), "k_weight")):
        rms = torch.sqrt(x[:, heads].pow(2).sum(-1, keepdim=True) / d + state["eps"])
        x[:, heads] = x[:, heads] / rms * state[name].double()
    first = torch.arange(0, rot, 2, device="cuda") if case["interleaved"] else torch.arange(rot // 2, device="cuda")
    second = first + (1 if case["interleaved"] else rot // 2)
    keys, values = state["k"].double(), state["v"].double()
    q = x[:, :hq].clone()
    for i, (n, held) in enumerate(zip(b["new"], b["held"])):
        rows = torch.arange(b["start"][i], b["start"][i + 1], device="cuda")
        own_at = torch.arange(held - n, held, device="cuda")
        at = (own_at + case["prefix"]).clamp_min(0)
        turn = torch.complex(state["cos"][at].double(), state["sin"][at].double())[:, None]
        y = x[rows][:, :hq + hk]
        pair = torch.complex(y[..., first], y[..., second]) * turn
        y[..., first], y[..., second] = pair.real, pair.imag
        q[rows] = y[:, :hq]
        if held:
            page_of, slot = b["pages"][i][own_at // page].long(), own_at % page
            keys[page_of, :, slot], values[page_of, :, slot] = y[:, hq:], x[rows][:, hq + hk:]
    return [q, keys, values]


def _exact_window(state):
    case, b = state["case"], state["batch"]
    hq, hk, d, page, prefix = case["q_heads"], case["kv_heads"], case["dim"], case["page"], case["prefix"]
    window, sinks = case["window"], case["sinks"]
    group, q = hq // hk, state["q"].double()
    out = torch.zeros_like(q)
    for i, (n, held) in enumerate(zip(b["new"], b["held"])):
        line = [b["prefix_pages"].repeat_interleave(page)[:prefix], b["pages"][i].repeat_interleave(page)[:held]]
        line = torch.cat(line).long()
        place = torch.cat([torch.arange(prefix, device="cuda"), torch.arange(held, device="cuda")]) % page
        for t in range(0, n, 256):           # 256 tokens of the sequence at a time
            rows = slice(b["start"][i] + t, b["start"][i] + min(n, t + 256))
            pos = [prefix + max(-1, held - n + t + j) for j in range(rows.stop - rows.start)]
            last, begin = pos[-1], max(0, pos[0] - window + 1)
            keys = torch.tensor(sorted({*range(min(sinks, last + 1)), *range(begin, last + 1)}), device="cuda")
            if not len(keys):
                continue
            p = torch.tensor(pos, device="cuda")[:, None]
            seen = (keys[None] <= p) & ((p - keys[None] < window) | (keys[None] < sinks))
            for h in range(hk):
                k, v = state["k"][line[keys], h, place[keys]].double(), state["v"][line[keys], h, place[keys]].double()
                heads = slice(h * group, (h + 1) * group)
                s = torch.einsum("tgd,kd->tgk", q[rows, heads], k) * state["scale"]
                out[rows, heads] = torch.softmax(s.masked_fill(~seen[:, None], -math.inf), -1) @ v
    return out


def _exact_adjust(state):
    """Row by row, on the host."""
    host = {k: x.cpu().double().numpy() if k == "logits" else x.cpu().numpy() for k, x in state.items() if k != "case"}
    z = host["logits"]
    for i, row in enumerate(z):
        n, n0 = host["history_len"][i], host["prompt_len"][i]
        r, f, p = (float(host[name][i]) for name in ("repetition", "frequency", "presence"))
        t = np.unique(host["history"][i, :n])
        row[t] = np.where(row[t] > 0, row[t] / r, row[t] * r)
        t, count = np.unique(host["history"][i, n0:n], return_counts=True)
        row[t] -= f * count + p
        if "bias" in host:
            named = host["bias_ids"][i] >= 0
            np.add.at(row, host["bias_ids"][i][named], host["bias"][i][named].astype(np.float64))
        if "allowed" in host and host["allowed_row"][i] >= 0:
            bits = np.unpackbits(host["allowed"][host["allowed_row"][i]].view(np.uint8), bitorder="little")
            row[bits[:len(row)] == 0] = -math.inf
    return torch.from_numpy(z).cuda()


def exact(case, seed):
    global own
    was, own = own, False
    try:
        state = prepare(case, seed)
    finally:
        own = was
    return {"pages": _exact_pages, "append": _exact_append, "window": _exact_window, "adjust": _exact_adjust}[case["op"]](state)
