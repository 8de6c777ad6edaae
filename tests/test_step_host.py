"""CPU: what a decoding step's calls check before anything runs on a GPU, the
oracle's definitions of them, and rules of their kernels on the source text."""
import ctypes
import re
import struct

import numpy as np
import pytest
import torch

import oracle as O
from test_kernel_protocols import _block, _source

BUFFER = ctypes.create_string_buffer(1 << 12)
AT = (ctypes.addressof(BUFFER) + 255) // 256 * 256       # an aligned address; nothing is read or written there

ADJUST = ("history", "history_len", "prompt_len", "repetition", "frequency", "presence", "bias_ids", "bias", "allowed", "allowed_row",
          "history_stride", "bias_ids_stride", "bias_stride", "allowed_stride", "history_max", "n_bias", "n_allowed")
PAGES = ("page_tokens", "n_pages", "n_seqs", "n_tokens", "page_columns", "page_stride", "prefix_len", "own_len", "new_len", "done",
         "pages", "free_pages", "n_free", "token_start", "own_out", "n_free_out", "slots", "positions")


def _adjust(sdq, call=(), **fields):
    f = dict.fromkeys(ADJUST, 0) | dict(history=AT, bias_ids=AT, bias=AT, allowed=AT, history_stride=8, bias_ids_stride=4, bias_stride=4,
                                        allowed_stride=4, history_max=8, n_bias=4, n_allowed=2) | fields
    c = dict(logits=AT, kind=0, rows=2, vocab=100, ld=100, out=AT + 1024, ldo=100) | dict(call)
    return sdq.lib().sdq_adjust_logits(c["logits"], c["kind"], c["rows"], c["vocab"], c["ld"],
                                       sdq._ADJUST.pack(*(f[n] for n in ADJUST)), c["out"], c["ldo"], None)


def test_adjust_refuses_before_it_runs(sdq):
    assert _adjust(sdq) != -1                                # (no GPU here, or one: not an argument's fault)
    for call in (dict(logits=None), dict(out=None), dict(kind=2), dict(kind=-1), dict(rows=0), dict(rows=65536), dict(vocab=0),
                 dict(vocab=393217, ld=393217, ldo=393217), dict(ld=99), dict(ldo=99), dict(logits=AT + 2), dict(out=AT + 1026),
                 dict(out=AT + 4), dict(out=AT + 796), dict(out=AT, ldo=104)):
        assert _adjust(sdq, call) == -1, call
    for call in (dict(out=AT), dict(out=AT + 800), dict(rows=1, out=AT, ldo=104)):      # in place; just behind
        assert _adjust(sdq, call, n_allowed=2) != -1, call
    for fields in (dict(history_max=-1), dict(history_stride=-1), dict(bias_stride=-4), dict(bias_ids_stride=-4), dict(allowed_stride=-4),
                   dict(n_bias=-1), dict(n_bias=4097), dict(bias=0), dict(bias_ids=0), dict(n_allowed=1),
                   dict(n_allowed=0, allowed_row=AT)):
        assert _adjust(sdq, **fields) == -1, fields
    for fields in (dict(n_allowed=1, allowed_row=AT), dict(allowed=0, n_allowed=0), dict(n_bias=0, bias=0, bias_ids=0), dict(history=0),
                   dict(history_stride=0, bias_stride=0, allowed_stride=0)):
        assert _adjust(sdq, **fields) != -1, fields
    assert sdq.lib().sdq_adjust_logits(AT, 0, 1, 10, 10, None, AT, 10, None) == -1


def test_pages_refuse_before_they_run(sdq):
    def call(**fields):
        f = dict.fromkeys(PAGES, AT) | dict(page_tokens=16, n_pages=8, n_seqs=2, n_tokens=4, page_columns=3, page_stride=3,
                                            prefix_len=0) | fields
        return sdq.lib().sdq_pages_step(sdq._PAGES.pack(*(f[n] or 0 for n in PAGES)), None)
    assert call() != -1 and call(done=None, slots=None, positions=None) != -1
    for fields in [{n: None} for n in ("own_len", "new_len", "pages", "free_pages", "n_free", "token_start", "own_out", "n_free_out")] + \
                  [dict(page_tokens=8), dict(page_tokens=48), dict(page_tokens=256), dict(n_pages=0), dict(n_pages=1 << 27),
                   dict(n_seqs=0), dict(n_seqs=65536), dict(n_tokens=0), dict(n_tokens=(1 << 20) + 1), dict(page_columns=0),
                   dict(page_stride=2), dict(page_columns=1 << 26, page_stride=1 << 26), dict(prefix_len=-1), dict(prefix_len=1 << 30)]:
        assert call(**fields) == -1, fields
    assert sdq.lib().sdq_pages_step(None, None) == -1


def test_windows_and_norms_without_handles_are_refused(sdq):
    L = sdq.lib()
    assert L.sdq_attention_window(None, None, 1, None, 0, 1.0, 4, 0, None, None, None, 0, None) == -1
    assert L.sdq_attention_window_workspace_bytes(None, None, 1, 4, 0) == 0
    assert L.sdq_cache_append_norm(None, None, 1, None, 0, None, 0, None, 0, 0, None, None, None, None) == -1


def test_the_structs_are_the_headers(sdq):
    """Sizes and places of the C structs' members, on the header's text."""
    text = re.sub(r"/\*.*?\*/", "", open(_header()).read(), flags=re.S)
    for name, packed in (("sdq_adjust", sdq._ADJUST), ("sdq_pages", sdq._PAGES)):
        body = re.search(r"typedef struct \{([^}]*)\} %s;" % name, text).group(1)
        kinds = "".join("P" * d.count(",") + "P" if "*" in d else ("q" if "int64_t" in d else "i") * (d.count(",") + 1)
                        for d in body.split(";") if d.strip())
        assert struct.calcsize("@" + kinds) <= packed.size and packed.size % 8 == 0
        flat = "".join(c * int(n or 1) for n, c in re.findall(r"(\d*)([Pqi])", packed.format))
        assert flat == kinds


def _header():
    import os
    return os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "sdq.h")


class _Elsewhere:
    """A tensor that says which GPU it is on."""

    def __init__(self, t, device=0):
        self.t, self.device = t, torch.device("cuda", device)

    is_cuda = True

    def get_device(self):
        return self.device.index

    def __getattr__(self, name):
        return getattr(self.t, name)


def test_tensors_on_other_devices_are_refused(sdq, monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(sdq, "_empty", lambda *a: pytest.fail("the call went on"))
    i, f = torch.zeros(2, dtype=torch.int32), torch.ones(2)
    z, h, p = torch.zeros((2, 10)), torch.zeros((2, 4), dtype=torch.int32), torch.zeros((2, 3), dtype=torch.int32)
    for other in (1, 0):
        with pytest.raises(ValueError):                      # one of them elsewhere; all of them, but not the current device
            sdq.adjust_logits(_Elsewhere(z, 1), _Elsewhere(h, other), repetition=_Elsewhere(f, 1))
        pool = sdq.PagePool.__new__(sdq.PagePool)
        pool.page_tokens, pool.free, pool.n_free = 16, _Elsewhere(i, other), _Elsewhere(i[:1], 1)
        with pytest.raises(ValueError):
            pool.step(_Elsewhere(i, 1), _Elsewhere(i.clone(), 1), _Elsewhere(p, 1), 4)
    norm = sdq.HeadNorm(_Elsewhere(torch.ones(64), 1))
    with pytest.raises(ValueError):
        norm.check(4, 2, 64, torch.device("cuda", 0))
    norm.check(4, 2, 64, torch.device("cuda", 1))


def test_oracle_norm_and_window_by_hand():
    assert np.allclose(O.serving.head_norm([[[3.0, 4.0]]], [1, 2], 0.0), np.array([3, 8]) / np.sqrt(12.5))
    keys = lambda i, w, s: O.serving.visible_keys(0, i, [0, 2], [5], [[7]], [9], 3, 16, w, s)
    # positions 0 .. 2 are the prefix's, the two new tokens stand at 6 and 7
    assert keys(0, 2, 0) == [(7, 2), (7, 3)] and keys(1, 2, 0) == [(7, 3), (7, 4)]
    assert keys(0, 5, 1) == [(9, 0), (9, 2), (7, 0), (7, 1), (7, 2), (7, 3)]
    assert keys(0, 1, 4) == [(9, 0), (9, 1), (9, 2), (7, 0), (7, 3)] and len(keys(1, 8, 0)) == 8
    assert O.serving.visible_keys(0, 0, [0, 1], [0], [[7]], [9], 3, 16, 2, 0) == [(9, 1), (9, 2)]   # an empty slot


def test_oracle_adjust_by_hand():
    z = O.serving.adjust_row([2.0, -2.0, 1.0, 4.0], [0, 1, 1, 3, 9, -1, 3], 2, 2.0, 0.5, 0.25, [(2, 1.0), (2, 0.5), (7, 9.0)], {0, 1, 2})
    # 0 and 1 stand in the prompt, 1 once and 3 twice in the answer
    assert z.tolist() == [1.0, -4.75, 2.5, -np.inf]


def test_oracle_pages_by_hand():
    start, own, free, slots, pos, tables = O.serving.pages_step(16, 6, [5, 4, 3], [16, 0, 20], [1, 17, 2], [0, 0, 1],
                                                                [[0, -1], [-1, -1], [1, 2]], 20, 100)
    # 1 and 2 come back on top; the first sequence takes 2, the second 1 and 3, the third 4
    assert tables == [[0, 2], [1, 3], [4, 2]] and free == [5] and own == [17, 17, 2] and start == [0, 1, 18, 20]
    assert slots == [32] + list(range(16, 32)) + [48, 64, 65] and pos == [116] + list(range(100, 117)) + [100, 101]


def _kernel(name, kernel):
    text = _source(name)
    m = re.search(r"__global__[^;{]*?\b%s\(" % kernel, text, re.S)
    a, b = _block(text, text.index("{", text.index(")", m.end())))
    return text[a:b]


def test_every_kernel_orders_itself_behind_the_grid_before():
    for name, kernel in (("cache.cu", "append_stream_kernel"), ("adjust.cu", "adjust_kernel"), ("pages.cu", "pages_kernel"),
                         ("attention_window.cu", "window_kernel")):
        body = _kernel(name, kernel)
        wait = body.index("pdl_wait()")
        assert wait < body.index("pdl_launch_dependents()")
        assert not re.search(r"__ldg|__ldcg|seq_span\(|find_item\(|call_record_start|atomic", body[:wait]), name


def test_window_kernel_waits_for_its_copies_and_products():
    body = _kernel("attention_window.cu", "window_kernel")
    load = body[body.index("per_piece = kSub"):body.index("kF32Bf16 =")]
    assert load.rindex("mbar_wait_warp(&full_v[") > load.rindex("mbar_wait_warp(&full_k[") > load.rindex("tma_load_2d_warp(")
    products = body[body.index("kF32Bf16 ="):body.index("setmaxnreg.inc")]
    tail = products[max(products.rindex("umma_bf16_ts_warp("), products.rindex("scores(")):]
    assert re.search(r"umma_commit_warp\(&mma_done\).*mbar_wait_warp\(&mma_done, 0\)", tail, re.S)
    assert body.rindex("__syncthreads();") < body.rindex("tmem_dealloc(")
    # whoever waits for an item's place to be free counts every reader of it
    assert body.count("item_done(it);") == 5 and "mbar_init(&item_empty[i], 11);" in body        # loads, values, products, and two ways out of the softmax
    # a register split within what the block was launched with
    dec, inc = (int(x) for x in re.findall(r"setmaxnreg\.(?:dec|inc)\.sync\.aligned\.u32 (\d+)", body))
    assert dec + 2 * inc <= 3 * 168 and dec % 8 == inc % 8 == 0


def test_append_stream_pieces_hold_whole_heads():
    """A ring of 16 warps fits in shared memory; pieces are whole heads of every type and size."""
    text = _source("cache.cu")
    warps, piece, stages = (int(re.search(r"\b%s = (\d+)" % n, text).group(1)) for n in ("kStreamWarps", "kPiece", "kStages"))
    assert warps * piece * stages <= 227 * 1024
    assert all(piece % (dim * size) == 0 and (dim * size) % 16 == 0 for dim in (64, 128) for size in (2, 4))
