"""CPU: rules of copies, waits and streams in the attention kernels, on the
source text (as test_kernel_protocols does for the linear layer's)."""
import re

from test_kernel_protocols import _block, _source


def test_wide_kernel_waits_for_its_copies_and_products():
    text = _source("attention_wide.cu")
    branches = {}
    for m in re.finditer(r"\bif \(warp == (8|9)\) \{", text):
        a, b = _block(text, m.end() - 1)
        branches.setdefault(m.group(1), []).append(text[a:b])
    load = [b for b in branches["9"] if "tma_load_2d_warp(" in b]
    assert len(load) == 1
    assert load[0].rindex("mbar_wait_warp(&full[") > load[0].rindex("tma_load_2d_warp(")
    mma = [b for b in branches["8"] if "umma_bf16_warp(" in b]
    assert len(mma) == 1
    tail = mma[0][max(mma[0].rindex("umma_bf16_ts_warp("), mma[0].rindex("umma_bf16_warp(")):]
    assert re.search(r"umma_commit_warp\(&mma_done\).*mbar_wait_warp\(&mma_done, 0\)", tail, re.S)
    # (the whole thread block meets before tensor memory is freed)
    assert text.rindex("__syncthreads();") < text.rindex("tmem_dealloc(")


def test_narrow_kernel_waits_for_its_copies():
    text = _source("attention_narrow.cu")
    last_issue = text.rindex("issue();")
    assert re.search(r"if \(!ok\)\s*for \(int i = max\(0, ki - ST\); i < ki; \+\+i\) mbar_wait_warp\(&full\[warp\]\[i % ST\]", text[last_issue:])


def test_every_kernel_orders_itself_behind_the_grid_before():
    """Launched early, a kernel waits for the grid before it ahead of its first global access; the one that may
    run beside its own call's other kernel waits for it at the end."""
    for name, kernel in (("cache.cu", "append_kernel"), ("attention.cu", "join_kernel"), ("attention_wide.cu", "wide_kernel"),
                         ("attention_narrow.cu", "narrow_kernel"), ("sample.cu", "sample_kernel")):
        text = _source(name)
        m = re.search(r"__global__[^;{]*?\b%s\(" % kernel, text, re.S)
        a, b = _block(text, text.index("{", text.index(")", m.end())))
        body = text[a:b]
        wait = body.index("pdl_wait()")
        assert wait < body.index("pdl_launch_dependents()")
        assert not re.search(r"__ldg|__ldcg|seq_span\(|call_record_start|atomic", body[:wait]), name
    assert re.search(r"if \(late\) pdl_wait\(\);\s*\}", _source("attention_narrow.cu"))
