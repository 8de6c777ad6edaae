"""CPU: rules of the window kernel on the source text."""
from test_kernel_protocols import _block, _source


def _loops(text):
    """Bodies of for loops, innermost last."""
    import re
    for m in re.finditer(r"\bfor \([^{};]*;[^{};]*;[^{};]*\) \{", text):
        a, b = _block(text, m.end() - 1)
        yield text[a:b]


def test_whole_warps_read_the_output():
    """Reads of tensor memory are a warp's together: after rows that some lanes have and others do not, the lanes
    meet again ahead of the next read."""
    text = _source("attention_window.cu")
    out = [b for b in _loops(text) if "tmem_ld32(" in b and "p.out" in b and "load_queries" not in b]
    assert len(out) == 1
    body = out[0]
    assert "__syncwarp();" in body[body.rindex("live"):]
    outer = body[body.rindex("if (live"):]                 # (a continue of the loop itself would pass the meeting by)
    assert "continue" not in outer and "if (!live)" not in body
