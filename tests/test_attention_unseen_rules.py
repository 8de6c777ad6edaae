"""CPU: rules of the attention kernels for rows that see no key, on the source
text (as test_serving_protocols does for their copies and waits)."""
import re

from test_kernel_protocols import _block, _source


def _rows_out(text):
    """The wide kernel's branch that writes rows of the output."""
    starts = [m.end() - 1 for m in re.finditer(r"\belse if \(ok\) \{", text)]
    assert len(starts) == 1
    a, b = _block(text, starts[0])
    return text[a:b]


def test_places_of_the_queries_are_other_warps_output_places():
    """128 rows of queries lie as halves of 64 elements, 128 bytes a row; rows of the output as whole rows, 32 of a warp
    together.  Both from the same address on, so that with 128 elements a warp's output place holds other warps' queries."""
    queries = lambda w: {h * 16384 + 4096 * w + i for h in range(2) for i in range(0, 4096, 16)}
    output = lambda w: {8192 * w + i for i in range(0, 8192, 16)}
    assert any(output(w) & queries(o) for w in range(4) for o in range(4) if o != w)


def test_wide_kernel_orders_its_output_behind_the_queries_copies():
    """A warp's wait for the last product covers every warp's copies of the queries (the products start behind all of
    them).  Without a tile there is no product: a barrier of the warps that copied takes its place."""
    rows = _rows_out(_source("attention_wide.cu"))
    barrier = re.search(r"if \(n == 0\) named_bar_sync\(1, 128 \* halves\);", rows)
    assert barrier and barrier.end() < rows.index("st_shared16(")
