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


def test_narrow_kernel_splits_rows_by_multiplication_within_its_range_only():
    """token_of is exact below 32 rows (a unit with keys has no more), and not far beyond; a sequence without keys may
    bring any number of rows and goes another way."""
    def token_of(r, group):
        return (r * (65536 // group + 1) & 0xFFFFFFFF) >> 16
    assert all(token_of(r, g) == r // g for g in range(1, 4097) for r in range(32))
    assert token_of(8199, 8) != 8199 // 8 and token_of(4111, 16) != 4111 // 16 and token_of(65536, 1) != 65536
    text = _source("attention_narrow.cu")
    assert "(uint32_t)r * p.group_inverse >> 16" in text and "65536u / (uint32_t)group + 1" in _source("attention.cu")
    m = re.search(r"for \(int s = blockIdx\.x; s < p\.b\.n_seqs; s \+= gridDim\.x\)", text)
    a, b = _block(text, m.end())
    assert "own > 0" in text[a:b] and not re.search(r"\b(finish|token_of|group_inverse)\b", text[a:b])
