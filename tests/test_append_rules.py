"""CPU: rules of the append's kernels on the source text."""
from test_step_host import _kernel


def test_append_of_many_tokens_orders_itself_behind_the_grid_before():
    body = _kernel("cache.cu", "append_many_kernel")
    wait = body.index("pdl_wait()")
    assert wait < body.index("pdl_launch_dependents()") < body.index("place_of(")
    assert "load4(" not in body[:wait] and "store4(" not in body[:wait]
