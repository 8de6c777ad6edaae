"""CPU: arguments of `adjust_logits` that leave nothing to look at are not taken
for arguments that were not given."""
import pytest
import torch

from test_serving_devices import _On, _Reached, fakes  # noqa: F401


def test_a_grammar_without_sets_is_refused(fakes, monkeypatch):  # noqa: F811
    """No memory, so no address: the C call would read it as no grammar, and every token would be allowed."""
    def reached(*a):
        raise _Reached
    monkeypatch.setattr(fakes, "sdq_adjust_logits", reached)
    z, ints = _On(torch.zeros((2, 100)), 0), lambda *shape: _On(torch.zeros(shape, dtype=torch.int32), 0)
    with pytest.raises(_Reached):
        fakes.adjust_logits(z, allowed=ints(2, 4))
    with pytest.raises(ValueError):
        fakes.adjust_logits(z, allowed=ints(0, 4))
    with pytest.raises(_Reached):                         # (each row says which set it has: none of those)
        fakes.adjust_logits(z, allowed=ints(0, 4), allowed_row=ints(2))
    # a history, or a list of biases, of no places is one that names nothing
    with pytest.raises(_Reached):
        fakes.adjust_logits(z, ints(2, 0), bias_ids=ints(2, 0), bias=_On(torch.zeros((2, 0)), 0))
