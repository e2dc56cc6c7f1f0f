"""What the binding of the layer operators and of the evaluation refuses before it asks the library (no GPU needed)."""
import pytest
import torch

from paper_2112_13935_b200 import api

SPEC = api.aet_dropout_spec(1, rate=0.5)


def broadcast_calls():
    x, row = torch.zeros(6, 8), torch.zeros(8).expand(6, 8)
    overlap = torch.zeros(64).as_strided((6, 8), (3, 1))            # rows that share elements
    labels = torch.zeros(6, dtype=torch.int32)
    for name, m in (("broadcast", row), ("overlapping", overlap)):
        yield name + " x", "x", lambda m=m: api.aet_dropout(SPEC, m, x)
        yield name + " y", "y", lambda m=m: api.aet_dropout(SPEC, x, m)
        yield name + " residual", "residual", lambda m=m: api.aet_dropout(SPEC, x, x, residual=m)
        yield name + " logits", "logits", lambda m=m: api.aet_cross_entropy(m, labels)
        yield name + " dlogits", "dlogits", lambda m=m: api.aet_cross_entropy(x, labels, dlogits=m)
        plan = api.aet_dense(8, 8, act="relu")
        yield name + " layer's x", "x", lambda m=m: api.aet_dense_forward(plan, m, torch.zeros(8, 8), None, x)
        yield name + " layer's residual", "residual", lambda m=m: api.aet_dense_forward(plan, x, torch.zeros(8, 8), None, x, residual=m)
        yield name + " layer's dy", "dy", lambda m=m: api.aet_dense_backward(plan, x, torch.zeros(8, 8), m, pre=x)


@pytest.mark.parametrize("what,call", [pytest.param(w, c, id=n) for n, w, c in broadcast_calls()])
def test_rows_that_share_elements_are_refused(what, call):
    with pytest.raises(api.AetError, match=rf"^AET_ERR_ARG: {what}: strides") as e:
        call()
    assert e.value.status == 1


def test_one_row_and_one_column_may_have_any_stride():
    """What an index of one value strides by does not matter: these get as far as the device's check."""
    one_row = torch.zeros(8).expand(1, 8)
    one_column = torch.zeros(6, 9)[:, :1]
    for call in (lambda: api.aet_dropout(SPEC, one_row, one_row), lambda: api.aet_dropout(SPEC, one_column, one_column, residual=one_column),
                 lambda: api.aet_cross_entropy(one_column, torch.zeros(6, dtype=torch.int32))):
        with pytest.raises(api.AetError, match="current CUDA device"):
            call()
