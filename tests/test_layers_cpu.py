"""Refusals of the layer operators' C entries: every call here is turned down before anything is launched (no GPU needed)."""
import ctypes as C

import pytest

from oracle import rng
from paper_2112_13935_b200 import _lib, api, build

P = 1 << 20      # an address nobody reads


@pytest.fixture(scope="module", autouse=True)
def built():
    build.build()


def refused(status, text):
    msg = _lib.load().aet_last_error(None).decode()
    assert status == 1 and text in msg, (status, msg)


def test_dropout_stream_of_the_generator():
    assert api.aet_debug_draw(5, 4, 7, 123) == rng.draw(rng.stream_key(5, 4, 7), 123)


def dropout(**over):
    a = dict(dtype=0, rows=2, cols=3, drop=api.aet_dropout_spec(1, rate=0.5), x=P, ld_x=0, residual=None, ld_residual=0, y=P, ld_y=0)
    a.update(over)
    d = a["drop"]
    return _lib.load().aet_dropout(a["dtype"], a["rows"], a["cols"], C.addressof(d) if d is not None else None, a["x"], a["ld_x"], a["residual"],
                                   a["ld_residual"], a["y"], a["ld_y"], None)


@pytest.mark.parametrize("over,text", [
    (dict(dtype=3), "dtype"), (dict(drop=None), "null"), (dict(drop=api.aet_dropout_spec(1, rate=-0.1)), "rate"), (dict(drop=api.aet_dropout_spec(1, rate=1.0)), "rate"),
    (dict(drop=api.aet_dropout_spec(1, rate=float("nan"))), "rate"), (dict(drop=api.aet_dropout_spec(1, rate=0.999999)), "rate"), (dict(cols=0), "columns"),
    (dict(cols=1 << 31), "columns"), (dict(rows=1 << 31), "rows"), (dict(x=None), "null"), (dict(y=None), "null"), (dict(ld_x=2), "ld"), (dict(ld_y=2), "ld"),
    (dict(ld_residual=1), "ld"), (dict(ld_x=(1 << 31) + 1), "ld"), (dict(x=P + 2), "element size"), (dict(y=P + 1, dtype=1), "element size"), (dict(residual=P + 1, dtype=2), "element size")])
def test_dropout_refusals(over, text):
    refused(dropout(**over), text)


def test_calls_on_no_rows_do_nothing():
    assert dropout(rows=0, x=None, y=None) == 0
    assert loss(rows=0, logits=None, labels=None) == 0
    assert forward(rows=0, x=None, w=None, y=None) == 0


def loss(**over):
    a = dict(dtype=0, rows=2, classes=3, logits=P, ld=0, labels=P, weight=None, loss=P, dlogits=P, ld_d=0, top=P)
    a.update(over)
    return _lib.load().aet_cross_entropy(a["dtype"], a["rows"], a["classes"], a["logits"], a["ld"], a["labels"], a["weight"], 1.0, a["loss"], a["dlogits"],
                                         a["ld_d"], a["top"], None)


@pytest.mark.parametrize("over,text", [
    (dict(dtype=9), "dtype"), (dict(classes=0), "classes"), (dict(classes=(1 << 30) + 1), "classes"), (dict(rows=1 << 31), "rows"), (dict(logits=None), "null"),
    (dict(labels=None), "null"), (dict(ld=2), "ld"), (dict(ld_d=1), "ld"), (dict(logits=P + 2), "element size"), (dict(labels=P + 2), "element size"),
    (dict(weight=P + 1), "element size"), (dict(loss=P + 2), "element size"), (dict(top=P + 2), "element size"), (dict(dlogits=P + 1, dtype=1), "element size")])
def test_loss_refusals(over, text):
    refused(loss(**over), text)


def forward(desc=None, **over):
    d = api.aet_dense(8, 4) if desc is None else desc
    a = dict(rows=2, x=P, w=P, bias=None, residual=None, y=P, pre=None, ws=P, size=1 << 40)
    a.update(over)
    return _lib.load().aet_dense_forward(C.addressof(d) if d != 0 else None, a["rows"], a["x"], a["w"], a["bias"], a["residual"], a["y"], a["pre"], a["ws"], a["size"], None)


def backward(desc=None, **over):
    d = api.aet_dense(8, 4, act="relu") if desc is None else desc
    a = dict(rows=2, x=P, w=P, pre=P, dy=P, dx=P, dw=P, db=P, ws=P, size=1 << 40)
    a.update(over)
    return _lib.load().aet_dense_backward(C.addressof(d), a["rows"], a["x"], a["w"], a["pre"], a["dy"], a["dx"], a["dw"], a["db"], a["ws"], a["size"], None)


def broken(**over):
    d = api.aet_dense(8, 4)
    for k, v in over.items():
        setattr(d, k, v)
    return d


BAD = [(dict(struct_size=4), "struct_size"), (dict(dtype=3), "dtype"), (dict(act=4), "activation"), (dict(flags=4), "flag"), (dict(n_in=0), "n_in"),
       (dict(n_out=0), "n_out"), (dict(n_in=1 << 31), "n_in"), (dict(ld_x=7), "ld"), (dict(ld_w=3), "ld"), (dict(ld_pre=1), "ld"), (dict(ld_dw=(1 << 31) + 1), "ld"),
       (dict(drop=api.aet_dropout_spec(1, rate=2.0)), "rate")]


@pytest.mark.parametrize("over,text", BAD)
def test_dense_descriptor_refusals(over, text):
    refused(forward(broken(**over)), text)
    refused(backward(broken(**over)), text)
    n = C.c_size_t(7)
    d = broken(**over)
    refused(_lib.load().aet_dense_workspace(C.addressof(d), 2, 0, C.addressof(n)), text)
    assert n.value == 7


@pytest.mark.parametrize("over,text", [
    (dict(desc=0), "null"), (dict(x=None), "null"), (dict(w=None), "null"), (dict(y=None), "null"), (dict(rows=1 << 31), "rows"), (dict(x=P + 4), "16-byte"),
    (dict(w=P + 8), "16-byte"), (dict(x=P + 1), "element size"), (dict(y=P + 2), "element size"), (dict(bias=P + 2), "element size"), (dict(residual=P + 2), "element size"), (dict(pre=P + 3), "element size")])
def test_dense_forward_refusals(over, text):
    refused(forward(**over), text)


@pytest.mark.parametrize("over,text", [
    (dict(dy=None), "null"), (dict(x=None), "null"), (dict(w=None), "null"), (dict(pre=None), "null"), (dict(dy=P + 4), "16-byte"), (dict(x=P + 4), "16-byte"),
    (dict(w=P + 4), "16-byte"), (dict(dx=P + 2), "element size"), (dict(dw=P + 2), "element size"), (dict(db=P + 1), "element size"), (dict(ws=None), "workspace"),
    (dict(ws=P + 16), "workspace"), (dict(size=16), "workspace"), (dict(rows=1 << 31), "rows")])
def test_dense_backward_refusals(over, text):
    refused(backward(**over), text)


def test_dense_workspace_refusals_and_sizes():
    d = api.aet_dense(8, 4)
    refused(_lib.load().aet_dense_workspace(C.addressof(d), 2, 0, None), "null")
    assert api.aet_dense_workspace(api.aet_dense(8, 4), 0, True) == 0
    sizes = [api.aet_dense_workspace(api.aet_dense(100, 50), r, True) for r in (1, 10, 1000, 100000)]
    assert sizes == sorted(sizes) and all(s % 256 == 0 for s in sizes)


def test_binding_refuses_what_does_not_fit():
    torch = pytest.importorskip("torch")
    with pytest.raises(api.AetError, match="activation"):
        api.aet_dense(3, 4, act="tanh")
    with pytest.raises(api.AetError, match="element type"):
        api.aet_dense(3, 4, dtype=torch.float64)
    with pytest.raises(api.AetError, match="unknown argument"):
        api.aet_dense(3, 4, ld_q=3)
    x = torch.zeros(2, 3)
    with pytest.raises(api.AetError, match="current CUDA device"):       # CPU tensors
        api.aet_dropout(api.aet_dropout_spec(1), x, x)
    with pytest.raises(api.AetError, match="y:"):
        api.aet_dropout(api.aet_dropout_spec(1), x, torch.zeros(2, 4))
    with pytest.raises(api.AetError, match="strides"):
        api.aet_dropout(api.aet_dropout_spec(1), x, torch.zeros(3, 2).t())
    with pytest.raises(api.AetError, match="labels"):
        api.aet_cross_entropy(x, torch.zeros(2, dtype=torch.int64))
    with pytest.raises(api.AetError, match="x:"):
        api.aet_dense_forward(api.aet_dense(4, 4), x, x, None, x)
    with pytest.raises(api.AetError, match="w:"):
        api.aet_dense_forward(api.aet_dense(3, 4), x, x, None, x)


def test_evaluation_binding_refuses_other_types():
    import numpy as np
    x, y = np.zeros((4, 3), dtype=np.float32), np.zeros(4, dtype=np.int32)
    for bad in (lambda: api.aet_evaluate(None, 0, x.astype(np.float64), y), lambda: api.aet_evaluate(None, 0, x, y.astype(np.int64)),
                lambda: api.aet_evaluate(None, 0, x, y[:3]), lambda: api.aet_predict(None, 0, x), lambda: api.aet_predict(None, 0, x, np.zeros((3, 2), dtype=np.float32))):
        with pytest.raises(api.AetError):
            bad()
