"""What the binding of the layer operators and of the evaluation refuses before it asks the library (no GPU needed)."""
import types

import numpy as np
import pytest
import torch

from paper_2112_13935_b200 import _lib, api

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


@pytest.fixture
def library(monkeypatch):
    """A library that has a model of 12 inputs, 5 classes and 65 parameters and answers every call."""
    calls = []
    fake = types.SimpleNamespace(aet_n_inputs=lambda h: 12, aet_n_classes=lambda h: 5, aet_n_params=lambda h: 65,
                                 aet_predict=lambda *a: calls.append(a) or 0, aet_evaluate=lambda *a: calls.append(a) or 0,
                                 aet_load_client_data=lambda *a: calls.append(a) or 0)
    monkeypatch.setattr(_lib, "load", lambda: fake)
    return calls


@pytest.mark.parametrize("make", [np.zeros, torch.zeros], ids=["numpy", "torch"])
def test_evaluation_holds_its_arrays_to_the_model(library, make):
    f32, i32 = (np.float32, np.int32) if make is np.zeros else (torch.float32, torch.int32)
    x, y, z = make((4, 12), dtype=f32), make(4, dtype=i32), make((4, 5), dtype=f32)
    for bad in (make((4, 11), dtype=f32), make((4, 13), dtype=f32), make((48,), dtype=f32), make((4, 12, 2), dtype=f32)):
        with pytest.raises(api.AetError, match="x:"):
            api.aet_predict(None, 0, bad, z, stream=0)
        with pytest.raises(api.AetError, match="x:"):
            api.aet_evaluate(None, 0, bad, y, stream=0)
    for bad in (make((4, 4), dtype=f32), make((4, 6), dtype=f32), make((20,), dtype=f32), make((3, 5), dtype=f32)):
        with pytest.raises(api.AetError, match="logits:"):
            api.aet_predict(None, 0, x, bad, stream=0)
    for classes in (4, 6):
        with pytest.raises(api.AetError, match="logits:"):
            api.aet_predict(None, 0, x, classes=classes, stream=0)
    for bad in (make(3, dtype=i32), make((4, 2), dtype=i32)):
        with pytest.raises(api.AetError, match="y:"):
            api.aet_evaluate(None, 0, x, bad, stream=0)
    assert not library
    api.aet_predict(None, 0, x, z, stream=0)
    assert api.aet_predict(None, 0, x, classes=5, stream=0).shape == (4, 5)
    api.aet_evaluate(None, 0, x.reshape(4, 3, 4), y, stream=0)          # (pictures lie as their rows do)
    assert [c[3] for c in library[:2]] == [4, 4] and library[2][4] == 4


def test_client_data_is_held_to_the_model(library):
    x, y = np.zeros((4, 12), dtype=np.float32), np.zeros(4, dtype=np.int32)
    for bad in (x[:, :11].copy(), np.zeros((4, 13), dtype=np.float32), x.astype(np.float64), np.zeros(48, dtype=np.float32)):
        with pytest.raises(api.AetError, match="x:"):
            api.aet_load_client_data(None, 0, bad, y, stream=0)
    for bad in (y[:3], y.astype(np.int64), np.zeros((4, 2), dtype=np.int32)):
        with pytest.raises(api.AetError, match="y:"):
            api.aet_load_client_data(None, 0, x, bad, stream=0)
    assert not library
    api.aet_load_client_data(None, 0, x.reshape(4, 3, 2, 2), y, stream=0)
    api.aet_load_client_data(None, 0, torch.from_numpy(x), torch.from_numpy(y), stream=0)
    api.aet_load_client_data(None, 0, x, y.astype(np.uint32), stream=0)
    assert [c[4] for c in library] == [4, 4, 4]


def test_widths_of_no_handle():
    assert api.aet_n_inputs(None) == api.aet_n_classes(None) == 0


def test_numbers_past_32_bits_are_refused(library, monkeypatch):
    """... where the library's argument has 32: they would arrive cut off, as a call on fewer columns or on another client."""
    monkeypatch.setattr(api, "_stream_of", lambda dev, t, stream: 0)
    fake = _lib.load()
    fake.aet_dropout = fake.aet_cross_entropy = lambda *a: library.append(a) or 0
    wide = torch.empty(1, 2 ** 32 + 5, device="meta")
    labels = torch.empty(1, dtype=torch.int32, device="meta")
    many = types.SimpleNamespace(dtype="float32", shape=(2 ** 32 + 1, 12), numel=lambda: (2 ** 32 + 1) * 12)
    few, y = np.zeros((4, 12), dtype=np.float32), np.zeros(4, dtype=np.int32)
    for call in (lambda: api.aet_dropout(SPEC, wide, wide), lambda: api.aet_cross_entropy(wide, labels), lambda: api.aet_dense(2 ** 32 + 8, 4),
                 lambda: api.aet_dense(8, 2 ** 32), lambda: api.aet_dense(8, 4, flags=2 ** 32), lambda: api.aet_dropout_spec(1, client=2 ** 32),
                 lambda: api.aet_predict(None, 0, many, np.zeros((4, 5), dtype=np.float32), stream=0), lambda: api.aet_evaluate(None, 2 ** 32, few, y, stream=0),
                 lambda: api.aet_predict(None, 2 ** 32, few, classes=5, stream=0)):
        with pytest.raises(api.AetError, match="32 bits") as e:
            call()
        assert e.value.status == 1
    assert not library


def test_evaluation_refuses_arrays_of_another_device(library, monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)

    def there(dtype, *shape, device=1):
        return types.SimpleNamespace(dtype=dtype, shape=shape, numel=lambda: int(np.prod(shape)), is_cuda=True, get_device=lambda: device, device=f"cuda:{device}",
                                     is_contiguous=lambda: True, data_ptr=lambda: 1 << 20)

    x, y, z = np.zeros((4, 12), dtype=np.float32), np.zeros(4, dtype=np.int32), np.zeros((4, 5), dtype=np.float32)
    for call in (lambda: api.aet_predict(None, 0, there("float32", 4, 12), z, stream=0), lambda: api.aet_predict(None, 0, x, there("float32", 4, 5), stream=0),
                 lambda: api.aet_evaluate(None, 0, there("float32", 4, 12), y, stream=0), lambda: api.aet_evaluate(None, 0, x, there("int32", 4), stream=0)):
        with pytest.raises(api.AetError, match="current CUDA device"):
            call()
    assert not library
    api.aet_predict(None, 0, there("float32", 4, 12, device=0), there("float32", 4, 5, device=0), stream=0)
    assert len(library) == 1
