"""Evaluation of a handle's model against the oracle's losses and gradients in 64 bits."""
import numpy as np
import pytest
import torch

import layer_helpers as lh
from oracle import models, sim
from paper_2112_13935_b200 import api, workloads

pytestmark = pytest.mark.gpu


def session(dims, precision=0, l2=0.0, topology=0, n_clients=3, seed=5):
    cfg = workloads.get_config("cfg3" if len(dims) > 2 else "cfg1", dims=list(dims), model=1 if len(dims) > 2 else 0, precision=precision, l2=l2, topology=topology,
                               n_clients=n_clients, batch=4 if len(dims) > 2 else 1, sched_a=4, sched_b=4, seed=seed, lr=0.01)
    r = np.random.default_rng(seed)
    data = [(np.maximum(r.standard_normal((40, dims[0])), 0).astype(np.float32), r.integers(0, dims[-1], 40).astype(np.int32)) for _ in range(n_clients)]
    w0 = np.concatenate([np.concatenate([(r.uniform(-1, 1, (i * o)) / np.sqrt(i)), r.uniform(-0.1, 0.1, o)]) for i, o in zip(dims, dims[1:])]).astype(np.float32)
    return cfg, api.Session(cfg, data, w0), r


def rows_of(r, n, dims):
    return np.maximum(r.standard_normal((n, dims[0])), 0).astype(np.float32), r.integers(0, dims[-1], n).astype(np.int32)


CASES = [((784, 10), 0, 0.0, 300), ((784, 10), 0, 1e-3, 1), ((785, 7), 0, 1e-4, 2100), ((784, 128, 10), 0, 0.0, 3000), ((60, 33, 17, 5), 0, 1e-3, 257),
         ((784, 256, 128, 10), 1, 1e-4, 900), ((64, 32, 3), 1, 0.0, 77)]


@pytest.mark.parametrize("dims,precision,l2,n", CASES)
@pytest.mark.parametrize("where", ["host", "device"])
def test_evaluation_against_the_oracle(dims, precision, l2, n, where):
    cfg, s, r = session(dims, precision, l2)
    with s:
        s.run(2)
        w = s.model()
        x, y = rows_of(r, n, dims)
        want_loss, want_grad = models.loss_and_grad(w.astype(np.float64), x, y, dims, sim.f32(l2), precision)
        put = (lambda a: torch.from_numpy(a).cuda()) if where == "device" else (lambda a: a)
        grad = put(np.full(w.size, 7.0, dtype=np.float32))
        loss, right = s.evaluate(put(x), put(y), gradient=grad)
        assert s.evaluate(put(x), put(y)) == (loss, right)          # with or without a gradient
        z = put(np.zeros((n, dims[-1]), dtype=np.float32))
        api.aet_predict(s.h, 1, put(x), z)
        grad, z = (lh.host(v) if where == "device" else v.astype(np.float64) for v in (grad, z))
        # fp32: sums of up to 785 terms in a few layers, some 1e-6.  bf16: roundings that the oracle's 64-bit sums and these fp32 sums take differently
        # (a hidden value by 2^-8 of itself, here and there) and ReLU masks that flip with them
        tol = 1e-5 if precision == 0 else 3e-2
        assert abs(loss - want_loss) <= (1e-6 if precision == 0 else 2e-4) * max(1.0, want_loss)
        scale = np.abs(want_grad).max()
        assert np.abs(grad - want_grad).max() <= tol * scale
        if precision == 1:
            assert (np.abs(grad - want_grad) > 3e-4 * scale).mean() <= 0.02
        p = models.softmax_rows(z)
        assert abs(models._ce(p, y).mean() + 0.5 * l2 * sum((a.astype(float) ** 2).sum() for a, _ in models.unpack(w, dims)) - loss) <= 1e-5 * max(1.0, loss)
        assert right == int((z.argmax(1) == y).sum())


def test_evaluation_leaves_a_run_as_it_was():
    cfg, s, r = session((784, 10))
    x, y = rows_of(r, 500, (784, 10))
    with s:
        for _ in range(3):          # (every call runs to quiescence: three of one round are not one of three)
            s.run(1)
        want, log = s.model(), s.log(raw=True)
    cfg, s, r = session((784, 10))
    with s:
        for _ in range(3):
            s.run(1)
            s.evaluate(x, y, gradient=np.empty(7850, dtype=np.float32))
        assert np.array_equal(s.model(), want) and s.log(raw=True) == log


def test_evaluation_of_a_ring_node():
    cfg, s, r = session((784, 10), topology=1, n_clients=5)
    x, y = rows_of(r, 64, (784, 10))
    with s:
        s.run(3)
        losses = []
        for node in range(5):
            w = api.aet_get_node_model(s.h, node)
            want = models.loss_and_grad(w.astype(np.float64), x, y, (784, 10))[0]
            losses.append(s.evaluate(x, y, node=node)[0])
            assert abs(losses[-1] - want) <= 1e-6 * max(1, want)
        assert len(set(losses)) > 1


def test_evaluation_in_chunks_with_dropout():
    """70,000 rows are more than one chunk: masks, loss and gradient as in one piece."""
    dims, n = (32, 24, 16, 4), 70000
    cfg, s, r = session(dims)
    x, y = rows_of(r, n, dims)
    with s:
        w = s.model().astype(np.float64)
        grad = np.empty(w.size, dtype=np.float32)
        loss, right = s.evaluate(x, y, dropout=api.aet_dropout_spec(seed=3, client=2, counter=100, rate=0.25), gradient=grad)
        leaf = torch.as_tensor(w).cuda().requires_grad_()
        a, at, counter = torch.as_tensor(x).cuda().double(), 0, 100
        for l, (i, o) in enumerate(zip(dims, dims[1:])):
            a = a @ leaf[at:at + i * o].view(i, o) + leaf[at + i * o:at + i * o + o]
            at += i * o + o
            if l < 2:
                mask, factor = lh.kept(n, o, 3, 2, counter, 0.25)
                counter += n * ((o + 3) // 4)
                a = torch.relu(a) * torch.as_tensor(mask).cuda() * factor
        want = torch.nn.functional.cross_entropy(a, torch.as_tensor(y).cuda().long())
        want.backward()
        want = float(want.detach())
        assert abs(loss - want) <= 1e-6 * max(1.0, want)
        g = leaf.grad.cpu().numpy()
        assert np.abs(grad - g).max() <= 1e-5 * np.abs(g).max()


def test_evaluation_refusals():
    cfg, s, r = session((784, 10))
    x, y = rows_of(r, 8, (784, 10))
    with s:
        grad = np.full(7850, 3.0, dtype=np.float32)

        def refused(status, f):
            with pytest.raises(api.AetError) as e:
                f()
            assert e.value.status == status
            assert (grad == 3.0).all()

        refused(1, lambda: s.evaluate(x, np.where(np.arange(8) == 5, 10, y).astype(np.int32), gradient=grad))
        refused(1, lambda: s.evaluate(x, np.where(np.arange(8) == 5, -1, y).astype(np.int32), gradient=grad))
        refused(1, lambda: s.evaluate(x, y, node=3, gradient=grad))
        refused(1, lambda: s.evaluate(x[:0], y[:0], gradient=grad))
        refused(1, lambda: s.evaluate(x, y, dropout=api.aet_dropout_spec(1, rate=1.5), gradient=grad))
        bad = x.copy()
        bad[3, 5] = np.nan
        refused(7, lambda: s.evaluate(bad, y, gradient=grad))
        s.evaluate(x, y)                               # the handle stays usable
        s.run(1)
    conv = workloads.get_config("cfg7", n_clients=1)
    with api.Session(conv, [], None) as s:
        with pytest.raises(api.AetError) as e:
            s.evaluate(np.zeros((4, 784), dtype=np.float32), np.zeros(4, dtype=np.int32))
        assert e.value.status == 2


def test_evaluation_of_rows_that_do_not_fit_the_model():
    cfg, s, r = session((784, 10))
    x, y = rows_of(r, 8, (784, 10))
    with s:
        assert (api.aet_n_inputs(s.h), api.aet_n_classes(s.h), api.aet_n_params(s.h)) == (784, 10, 7850)
        for bad in (x[:, :783].copy(), np.zeros((8, 785), dtype=np.float32), torch.zeros(8, 783, device="cuda")):
            for call in (lambda: s.evaluate(bad, y), lambda: s.predict(bad)):
                with pytest.raises(api.AetError, match="x:") as e:
                    call()
                assert e.value.status == 1
        for classes in (9, 11):
            with pytest.raises(api.AetError, match="logits:"):
                api.aet_predict(s.h, 0, x, classes=classes)
            with pytest.raises(api.AetError, match="logits:"):
                api.aet_predict(s.h, 0, x, torch.zeros(8, classes, device="cuda"))
        assert s.predict(x).shape == (8, 10)
    conv = workloads.get_config("cfg7", n_clients=1)
    with api.Session(conv, [], None) as s:
        assert (api.aet_n_inputs(s.h), api.aet_n_classes(s.h)) == (784, 10)


@pytest.mark.parametrize("dims", [(784, 10), (784, 128, 10)])
def test_evaluation_of_a_whole_training_set(dims):
    """60,000 rows of the 28x28 sets: the products that many rows take, ten columns among them, against 64 bits."""
    cfg, s, r = session(dims, l2=1e-4)
    x, y = rows_of(r, 60000, dims)
    x, y = torch.as_tensor(x).cuda(), torch.as_tensor(y).cuda()
    with s:
        w = s.model()
        grad = torch.empty(w.size, device="cuda")
        loss, right = s.evaluate(x, y, gradient=grad)
        z = torch.empty(60000, dims[-1], device="cuda")
        api.aet_predict(s.h, 0, x, z)
        leaf = torch.as_tensor(w.astype(np.float64)).cuda().requires_grad_()
        a, at, norm = x.double(), 0, 0
        for l, (i, o) in enumerate(zip(dims, dims[1:])):
            m = leaf[at:at + i * o].view(i, o)
            a, norm = a @ m + leaf[at + i * o:at + i * o + o], norm + (m * m).sum()
            at += i * o + o
            if l + 2 < len(dims):
                a = torch.relu(a)
        want = torch.nn.functional.cross_entropy(a, y.long()) + 0.5 * sim.f32(1e-4) * norm
        want.backward()
        assert abs(loss - float(want.detach())) <= 1e-6 * max(1.0, float(want.detach()))
        # sums of 784 terms of a few tenths each: 800 2^-23 of their magnitudes at the very most
        assert float((z - a.detach()).abs().max()) <= 800 * 2.0 ** -23 * 40
        assert right == int((z.argmax(1) == y).sum())
        g = leaf.grad
        assert float((grad - g).abs().max()) <= 1e-5 * float(g.abs().max())
