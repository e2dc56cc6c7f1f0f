"""Performance cases of the layer operators: a dense layer and its gradient, the classification loss with its gradient,
and dropout from the counter-based generator.

A case names one call: its operator, element type, sizes and options.

  dense       y = residual + dropout(act(x w + bias)); x [rows, n_in], w [n_in, n_out] as the models of this library keep it
  dense_back  dx, dw, dbias of the same layer from dy, with x, w and the kept pre-activations at hand
  loss        softmax cross-entropy of [rows, n_out] logits: loss and prediction a row, and the gradient
  dropout     y = residual + dropout(x); without a residual it is its own gradient

Every matrix is row-major, its rows n + pad elements apart; types are f32, bf16 and f16.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = dict(f32=torch.float32, bf16=torch.bfloat16, f16=torch.float16)
LARGEST = 8192 * 4096 * 16384      # rows * n_in * n_out of the largest dense case


def _case(name, op, **over):
    c = dict(op=op, type="f32", rows=1, n_in=0, n_out=10, act="none", bias=True, residual=False, pre=False, rate=0.0, pad=0)
    assert set(over) <= set(c), over
    c.update(over)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # One row through a wide layer, as a server answers a single request: bound by reading the weights.
        _case("dense_one_row", "dense", type="bf16", rows=1, n_in=4096, n_out=16384, act="silu"),
        # A minibatch through the hidden layer of the 784-128-10 perceptron, pre-activations kept: the smallest training call.
        _case("dense_minibatch", "dense", rows=32, n_in=784, n_out=128, act="relu", pre=True),
        # The whole 28x28 training set through the same layer: evaluating a model.
        _case("dense_evaluation", "dense", rows=60000, n_in=784, n_out=128, act="relu"),
        # A large batch through a wide layer with everything in its epilogue: training at scale, the largest call.
        _case("dense_large", "dense", type="bf16", rows=8192, n_in=4096, n_out=16384, act="gelu", residual=True, pre=True, rate=0.1),
        # Odd sizes and rows that start on no boundary.
        _case("dense_ragged", "dense", type="f16", rows=1003, n_in=785, n_out=1017, act="silu", residual=True, rate=0.25, pad=2),
        # The gradient of a large square layer.
        _case("dense_back_large", "dense_back", type="bf16", rows=8192, n_in=4096, n_out=4096, act="gelu"),
        # The gradient of an odd fp32 layer with dropout, a batch of a few hundred.
        _case("dense_back_ragged", "dense_back", rows=777, n_in=785, n_out=131, act="relu", rate=0.5, pad=1),
        # Ten classes over the whole 28x28 training set: many short rows.
        _case("loss_ten_classes", "loss", rows=60000, n_out=10),
        # A large vocabulary: long rows, each read once.
        _case("loss_large", "loss", type="bf16", rows=8192, n_out=65536),
        # A handful of long odd rows.
        _case("loss_few_rows", "loss", type="f32", rows=5, n_out=50001, pad=3),
        # Hidden states of a large batch on their way to the residual stream.
        _case("dropout_large", "dropout", type="bf16", rows=8192, n_out=8192, rate=0.1, residual=True),
        # The activations of a small odd batch.
        _case("dropout_odd", "dropout", rows=129, n_out=1001, rate=0.5, pad=1),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(["dense", "dense", "dense_back", "loss", "dropout"])
    c = dict(type=rng.choice(["f32", "bf16", "bf16", "f16"]), pad=rng.choice([0, 0, 0, 1, 2, 8]))
    if op in ("dense", "dense_back"):
        while True:
            r, i, o = _log_int(rng, 1, 60000), _log_int(rng, 8, 8192), _log_int(rng, 2, 16384)
            if r * i * o <= LARGEST // (8 if op == "dense_back" else 4) and r * max(i, o) <= 1 << 27:
                break
        if rng.random() < 0.5:      # widths of models are often multiples of sixteen
            i, o = -(-i // 16) * 16, -(-o // 16) * 16
        c.update(rows=r, n_in=i, n_out=o, act=rng.choice(["none", "relu", "relu", "gelu", "silu"]), rate=rng.choice([0.0, 0.0, 0.1, 0.5]))
        if op == "dense":
            c.update(residual=rng.random() < 0.4, pre=rng.random() < 0.4, bias=rng.random() < 0.8)
    elif op == "loss":
        n = _log_int(rng, 2, 131072)
        c.update(n_out=n, rows=_log_int(rng, 1, min(100000, (1 << 28) // n)))
    else:
        n = _log_int(rng, 1, 16384)
        c.update(n_out=n, rows=_log_int(rng, 1, min(100000, (1 << 26) // n)), rate=rng.choice([0.1, 0.2, 0.5, rng.uniform(0.01, 0.9)]),
                 residual=rng.random() < 0.5)
    return _case(None, op, **c)


def _matrix(rows, cols, pad, dtype, fill=None):
    """[rows, cols] of rows cols + pad elements apart."""
    m = torch.empty(rows, cols + pad, dtype=dtype, device="cuda")[:, :cols]
    if fill is not None:
        m.copy_(fill)
    return m


def _inputs(case, seed):
    """The tensors of a case, from the seed alone."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    t, pad = TYPES[case["type"]], case["pad"]
    r, i, o = case["rows"], case["n_in"], case["n_out"]

    def normal(rows, cols, scale=1.0):
        return _matrix(rows, cols, pad, t, torch.randn(rows, cols, generator=g, device="cuda") * scale)

    d = {}
    if case["op"] in ("dense", "dense_back"):
        # inputs as a layer behind another sees them: about half of them at zero
        d["x"] = _matrix(r, i, pad, t, torch.randn(r, i, generator=g, device="cuda").clamp_(min=0.0))
        d["w"] = _matrix(i, o, pad, t, (torch.rand(i, o, generator=g, device="cuda") * 2 - 1) * (3.0 / i) ** 0.5)
        if case["op"] == "dense":
            d["bias"] = (torch.randn(o, generator=g, device="cuda") * 0.1).to(t) if case["bias"] else None
            d["residual"] = normal(r, o) if case["residual"] else None
        else:
            d["z"] = normal(r, o, 0.7)
            d["dy"] = normal(r, o, 0.01)
    elif case["op"] == "loss":
        d["logits"] = normal(r, o, 2.0)
        d["labels"] = torch.randint(0, max(1, o - o // 50), (r,), generator=g, device="cuda", dtype=torch.int32)
        d["labels"][torch.rand(r, generator=g, device="cuda") < 0.05] = -1      # rows without an answer
        if o // 50:
            d["logits"][:, o - o // 50:] = float("-inf")                        # entries a vocabulary is padded with
    else:
        d["x"] = normal(r, o)
        d["residual"] = normal(r, o) if case["residual"] else None
    return d


def prepare(case, seed):
    s = dict(case=case, seed=seed, **_inputs(case, seed))
    if own:
        from paper_2112_13935_b200 import api
        t, pad = TYPES[case["type"]], case["pad"]
        r, i, o = case["rows"], case["n_in"], case["n_out"]
        drop = api.aet_dropout_spec(seed=seed, client=7, counter=1 << 33, rate=case["rate"])
        if case["op"] in ("dense", "dense_back"):
            s["plan"] = api.aet_dense(i, o, dtype=t, act=case["act"], dropout=drop, ld_in=i + pad, ld_out=o + pad, ld_w=o + pad)
            need = api.aet_dense_workspace(s["plan"], r, backward=case["op"] == "dense_back")
            s["workspace"] = torch.empty(need, dtype=torch.uint8, device="cuda")
        s["drop"] = drop
        if case["op"] == "dense":
            s["y"], s["pre"] = _matrix(r, o, pad, t), _matrix(r, o, pad, t) if case["pre"] else None
        elif case["op"] == "dense_back":
            s["dx"], s["dw"], s["db"] = _matrix(r, i, pad, t), _matrix(i, o, pad, t), torch.empty(o, dtype=t, device="cuda")
        elif case["op"] == "loss":
            s["loss"], s["top"] = torch.empty(r, device="cuda"), torch.empty(r, dtype=torch.int32, device="cuda")
            s["grad"] = _matrix(r, o, pad, t)
        else:
            s["y"] = _matrix(r, o, pad, t)
    return s


# ---- the plain forms ----------------------------------------------------------------------------------------------------

_M64 = (1 << 64) - 1


def _signed(v):
    v &= _M64
    return v - (1 << 64) if v >> 63 else v


def _mix(z):
    """The SplitMix64 output function on int64 tensors (products wrap; shifts without the sign)."""
    z = (z ^ ((z >> 30) & ((1 << 34) - 1))) * _signed(0xBF58476D1CE4E5B9)
    z = (z ^ ((z >> 27) & ((1 << 37) - 1))) * _signed(0x94D049BB133111EB)
    return z ^ ((z >> 31) & ((1 << 33) - 1))


_GAMMA = 0x9E3779B97F4A7C15


def _kept(case, seed):
    """Which elements stay: sixteen bits each, four to a draw, a row's draws one after another; and the factor of those that do."""
    rows, cols = case["rows"], case["n_out"]
    q = int(math.floor(float(torch.tensor(case["rate"], dtype=torch.float32)) * 65536 + 0.5))
    one = lambda v: int(_mix(torch.tensor(_signed(v), dtype=torch.int64)))      # noqa: E731
    key = one(one(seed + _GAMMA * 5) + _GAMMA * 8)                              # stream 4, client 7
    groups = (cols + 3) // 4
    n = torch.arange(rows * groups, device="cuda", dtype=torch.int64)
    bits = _mix(n * _signed(_GAMMA) + _signed(key + _GAMMA * ((1 << 33) + 1)))
    lanes = torch.arange(4, device="cuda", dtype=torch.int64) * 16
    kept = (((bits.view(rows, groups, 1) >> lanes) & 0xFFFF) >= q).view(rows, groups * 4)[:, :cols]
    return kept, 65536.0 / (65536 - q)


def _act(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * 0.5 ** 0.5))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * 0.5 ** 0.5)) + z * torch.exp(-0.5 * z * z) * (2 * math.pi) ** -0.5
    if act == "silu":
        s = 1 / (1 + torch.exp(-z))
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


def _plain(s):
    c = s["case"]
    t = TYPES[c["type"]]
    if c["op"] == "dense":
        z = s["x"].float() @ s["w"].float()
        if s["bias"] is not None:
            z = z + s["bias"].float()
        y = _act(z, c["act"])
        if c["rate"]:
            kept, factor = _kept(c, s["seed"])
            y = torch.where(kept, y * factor, 0.0)
        if s["residual"] is not None:
            y = y + s["residual"].float()
        return dict(y=y.to(t), **(dict(pre=z.to(t)) if c["pre"] else {}))
    if c["op"] == "dense_back":
        dz = s["dy"].float() * _slope(s["z"].float(), c["act"])
        if c["rate"]:
            kept, factor = _kept(c, s["seed"])
            dz = torch.where(kept, dz * factor, 0.0)
        return dict(dx=(dz @ s["w"].float().t()).to(t), dw=(s["x"].float().t() @ dz).to(t), db=dz.sum(0).to(t))
    if c["op"] == "loss":
        z, labels = s["logits"].float(), s["labels"].long()
        used = labels >= 0
        at = labels.clamp(min=0)[:, None]
        top = z.amax(1, keepdim=True)
        e = torch.exp(z - top)
        total = e.sum(1, keepdim=True)
        loss = (torch.log(total) + top - z.gather(1, at))[:, 0]
        grad = e / total
        grad.scatter_add_(1, at, torch.full_like(total, -1.0))
        places = torch.arange(z.shape[1], device="cuda", dtype=torch.int32)
        best = torch.where(z == top, places, z.shape[1]).amin(1).to(torch.int32)
        grad = grad * (1.0 / c["rows"])
        return dict(loss=torch.where(used, loss, 0.0), grad=torch.where(used[:, None], grad, 0.0).to(t), top=torch.where(used, best, -1))
    kept, factor = _kept(c, s["seed"])
    y = torch.where(kept, s["x"].float() * factor, 0.0)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return dict(y=y.to(t))


def run(s):
    if not own:
        return _plain(s)
    from paper_2112_13935_b200 import api
    c = s["case"]
    if c["op"] == "dense":
        api.aet_dense_forward(s["plan"], s["x"], s["w"], s["bias"], s["y"], residual=s["residual"], pre=s["pre"], workspace=s["workspace"])
        return dict(y=s["y"], **(dict(pre=s["pre"]) if c["pre"] else {}))
    if c["op"] == "dense_back":
        api.aet_dense_backward(s["plan"], s["x"], s["w"], s["dy"], pre=s["z"], dx=s["dx"], dw=s["dw"], db=s["db"], workspace=s["workspace"])
        return dict(dx=s["dx"], dw=s["dw"], db=s["db"])
    if c["op"] == "loss":
        api.aet_cross_entropy(s["logits"], s["labels"], loss=s["loss"], dlogits=s["grad"], top=s["top"], scale=1.0 / c["rows"])
        return dict(loss=s["loss"], grad=s["grad"], top=s["top"])
    api.aet_dropout(s["drop"], s["x"], s["y"], residual=s["residual"])
    return dict(y=s["y"])


def work(case):
    b = 4 if case["type"] == "f32" else 2
    r, i, o = case["rows"], case["n_in"], case["n_out"]
    if case["op"] == "dense":
        return dict(bytes=b * (r * i + i * o + o * case["bias"] + r * o * (1 + case["residual"] + case["pre"])), flops=2 * r * i * o)
    if case["op"] == "dense_back":
        return dict(bytes=b * (2 * (r * i + i * o + r * o) + o), flops=4 * r * i * o)
    if case["op"] == "loss":
        return dict(bytes=2 * b * r * o + 12 * r, flops=5 * r * o)
    return dict(bytes=b * r * o * (2 + case["residual"]), flops=2 * r * o)


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------------

def _mask64(case, seed):
    """dropout's factor an element, in 64 bits: numpy's unsigned arithmetic, from the definition of the generator."""
    import numpy as np

    def mix(z):
        z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
        z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
        return z ^ (z >> np.uint64(31))

    with np.errstate(over="ignore"):
        gamma = np.uint64(0x9E3779B97F4A7C15)
        key = mix(mix(np.uint64(seed) + gamma * np.uint64(5)) + gamma * np.uint64(8))
        rows, cols = case["rows"], case["n_out"]
        per = (cols + 3) // 4
        draws = mix(key + gamma * (np.arange(rows * per, dtype=np.uint64) + np.uint64((1 << 33) + 1)))
    words = draws.astype("<u8").view("<u2").reshape(rows, per * 4)[:, :cols]
    q = int(math.floor(float(np.float32(case["rate"])) * 65536 + 0.5))
    return torch.from_numpy(np.ascontiguousarray(words).astype(np.int32)).cuda().ge(q).double() * (65536.0 / (65536 - q))


def exact(case, seed):
    s = _inputs(case, seed)
    d = {k: v.double() if v is not None and v.is_floating_point() else v for k, v in s.items()}
    act = case["act"]
    if case["op"] == "dense":
        z = torch.mm(d["x"], d["w"])
        if d["bias"] is not None:
            z += d["bias"]
        if act == "relu":
            y = torch.where(z > 0, z, 0.0)
        elif act == "gelu":
            y = z * torch.special.ndtr(z)
        elif act == "silu":
            y = z * torch.sigmoid(z)
        else:
            y = z.clone()
        if case["rate"]:
            y *= _mask64(case, seed)
        if d["residual"] is not None:
            y += d["residual"]
        return dict(y=y, pre=z) if case["pre"] else dict(y=y)
    if case["op"] == "dense_back":
        z = d["z"]
        if act == "relu":
            slope = torch.where(z > 0, 1.0, 0.0).double()
        elif act == "gelu":
            slope = torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
        elif act == "silu":
            slope = torch.sigmoid(z) + z * torch.sigmoid(z) * torch.sigmoid(-z)
        else:
            slope = torch.ones_like(z)
        dz = slope * d["dy"]
        if case["rate"]:
            dz *= _mask64(case, seed)
        return dict(dx=torch.mm(dz, d["w"].t()), dw=torch.mm(d["x"].t(), dz), db=dz.sum(0))
    if case["op"] == "loss":
        rows, step = case["rows"], max(1, (1 << 27) // case["n_out"])
        loss, grad = torch.zeros(rows, dtype=torch.float64, device="cuda"), torch.zeros(rows, case["n_out"], dtype=torch.float64, device="cuda")
        for a in range(0, rows, step):
            z, y = s["logits"][a:a + step].double(), s["labels"][a:a + step].long()
            logp = torch.log_softmax(z, 1)
            used = y >= 0
            n = torch.arange(z.shape[0], device="cuda")
            loss[a:a + step] = torch.where(used, -logp[n, y.clamp(min=0)], 0.0)
            p = logp.exp_()
            p[n, y.clamp(min=0)] -= 1
            grad[a:a + step] = torch.where(used[:, None], p / rows, 0.0)
        return dict(loss=loss, grad=grad, top=None)
    y = d["x"] * _mask64(case, seed)
    if d["residual"] is not None:
        y = y + d["residual"]
    return dict(y=y)
