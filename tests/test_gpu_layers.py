"""Layer operators against plain 64-bit forms: every type, odd sizes, gaps between rows, odd addresses, each option."""
import numpy as np
import pytest
import torch

import layer_helpers as lh
from paper_2112_13935_b200 import api

pytestmark = pytest.mark.gpu

STEP = 2.0 ** -23


def layer_inputs(rows, n_in, n_out, dtype, seed):
    r = np.random.default_rng(seed)
    q = lambda a: torch.as_tensor(a).to(dtype).double().numpy()   # noqa: E731  the values the type holds
    return dict(x=q(np.maximum(r.standard_normal((rows, n_in)), 0)), w=q(r.uniform(-1, 1, (n_in, n_out)) * (3 / n_in) ** 0.5),
                bias=q(r.standard_normal(n_out) * 0.1), residual=q(r.standard_normal((rows, n_out))), dy=q(r.standard_normal((rows, n_out))),
                pre=q(r.standard_normal((rows, n_out))))


def workspace(plan, rows, backward):
    n = api.aet_dense_workspace(plan, rows, backward)
    return torch.full((n + 256,), 0xFF, dtype=torch.uint8, device="cuda")[:n]     # (NaN in every type)


def check_forward(rows, n_in, n_out, type, act="none", bias=True, residual=False, pre=False, rate=0.0, pad=0, shift=0, seed=1, in_place=False):
    t = lh.TYPES[type]
    d = layer_inputs(rows, n_in, n_out, t, seed)
    drop = api.aet_dropout_spec(seed=seed, client=3, counter=2 ** 40 + 5, rate=rate)
    plan = api.aet_dense(n_in, n_out, dtype=t, act=act, dropout=drop, ld_in=n_in + pad, ld_out=n_out + pad, ld_w=n_out + pad,
                         flags=api.DENSE_ANY_ADDRESS if shift else 0)
    x, _ = lh.matrix(d["x"], t, pad, shift)
    w, _ = lh.matrix(d["w"], t, pad, shift)
    b = torch.as_tensor(d["bias"]).to(t).cuda() if bias else None
    res = lh.matrix(d["residual"], t, pad, shift) if residual else (None, None)
    y, ybuf = res if in_place else lh.matrix(np.zeros((rows, n_out)), t, pad, shift)
    z, zbuf = lh.matrix(np.zeros((rows, n_out)), t, pad, shift) if pre else (None, None)
    api.aet_dense_forward(plan, x, w, b, y, residual=res[0], pre=z, workspace=workspace(plan, rows, False))
    torch.cuda.synchronize()
    size = np.abs(d["x"]) @ np.abs(d["w"]) + (np.abs(d["bias"]) if bias else 0)
    slack = (n_in + 16) * STEP * size
    want = d["x"] @ d["w"] + (d["bias"] if bias else 0)
    if pre:
        lh.assert_close(z, want, t, slack, "pre")
        assert lh.gaps_untouched(z, zbuf, pad, shift)
    # the activations' slopes stay below 1.13 and their own error below four steps of their argument's magnitude
    want, slack = lh.act(want, act), 1.13 * slack + 4 * STEP * size
    if rate:
        mask, factor = lh.kept(rows, n_out, seed, 3, 2 ** 40 + 5, rate)
        want, slack = np.where(mask, want * factor, 0), np.where(mask, slack * factor + 2 * STEP * np.abs(want * factor), 0)
    if residual:
        want, slack = want + d["residual"], slack + STEP * (np.abs(want) + np.abs(d["residual"]))
    lh.assert_close(y, want, t, slack, "y")
    assert lh.gaps_untouched(y, ybuf, pad, shift)


SHAPES = [(1, 1, 1), (1, 7, 3), (2, 64, 64), (5, 65, 130), (33, 784, 10), (64, 100, 37), (65, 785, 128), (130, 33, 257), (300, 256, 65)]


@pytest.mark.parametrize("type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,n_in,n_out", SHAPES)
def test_dense_forward_sizes(rows, n_in, n_out, type):
    check_forward(rows, n_in, n_out, type, act="relu", pre=True)


@pytest.mark.parametrize("type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,n_in,n_out", [(1, 1, 1000), (1, 520, 8), (2, 16384, 70), (3, 5000, 2049), (8, 300, 1000), (8, 16384, 9), (1, 20000, 300), (7, 64, 20000)])
@pytest.mark.parametrize("over", [dict(act="silu", pre=True), dict(pad=1, residual=True, rate=0.2), dict(pad=8, shift=1, residual=True, in_place=True)])
def test_dense_forward_few_rows(rows, n_in, n_out, type, over):
    check_forward(rows, n_in, n_out, type, **over)


@pytest.mark.parametrize("type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("over", [
    dict(act="none", bias=False), dict(act="gelu", residual=True), dict(act="silu", rate=0.3), dict(act="relu", rate=0.5, residual=True, pre=True),
    dict(pad=1, act="gelu", residual=True, pre=True), dict(pad=3, shift=1, rate=0.1, residual=True, pre=True), dict(pad=8, act="silu"),
    dict(residual=True, in_place=True, act="relu"), dict(rate=0.9999), dict(rate=2.0 ** -18)])
def test_dense_forward_options(type, over):
    check_forward(70, 131, 94, type, **over)


# products the tensor cores take: odd edges of tiles and of k, few rows, a long k in parts, enough tiles for pairs of CTAs
LARGE = [(300, 785, 300), (129, 1000, 640), (1, 8192, 8200), (70, 20000, 200), (4001, 131, 130), (2305, 72, 2100), (257, 513, 1024), (2049, 2048, 2056)]


@pytest.mark.parametrize("type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,n_in,n_out", LARGE)
def test_dense_forward_large(rows, n_in, n_out, type):
    check_forward(rows, n_in, n_out, type, act="relu", pre=True)


@pytest.mark.parametrize("type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,n_in,n_out", [(300, 785, 300), (100, 9000, 130), (2305, 72, 2100), (9, 5000, 3001), (65, 700, 5002)])
@pytest.mark.parametrize("over", [dict(pad=1, residual=True, act="silu", pre=True), dict(pad=3, shift=1, rate=0.1, residual=True), dict(pad=8, bias=False, residual=True, in_place=True)])
def test_dense_forward_large_options(rows, n_in, n_out, type, over):
    check_forward(rows, n_in, n_out, type, **over)


def check_backward(rows, n_in, n_out, type, act="none", rate=0.0, pad=0, shift=0, accumulate=False, want=("dx", "dw", "db"), seed=2):
    t = lh.TYPES[type]
    d = layer_inputs(rows, n_in, n_out, t, seed)
    drop = api.aet_dropout_spec(seed=seed, client=0, counter=9, rate=rate)
    flags = (api.DENSE_ANY_ADDRESS if shift else 0) | (api.DENSE_ACCUMULATE if accumulate else 0)
    plan = api.aet_dense(n_in, n_out, dtype=t, act=act, dropout=drop, ld_in=n_in + pad, ld_out=n_out + pad, ld_w=n_out + pad, flags=flags)
    at = {k: lh.matrix(d[k], t, pad, shift)[0] for k in ("x", "w", "dy", "pre")}
    before = dict(dx=np.zeros((rows, n_in)), dw=d["w"] * 3, db=d["bias"][None])
    before = {k: torch.as_tensor(v).to(t).double().numpy() for k, v in before.items()}
    out = {k: lh.matrix(before[k], t, 0 if k == "db" else pad, shift) for k in want}
    args = {k: (v[0][0] if k == "db" else v[0]) for k, v in out.items()}
    api.aet_dense_backward(plan, at["x"] if "dw" in want else None, at["w"] if "dx" in want else None, at["dy"],
                           pre=None if act == "none" else at["pre"], workspace=workspace(plan, rows, True), **args)
    torch.cuda.synchronize()
    dz = d["dy"] * lh.slope(d["pre"], act)
    off = 8 * STEP * np.abs(d["dy"])              # the slopes are below 1.13, and off by a few steps
    if rate:
        mask, factor = lh.kept(rows, n_out, seed, 0, 9, rate)
        dz, off = np.where(mask, dz * factor, 0), np.where(mask, off * factor + 2 * STEP * np.abs(dz * factor), 0)
    in_type = off + (0 if act == "none" and not rate else lh.HALF_STEP[t] * np.abs(dz) + lh.TINY[t])   # dz as the products take it
    plus = {k: before[k] if accumulate and k != "dx" else 0 for k in before}
    if "dx" in want:
        size = np.abs(dz) @ np.abs(d["w"]).T
        lh.assert_close(out["dx"][0], dz @ d["w"].T, t, in_type @ np.abs(d["w"]).T + (n_out + 16) * STEP * size, "dx")
    if "dw" in want:
        size = np.abs(d["x"]).T @ np.abs(dz) + np.abs(plus["dw"])
        lh.assert_close(out["dw"][0], d["x"].T @ dz + plus["dw"], t, np.abs(d["x"]).T @ in_type + (rows + 16) * STEP * size, "dw")
    if "db" in want:
        size = np.abs(dz).sum(0)[None] + np.abs(plus["db"])
        lh.assert_close(out["db"][0], dz.sum(0)[None] + plus["db"], t, off.sum(0)[None] + (rows + 16) * STEP * size, "db")
    for k, (m, buf) in out.items():
        assert lh.gaps_untouched(m, buf, 0 if k == "db" else pad, shift), k


@pytest.mark.parametrize("type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,n_in,n_out", SHAPES)
def test_dense_backward_sizes(rows, n_in, n_out, type):
    check_backward(rows, n_in, n_out, type, act="relu")


@pytest.mark.parametrize("type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("over", [
    dict(), dict(act="gelu"), dict(act="silu", rate=0.3), dict(act="relu", rate=0.5, pad=1), dict(act="gelu", pad=3, shift=1),
    dict(act="relu", accumulate=True, pad=8), dict(accumulate=True), dict(want=("dw",)), dict(want=("dx",), act="silu"), dict(want=("db",), act="relu"),
    dict(want=("dw", "db"), rate=0.2)])
def test_dense_backward_options(type, over):
    check_backward(90, 77, 139, type, **over)


@pytest.mark.parametrize("type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,n_in,n_out", LARGE)
def test_dense_backward_large(rows, n_in, n_out, type):
    check_backward(rows, n_in, n_out, type, act="relu")


@pytest.mark.parametrize("type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,n_in,n_out", [(300, 785, 300), (9000, 100, 130), (72, 2305, 2100)])
@pytest.mark.parametrize("over", [dict(), dict(pad=1), dict(pad=8), dict(pad=3, shift=1, act="silu", rate=0.1), dict(accumulate=True, act="relu"), dict(want=("dw",), pad=8), dict(want=("dx", "db"))])
def test_dense_backward_large_options(rows, n_in, n_out, type, over):
    check_backward(rows, n_in, n_out, type, **over)


def test_dense_backward_over_no_rows_is_zero():
    plan = api.aet_dense(5, 3, ld_w=4)
    dw, buf = lh.matrix(np.ones((5, 3)), torch.float32, 1)
    db = torch.ones(3, device="cuda")
    empty = lambda n: torch.empty(0, n, device="cuda")   # noqa: E731
    w, _ = lh.matrix(np.ones((5, 3)), torch.float32, 1)
    api.aet_dense_backward(plan, empty(5), w, empty(3), dx=empty(5), dw=dw, db=db)
    api.aet_dense_forward(plan, empty(5), w, None, empty(3))
    torch.cuda.synchronize()
    assert not dw.any() and not db.any() and lh.gaps_untouched(dw, buf, 1, 0)


def test_dense_gradient_agrees_with_differences():
    """fp32 forward passes at both sides of a step against the backward pass: F = sum of dy * y."""
    rows, n_in, n_out = 9, 20, 14
    d = layer_inputs(rows, n_in, n_out, torch.float32, 5)
    c = {k: torch.as_tensor(v).float().cuda() for k, v in d.items()}
    plan = api.aet_dense(n_in, n_out, act="silu", dropout=api.aet_dropout_spec(seed=1, rate=0.25))
    y, pre = torch.empty(rows, n_out, device="cuda"), torch.empty(rows, n_out, device="cuda")

    def F(x, w, b):
        api.aet_dense_forward(plan, x, w, b, y, pre=pre)
        return float((y.double() * c["dy"].double()).sum())

    F(c["x"], c["w"], c["bias"])
    g = dict(dx=torch.empty_like(c["x"]), dw=torch.empty_like(c["w"]), db=torch.empty_like(c["bias"]))
    api.aet_dense_backward(plan, c["x"], c["w"], c["dy"], pre=pre, workspace=workspace(plan, rows, True), **g)
    # a step of 2^-6: the third derivative of silu stays below 0.31 and |x|, |w| below 4, so the difference quotient is off by at most
    # 2^-12 / 6 * 0.31 * 64 * sum |dy| factor < 0.002 sum |dy|; fp32 rounding adds 2^-20 sum |y dy| * 2^6
    h = 2.0 ** -6
    for k, name in enumerate(("x", "w", "bias")):
        for at in [(0,), (3,)] if name == "bias" else [(0, 0), (4, 7), (8, 13)]:
            side = []
            for sign in (1, -1):
                v = [c["x"].clone(), c["w"].clone(), c["bias"].clone()]
                v[k][at] += sign * h
                side.append(F(*v))
            got = float(g["d" + {"x": "x", "w": "w", "bias": "b"}[name]][at])
            assert abs((side[0] - side[1]) / (2 * h) - got) <= 0.003 * float(c["dy"].abs().sum()) / n_out + 2.0 ** -13, (name, at)


@pytest.mark.parametrize("type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
def test_activations_and_slopes_at_extreme_values(act, type):
    """The type's largest and lowest values and zeros of both signs through a 1 x 1 layer of weight 1: finite, and a slope of 0 or 1 far out."""
    t = lh.TYPES[type]
    top = torch.finfo(t).max
    z = torch.tensor([top, -top, 0.0, -0.0, 60.0, -60.0], device="cuda").to(t)[:, None]
    rows, one = z.shape[0], torch.ones(1, 1, dtype=t, device="cuda")
    plan = api.aet_dense(1, 1, dtype=t, act=act)
    y, dx = torch.empty_like(z), torch.empty_like(z)
    for n in (rows, 1):                                      # the FMA kernel's rows stand for all kernels: one epilogue; a single row has its own
        api.aet_dense_forward(plan, z[:n], one, None, y[:n], workspace=workspace(plan, n, False))
    api.aet_dense_backward(plan, z, one, torch.ones_like(z), pre=z, dx=dx, workspace=workspace(plan, rows, True))
    assert torch.equal(y[:2, 0], torch.stack([z[0, 0], torch.zeros_like(z[0, 0])])) and not y[2:4].any()
    assert dx[0] == 1 and dx[1] == 0 and float(dx[2]) == float(dx[3]) == {"relu": 0.0, "gelu": 0.5, "silu": 0.5}[act]
    assert y[4] == z[4] and dx[4] == 1 and abs(float(y[5])) <= 1e-20 and abs(float(dx[5])) <= 1e-20


# ---- loss ----------------------------------------------------------------------------------------------------------------

def loss_reference(z, labels, scale, weight):
    """loss, gradient and top in 64 bits, with the rules for rows that have none."""
    rows, n = z.shape
    loss, grad, top = np.zeros(rows), np.zeros((rows, n)), np.full(rows, -1)
    for r in range(rows):
        y = labels[r]
        if y < 0:
            continue
        if not np.isnan(z[r]).any():
            top[r] = int(np.argmax(z[r]))
        m = z[r].max()
        if np.isnan(z[r]).any() or np.isinf(m) or y >= n:
            loss[r], grad[r] = np.nan, np.nan
            continue
        e = np.exp(z[r] - m)
        with np.errstate(divide="ignore"):
            loss[r] = np.log(e.sum()) + m - z[r, y]
        grad[r] = e / e.sum()
        grad[r, y] -= 1
        grad[r] *= scale * (1 if weight is None else weight[r])
    return loss, grad, top


def check_loss(z, labels, type, scale=1.0, weight=None, pad=0, shift=0, in_place=False, outs=("loss", "dlogits", "top")):
    t = lh.TYPES[type]
    rows, n = z.shape
    with np.errstate(invalid="ignore"):
        z = torch.as_tensor(z).to(t).double().numpy()
    logits, lbuf = lh.matrix(z, t, pad, shift)
    y = torch.as_tensor(np.asarray(labels, dtype=np.int32)).cuda()
    w = None if weight is None else torch.as_tensor(weight).float().cuda()
    got = dict(loss=torch.full((rows,), 5.0, device="cuda"), top=torch.full((rows,), 5, dtype=torch.int32, device="cuda"))
    got["dlogits"], gbuf = (logits, lbuf) if in_place else lh.matrix(np.ones((rows, n)), t, pad, shift)
    api.aet_cross_entropy(logits, y, weight=w, scale=scale, **{k: got[k] for k in outs})
    torch.cuda.synchronize()
    want = dict(zip(("loss", "dlogits", "top"), loss_reference(z, labels, scale, None if weight is None else np.asarray(weight, np.float32).astype(float))))
    # exp is off by 2^-22 of itself and the difference under it by 2^-24 of itself; adding n of them in any order by n 2^-24
    spread = np.nan_to_num(np.where(np.isinf(z), 0, np.abs(z)).max(1), nan=0.0) * 2
    rel = (n + 16) * 2.0 ** -24 + 2.0 ** -21 + spread * 2.0 ** -23
    for k in outs:
        if k == "top":
            assert np.array_equal(got["top"].cpu().numpy(), want["top"])
            continue
        a, b = lh.host(got[k]), want[k]
        assert np.array_equal(np.isnan(a), np.isnan(b)), k
        assert np.array_equal(np.isinf(a), np.isinf(b)) and (a[np.isinf(b)] > 0).all(), k
        fine = np.isfinite(b)
        if k == "loss":
            slack = rel + 2.0 ** -22 * (np.abs(np.where(fine, b, 0)) + spread)
            off = np.abs(a[fine] - b[fine])
            assert (off <= slack[fine]).all(), (off / slack[fine]).max()
        else:
            wgt = scale * (np.ones(rows) if weight is None else np.abs(weight))
            with np.errstate(invalid="ignore"):
                slack = (4 * rel * wgt)[:, None] * (np.abs(b) / np.maximum(wgt, 1e-300)[:, None]) + (2.0 ** -22 * wgt)[:, None] * (np.arange(n)[None] == np.asarray(labels)[:, None])
            lh.assert_close(a[fine], b[fine], t, slack[fine], k)
    if "dlogits" in outs:
        assert lh.gaps_untouched(got["dlogits"], gbuf, pad, shift)


@pytest.mark.parametrize("type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,n", [(1, 1), (3, 2), (7, 10), (300, 10), (33, 31), (40, 33), (9, 100), (5, 257), (3, 1000), (2, 1025), (3, 4099), (2, 30001), (1, 131072), (200, 9000), (1, 300007), (1, 1000003), (2400, 3000), (1200, 5003)])
def test_loss_sizes(rows, n, type):
    r = np.random.default_rng(rows * 1000 + n)
    z = r.standard_normal((rows, n)) * 2
    labels = r.integers(0, n, rows)
    labels[rows // 2] = -1 if rows > 2 else labels[rows // 2]
    check_loss(z, labels, type, scale=1.0 / rows)


@pytest.mark.parametrize("type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n", [10, 37, 700, 5003])
@pytest.mark.parametrize("over", [dict(pad=1), dict(pad=3, shift=1), dict(pad=8), dict(in_place=True), dict(weighted=True), dict(outs=("loss",)),
                                  dict(outs=("dlogits",)), dict(outs=("top",))])
def test_loss_options(type, n, over):
    r = np.random.default_rng(n)
    over = dict(over)
    if over.pop("weighted", False):
        over["weight"] = r.uniform(0, 2, 12).astype(np.float32)
    check_loss(r.standard_normal((12, n)), r.integers(-1, n, 12), type, scale=0.125, **over)


@pytest.mark.parametrize("type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n", [2, 10, 70, 2500, 9001])
def test_loss_of_odd_rows(n, type):
    """Infinities, NaN, the type's lowest value, ties, labels that are none: every rule of the header."""
    r = np.random.default_rng(7)
    low = torch.finfo(lh.TYPES[type]).min
    z = r.standard_normal((14, n))
    labels = np.full(14, n - 1)
    z[0, : n - 1] = -np.inf                     # one class left
    z[1] = -np.inf                              # none left
    z[2, 0] = np.inf
    z[3, n // 2] = np.nan
    z[4] = np.nan; labels[4] = -1               # not read
    z[5] = low                                  # a mask of the lowest value that leaves nothing: uniform
    z[6, : n - 1] = low
    z[7] = 1.0                                  # ties: the first
    labels[8] = n                               # no such class
    labels[9] = -2 ** 31
    z[10, n - 1] = -np.inf                      # the label itself cannot be: loss inf
    z[11, 0] = -torch.finfo(lh.TYPES[type]).min / 2    # one class far above the rest
    labels[11] = 0
    z[12] = r.standard_normal(n) * 1e-3 + 500   # far from zero
    z[13, 1] = np.nan
    z[13, 0] = np.inf
    check_loss(z, labels, type)


# ---- dropout -------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 3), (3, 4), (5, 9), (129, 1001), (64, 64), (700, 128), (2, 70000), (30000, 12)])
@pytest.mark.parametrize("over", [dict(rate=0.5), dict(rate=0.1, residual=True), dict(rate=0.0), dict(rate=0.9999, pad=1, shift=1, residual=True), dict(rate=0.3, pad=4, in_place="x"), dict(rate=0.3, residual=True, in_place="residual")])
def test_dropout(rows, cols, type, over):
    t = lh.TYPES[type]
    r = np.random.default_rng(cols)
    q = lambda a: torch.as_tensor(a).to(t).double().numpy()   # noqa: E731
    pad, shift, rate = over.get("pad", 0), over.get("shift", 0), over["rate"]
    xv, rv = q(r.standard_normal((rows, cols))), q(r.standard_normal((rows, cols)))
    if rate:
        mask, factor = lh.kept(rows, cols, 11, 5, 2 ** 64 - 3, rate)    # (the counter wraps)
        xv[~mask] = np.nan                                     # a dropped element is zero whatever it was
    else:
        mask, factor = np.ones((rows, cols), bool), 1.0
    x, xbuf = lh.matrix(xv, t, pad, shift)
    res, rbuf = lh.matrix(rv, t, pad, shift) if over.get("residual") else (None, None)
    place = over.get("in_place")
    y, ybuf = (x, xbuf) if place == "x" else (res, rbuf) if place else lh.matrix(np.zeros((rows, cols)), t, pad, shift)
    api.aet_dropout(api.aet_dropout_spec(11, 5, 2 ** 64 - 3, rate), x, y, residual=res)
    torch.cuda.synchronize()
    want = np.where(mask, xv * factor, 0)
    slack = 2 * STEP * np.abs(want)
    if res is not None:
        want, slack = want + rv, slack + STEP * (np.abs(want) + np.abs(rv))
    lh.assert_close(y, want, t, slack)
    assert lh.gaps_untouched(y, ybuf, pad, shift)


def test_dropout_rate_is_what_was_asked():
    """q of 65,536 in expectation; five standard deviations either way, and rows, columns and lanes alike."""
    rows, cols = 512, 1024
    y = torch.empty(rows, cols, device="cuda")
    for rate in (0.1, 0.5, 0.75):
        api.aet_dropout(api.aet_dropout_spec(3, rate=rate), torch.ones(rows, cols, device="cuda"), y)
        gone = (y == 0).double()
        for share, n in ((gone.mean(), rows * cols), (gone[:, ::4].mean(), rows * cols / 4), (gone[:, 3::4].mean(), rows * cols / 4)):
            assert abs(float(share) - rate) <= 5 * (rate * (1 - rate) / n) ** 0.5 + 2.0 ** -17


# ---- together, streams, graphs -------------------------------------------------------------------------------------------

def training_step(c, plans, ws, out):
    """Two layers, the loss, and all gradients."""
    p1, p2 = plans
    api.aet_dense_forward(p1, c["x"], c["w1"], c["b1"], out["h"], pre=out["z"], workspace=ws[0])
    api.aet_dense_forward(p2, out["h"], c["w2"], c["b2"], out["logits"], workspace=ws[1])
    api.aet_cross_entropy(out["logits"], c["labels"], loss=out["loss"], dlogits=out["g"], top=out["top"], scale=1 / c["x"].shape[0])
    api.aet_dense_backward(p2, out["h"], c["w2"], out["g"], dx=out["gh"], dw=out["dw2"], db=out["db2"], workspace=ws[2])
    api.aet_dense_backward(p1, c["x"], c["w1"], out["gh"], pre=out["z"], dw=out["dw1"], db=out["db1"], workspace=ws[3])


def step_state(rows, dims, dtype, seed, rate):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n0, n1, n2 = dims
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")   # noqa: E731
    c = dict(x=rnd(rows, n0).to(dtype), w1=(rnd(n0, n1) / n0 ** 0.5).to(dtype), b1=rnd(n1).to(dtype), w2=(rnd(n1, n2) / n1 ** 0.5).to(dtype),
             b2=rnd(n2).to(dtype), labels=torch.randint(0, n2, (rows,), generator=g, device="cuda", dtype=torch.int32))
    plans = (api.aet_dense(n0, n1, dtype=dtype, act="gelu", dropout=api.aet_dropout_spec(seed, rate=rate)), api.aet_dense(n1, n2, dtype=dtype))
    ws = [torch.empty(api.aet_dense_workspace(p, rows, b), dtype=torch.uint8, device="cuda") for b in (False, True) for p in plans]
    ws = [ws[0], ws[1], ws[3], ws[2]]
    e = lambda *s: torch.empty(*s, dtype=dtype, device="cuda")   # noqa: E731
    out = dict(h=e(rows, n1), z=e(rows, n1), logits=e(rows, n2), g=e(rows, n2), gh=e(rows, n1), dw1=e(n0, n1), db1=e(n1), dw2=e(n1, n2), db2=e(n2),
               loss=torch.empty(rows, device="cuda"), top=torch.empty(rows, dtype=torch.int32, device="cuda"))
    return c, plans, ws, out


@pytest.mark.parametrize("rows,dims,rate", [(50, (100, 64, 10), 0.0), (257, (784, 130, 37), 0.2)])
def test_a_training_step_against_autograd_in_64_bits(rows, dims, rate):
    c, plans, ws, out = step_state(rows, dims, torch.float32, 4, rate)
    training_step(c, plans, ws, out)
    leaf = {k: c[k].double().requires_grad_() for k in ("w1", "b1", "w2", "b2")}
    h = torch.nn.functional.gelu(c["x"].double() @ leaf["w1"] + leaf["b1"])
    if rate:
        mask, factor = lh.kept(rows, dims[1], 4, 0, 0, rate)
        h = h * torch.as_tensor(mask).cuda() * factor
    logits = h @ leaf["w2"] + leaf["b2"]
    loss = torch.nn.functional.cross_entropy(logits, c["labels"].long(), reduction="none")
    loss.mean().backward()
    # fp32 sums of up to 784 terms twice on the way in and as many on the way back: some 1e-6, against the largest entry
    for got, want in [(out["loss"], loss)] + [(out["d" + k], leaf[k].grad) for k in leaf]:
        want = want.detach()
        assert float((got.double() - want).abs().max() / want.abs().max()) <= 2e-5
    assert torch.equal(out["top"].long(), out["logits"].argmax(1))


def test_a_training_step_repeats_bit_for_bit_on_streams_and_in_graphs():
    c, plans, ws, out = step_state(200, (300, 96, 33), torch.bfloat16, 8, 0.1)
    training_step(c, plans, ws, out)
    torch.cuda.synchronize()
    first = {k: v.clone() for k, v in out.items()}
    side = torch.cuda.Stream()
    for v in out.values():
        v.zero_()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        training_step(c, plans, ws, out)
    side.synchronize()
    assert all(torch.equal(first[k], out[k]) for k in out)
    # two graphs of two states, each with its own workspaces, replayed at the same time
    states = [(c, plans, ws, out), step_state(200, (300, 96, 33), torch.bfloat16, 9, 0.3)]
    training_step(*states[1])
    torch.cuda.synchronize()
    want = [first, {k: v.clone() for k, v in states[1][3].items()}]
    graphs = []
    for st in states:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            training_step(*st)
        graphs.append(g)
    for st in states:
        for v in st[3].values():
            v.zero_()
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    for _ in range(3):
        graphs[0].replay()
        with torch.cuda.stream(other):
            graphs[1].replay()
        torch.cuda.synchronize()
    for st, w in zip(states, want):
        assert all(torch.equal(w[k], st[3][k]) for k in w)


# ---- offsets past 32 bits, first calls in a capture -----------------------------------------------------------------------

def far(rows, cols, ld, dtype, values=None):
    """A matrix whose last row starts more than 2^31 elements behind its first."""
    assert (rows - 1) * ld >= 2 ** 31
    m = torch.empty((rows - 1) * ld + cols, dtype=dtype, device="cuda").as_strided((rows, cols), (ld, 1))
    if values is not None:
        m.copy_(values)
    return m


@pytest.mark.parametrize("rows,n_in,n_out,type", [(3, 200, 90, "bf16"), (20, 70, 33, "bf16"), (130, 640, 900, "f16"), (130, 1024, 1100, "f32")])
def test_dense_of_rows_far_apart(rows, n_in, n_out, type):
    """Few rows, FMAs, tensor cores: the same bits as with rows side by side."""
    t = lh.TYPES[type]
    ld = -(-2 ** 31 // (rows - 1)) // 8 * 8 + 8
    g = torch.Generator(device="cuda").manual_seed(1)
    x, w, dy = (torch.randn(a, b, generator=g, device="cuda").to(t) for a, b in ((rows, n_in), (n_in, n_out), (rows, n_out)))
    near = api.aet_dense(n_in, n_out, dtype=t, act="silu")
    apart = api.aet_dense(n_in, n_out, dtype=t, act="silu", ld_x=ld, ld_pre=ld)
    got = []
    for plan, xx, pre in ((near, x, torch.empty(rows, n_out, dtype=t, device="cuda")), (apart, far(rows, n_in, ld, t, x), far(rows, n_out, ld, t))):
        y, dx, dw = torch.empty_like(dy), torch.empty_like(x), torch.empty_like(w)
        api.aet_dense_forward(plan, xx, w, None, y, pre=pre, workspace=workspace(plan, rows, False))
        api.aet_dense_backward(plan, xx, w, dy, pre=pre, dx=dx, dw=dw, workspace=workspace(plan, rows, True))
        got.append((y, pre, dx, dw))
    for a, b in zip(*got):
        assert torch.equal(a, b)


def test_loss_and_dropout_of_rows_far_apart():
    ld, t = 2 ** 30 + 4, torch.bfloat16
    g = torch.Generator(device="cuda").manual_seed(2)
    z = torch.randn(3, 1001, generator=g, device="cuda").to(t)
    labels = torch.tensor([3, 0, 1000], dtype=torch.int32, device="cuda")
    zz = far(3, 1001, ld, t, z)
    out = []
    for m in (z, zz):
        loss, grad = torch.empty(3, device="cuda"), torch.empty(3, 1001, dtype=t, device="cuda")
        api.aet_cross_entropy(m, labels, loss=loss, dlogits=grad)
        y = torch.empty(3, 1001, dtype=t, device="cuda")
        api.aet_dropout(api.aet_dropout_spec(1, rate=0.5), m, y)
        out.append((loss, grad, y))
    for a, b in zip(*out):
        assert torch.equal(a, b)
    api.aet_cross_entropy(zz, labels, dlogits=zz)
    assert torch.equal(zz, out[0][1])


FIRST_CALLS = """
import sys, torch
sys.path[:0] = [%r]
from paper_2112_13935_b200 import api
t = torch.bfloat16
x, w, dy = (torch.ones(a, b, dtype=t, device='cuda') for a, b in ((512, 768), (768, 640), (512, 640)))
plan = api.aet_dense(768, 640, dtype=t, act='relu')
ws = [torch.empty(api.aet_dense_workspace(plan, 512, b), dtype=torch.uint8, device='cuda') for b in (False, True)]
y, dx, dw, db = dy.clone(), x.clone(), w.clone(), dy[0].clone()
labels, grad = torch.zeros(512, dtype=torch.int32, device='cuda'), dy.clone()
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    api.aet_dense_forward(plan, x, w, None, y, workspace=ws[0])
    api.aet_cross_entropy(y, labels, dlogits=grad)
    api.aet_dense_backward(plan, x, w, dy, pre=y, dx=dx, dw=dw, db=db, workspace=ws[1])
    api.aet_dropout(api.aet_dropout_spec(1, rate=0.5), dx, dx)
g.replay()
torch.cuda.synchronize()
assert (y == 768).all() and (dw == 512).all() and (db == 512).all() and set(dx.unique().tolist()) == {0.0, 1280.0}
print('fine')
"""


def test_first_calls_of_a_process_inside_a_capture():
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST_CALLS % root], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "fine" in r.stdout, r.stderr[-2000:]


def test_two_streams_at_once():
    """Calls that overlap on the GPU, each with its own workspace, give what they give alone."""
    states = [step_state(700, (900, 640, 70), torch.bfloat16, seed, 0.2) for seed in (1, 2)]
    want = []
    for st in states:
        training_step(*st)
        torch.cuda.synchronize()
        want.append({k: v.clone() for k, v in st[3].items()})
    streams = [torch.cuda.Stream() for _ in states]
    for _ in range(5):
        for st, s in zip(states, streams):
            with torch.cuda.stream(s):
                training_step(*st)
    torch.cuda.synchronize()
    for st, w in zip(states, want):
        assert all(torch.equal(w[k], st[3][k]) for k in w)


# ---- a wait that gives up ------------------------------------------------------------------------------------------------

# type, rows, n_in, n_out; stages a tile has, tiles of the first CTA (or pair), and the sums of a tile
LOST = [("bf16", 2560, 640, 2304, 10, 2, 256 * 256),        # pairs of CTAs
        ("f16", 1536, 320, 1536, 5, 1, 128 * 128),          # single CTAs
        ("f16", 1024, 768, 1024, 6, 1, 128 * 128),          # ... and k in two parts
        ("f32", 20000, 256, 128, 8, 2, 128 * 128),
        ("f32", 8000, 512, 64, 8, 1, 128 * 64),             # 64 columns at a time, k in two parts
        ("f32", 64, 1024, 4096, 8, 1, 128 * 64)]            # transposed, k in four


@pytest.mark.parametrize("type,rows,n_in,n_out,stages,tiles,sums", LOST)
def test_lost_copies_leave_nan_in_their_tiles_alone(type, rows, n_in, n_out, stages, tiles, sums):
    t = lh.TYPES[type]
    g = torch.Generator(device="cuda").manual_seed(rows)
    x, w = (torch.randn(n, generator=g, device="cuda").to(t) for n in ((rows, n_in), (n_in, n_out)))
    plan = api.aet_dense(n_in, n_out, dtype=t)
    ws = workspace(plan, rows, False)
    want, y = torch.empty(rows, n_out, dtype=t, device="cuda"), torch.empty(rows, n_out, dtype=t, device="cuda")
    api.aet_dense_forward(plan, x, w, None, want, workspace=ws)
    assert not want.isnan().any()
    for lost in (0, 1, stages - 1, stages, stages + 1, tiles * stages):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        api.aet_debug_dense_lost_copies(plan, x, w, y, ws, lost, 2000)
        b.record()
        torch.cuda.synchronize()
        assert a.elapsed_time(b) < 2000
        none = y.isnan()
        assert int(none.sum()) == (tiles - min(tiles, lost // stages)) * sums, lost
        assert torch.equal(y[~none], want[~none])
        y.fill_(3.0)
        api.aet_dense_forward(plan, x, w, None, y, workspace=ws)       # the next call is as ever
        assert torch.equal(y, want)


def test_lost_copies_refusals():
    x = torch.zeros(4, 8, device="cuda")
    for status, args in ((2, (0, 100)), (1, (0, 0)), (1, (0, 10 ** 6 + 1))):      # (a small product waits for nothing)
        with pytest.raises(api.AetError) as e:
            api.aet_debug_dense_lost_copies(api.aet_dense(8, 8), x, torch.zeros(8, 8, device="cuda"), x, None, *args)
        assert e.value.status == status


@pytest.mark.parametrize("type,rows,n_in,n_out", [("bf16", 2 ** 26 + 5, 8, 8), ("f16", 2 ** 22 + 3, 1024, 2400), ("f32", 2 ** 26 + 5, 8, 8)])
def test_weight_gradient_over_very_many_rows(type, rows, n_in, n_out):
    """Terms of one sign, where every addition that cuts loses a little: at most 2^17 of k go into one sum in tensor memory, 16 at a time, and
    each addition there loses less than 2^-23 of the sum; the parts are added up rounded to nearest (fp32: sums of 64 are)."""
    t = lh.TYPES[type]
    g = torch.Generator(device="cuda").manual_seed(rows)
    x, dy = (torch.empty(rows, n, dtype=t, device="cuda") for n in (n_in, n_out))
    for m in (x, dy):
        for part in m.split(1 << 22):
            part.copy_(torch.rand(part.shape, generator=g, device="cuda") * 2 ** -6)
    want = sum(a.double().t() @ b.double() for a, b in zip(x[:, :16].split(1 << 22), dy[:, :16].split(1 << 22)))
    plan = api.aet_dense(n_in, n_out, dtype=t)
    dw = torch.empty(n_in, n_out, dtype=t, device="cuda")
    api.aet_dense_backward(plan, x, None, dy, dw=dw, workspace=workspace(plan, rows, True))
    parts = -(-rows // 2 ** 17)
    cut = (parts + (2 ** 17 / 64 if type == "f32" else 0)) * 2.0 ** -24 + (24 * 2.0 ** -23 if type == "f32" else 2 ** 17 / 16 * 2.0 ** -23)
    off = float(((dw[:16, :16].double() - want) / want).abs().max())
    assert off <= cut + lh.HALF_STEP[t]


@pytest.mark.parametrize("type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,n_in,n_out", [(3, 100, 300), (40, 70, 90), (300, 785, 300), (8000, 512, 64), (70, 1024, 4100), (2560, 640, 2304)])
@pytest.mark.parametrize("value", [float("inf"), float("nan")])
def test_infinities_stay_in_their_rows_and_columns(rows, n_in, n_out, type, value):
    """Non-finite operands: their row or column of sums is not finite, every other sum as without them; every product kernel."""
    t = lh.TYPES[type]
    g = torch.Generator(device="cuda").manual_seed(rows)
    x, w, dy = (torch.randn(n, generator=g, device="cuda").to(t) for n in ((rows, n_in), (n_in, n_out), (rows, n_out)))
    plan = api.aet_dense(n_in, n_out, dtype=t)

    def run(x, w, dy):
        y, dx, dw, db = (torch.empty(n, dtype=t, device="cuda") for n in ((rows, n_out), (rows, n_in), (n_in, n_out), (n_out,)))
        api.aet_dense_forward(plan, x, w, None, y, workspace=workspace(plan, rows, False))
        api.aet_dense_backward(plan, x, w, dy, dx=dx, dw=dw, db=db, workspace=workspace(plan, rows, True))
        return y, dx, dw, db

    want = run(x, w, dy)
    assert all(v.isfinite().all() for v in want)
    r, i, o = rows - 1, n_in // 2, n_out - 1
    for name, at in (("x", (r, i)), ("w", (i, o)), ("dy", (r, o))):
        m = dict(x=x.clone(), w=w.clone(), dy=dy.clone())
        m[name][at] = value
        got = run(**m)
        hit = [torch.zeros_like(v, dtype=torch.bool) for v in want]
        if name == "x":
            hit[0][r], hit[2][i] = True, True
        elif name == "w":
            hit[0][:, o], hit[1][:, i] = True, True
        else:
            hit[1][r], hit[2][:, o], hit[3][o] = True, True, True
        for v, u, h in zip(got, want, hit):
            assert not v[h].isfinite().any() and torch.equal(v[~h], u[~h]), name
