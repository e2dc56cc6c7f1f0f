"""Classification loss of rows whose largest logit is far from zero but not the type's lowest value: masks of -1e9, -1e10 or -1e30 over a whole
row, one large logit among ordinary ones, neighbours a step of the type apart.  Every path: lanes, one CTA, a cluster, rows read again."""
import numpy as np
import pytest
import torch

import layer_helpers as lh
from paper_2112_13935_b200 import api

pytestmark = pytest.mark.gpu

# 2^20 and 2^24 with their neighbours among them: where fp32 values are a sixteenth, and one and two, apart
FAR = [6e4, 1e5, 2.0 ** 20, 1.1e6, 2.0 ** 24, 1.7e7, 1e8, 1e9, 3e9, 1e10, 1e20, 1e30]


def far_rows(n, t, r):
    """(rows, labels): for each distance and sign a row all there, one logit there (the label and not), all but one there, and the label
    there; steps of the type below it."""
    z, labels = [], []

    def add(row, label):
        z.append(row)
        labels.append(label)

    for f in FAR:
        if f > torch.finfo(t).max:
            continue
        f = float(torch.tensor(f).to(t))
        for v in (f, -f):
            add(np.full(n, v), int(r.integers(n)))
            for label in range(2):
                row, at = r.standard_normal(n), int(r.integers(n))
                row[at] = v
                add(row, at if label else (at + 1) % n)
                row = np.full(n, v)
                row[at] = r.standard_normal()
                add(row, at if label else (at + 1) % n)
        step = float(torch.finfo(t).eps) * f          # a step of the type above f's power of two, two below it
        add(f + step * r.integers(-4, 5, n), int(r.integers(n)))
        add(-f + step * r.integers(-4, 5, n), int(r.integers(n)))
    return torch.as_tensor(np.stack(z)).to(t).double().numpy(), np.array(labels, dtype=np.int32)


@pytest.mark.parametrize("type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n", [2, 10, 700, 2500, 5003, 30001, 1000003])
@pytest.mark.parametrize("in_place", [False, True])
def test_loss_of_far_logits(n, type, in_place):
    t = lh.TYPES[type]
    z, labels = far_rows(n, t, np.random.default_rng(n))
    rows = len(labels)
    logits, _ = lh.matrix(z, t)
    grad = logits if in_place else torch.full((rows, n), 3.0, dtype=t, device="cuda")
    loss, top = torch.full((rows,), 5.0, device="cuda"), torch.full((rows,), 5, dtype=torch.int32, device="cuda")
    api.aet_cross_entropy(logits, torch.as_tensor(labels).cuda(), loss=loss, dlogits=grad, top=top, scale=0.5)
    loss, grad = lh.host(loss), lh.host(grad)
    # u = 2^-24.  An exponent x of a power of two has three roundings, 3 u |x|, and matters up to |x| = 152 (2^-150 is nothing in fp32);
    # twice that where the parts of a row are joined.  The power is off by 4 u, a sum of n by n u, products by a few more.
    rel = (n + 2 * 3 * 152 + 24) * 2.0 ** -24
    assert np.array_equal(top.cpu().numpy(), z.argmax(1))
    for r in range(rows):
        m = z[r].max()
        e = np.exp(z[r] - m)
        want = np.log(e.sum()) + (m - z[r, labels[r]])
        assert abs(loss[r] - want) <= rel + 2.0 ** -22 * (abs(want) + 1), (r, z[r, :4], loss[r], want)
        p = e / e.sum()
        slack = 0.5 * (rel * p + 2.0 ** -120)
        slack[labels[r]] += 0.5 * 2.0 ** -22
        p[labels[r]] -= 1
        lh.assert_close(grad[r], 0.5 * p, t, slack, (r, m))
