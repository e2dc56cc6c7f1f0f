"""Plain 64-bit forms of the layer operators, and how far the library may be from them.

Rounding to a type is off by at most half a step, u = finfo(type).eps / 2 relative (and half of the smallest subnormal).
fp32 sums of K terms are off by at most K + 16 steps of 2^-23 of the sum of the terms' magnitudes: every addition loses less than
a step of its result (tensor cores cut, they do not round), a product of three-part operands 2^-22 of itself."""
import math

import numpy as np
import torch

TYPES = dict(f32=torch.float32, bf16=torch.bfloat16, f16=torch.float16)
HALF_STEP = {t: torch.finfo(t).eps / 2 for t in TYPES.values()}
TINY = {torch.float32: 2.0 ** -140, torch.bfloat16: 2.0 ** -130, torch.float16: 2.0 ** -25}


def kept(rows, cols, seed, client, counter, rate):
    """(mask [rows, cols], factor) by the definition: oracle arithmetic on the framework's generator."""
    from oracle import rng
    q = int(math.floor(float(np.float32(rate)) * 65536 + 0.5))
    per = (cols + 3) // 4
    with np.errstate(over="ignore"):
        z = np.uint64(rng.stream_key(seed, 4, client)) + np.uint64(0x9E3779B97F4A7C15) * (
            np.uint64(counter & (2 ** 64 - 1)) + np.arange(rows * per, dtype=np.uint64) + np.uint64(1))
        z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
        z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
        z = z ^ (z >> np.uint64(31))
    bits = np.stack([(z >> np.uint64(16 * i)) & np.uint64(0xFFFF) for i in range(4)], 1).reshape(rows, per * 4)[:, :cols]
    return bits >= q, 65536.0 / (65536 - q)


_erf = np.vectorize(math.erf, otypes=[float])


def act(z, name):
    if name == "relu":
        return np.where(z > 0, z, 0.0)
    if name == "gelu":
        return 0.5 * z * (1 + _erf(z / math.sqrt(2)))
    if name == "silu":
        return z / (1 + np.exp(-z))
    return z


def slope(z, name):
    if name == "relu":
        return (z > 0).astype(float)
    if name == "gelu":
        return 0.5 * (1 + _erf(z / math.sqrt(2))) + z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "silu":
        s = 1 / (1 + np.exp(-z))
        return s * (1 + z * (1 - s))
    return np.ones_like(z)


def matrix(values, dtype, pad=0, shift=0):
    """A CUDA matrix with these values, rows `pad` elements longer than its columns, `shift` elements off the buffer's start, and its
    buffer (the elements between rows hold 77)."""
    rows, cols = values.shape
    ld = cols + pad
    buf = torch.full((rows * ld + shift + 8,), 77.0, dtype=dtype, device="cuda")
    m = buf[shift:shift + rows * ld].view(rows, ld)[:, :cols]
    m.copy_(torch.as_tensor(values))
    return m, buf


def gaps_untouched(m, buf, pad, shift):
    """The elements around and between the rows of a matrix() still hold 77."""
    rows, cols = m.shape
    b = buf.clone()
    b[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols] = 77.0
    return bool((b == 77.0).all())


def host(t):
    return t.detach().cpu().double().numpy()


def assert_close(got, want, dtype, slack, what=""):
    """|got - want| <= slack + half a step of the type, entry by entry."""
    got = host(got) if torch.is_tensor(got) else got
    bound = slack + HALF_STEP[dtype] * (np.abs(want) + slack) + TINY[dtype]
    err = np.abs(got - want)
    bad = ~(err <= bound)
    assert not bad.any(), (what, int(bad.sum()), float(np.nanmax(err / bound)), tuple(np.argwhere(bad)[0]))
