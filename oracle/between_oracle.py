"""CPU oracle of what stands between a block's linears: norm of the residual stream, rotary positions, gated product, and
their gradients.  numpy, float64, from the formulas; decisions that the definitions take in binary32 (codes) are taken there.
Values of bf16 tensors come in as the float64 or float32 numbers that they stand for."""
import math

import numpy as np

E4M3_TOP, INT8_TOP = 448.0, 127.0
SMALL_GROUP = 2.0 ** -110


def erfc(x):
    return np.vectorize(math.erfc, otypes=[np.float64])(x)


# ---------------------------------------------------------------------------------------------- norm
def norm_scale(h, eps):
    h = np.asarray(h, np.float64)
    return 1.0 / np.sqrt((h * h).mean(-1, keepdims=True) + eps)


def norm_fwd(h, w, eps):
    return np.asarray(h, np.float64) * np.asarray(w, np.float64) * norm_scale(h, eps)


def e4m3(x):
    """Nearest e4m3 number, half to even, saturated: 3 mantissa bits, least exponent -6."""
    x = np.asarray(x, np.float64)
    exponent = np.maximum(np.floor(np.log2(np.where(x == 0, 1.0, np.abs(x)))), -6)
    step = 2.0 ** (exponent - 3)
    return np.clip(np.rint(x / step) * step, -E4M3_TOP, E4M3_TOP)


def norm_codes(h, w, eps, group, top):
    """The numbers that the codes are (whole, or e4m3), and the scales [rows, groups] in float64."""
    t = np.asarray(h, np.float32) * np.asarray(w, np.float32)
    t = t.reshape(t.shape[0], -1, group)
    most = np.abs(t).max(-1)
    most = np.where(most < np.float32(SMALL_GROUP), np.float32(0), most)
    up = np.divide(np.float32(top), most, out=np.zeros_like(most), where=most > 0)
    q = t * up[..., None]                                           # binary32
    assert q.dtype == np.float32
    q = np.rint(q).astype(np.float64) if top == INT8_TOP else e4m3(q)
    return q.reshape(np.shape(h)), most.astype(np.float64) * norm_scale(h, eps) / top


def norm_bwd(dy, h, w, eps, dr=None):
    """dx, dw."""
    dy, h, w = (np.asarray(x, np.float64) for x in (dy, h, w))
    c = norm_scale(h, eps)
    v = dy * w
    dx = c * (v - h * c * c * (v * h).mean(-1, keepdims=True))
    return (dx if dr is None else dx + np.asarray(dr, np.float64)), (dy * h * c).sum(0)


# ---------------------------------------------------------------------------------------------- rotary positions
def frequencies(rotary_dim, base=10000.0, kind="plain", factor=1.0, low=0.0, high=0.0, length=0.0):
    out = []
    for i in range(rotary_dim // 2):
        b = base
        if kind == "base" and rotary_dim > 2:
            b = base * factor ** (rotary_dim / (rotary_dim - 2))
        f = b ** (-2 * i / rotary_dim)
        if kind == "linear":
            f = f / factor
        if kind == "ramp":
            k = min(1.0, max(0.0, (length * f / (2 * math.pi) - low) / (high - low)))
            f = k * f + (1 - k) * f / factor
        out.append(f)
    return out


def turns_at(turns, position):
    """The angle of integer turns at a position, radians, from exact integers."""
    return [((int(f) * int(position)) % 2 ** 64) / 2.0 ** 64 * 2 * math.pi for f in turns]


def rotate(x, angles, layout, amplitude=1.0):
    """x [rows, heads, head_dim], angles [rows, pairs]."""
    y = np.array(x, np.float64)
    n = angles.shape[-1]
    ia, ib = (slice(0, n), slice(n, 2 * n)) if layout == "halves" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    a, b = y[..., ia].copy(), y[..., ib].copy()
    c, s = np.cos(angles)[:, None], np.sin(angles)[:, None]
    y[..., ia], y[..., ib] = amplitude * (a * c - b * s), amplitude * (b * c + a * s)
    return y


# ---------------------------------------------------------------------------------------------- gated product
def activation(g, kind):
    """act(g), act'(g), and the sum of the sizes of the derivative's terms."""
    g = np.asarray(g, np.float64)
    with np.errstate(over="ignore"):
        if kind == "silu":
            s = 1 / (1 + np.exp(-g))
            return g * s, s + g * s * (1 - s), s + np.abs(g) * s * (1 - s)
        if kind == "gelu":
            phi, p = erfc(-g / math.sqrt(2)) / 2, np.exp(-g * g / 2) / math.sqrt(2 * math.pi)
            return g * phi, phi + g * p, phi + np.abs(g) * p
        k = 2 * math.sqrt(2 / math.pi)
        s = 1 / (1 + np.exp(-k * (g + 0.044715 * g ** 3)))
        d = k * (1 + 3 * 0.044715 * g * g)
        return g * s, s + g * s * (1 - s) * d, s + np.abs(g) * s * (1 - s) * d


def gated_bwd(dh, g, u, kind):
    """dg, du."""
    dh, u = np.asarray(dh, np.float64), np.asarray(u, np.float64)
    a, slope, _ = activation(g, kind)
    return dh * u * slope, dh * a
