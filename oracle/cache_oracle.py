"""CPU oracle of the 4-bit key/value cache and the attention over it (numpy, fp64 sums).

One function per definition of include/eqat.h.  The decisions of the quantiser (step, quotient, code) are taken in binary32
as they are defined; everything else is float64.  It imports nothing from the package.
"""
import numpy as np

f32 = np.float32
STEP_MIN = f32(2.0 ** -126)


def bf16(x):
    """Nearest bf16 value (half to even) of float32 numbers, as float32; NaN stays NaN."""
    x = np.ascontiguousarray(x, f32)
    b = x.view(np.uint32).astype(np.uint64)
    r = (((b + 0x7FFF + ((b >> 16) & 1)) >> 16) << 16).astype(np.uint32).view(f32)
    return np.where(np.isnan(x), f32(np.nan), r).astype(f32)


def quantise(x, group):
    """bf16 values [..., D] (as float32) -> codes [..., D] u8, step and minimum [..., D/group] float32."""
    x = np.asarray(x, f32)
    x = x.reshape(*x.shape[:-1], x.shape[-1] // group, group)
    with np.errstate(all="ignore"):
        low, high = x.min(-1), x.max(-1)                    # NaN if the group holds one
        step = bf16((high - low).astype(f32) * (f32(1) / f32(15)))
        step = np.where(step < STEP_MIN, f32(0), step)
        step = np.where(np.isfinite(step), step, f32(np.nan)).astype(f32)
        inverse = np.where(step > 0, f32(1) / np.where(step > 0, step, f32(1)), f32(0)).astype(f32)
        q = np.rint((x - low[..., None]).astype(f32) * inverse[..., None])
    q = np.clip(np.nan_to_num(q, nan=0.0, posinf=0.0, neginf=0.0), 0, 15).astype(np.uint8)
    return q.reshape(*q.shape[:-2], q.shape[-2] * group), step, low.astype(f32)


def pack(codes):
    """Two codes a byte, the even element in the low half."""
    return (codes[..., 0::2] | (codes[..., 1::2] << 4)).astype(np.uint8)


def unpack(packed):
    return np.stack([packed & 15, packed >> 4], -1).reshape(*packed.shape[:-1], 2 * packed.shape[-1])


def values(codes, step, low):
    """q s + m, float64 [..., D]."""
    g = codes.shape[-1] // step.shape[-1]
    with np.errstate(all="ignore"):
        return codes.astype(np.float64) * np.repeat(step.astype(np.float64), g, -1) + np.repeat(low.astype(np.float64), g, -1)


def places(row_offsets, lengths, page_table, page_size, pages, rows):
    """Sequence, page and place in the page of every row; page -1 where the row has no place, sequence -1 where it belongs
    to none."""
    seq, page, at = np.full(rows, -1), np.full(rows, -1), np.zeros(rows, int)
    for b in range(len(lengths)):
        n = row_offsets[b + 1] - row_offsets[b]
        for i in range(n):
            r, pos = row_offsets[b] + i, lengths[b] - n + i
            seq[r] = b
            if pos >= 0 and 0 <= page_table[b][pos // page_size] < pages:
                page[r], at[r] = page_table[b][pos // page_size], pos % page_size
    return seq, page, at


def attention(Q, keys, vals, lengths, row_offsets, scale, window=0, key_sizes=None, val_sizes=None):
    """Q [rows, q_heads, D], keys/vals: one [length, kv_heads, D] array per sequence (float64) -> O, lse, and what error
    bounds are made of: sum p |v| per output element and the largest |scale| sum_d |Q_d K_jd| of a row, with the given sizes
    (of what a kernel adds up) in the place of |v| and |K|."""
    rows, hq, D = Q.shape
    key_sizes = key_sizes or [np.abs(k) for k in keys]
    val_sizes = val_sizes or [np.abs(v) for v in vals]
    O, lse = np.zeros((rows, hq, D)), np.full((rows, hq), -np.inf)
    mass, size = np.zeros((rows, hq, D)), np.zeros((rows, hq))
    for b, n_keys in enumerate(lengths):
        n, kv = row_offsets[b + 1] - row_offsets[b], keys[b].shape[1]
        for i in range(n):
            pos = n_keys - n + i
            first = max(0, pos - window + 1) if window else 0
            if pos < 0:
                continue
            for h in range(hq):
                r, at = row_offsets[b] + i, (slice(first, pos + 1), h * kv // hq)
                k, v = keys[b][at], vals[b][at]
                z = scale * (k @ Q[r, h])
                p = np.exp(z - z.max())
                lse[r, h] = z.max() + np.log(p.sum())
                p /= p.sum()
                O[r, h], mass[r, h] = p @ v, p @ val_sizes[b][at]
                size[r, h] = abs(scale) * (key_sizes[b][at] @ np.abs(Q[r, h])).max()
    return O, lse, mass, size
