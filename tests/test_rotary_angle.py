"""The header's bound on a rotary angle, against the arithmetic that the kernel does with it (csrc/rotary.cu, read in the source)."""
import os
import re

import numpy as np

from conftest import ROOT


def read(*path):
    return open(os.path.join(ROOT, *path)).read()


def test_the_bound_of_an_angle():
    kernel = read("paper_2407_11062_b200", "csrc", "rotary.cu")
    assert "+ 0x80000000ull;" in kernel and "sincospif((float)(int32_t)(angle >> 32) * 0x1p-31f, &sn, &cs);" in kernel
    text = re.sub(r"\s*\n \* ", " ", read("include", "eqat.h"))
    assert "at most 2^-26 + 2^-33 of a turn" in text
    rng = np.random.default_rng(1)
    exact = np.concatenate([rng.integers(0, 2 ** 64, 200000, dtype=np.uint64), rng.integers(2 ** 62, 2 ** 62 + 2 ** 61, 200000, dtype=np.uint64)])
    rounded = ((exact + np.uint64(2 ** 31)) >> np.uint64(32)).astype(np.uint32).view(np.int32)
    held = rounded.astype(np.float32).astype(np.float64) * 2.0 ** -32
    off = np.abs(held - exact.view(np.int64).astype(np.float64) * 2.0 ** -64)
    off = np.minimum(off, 1 - off)                                  # half a turn either way is the same
    assert off.max() <= 2.0 ** -26 + 2.0 ** -33 + 2.0 ** -53
    assert off.max() > 2.0 ** -28                                   # and not 2^-32 of a turn
