"""The norm's gradient where the factor c of a row is far from 1: no power of c may be formed that binary32 does not hold.

Bounds.  As in test_gpu_norm.py c is right to 2^-18 of itself where squares are ordinary numbers.  Rows of root mean square 2^-66 have
squares around 2^-132, in steps of 2^-149: rounding each, and their mean, moves the mean by 2^-18 of itself twice, c by half of that.
c enters dx to the third power: 2^-15 covers all of it."""
import numpy as np
import pytest
import torch

from helpers import Guarded, assert_elementwise, torch_to_f64
from oracle import between_oracle as B

pytestmark = pytest.mark.gpu
HALF_STEP, STATS = 2.0 ** -8, 2.0 ** -15


@pytest.fixture(scope="module")
def eqat():
    from paper_2407_11062_b200.build import build_library
    build_library()
    from paper_2407_11062_b200 import binding
    return binding


def normal(*shape, seed):
    return torch.randn(*shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))


# one width of each way to share a row out
@pytest.mark.parametrize("rows,n", [(9, 128), (3, 264), (5, 4096), (2, 16384), (2, 32768)])
@pytest.mark.parametrize("std,eps", [(2.0 ** -66, 0.0), (2.0 ** -64, 0.0), (2.0 ** -40, 1e-30), (0.0, 1e-40), (0.0, 1e-5), (2.0 ** 50, 0.0)])
def test_gradient_of_rows_far_from_one(eqat, rows, n, std, eps):
    H, dY, W = ((normal(rows, n, seed=1) * std).to(torch.bfloat16), normal(rows, n, seed=2).to(torch.bfloat16),
                (1 + 0.3 * normal(n, seed=3)).to(torch.bfloat16))
    dR, buf, d = normal(rows, n, seed=4).to(torch.bfloat16), Guarded(), eqat.make_norm_desc(rows, n, eps)
    dX, Y, dW = (buf.empty(*s, dtype=t) for s, t in (((rows, n), torch.bfloat16), ((rows, n), torch.bfloat16), ((n,), torch.float32)))
    eqat.eqat_rms_norm_fwd(d, H, None, W, None, Y)
    eqat.eqat_rms_norm_bwd(d, dY, H, W, dR, dX, dW, buf.empty(eqat.rms_norm_workspace_bytes(d), dtype=torch.uint8))
    buf.check()
    h, dy, w, dr, eps = (*(torch_to_f64(t) for t in (H, dY, W, dR)), float(np.float32(eps)))
    c = B.norm_scale(h, eps)
    y, (dx, dw), v = B.norm_fwd(h, w, eps), B.norm_bwd(dy, h, w, eps, dr), np.abs(dy * w)
    terms = c * (v + np.abs(h) * c * c * (v * np.abs(h)).mean(-1, keepdims=True)) + np.abs(dr)
    assert_elementwise(torch_to_f64(Y), y, (HALF_STEP + STATS) * np.abs(y) + 2.0 ** -133, "Y")
    assert_elementwise(torch_to_f64(dX), dx, HALF_STEP * np.abs(dx) + STATS * terms + 2.0 ** -133, "dX")
    assert_elementwise(torch_to_f64(dW), dw, STATS * (np.abs(dy * h) * c).sum(0) + 1e-37, "dW")
