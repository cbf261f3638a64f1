"""Every shape of tile that the gradient of a gated feed-forward block takes, its contraction whole and in parts.

Which tiles, and how many parts, follow the sizes and the number of SMs; the host tells (eqat_packed_gated_tile).  The problems below
reach every kernel that the library has for a B200 of 148 SMs, which is checked without a GPU, and on a GPU each has to take the
same tiles there.  Bounds as in test_gpu_gated.py."""
import ctypes

import numpy as np
import pytest
import torch

from helpers import Guarded, assert_elementwise, contraction_bound, torch_to_f64
from test_gpu_gated import act_code, both_weights, check_grads, eqat, normal  # noqa: F401

SMS = 148
SINGLE, WIDE, PAIR = (128, 128, 1), (256, 256, 1), (256, 256, 2)
# tokens, out, width, bits, group, fp16 zero points, activation: tile, parts
CASES = {
    (1, 64, 128, 2, 64, False, "silu"): (SINGLE, 1), (1, 1088, 128, 2, 128, True, "gelu"): (SINGLE, 2),
    (3, 64, 128, 3, 32, True, "gelu_tanh"): (SINGLE, 1), (5, 1088, 128, 3, 64, False, "silu"): (SINGLE, 2),
    (2, 64, 128, 4, 128, True, "silu"): (SINGLE, 1), (7, 1088, 128, 4, 32, False, "gelu"): (SINGLE, 2),
    # 256 rows on one CTA: 129 to 256 tokens of most models' blocks; parts of one length, and of two
    (640, 64, 9600, 2, 64, True, "silu"): (WIDE, 1), (640, 64, 9600, 3, 128, False, "gelu"): (WIDE, 1), (640, 64, 9600, 4, 32, True, "silu"): (WIDE, 1),
    (129, 2624, 5120, 2, 64, False, "silu"): (WIDE, 5), (250, 1600, 9600, 3, 128, True, "gelu_tanh"): (WIDE, 3), (150, 1600, 9600, 4, 64, False, "silu"): (WIDE, 3),
    (130, 11008, 4096, 2, 64, False, "silu"): (WIDE, 8), (200, 11008, 4096, 3, 128, False, "silu"): (WIDE, 8), (256, 11008, 4096, 4, 32, True, "silu"): (WIDE, 8),
    # pairs of CTAs
    (130, 64, 9600, 2, 128, False, "silu"): (PAIR, 1), (130, 64, 9600, 3, 64, True, "silu"): (PAIR, 1), (130, 64, 9600, 4, 128, True, "gelu"): (PAIR, 1),
    (1029, 2112, 768, 2, 256, True, "silu"): (PAIR, 4), (1029, 2240, 768, 3, 32, False, "gelu"): (PAIR, 4), (1029, 2368, 768, 4, 768, True, "gelu_tanh"): (PAIR, 4),
    (512, 11008, 4096, 3, 128, False, "silu"): (PAIR, 4),
}


def described(eqat, case):  # noqa: F811
    T, out, width, bits, group, fp16, _ = case
    return eqat.make_desc(bits, group, out, width, T, 0, eqat.EQAT_ZP_FP16 if fp16 else eqat.EQAT_ZP_U8)


def test_the_cases_are_every_kernel(eqat):  # noqa: F811
    reached = set()
    for case, (tile, parts) in CASES.items():
        d = described(eqat, case)
        assert eqat.eqat_packed_gated_tile(d, eqat.EQAT_OP_PACKED_GATED_BWD, SMS) == (*tile, parts), case
        reached.add((case[3], tile, parts > 1))
    every = set()
    for bits in (2, 3, 4):
        for out in (64, 320, 1088, 2048, 4096, 11008, 28672):
            for width in (128, 768, 2048, 4096, 9600):
                for T in (1, 64, 130, 200, 257, 512, 640, 1029, 2500, 20000):
                    *tile, parts = eqat.eqat_packed_gated_tile(eqat.make_desc(bits, 128, out, width, T), eqat.EQAT_OP_PACKED_GATED_BWD, SMS)
                    every.add((bits, tuple(tile), parts > 1))
    assert reached == every and len(every) == 18


def test_the_parts_are_those_of_the_workspace(eqat):  # noqa: F811
    for T, out, width in ((1, 64, 128), (200, 11008, 4096), (700, 11008, 4096), (4096, 11008, 4096)):
        d = eqat.make_desc(2, 64, out, width, T)
        parts = eqat.eqat_packed_gated_tile(d, eqat.EQAT_OP_PACKED_GATED_BWD)[3]
        assert eqat.workspace_bytes(d, eqat.EQAT_OP_PACKED_GATED_BWD) == (4 * parts * T * width if parts > 1 else 0)


def test_what_the_diagnostic_refuses(eqat):  # noqa: F811
    d, tile = eqat.make_desc(2, 64, 256, 256, 100), (ctypes.c_int * 4)()
    call = lambda d, op, sms, t: eqat.lib.eqat_packed_gated_tile(d and ctypes.byref(d), op, sms, t)  # noqa: E731
    for op in (0, eqat.EQAT_OP_FAKEQUANT_BWD, eqat.EQAT_OP_PACKED_BWD_DS, 5):
        assert call(d, op, 0, tile) == eqat.EQAT_ERR_UNSUPPORTED
    for op in (eqat.EQAT_OP_PACKED_GATED_FWD, eqat.EQAT_OP_PACKED_GATED_BWD):
        assert call(None, op, 0, tile) == call(d, op, 0, None) == eqat.EQAT_ERR_NULL
        assert call(d, op, -1, tile) == eqat.EQAT_ERR_SHAPE
        assert call(eqat.make_desc(2, 64, 96, 256, 100), op, 0, tile) == eqat.EQAT_ERR_SHAPE
    assert eqat.eqat_packed_gated_tile(eqat.make_desc(2, 64, 11008, 4096, 4096), eqat.EQAT_OP_PACKED_GATED_FWD, SMS) == (256, 256, 2, 1)


@pytest.mark.gpu
@pytest.mark.parametrize("case", list(CASES))
def test_gradient(eqat, case):  # noqa: F811
    T, out, width, bits, group, fp16, kind = case
    d, act = described(eqat, case), act_code(eqat, kind)
    assert eqat.eqat_packed_gated_tile(d, eqat.EQAT_OP_PACKED_GATED_BWD) == (*CASES[case][0], CASES[case][1])
    gate, up = both_weights(out, width, bits, group, fp16)
    dH, G, U, buf = normal(T, out, seed=4, std=0.1), normal(T, out, seed=5, std=1.5), normal(T, out, seed=6), Guarded()
    dX, dG, dU = buf.empty(T, width, dtype=torch.bfloat16, shift_bytes=16), *(buf.empty(T, out, dtype=torch.bfloat16) for _ in range(2))
    need = eqat.workspace_bytes(d, eqat.EQAT_OP_PACKED_GATED_BWD)
    ws = buf.empty(need, dtype=torch.uint8) if need else None
    eqat.qlinear_packed_gated_bwd(d, act, dH, G, U, gate.on, up.on, dX, dG, dU, ws)
    buf.check()
    assert eqat.device_status() == (0, 0)
    few = slice(0, 64)                                              # the element-wise part has tests of its own
    check_grads(*(torch_to_f64(t[few]) for t in (dG, dU, dH, G, U)), kind)
    dev = [(t.double(), torch.from_numpy(np.asarray(w.value, np.float64)).cuda()) for t, w in ((dG, gate), (dU, up))]
    ref, size, square = (sum(f(y) @ f(w) for y, w in dev).cpu().numpy() for f in (lambda t: t, torch.abs, torch.square))
    assert_elementwise(torch_to_f64(dX), ref, contraction_bound(ref, size, square), "dX")
    if need:                                                        # nothing is kept in the workspace: the same bits again
        first = dX.clone()
        ws.fill_(0xFF)
        eqat.qlinear_packed_gated_bwd(d, act, dH, G, U, gate.on, up.on, dX.zero_(), dG, dU, ws)
        assert torch.equal(dX, first)
