"""Results in place of operands: with another pitch rows would overwrite rows that are still to be read, so the call is refused.
Addresses that nothing is launched with."""
import ctypes
import itertools

import pytest

A, B, C, D, E = (0x10000 * (i + 1) for i in range(5))


@pytest.fixture(scope="module")
def eqat():
    from paper_2407_11062_b200.build import build_library
    build_library()
    from paper_2407_11062_b200 import binding
    return binding


@pytest.mark.parametrize("which", ["q", "k"])
@pytest.mark.parametrize("pitches", [(256, 512), (768, 256), (264, 256)])
def test_rotary(eqat, which, pitches):
    d = eqat.make_rotary_desc(2, 4, 4, 64)
    for f in (eqat.lib.eqat_rotary_fwd, eqat.lib.eqat_rotary_bwd):
        q, k, q_out, k_out = (A, pitches[0]), (B, 256), (C, 256), (D, 256)
        if which == "q":
            q_out = (A, pitches[1])
        else:
            q, k, k_out = (A, 256), (B, pitches[0]), (B, pitches[1])
        assert f(ctypes.byref(d), *q, *k, E, E, None, None, *q_out, *k_out, None) == eqat.EQAT_ERR_SHAPE


def test_gated(eqat):
    d = eqat.make_gated_desc(2, 64)
    fwd, bwd = (lambda *p, f=f: f(ctypes.byref(d), *p, None) for f in (eqat.lib.eqat_gated_fwd, eqat.lib.eqat_gated_bwd))
    assert fwd(A, 128, B, 64, A) == fwd(A, 64, B, 72, B) == eqat.EQAT_ERR_SHAPE           # H is dense
    for source, out in itertools.product(range(3), range(2)):
        ins, outs = [[A, 64], [B, 128], [C, 136]], [[D, 64], [E, 64]]
        outs[out] = [ins[source][0], ins[source][1] + 64]
        assert bwd(A, *ins[1], *ins[2], *outs[0], *outs[1]) == eqat.EQAT_ERR_SHAPE
