"""Norm, rotary positions and gated product without a device: what the library refuses before it launches anything, the tables of
turns, how a gated call is divided, and the oracle's gradients against differences."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import between_oracle as B


@pytest.fixture(scope="module")
def eqat():
    from paper_2407_11062_b200.build import build_library
    build_library()
    from paper_2407_11062_b200 import binding
    return binding


A = 0x1000                       # an aligned address: nothing is launched where it is refused
ODD = 0x1008


# ---------------------------------------------------------------------------------------------- refusals
NORM = dict(rows=4, features=256, eps=1e-5, codes=0, group=0)


@pytest.mark.parametrize("kw,status", [
    (dict(rows=0), -2), (dict(rows=-1), -2), (dict(rows=(1 << 30) + 1), -2), (dict(features=0), -2), (dict(features=12), -2),
    (dict(features=32776), -2), (dict(eps=-1e-9), -4), (dict(eps=float("nan")), -4), (dict(eps=float("inf")), -4),
    (dict(codes=3), -4), (dict(codes=-1), -4), (dict(group=64), -2), (dict(codes=1), -4), (dict(codes=1, group=48), -4),
    (dict(codes=2, group=16), -4), (dict(codes=2, group=512), -4), (dict(codes=1, group=128, features=192), -2),
])
def test_norm_descriptors(eqat, kw, status):
    d = eqat.make_norm_desc(**{**NORM, **kw})
    codes = (A, A) if kw.get("codes", 0) else (None, None)
    assert eqat.lib.eqat_rms_norm_fwd(ctypes.byref(d), A, A, A, A, A, *codes, None) == status
    assert eqat.lib.eqat_rms_norm_bwd(ctypes.byref(d), A, A, A, A, A, None, None, 0, None) == status
    with pytest.raises(eqat.EqatError):
        eqat.rms_norm_workspace_bytes(d)


def test_norm_pointers(eqat):
    lib, plain = eqat.lib, eqat.make_norm_desc(**NORM)
    coded = eqat.make_norm_desc(4, 256, 1e-5, eqat.EQAT_CODES_INT8, 64)
    fwd = lambda d, *p: lib.eqat_rms_norm_fwd(ctypes.byref(d), *p, None)  # noqa: E731
    bwd = lambda *p: lib.eqat_rms_norm_bwd(ctypes.byref(plain), *p, None)  # noqa: E731
    assert lib.eqat_rms_norm_fwd(None, A, A, A, A, A, None, None, None) == eqat.EQAT_ERR_NULL
    for i in (0, 2, 4):
        p = [A, None, A, None, A, None, None]
        p[i] = None
        assert fwd(plain, *p) == eqat.EQAT_ERR_NULL
    for i in range(5):
        p = [A, A, A, A, A, None, None]
        p[i] = ODD
        assert fwd(plain, *p) == eqat.EQAT_ERR_ALIGN
    assert fwd(plain, A, A, A, A, A, A, None) == eqat.EQAT_ERR_UNSUPPORTED
    assert fwd(plain, A, A, A, A, A, None, A) == eqat.EQAT_ERR_UNSUPPORTED
    assert fwd(coded, A, A, A, A, A, None, A) == eqat.EQAT_ERR_NULL
    assert fwd(coded, A, A, A, A, A, A, None) == eqat.EQAT_ERR_NULL
    assert fwd(coded, A, A, A, A, ODD, A, A) == eqat.EQAT_ERR_ALIGN
    for i in (0, 1, 2, 4):
        p = [A, A, A, None, A, None, None, 0]
        p[i] = None
        assert bwd(*p) == eqat.EQAT_ERR_NULL
    assert bwd(A, A, A, ODD, A, None, None, 0) == eqat.EQAT_ERR_ALIGN
    need = eqat.rms_norm_workspace_bytes(plain)
    assert need > 0
    for ws in ((None, 0), (A, need - 1), (A + 16, need)):
        assert bwd(A, A, A, A, A, A, *ws) == eqat.EQAT_ERR_WORKSPACE


ROTARY = dict(rows=4, q_heads=4, kv_heads=2, head_dim=64, rotary_dim=64, layout=0, amplitude=1.0, sequences=0)


def _rotary(eqat, d, q=A, qp=256, k=A, kp=128, turns=A, pos=A, off=None, lens=None, qo=A, qop=256, ko=A, kop=128):
    got = {f(ctypes.byref(d) if d else None, q, qp, k, kp, turns, pos, off, lens, qo, qop, ko, kop, None)
           for f in (eqat.lib.eqat_rotary_fwd, eqat.lib.eqat_rotary_bwd)}
    assert len(got) == 1
    return got.pop()


@pytest.mark.parametrize("kw,status", [
    (dict(rows=0), -2), (dict(rows=(1 << 30) + 1), -2), (dict(q_heads=0), -2), (dict(kv_heads=-1), -2), (dict(head_dim=60), -2),
    (dict(head_dim=520, rotary_dim=64), -2), (dict(rotary_dim=0), -2), (dict(rotary_dim=33), -2), (dict(rotary_dim=66), -2), (dict(layout=2), -4),
    (dict(sequences=-1), -2), (dict(sequences=(1 << 20) + 1), -2), (dict(amplitude=float("nan")), -4), (dict(amplitude=float("inf")), -4),
])
def test_rotary_descriptors(eqat, kw, status):
    assert _rotary(eqat, eqat.make_rotary_desc(**{**ROTARY, **kw})) == status


def test_rotary_arguments(eqat):
    d = eqat.make_rotary_desc(**ROTARY)
    assert _rotary(eqat, None) == eqat.EQAT_ERR_NULL
    for name in ("q", "k", "turns", "qo", "ko"):
        assert _rotary(eqat, d, **{name: None}) == eqat.EQAT_ERR_NULL
        assert _rotary(eqat, d, **{name: ODD}) == eqat.EQAT_ERR_ALIGN
    for name in ("qp", "kp", "qop", "kop"):
        assert _rotary(eqat, d, **{name: 120}) == eqat.EQAT_ERR_SHAPE
        assert _rotary(eqat, d, **{name: 260}) == eqat.EQAT_ERR_SHAPE
    assert _rotary(eqat, d, pos=ODD) == eqat.EQAT_ERR_ALIGN
    assert _rotary(eqat, d, off=A, lens=A) == eqat.EQAT_ERR_UNSUPPORTED          # both ways to give positions
    assert _rotary(eqat, d, pos=None) == eqat.EQAT_ERR_SHAPE                     # neither
    seqs = eqat.make_rotary_desc(**{**ROTARY, "sequences": 2})
    assert _rotary(eqat, seqs, pos=None, off=A) == eqat.EQAT_ERR_NULL
    assert _rotary(eqat, seqs, pos=None, lens=A) == eqat.EQAT_ERR_NULL


@pytest.mark.parametrize("kw,status", [(dict(rows=0), -2), (dict(features=0), -2), (dict(features=4), -2), (dict(activation=3), -4),
                                       (dict(activation=-1), -4), (dict(rows=(1 << 30) + 1), -2)])
def test_gated_descriptors(eqat, kw, status):
    d = eqat.make_gated_desc(**{**dict(rows=3, features=64, activation=0), **kw})
    assert eqat.lib.eqat_gated_fwd(ctypes.byref(d), A, 64, A, 64, A, None) == status
    assert eqat.lib.eqat_gated_bwd(ctypes.byref(d), A, A, 64, A, 64, A, 64, A, 64, None) == status


def test_gated_arguments(eqat):
    d = eqat.make_gated_desc(3, 64)
    fwd, bwd = (lambda *p, f=f: f(ctypes.byref(d), *p, None) for f in (eqat.lib.eqat_gated_fwd, eqat.lib.eqat_gated_bwd))
    assert eqat.lib.eqat_gated_fwd(None, A, 64, A, 64, A, None) == eqat.EQAT_ERR_NULL
    for pitch in (56, 68, 0, -64):
        assert fwd(A, pitch, A, 64, A) == fwd(A, 64, A, pitch, A) == eqat.EQAT_ERR_SHAPE
        for i in (2, 4, 6, 8):
            p = [A, A, 64, A, 64, A, 64, A, 64]
            p[i] = pitch
            assert bwd(*p) == eqat.EQAT_ERR_SHAPE
    for i in (0, 2, 4):
        for value, status in ((None, -1), (ODD, -3)):
            p = [A, 64, A, 64, A]
            p[i] = value
            assert fwd(*p) == status
    for i in (0, 1, 3, 5, 7):
        for value, status in ((None, -1), (ODD, -3)):
            p = [A, A, 64, A, 64, A, 64, A, 64]
            p[i] = value
            assert bwd(*p) == status


def test_packed_gated_arguments(eqat):
    W = eqat.eqat_packed_weight
    good, desc = W(A, A, A), eqat.make_desc(2, 64, 128, 256, 5)

    def fwd(d=desc, act=0, X=A, gate=good, up=good, H=A, G=A, U=A):
        return eqat.lib.qlinear_packed_gated_fwd(d and ctypes.byref(d), act, X, gate and ctypes.byref(gate), up and ctypes.byref(up), H, G, U, None, 0, None)

    def bwd(d=desc, act=0, dH=A, G=A, U=A, gate=good, up=good, dX=A, dG=A, dU=A, w=A, n=1 << 30):
        return eqat.lib.qlinear_packed_gated_bwd(d and ctypes.byref(d), act, dH, G, U, gate and ctypes.byref(gate), up and ctypes.byref(up), dX, dG, dU, w, n, None)

    for call, names in ((fwd, ("d", "X", "gate", "up", "H", "G", "U")), (bwd, ("d", "dH", "G", "U", "gate", "up", "dX", "dG", "dU"))):
        for name in names:
            assert call(**{name: None}) == eqat.EQAT_ERR_NULL
            if name not in ("d", "gate", "up"):
                assert call(**{name: ODD}) == eqat.EQAT_ERR_ALIGN
        for weight in ("gate", "up"):
            for i in range(3):
                for value, status in ((None, -1), (ODD, -3)):
                    assert call(**{weight: W(*[value if j == i else A for j in range(3)])}) == status
        for act in (-1, 3):
            assert call(act=act) == eqat.EQAT_ERR_UNSUPPORTED
        for d, status in ((eqat.make_desc(5, 64, 128, 256, 5), -4), (eqat.make_desc(2, 64, 96, 256, 5), -2), (eqat.make_desc(2, 64, 128, 200, 5), -2),
                          (eqat.make_desc(2, 64, 128, 256, 0), -2), (eqat.make_desc(2, 512, 128, 1024, 5), -4)):
            assert call(d=d) == status


def test_a_workspace_is_needed_where_the_projections_pass_through_memory(eqat):
    """Checked before any launch, and so without a device."""
    W, seen = eqat.eqat_packed_weight(A, A, A), set()
    for bits in (2, 3, 4):
        for T in (1, 8, 37, 64, 100, 300, 600, 5000, 20000):
            d = eqat.make_desc(bits, 64, 11008, 4096, T)
            need, route = eqat.workspace_bytes(d, eqat.EQAT_OP_PACKED_GATED_FWD), eqat.eqat_packed_gated_route(d, 148)
            seen.add(route)
            rows = eqat.eqat_packed_fwd_route(eqat.make_desc(bits, 64, 22016, 4096, T), 148)[0]
            assert route == rows or (rows, route) == (eqat.EQAT_ROUTE_WEIGHT_ROW_PAIRS, eqat.EQAT_ROUTE_TILED)
            assert (need > 0) == (route == eqat.EQAT_ROUTE_WEIGHT_ROW_PAIRS)
            if need:
                assert need >= 2 * T * 11008 * 2 and need % 512 == 0
                for ws in ((None, need), (A, need - 1), (A + 128, need)):
                    assert eqat.lib.qlinear_packed_gated_fwd(ctypes.byref(d), 0, A, ctypes.byref(W), ctypes.byref(W), A, None, None, *ws, None) == eqat.EQAT_ERR_WORKSPACE
    assert seen == {eqat.EQAT_ROUTE_MATRIX_VECTOR, eqat.EQAT_ROUTE_WEIGHT_ROWS, eqat.EQAT_ROUTE_WEIGHT_ROW_PAIRS, eqat.EQAT_ROUTE_TILED}
    assert eqat.lib.eqat_packed_gated_route(ctypes.byref(eqat.make_desc(2, 64, 256, 256, 4)), -1) == eqat.EQAT_ERR_SHAPE
    for op in (eqat.EQAT_OP_PACKED_GATED_FWD, eqat.EQAT_OP_PACKED_GATED_BWD):
        with pytest.raises(eqat.EqatError):
            eqat.workspace_bytes(eqat.make_desc(2, 64, 96, 256, 5), op)


def test_few_tokens_split_the_contraction(eqat):
    """The parts of the backward pass's sums: at most eight, each with work, none for batches that fill the chip."""
    W = eqat.eqat_packed_weight(A, A, A)
    for out, width in ((64, 128), (192, 384), (1408, 2048), (11008, 4096), (28672, 8192), (64, 9600)):
        for T in (1, 128, 129, 256, 300, 600, 1000, 2000, 4096, 20000):
            d = eqat.make_desc(2, 64, out, width, T)
            need = eqat.workspace_bytes(d, eqat.EQAT_OP_PACKED_GATED_BWD)
            parts, rest = divmod(need, 4 * T * width)
            assert rest == 0 and parts != 1 and parts <= 8 and 2 * out // 64 >= 16 * parts and need <= 64e6
            assert T > 128 or out < 1408 or parts >= 2
            if need:
                for ws in ((None, need), (A, need - 1), (A + 128, need)):
                    assert eqat.lib.qlinear_packed_gated_bwd(ctypes.byref(d), 0, A, A, A, ctypes.byref(W), ctypes.byref(W), A, A, A, *ws, None) == eqat.EQAT_ERR_WORKSPACE


def test_tensors_are_checked_before_the_call(eqat):
    """Types and sizes, without a device: a tensor of the host is refused as such only after them."""
    b = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    d = eqat.make_norm_desc(3, 64, 1e-5, eqat.EQAT_CODES_E4M3, 32)
    for bad in (b(2, 64), torch.zeros(3, 64)):
        with pytest.raises((TypeError, ValueError), match="fewer elements|type"):
            eqat.eqat_rms_norm_fwd(d, bad, None, b(64), None, b(3, 64))
    with pytest.raises(ValueError, match="contiguous CUDA tensor"):
        eqat.eqat_rms_norm_fwd(d, b(3, 64), None, b(64), None, b(3, 64))
    r = eqat.make_rotary_desc(3, 4, 2, 64)
    for q, k in ((b(3, 4, 32), b(3, 2, 64)), (b(2, 4, 64), b(3, 2, 64)), (b(3, 256), b(3, 2, 64))):
        with pytest.raises(ValueError, match="shape"):
            eqat.eqat_rotary_fwd(r, q, k, torch.zeros(32, dtype=torch.int64), q, k, torch.zeros(3, dtype=torch.int32))
    g = eqat.make_gated_desc(3, 64)
    for bad in (b(3, 56), b(2, 64), b(192)):
        with pytest.raises(ValueError, match="shape"):
            eqat.eqat_gated_fwd(g, bad, b(3, 64), b(3, 64))
    with pytest.raises(TypeError, match="a weight"):
        eqat.qlinear_packed_gated_fwd(eqat.make_desc(2, 64, 128, 256, 5), 0, None, [None] * 3, None, None)
    with pytest.raises(TypeError):
        eqat.qlinear_packed_gated_fwd(g, 0, *[None] * 4)


# ---------------------------------------------------------------------------------------------- turns
def _near(turns, frequencies):
    """2^64 f / 2 pi mod 1, to what a frequency in 64 bits leaves: 2^-50 of itself, and a unit."""
    for t, f in zip((int(x) % 2 ** 64 for x in turns), frequencies):
        want = f / (2 * math.pi) * 2.0 ** 64
        assert abs((t - int(want) + 2 ** 63) % 2 ** 64 - 2 ** 63) <= abs(want) * 2.0 ** -48 + 1, (t, want)


@pytest.mark.parametrize("kind", ["plain", "linear", "base", "ramp"])
@pytest.mark.parametrize("dim", [2, 4, 22, 64, 128, 512])
@pytest.mark.parametrize("base", [10000.0, 500000.0])
def test_turns_are_the_frequencies(eqat, kind, dim, base):
    code = {"plain": eqat.EQAT_ROTARY_PLAIN, "linear": eqat.EQAT_ROTARY_LINEAR, "base": eqat.EQAT_ROTARY_BASE, "ramp": eqat.EQAT_ROTARY_RAMP}[kind]
    more = dict(factor=16.0, low=1.0, high=32.0, length=8192.0)
    got = eqat.rotary_turns(dim, base, code, **more)
    assert got.dtype == torch.int64 and got.shape == (dim // 2,)
    want = B.frequencies(dim, base, kind, **more)
    _near(got.tolist(), want)
    _near(eqat.rotary_turns_of(want).tolist(), want)
    if kind == "base" and dim > 2:                                    # the ends: as it was, and divided by the factor
        plain = B.frequencies(dim, base)
        assert want[0] == plain[0] and math.isclose(want[-1], plain[-1] / 16, rel_tol=1e-12)
    if kind == "ramp" and dim == 128 and base == 10000.0:
        plain = B.frequencies(dim, base)
        ratio = [w / p for w, p in zip(want, plain)]
        assert ratio[0] == 1 and math.isclose(ratio[-1], 1 / 16) and all(a >= b for a, b in zip(ratio, ratio[1:]))


def test_turns_of_any_frequency(eqat):
    f = [0.0, 2 * math.pi, -2 * math.pi, 1e-300, -1e-300, 7.0, -0.25, 1e6]
    got = [int(x) % 2 ** 64 for x in eqat.rotary_turns_of(f)]
    assert got[0] == got[3] == got[4] == 0
    _near(got[5:7], f[5:7])
    assert (got[5] + int(eqat.rotary_turns_of([-7.0])[0])) % 2 ** 64 in (0, 1, 2 ** 64 - 1)
    for bad in (float("nan"), float("inf")):
        with pytest.raises(eqat.EqatError):
            eqat.rotary_turns_of([1.0, bad])
    with pytest.raises(eqat.EqatError):
        eqat.rotary_turns_of([])


@pytest.mark.parametrize("kw", [dict(rotary_dim=0), dict(rotary_dim=7), dict(rotary_dim=514), dict(base=0.0), dict(base=-1.0), dict(base=float("nan")),
                                dict(kind=4), dict(kind=-1), dict(kind=1, factor=0.0), dict(kind=2, factor=float("inf")),
                                dict(kind=3, factor=2.0, low=1.0, high=1.0, length=8.0), dict(kind=3, factor=2.0, low=-1.0, high=1.0, length=8.0),
                                dict(kind=3, factor=2.0, low=0.0, high=1.0, length=0.0), dict(kind=3, factor=2.0, low=0.0, high=float("nan"), length=1.0)])
def test_scalings_that_are_none(eqat, kw):
    with pytest.raises(eqat.EqatError):
        eqat.rotary_turns(**{"rotary_dim": 64, **kw})


# ---------------------------------------------------------------------------------------------- the oracle's gradients
@pytest.mark.parametrize("kind", ["silu", "gelu", "gelu_tanh"])
def test_oracle_activation_against_differences(kind):
    """Central differences, error h^2/6 times a third derivative below 3, and 2^-52 of the values over h."""
    g, h = np.linspace(-12, 12, 2001), 2.0 ** -17
    slope = (B.activation(g + h, kind)[0] - B.activation(g - h, kind)[0]) / (2 * h)
    assert np.abs(slope - B.activation(g, kind)[1]).max() <= h * h / 2 + 2.0 ** -51 * 12 / h


def test_oracle_norm_against_differences():
    rng = np.random.default_rng(1)
    x, w, dy, dr = rng.standard_normal((3, 16)), rng.standard_normal(16), rng.standard_normal((3, 16)), rng.standard_normal((3, 16))
    loss = lambda x, w: (dy * B.norm_fwd(x, w, 1e-3)).sum() + (dr * x).sum()  # noqa: E731
    dx, dw = B.norm_bwd(dy, x, w, 1e-3, dr)
    h = 2.0 ** -17
    for grad, at in ((dx, 0), (dw, 1)):
        for i in np.ndindex(grad.shape):
            lo, hi = [x.copy(), w.copy()], [x.copy(), w.copy()]
            lo[at][i] -= h
            hi[at][i] += h
            assert abs((loss(*hi) - loss(*lo)) / (2 * h) - grad[i]) <= 1e-7


@pytest.mark.parametrize("layout", ["halves", "pairs"])
def test_oracle_rotation(layout):
    """Turning back is the transpose: lengths and inner products stay, positions add up."""
    rng = np.random.default_rng(2)
    x, y = rng.standard_normal((2, 5, 3, 8))
    t = rng.standard_normal((5, 3))
    r = B.rotate(x, t, layout)
    assert np.array_equal(r[..., 6:], x[..., 6:])
    assert np.allclose((r * y).sum(), (x * B.rotate(y, -t, layout)).sum(), rtol=1e-13)
    assert np.allclose(B.rotate(r, t, layout), B.rotate(x, 2 * t, layout), rtol=1e-13)
    i, j = (0, 3) if layout == "halves" else (0, 1)
    one = np.zeros((1, 1, 8))
    one[..., i] = 1
    quarter = B.rotate(one, np.full((1, 3), np.pi / 2), layout)
    assert np.argmax(quarter) == j and np.isclose(quarter.max(), 1)


def test_oracle_e4m3():
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    every = np.sort(every[np.isfinite(every)])
    rng = np.random.default_rng(3)
    x = np.concatenate([every, (every[1:] + every[:-1]) / 2, rng.uniform(-448, 448, 4000), rng.uniform(-0.02, 0.02, 4000)]).astype(np.float32)
    assert np.array_equal(B.e4m3(x), torch.from_numpy(x).to(torch.float8_e4m3fn).double().numpy())


def test_rows_of_many_heads(eqat):
    """What a row may hold at most fits the grid; more is refused."""
    most = dict(head_dim=512, rotary_dim=2, layout=0)
    for q, k in ((16385, 1), (1, 16385), (65536, 0)):
        d = eqat.make_rotary_desc(**{**ROTARY, **most, "q_heads": q, "kv_heads": k})
        assert _rotary(eqat, d, qp=512 << 17, kp=512 << 17, qop=512 << 17, kop=512 << 17) == eqat.EQAT_ERR_SHAPE
    assert (2 * 16384 * (1 + 510) + 255) // 256 < 1 << 16
