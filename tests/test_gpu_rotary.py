"""Rotary positions against the oracle: layouts, parts of a head, far positions, ways to give them, slices, in place.

Bound.  The angle is exact up to 2^-33 of a turn and the conversion to 24 bits (2^-24 radians); sine, cosine and the two products
and the sum add a few units of 2^-24 of |a| + |b|: 2^-20 of it, times the amplitude, is above all of them (2^-19 of a head's largest
element, at least half of |a| + |b|).  Then half a step."""
import numpy as np
import pytest
import torch

from helpers import Guarded, assert_elementwise, torch_to_f64
from oracle import between_oracle as B

pytestmark = pytest.mark.gpu
HALF_STEP = 2.0 ** -8


@pytest.fixture(scope="module")
def eqat():
    from paper_2407_11062_b200.build import build_library
    build_library()
    from paper_2407_11062_b200 import binding
    return binding


def heads(rows, h, d, seed):
    return torch.randn(rows, h, d, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).to(torch.bfloat16)


def layout_code(eqat, layout):
    return eqat.EQAT_ROTARY_HALVES if layout == "halves" else eqat.EQAT_ROTARY_PAIRS


def check(got, x, turns, positions, layout, sign=1, amplitude=1.0):
    t = sign * np.array([B.turns_at(turns.tolist(), p) for p in positions])
    want = B.rotate(torch_to_f64(x), t, layout, amplitude)
    n = 2 * t.shape[1]
    room = np.zeros_like(want)
    room[..., :n] = HALF_STEP * np.abs(want[..., :n]) + 2.0 ** -19 * abs(amplitude) * np.abs(torch_to_f64(x)).max(-1, keepdims=True)
    assert_elementwise(torch_to_f64(got), want, room + 2.0 ** -133, layout)


POSITIONS = [0, 1, -1, 2, 4095, 100001, 2 ** 20 + 7, 2 ** 31 - 1, -2 ** 31, 12345678]


@pytest.mark.parametrize("head_dim,rotary_dim", [(8, 2), (8, 8), (64, 64), (64, 32), (96, 96), (96, 24), (128, 128), (128, 32), (128, 50), (128, 126), (256, 256), (256, 64),
                                                 (512, 512), (104, 88), (80, 40)])
@pytest.mark.parametrize("layout", ["halves", "pairs"])
@pytest.mark.parametrize("q_heads,kv_heads", [(4, 2), (1, 0), (5, 1)])
def test_against_oracle(eqat, head_dim, rotary_dim, layout, q_heads, kv_heads):
    rows, buf = len(POSITIONS), Guarded()
    turns = eqat.rotary_turns(rotary_dim, 500000.0)
    pos = torch.tensor(POSITIONS, dtype=torch.int32, device="cuda")
    Q, K = heads(rows, q_heads, head_dim, 1), heads(rows, kv_heads, head_dim, 2) if kv_heads else None
    d = eqat.make_rotary_desc(rows, q_heads, kv_heads, head_dim, rotary_dim, layout_code(eqat, layout), 1.25)
    for call, sign in ((eqat.eqat_rotary_fwd, 1), (eqat.eqat_rotary_bwd, -1)):
        Qo = buf.empty(rows, q_heads, head_dim, dtype=torch.bfloat16, shift_bytes=16)
        Ko = buf.empty(rows, kv_heads, head_dim, dtype=torch.bfloat16) if kv_heads else None
        call(d, Q, K, turns.cuda(), Qo, Ko, pos)
        buf.check()
        for x, y in ((Q, Qo), (K, Ko)):
            if x is not None:
                check(y, x, turns, POSITIONS, layout, sign, 1.25)
                assert torch.equal(y[..., rotary_dim:], x[..., rotary_dim:])
        # in place
        q, k = Q.clone(), K.clone() if kv_heads else None
        call(d, q, k, turns.cuda(), q, k, pos)
        assert torch.equal(q, Qo) and (k is None or torch.equal(k, Ko))


@pytest.mark.parametrize("layout", ["halves", "pairs"])
@pytest.mark.parametrize("lens,news", [([5], [1]), ([700, 3, 90000, 1], [1, 3, 16, 0]), ([40] * 70, [1] * 70), ([1500, 900], [1500, 900]), ([3] * 2000, [1, 0] * 1000)])
def test_positions_of_a_cache(eqat, layout, lens, news):
    """The rows stand where the cache's calls put them; rows of no sequence are left alone."""
    rows = sum(news) + 3
    off = np.concatenate([[0], np.cumsum(news)])
    where = [n - k + i for n, k in zip(lens, news) for i in range(k)]
    Q, K = heads(rows, 3, 64, 3), heads(rows, 1, 64, 4)
    turns = eqat.rotary_turns(64, 10000.0)
    args = [torch.tensor(x, dtype=torch.int32, device="cuda") for x in (off, lens)]
    d = eqat.make_rotary_desc(rows, 3, 1, 64, 64, layout_code(eqat, layout), sequences=len(lens))
    Qo, Ko = torch.full_like(Q, 7), torch.full_like(K, 7)
    eqat.eqat_rotary_fwd(d, Q, K, turns.cuda(), Qo, Ko, None, *args)
    n = len(where)
    check(Qo[:n], Q[:n], turns, where, layout)
    check(Ko[:n], K[:n], turns, where, layout)
    assert (Qo[n:] == 7).all() and (Ko[n:] == 7).all()
    same = [torch.full_like(x, 7) for x in (Q, K)]
    pos = torch.tensor(where + [0] * 3, dtype=torch.int32, device="cuda")
    eqat.eqat_rotary_fwd(eqat.make_rotary_desc(rows, 3, 1, 64, 64, layout_code(eqat, layout)), Q, K, turns.cuda(), *same, pos)
    assert torch.equal(same[0][:n], Qo[:n]) and torch.equal(same[1][:n], Ko[:n])


def test_arrays_that_say_nothing_sensible(eqat):
    """No access leaves the tensors, whatever offsets and lengths say."""
    buf, rows = Guarded(), 40
    for off, lens in (([0, 100, 2000], [5, 6]), ([-7, -3, -1], [1, 1]), ([0, 1 << 30, 1 << 30], [-5, 1 << 30]), ([50, 50, 50], [1, 1])):
        Q, K = heads(rows, 2, 64, 5), heads(rows, 1, 64, 6)
        Qo, Ko = buf.empty(rows, 2, 64, dtype=torch.bfloat16), buf.empty(rows, 1, 64, dtype=torch.bfloat16)
        d = eqat.make_rotary_desc(rows, 2, 1, 64, sequences=2)
        eqat.eqat_rotary_fwd(d, Q, K, eqat.rotary_turns(64).cuda(), Qo, Ko, None, *[torch.tensor(x, dtype=torch.int32, device="cuda") for x in (off, lens)])
    buf.check()


@pytest.mark.parametrize("layout", ["halves", "pairs"])
@pytest.mark.parametrize("rows", [1, 2, 333, 6000])
def test_slices_of_a_projection(eqat, layout, rows):
    """Queries and keys side by side with the values, in place and out of it: pitches of their own; what is between stays."""
    qkv = heads(rows, 8 + 2 + 2, 128, 7)
    was, Q, K = qkv.clone(), qkv[:, :8], qkv[:, 8:10]
    turns = eqat.rotary_turns(96, 10000.0).cuda()
    pos = torch.arange(rows, device="cuda", dtype=torch.int32) * 17
    d = eqat.make_rotary_desc(rows, 8, 2, 128, 96, layout_code(eqat, layout))
    Qo, Ko = torch.empty(rows, 8, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(rows, 2, 128, dtype=torch.bfloat16, device="cuda")
    eqat.eqat_rotary_fwd(d, Q, K, turns, Qo, Ko, pos)
    assert torch.equal(qkv, was)
    eqat.eqat_rotary_fwd(d, Q, K, turns, Q, K, pos)
    assert torch.equal(Q, Qo) and torch.equal(K, Ko) and torch.equal(qkv[:, 10:], was[:, 10:])
    some = sorted({0, rows // 2, rows - 1})
    check(Qo[some], was[some, :8], turns.cpu(), [17 * i for i in some], layout)
    back = torch.empty_like(qkv)
    eqat.eqat_rotary_bwd(d, Q, K, turns, back[:, :8], back[:, 8:10], pos)
    # there and back: two roundings of each element of a pair
    assert ((back[:, :10].float() - was[:, :10].float()).abs().amax() <= 2.1 * 2 ** -8 * was.float().abs().amax() * 2 ** 0.5)


def test_gradient_is_the_transpose(eqat):
    """<rotate(x), y> = <x, back(y)>, up to the roundings of both (a random walk over the elements, eight deviations)."""
    rows, pos = 64, torch.arange(64, dtype=torch.int32, device="cuda") * 1001 - 30000
    for layout in ("halves", "pairs"):
        d = eqat.make_rotary_desc(rows, 4, 0, 128, 128, layout_code(eqat, layout), 0.75)
        x, y, turns = heads(rows, 4, 128, 8), heads(rows, 4, 128, 9), eqat.rotary_turns(128).cuda()
        rx, by = torch.empty_like(x), torch.empty_like(y)
        eqat.eqat_rotary_fwd(d, x, None, turns, rx, None, pos)
        eqat.eqat_rotary_bwd(d, y, None, turns, by, None, pos)
        a, b = (rx.double() * y.double()), (x.double() * by.double())
        assert abs(float(a.sum() - b.sum())) <= 8 * HALF_STEP * float((a.square().sum() + b.square().sum()).sqrt())


def test_without_keys_nothing_is_asked_of_them(eqat):
    Q, pos = heads(5, 2, 64, 12), torch.arange(5, dtype=torch.int32, device="cuda")
    turns, d = eqat.rotary_turns(64).cuda(), eqat.make_rotary_desc(5, 2, 0, 64)
    got = [torch.empty_like(Q) for _ in range(2)]
    eqat.eqat_rotary_fwd(d, Q, None, turns, got[0], None, pos)
    eqat.eqat_rotary_fwd(d, Q, torch.empty(0), turns, got[1], Q, pos)
    assert torch.equal(*got)


def test_captured(eqat):
    """A captured call serves other lengths and tables."""
    off, lens = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, 1, 2], [9, 100]))
    Q, K, turns = heads(2, 4, 128, 10), heads(2, 2, 128, 11), eqat.rotary_turns(128).cuda()
    Qo, Ko = torch.empty_like(Q), torch.empty_like(K)
    d = eqat.make_rotary_desc(2, 4, 2, 128, sequences=2)
    eqat.eqat_rotary_fwd(d, Q, K, turns, Qo, Ko, None, off, lens)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        eqat.eqat_rotary_fwd(d, Q, K, turns, Qo, Ko, None, off, lens)
    for a, b in ((10, 101), (5000, 1)):
        lens.copy_(torch.tensor([a, b], dtype=torch.int32))
        Q.copy_(heads(2, 4, 128, a))
        g.replay()
        check(Qo, Q, turns.cpu(), [a - 1, b - 1], "halves")
        check(Ko, K, turns.cpu(), [a - 1, b - 1], "halves")
