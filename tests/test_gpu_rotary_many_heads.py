"""As many heads in a row as a call may have: the grid holds the items of every part of a head, in place and not.

Bound as in test_gpu_rotary.py: half a step of the result, and 2^-19 of a head's largest element."""
import numpy as np
import pytest
import torch

from oracle import between_oracle as B

pytestmark = pytest.mark.gpu
HEADS, DIM, POSITION = 16384, 512, 100001


@pytest.fixture(scope="module")
def eqat():
    from paper_2407_11062_b200.build import build_library
    build_library()
    from paper_2407_11062_b200 import binding
    return binding


# parts of a head with the most items, moved one, two, four, eight elements at a time, and a small one with most of the head handed on
@pytest.mark.parametrize("rotary_dim,layout", [(510, "halves"), (508, "halves"), (504, "halves"), (496, "halves"), (512, "halves"), (2, "halves"), (4, "halves"), (510, "pairs"), (2, "pairs")])
def test_the_most_heads(eqat, rotary_dim, layout):
    gen = torch.Generator(device="cuda").manual_seed(rotary_dim)
    # keys off 32 bytes, so that pieces of 16 elements are not taken
    raw = torch.randn(2 * HEADS * DIM + 8, device="cuda", generator=gen).to(torch.bfloat16)
    Q, K = raw[8:8 + HEADS * DIM].view(1, HEADS, DIM), raw[8 + HEADS * DIM:].view(1, HEADS, DIM)
    turns, pos = eqat.rotary_turns(rotary_dim), torch.tensor([POSITION], dtype=torch.int32, device="cuda")
    d = eqat.make_rotary_desc(1, HEADS, HEADS, DIM, rotary_dim, eqat.EQAT_ROTARY_HALVES if layout == "halves" else eqat.EQAT_ROTARY_PAIRS)
    angle = torch.tensor(B.turns_at(turns.tolist(), POSITION), dtype=torch.float64, device="cuda")
    c, s, n = angle.cos(), angle.sin(), rotary_dim // 2
    out = torch.full((2 * HEADS * DIM + 8,), float("nan"), dtype=torch.bfloat16, device="cuda")
    Qo, Ko = out[8:8 + HEADS * DIM].view(1, HEADS, DIM), out[8 + HEADS * DIM:].view(1, HEADS, DIM)
    eqat.eqat_rotary_fwd(d, Q, K, turns.cuda(), Qo, Ko, pos)
    for x, got in ((Q, Qo), (K, Ko)):
        a, b = (slice(0, n), slice(n, 2 * n)) if layout == "halves" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
        want = x.double()
        want[..., a], want[..., b] = x[..., a].double() * c - x[..., b].double() * s, x[..., b].double() * c + x[..., a].double() * s
        room = 2.0 ** -8 * want.abs() + 2.0 ** -19 * x.double().abs().amax(-1, keepdim=True)
        room[..., 2 * n:] = 0
        assert bool(((got.double() - want).abs() <= room).all())
    Q2, K2 = Q.clone(), K.clone()
    eqat.eqat_rotary_fwd(d, Q2, K2, turns.cuda(), Q2, K2, pos)
    assert torch.equal(Q2, Qo) and torch.equal(K2, Ko)
    assert not np.isnan(float(out[8:].float().sum()))
