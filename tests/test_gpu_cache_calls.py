"""The cache's calls with tensors that are laid out or placed in ways that the other tests do not have."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def eqat():
    from paper_2407_11062_b200.build import build_library
    build_library()
    from paper_2407_11062_b200 import binding
    return binding


class Step:
    """One new token of one sequence, keys and values written and read, one row of attention."""

    def __init__(self, eqat, device="cuda"):
        gen = torch.Generator().manual_seed(1)
        def rows(h):
            return torch.randn(1, h, 64, generator=gen).to(torch.bfloat16).to(device)
        self.eqat = eqat
        self.K, self.V, self.Q = rows(2), rows(2), rows(4)
        self.pool = tuple(torch.zeros(3, 2, 16, *shape, dtype=t, device=device) for _ in range(2)
                          for shape, t in (((32,), torch.uint8), ((1, 2), torch.bfloat16)))
        self.where = [torch.tensor(x, dtype=torch.int32, device=device) for x in ([0, 1], [5], [[2]])]
        self.O = torch.zeros_like(self.Q)
        self.hat = [torch.zeros_like(self.K) for _ in range(2)]
        self.desc, self.attn = eqat.make_cache_desc(64, 64, 2, 16, 3, 1, 1, 1), eqat.make_attention_desc(4, 1, 0.125)

    def append(self):
        self.eqat.eqat_cache_append(self.desc, self.K, self.V, *self.where, self.pool, *self.hat)

    def read(self):
        self.eqat.eqat_cache_read(self.desc, *self.where, self.pool, *self.hat)

    def attend(self):
        self.eqat.eqat_cache_attention(self.desc, self.attn, self.Q, *self.where, self.pool, self.O,
                                       None, torch.empty(1 << 20, dtype=torch.uint8, device=self.Q.device))


@pytest.mark.skipif(torch.cuda.device_count() < 2, reason="needs two devices")
def test_tensors_of_another_device_are_refused(eqat):
    """All of them, or one: nothing is launched."""
    away, here = Step(eqat, "cuda:1"), Step(eqat, "cuda:0")
    with torch.cuda.device(0):
        for call in (away.append, away.read, away.attend):
            with pytest.raises(ValueError, match="current device"):
                call()
        for name in ("V", "Q", "O"):
            mixed = Step(eqat, "cuda:0")
            setattr(mixed, name, getattr(away, name))
            with pytest.raises(ValueError, match="current device"):
                (mixed.append if name == "V" else mixed.attend)()
        here.append()
        here.attend()
    with torch.cuda.device(1):
        away.append()
        away.attend()
    assert torch.equal(here.O.cpu(), away.O.cpu())


@pytest.mark.parametrize("stride", [1, 129, 1003, 4096])
def test_the_stride_of_a_single_row_does_not_matter(eqat, stride):
    want, got = Step(eqat), Step(eqat)
    for name in ("K", "V", "Q", "O"):
        t = getattr(got, name)
        setattr(got, name, t.as_strided(t.shape, (stride, *t.stride()[1:])))
    for step in (want, got):
        step.append()
        step.attend()
    assert all(torch.equal(x, y) for x, y in zip(want.pool, got.pool)) and torch.equal(want.O, got.O) and bool((got.O != 0).any())
