"""Attention over the cache for prompts: keys, values and queries at the ends of the numbers' range."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as C
from test_gpu_cache import Cache, check_prompt, host, run_attention

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def eqat():
    from paper_2407_11062_b200.build import build_library
    build_library()
    from paper_2407_11062_b200 import binding
    return binding


def sixteen(eqat, D, group, seed):
    """Sixteen sequences of 400 tokens, the last 250 of them new; sequence b is to have something at position 160 + b, which
    is in the middle of a step for nearly all rows behind it."""
    c = Cache(eqat, D, group, 2, 16, [400] * 16, [250] * 16, seed=seed)
    held = c.fill()
    assert eqat.eqat_cache_attention_plan(c.desc(), eqat.make_attention_desc(8, 250, 0.1))[1] == 1
    return c, held


def check_nan_behind(c, O, lse, heads=slice(None)):
    """Rows from the position on are NaN, those before it are not."""
    got, lse = host(O), lse.cpu().numpy()
    for b in range(16):
        mine, sums = got[c.offsets[b]:c.offsets[b + 1]], lse[c.offsets[b]:c.offsets[b + 1]]
        first = 160 + b - 150
        assert np.isnan(mine[first:, heads]).all() and np.isnan(sums[first:, heads]).all(), b
        assert np.isfinite(mine[:first]).all() and np.isfinite(sums[:first]).all(), b


@pytest.mark.parametrize("D,group", [(128, 128), (128, 32), (64, 64)])
@pytest.mark.parametrize("bad", ["nan", "infinite minimum", "minus infinite minimum"])
def test_a_key_that_is_not_finite_reaches_every_row_behind_it(eqat, D, group, bad):
    c, _ = sixteen(eqat, D, group, D + group)
    step, low = {"nan": (np.nan, np.nan), "infinite minimum": (0.5, np.inf), "minus infinite minimum": (0.5, -np.inf)}[bad]
    for b in range(16):
        page, at = c.table[b][(160 + b) // 16], (160 + b) % 16
        c.params[0][page, :, at, -1, 0], c.params[0][page, :, at, -1, 1] = step, low
    c.upload()
    _, O, lse = run_attention(eqat, c, 8)
    check_nan_behind(c, O, lse)


@pytest.mark.parametrize("D,group", [(128, 128), (64, 32)])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_a_score_beyond_fp32_makes_its_row_nan(eqat, D, group, sign):
    """Keys of 2^126 in one position, all queries positive and of some units: sums of 2^131 and more."""
    c, _ = sixteen(eqat, D, group, D + group)
    for b in range(16):
        page, at = c.table[b][(160 + b) // 16], (160 + b) % 16
        c.params[0][page, :, at, :, 0], c.params[0][page, :, at, :, 1] = 0.0, sign * 2.0 ** 126
    c.upload()
    Q = C.bf16((c.rng.random((c.rows, 8, D)) * 2 + 4).astype(np.float32))
    _, O, lse = run_attention(eqat, c, 8, Q=Q)
    check_nan_behind(c, O, lse)


@pytest.mark.parametrize("D,group", [(128, 128), (128, 32), (64, 64)])
@pytest.mark.parametrize("power", [-12, -10, -9, -8])
def test_small_steps_keep_what_is_promised_of_a_key(eqat, D, group, power):
    """Steps of 2^-12 to 2^-8 and minima of 33 * 2^-25, which lie between two fp16 numbers, everywhere but in one element that
    the queries leave out: a key is off by 2^-11 of itself or 2^-19 of its largest element at most."""
    c = Cache(eqat, D, group, 4, 16, [300], [300], seed=D + group)
    held = c.fill()
    for t in range(300):
        page, at = c.table[0][t // 16], t % 16
        c.codes[0][page, :, at] = 0
        c.codes[0][page, :, at, 0] = 15
        c.params[0][page, :, at, :, 0], c.params[0][page, :, at, :, 1] = 2.0 ** power, 33 * 2.0 ** -25
    held[0][0][:] = 33 * 2.0 ** -25
    held[0][0][:, :, 0] += 15 * 2.0 ** power
    c.upload()
    Q = C.bf16(((1 + c.rng.random((300, 32, D))) * 2.0 ** 12).astype(np.float32))
    Q[..., 0] = 0
    _, O, lse = run_attention(eqat, c, 32, Q=Q)
    _, want, _, size = C.attention(Q.astype(np.float64), held[0], held[1], c.lengths, c.offsets, D ** -0.5)
    most = np.abs(Q).sum(-1) * held[0][0].max() * D ** -0.5
    # as for keys of every size; the queries are exact
    delta = size * (2.0 ** -11 + 2.0 ** -16) + most * 2.0 ** -18
    assert (np.abs(lse.cpu().numpy() - want) <= delta + 2.0 ** -18 * (1 + np.abs(want))).all()


@pytest.mark.parametrize("D,group", [(128, 128), (128, 32), (64, 64)])
def test_values_that_round_to_an_infinity_reach_those_who_see_them_only(eqat, D, group):
    """A group of finite numbers from 2^119 to bf16's largest: step 17 * 2^120, the largest code stands for 255.5 * 2^120."""
    c, held = sixteen(eqat, D, group, D + group)
    x = np.full(D, 2.0 ** 119, np.float32)
    x[-1] = 255 * 2.0 ** 120
    q, s, m = C.quantise(x, group)
    assert np.isfinite(C.bf16(x)).all() and np.isinf(C.bf16(C.values(q, s, m).astype(np.float32))[-1])
    for b in range(16):
        page, at = c.table[b][(160 + b) // 16], (160 + b) % 16
        c.codes[1][page, :, at], c.params[1][page, :, at] = C.pack(q), np.stack([s, m], -1)
    c.upload()
    Q, O, lse = run_attention(eqat, c, 8)
    got, before = host(O), []
    for b in range(16):
        first = c.offsets[b] + 10 + b
        assert np.isnan(got[first:c.offsets[b + 1]]).all()
        before += range(c.offsets[b], first)
    assert np.isfinite(lse.cpu().numpy()).all()
    for b in range(16):
        held[1][b][160 + b] = 0.0
    check_prompt(c, O, None, Q, held, rows=before)


@pytest.mark.parametrize("D,group,ratio", [(128, 128, 8), (128, 32, 8), (64, 64, 3), (128, 64, 4)])
def test_decoding_beside_a_prompt(eqat, D, group, ratio):
    """Both kernels, the one for few rows in tiles of one token's rows; some sequences have more than a tile."""
    lengths, news = [3000, 260, 17, 900, 1, 2100, 0, 64], [1, 200, 2, 1, 1, 1, 0, 4]
    c = Cache(eqat, D, group, 8, 16, lengths, news, seed=D + group, pad_rows=1)
    held = c.fill()
    # by the number of sequences and rows an ordinary one has one or two tokens
    plan = eqat.eqat_cache_attention_plan(c.desc(), eqat.make_attention_desc(8 * ratio, 200, 0.1))
    assert plan[1] == 33 and plan[0] < 32
    Q, O, lse = run_attention(eqat, c, 8 * ratio)
    check_prompt(c, O, lse, Q, held)
