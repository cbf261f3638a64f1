"""Softmax weights of the attention over the cache, few rows: long stretches of a sequence in one worker, tokens that take
nearly all of a row's softmax, tokens with far larger or smaller values than the others'.  Outputs are compared by the norm of
each row and head."""
import numpy as np
import pytest
import torch

from helpers import TOL
from oracle import cache_oracle as C
from test_gpu_cache import GEOMETRIES, Cache, dev, host, run_attention

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def eqat():
    from paper_2407_11062_b200.build import build_library
    build_library()
    from paper_2407_11062_b200 import binding
    return binding


def put(c, held, i, head, pos, x):
    """Another key (i = 0) or value (1) of one head at a position of sequence 0."""
    q, s, m = C.quantise(C.bf16(np.asarray(x, np.float32))[None, None], c.group)
    page, at = c.table[0][pos // c.page], pos % c.page
    c.codes[i][page, head, at] = C.pack(q)[0, 0]
    c.params[i][page, head, at] = np.stack([s, m], -1)[0, 0]
    held[i][0][pos, head] = C.values(q, s, m)[0, 0]


def repeated(eqat, c, copies, Q):
    """Decoding by `copies` sequences that all read the pages of sequence 0: as many tokens as possible for a worker."""
    d = eqat.make_cache_desc(c.group, c.D, c.H, c.page, c.pages, copies, c.max_pages, copies)
    a = eqat.make_attention_desc(Q.shape[1], 1, c.D ** -0.5)
    c.upload()
    off = torch.arange(copies + 1, dtype=torch.int32, device="cuda")
    lengths = torch.full((copies,), c.lengths[0], dtype=torch.int32, device="cuda")
    table = torch.from_numpy(c.table[:1]).cuda().repeat(copies, 1)
    O = torch.empty(copies, Q.shape[1], c.D, dtype=torch.bfloat16, device="cuda")
    lse = torch.empty(copies, Q.shape[1], device="cuda")
    need = eqat.cache_workspace_bytes(d, a)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    eqat.eqat_cache_attention(d, a, dev(Q), off, lengths, table, tuple(c.pool), O, lse, ws)
    assert eqat.device_status() == (0, 0)
    return O, lse


def expected(c, held, Q):
    """Outputs of `repeated` in 64 bits, the log-sum-exp and the largest weight of each row."""
    k, v = (torch.from_numpy(h[0]).cuda().repeat_interleave(Q.shape[1] // c.H, 1).transpose(0, 1) for h in held)      # [q_heads, tokens, D]
    z = torch.from_numpy(Q).cuda().double().transpose(0, 1) @ k.transpose(1, 2) * c.D ** -0.5                        # [q_heads, copies, tokens]
    top = z.amax(-1, keepdim=True)
    p = torch.exp(z - top)
    total = p.sum(-1, keepdim=True)
    p /= total
    return [x.transpose(0, 1).cpu().numpy() for x in (p @ v, (top + torch.log(total))[..., 0], p.amax(-1))]


def check_norms(got, want):
    """Each row and head by itself.  The rounding to bf16 is 2^-8 of an element at most; the rest of TOL is what scores (some
    2^-14 of the sums of sizes, which are at most a few times the outputs here) and the weights' integers (sqrt(tokens) halves
    of 15 units, of which the largest product of weight and step has 2^20) add."""
    err, size = np.linalg.norm(got - want, axis=-1), np.linalg.norm(want, axis=-1)
    bad = ~(err <= TOL * size)
    assert not bad.any(), (bad.sum(), np.argwhere(bad)[:5].tolist(), (err / size)[bad][:5])


# 600 segments for 592 workers: a stretch is longer than a segment, and most of a segment lies in one
COPIES, HEADS = 75, 8


@pytest.mark.parametrize("D,group,ratio", [(128, 128, 1), (128, 128, 8), (128, 32, 1), (64, 64, 4), (256, 64, 1)])
@pytest.mark.parametrize("at", [0, 6001, 14079])
@pytest.mark.parametrize("shrink", [64, 1024])
def test_a_dominant_token_with_small_values(eqat, D, group, ratio, at, shrink):
    """One of 14080 tokens takes from half to 99.99 % of the softmax; its values are 1/64 or 1/1024 of the others'."""
    N = 14080
    c = Cache(eqat, D, group, HEADS, 64, [N], [1], seed=D + group + at + shrink)
    held = c.fill()
    u = c.rng.standard_normal((HEADS, D)).astype(np.float32)
    u *= np.float32(D ** 0.5) / np.linalg.norm(u, axis=-1, keepdims=True)
    for h in range(HEADS):
        put(c, held, 0, h, at, u[h] * 1.5)
        put(c, held, 1, h, at, held[1][0][at, h] / shrink)
    # the queries' part along u from 6 to 12 (over D^1/2): scores of the token 1.5 times that above the mean
    along = np.linspace(0.55, 1.15, COPIES * ratio).reshape(COPIES, 1, ratio, 1).astype(np.float32) * np.float32((128 / D) ** 0.5)
    Q = along * u[None, :, None] + 0.2 * c.rng.standard_normal((COPIES, HEADS, ratio, D)).astype(np.float32)
    Q = C.bf16(Q.reshape(COPIES, HEADS * ratio, D))
    want, lse, share = expected(c, held, Q)
    assert (share > 0.5).mean() > 0.5 and share.max() > 0.99
    O, got_lse = repeated(eqat, c, COPIES, Q)
    check_norms(host(O).astype(np.float64), want)
    assert np.abs(got_lse.cpu().numpy() - lse).max() < 1e-3


@pytest.mark.parametrize("D,group,ratio", [(128, 128, 1), (128, 128, 8), (128, 32, 4), (64, 64, 1), (256, 128, 1)])
@pytest.mark.parametrize("power", [12, 16, 20, 30])
def test_a_token_that_is_hardly_seen_with_large_values(eqat, D, group, ratio, power):
    """Its weight is below 2^-45 of the others', its values 2^12 to 2^30 times theirs."""
    N = 1024
    c = Cache(eqat, D, group, HEADS, 64, [N], [1], seed=D + group + power)
    held = c.fill()
    u = c.rng.standard_normal((HEADS, D)).astype(np.float32)
    u *= np.float32(D ** 0.5) / np.linalg.norm(u, axis=-1, keepdims=True)
    for h in range(HEADS):
        put(c, held, 0, h, 300, u[h] * -10.0)
        put(c, held, 1, h, 300, held[1][0][300, h] * 2.0 ** power)
    Q = 0.6 * np.float32((128 / D) ** 0.5) * u[None, :, None] + 0.05 * c.rng.standard_normal((COPIES, HEADS, ratio, D)).astype(np.float32)
    Q = C.bf16(Q.reshape(COPIES, HEADS * ratio, D))
    want, lse, _ = expected(c, held, Q)
    O, _ = repeated(eqat, c, COPIES, Q)
    check_norms(host(O).astype(np.float64), want)


@pytest.mark.parametrize("D,group,H,page", GEOMETRIES)
@pytest.mark.parametrize("ratio", [1, 8])
def test_decoding_by_norm(eqat, D, group, H, page, ratio):
    lengths = [1, 2, 17, 33, 129, 300, 777, 2500]
    c = Cache(eqat, D, group, H, page, lengths, [1] * len(lengths), seed=D + ratio)
    held = c.fill()
    Q, O, _ = run_attention(eqat, c, H * ratio)
    check_norms(host(O).astype(np.float64), C.attention(Q.astype(np.float64), held[0], held[1], c.lengths, c.offsets, D ** -0.5)[0])


@pytest.mark.parametrize("D,group,H,page", GEOMETRIES)
@pytest.mark.parametrize("window,scale", [(0, 1.0), (50, 1.0), (0, 6.0), (0, -3.0)])
def test_drafts_by_norm(eqat, D, group, H, page, window, scale):
    """Also with sharp softmaxes, whose maxima rise along a sequence."""
    c = Cache(eqat, D, group, H, page, [9, 40, 300, 3, 129, 75, 0, 1500], [5, 0, 7, 5, 1, 15, 2, 16], seed=D + group, pad_rows=2)
    held, scale = c.fill(), scale * D ** -0.5
    Q, O, _ = run_attention(eqat, c, H * 2, window=window, scale=scale)
    rows = int(c.offsets[-1])
    check_norms(host(O).astype(np.float64)[:rows], C.attention(Q.astype(np.float64), held[0], held[1], c.lengths, c.offsets, scale, window)[0][:rows])


@pytest.mark.parametrize("ratio", [1, 4, 8])
def test_a_sequence_in_many_pieces_by_norm(eqat, ratio):
    c = Cache(eqat, 128, 128, 1, 64, [20011], [1], seed=3)
    held = c.fill()
    Q, O, _ = run_attention(eqat, c, ratio)
    check_norms(host(O).astype(np.float64), C.attention(Q.astype(np.float64), held[0], held[1], c.lengths, c.offsets, 128 ** -0.5)[0])


@pytest.mark.parametrize("ratio", [1, 8])
@pytest.mark.parametrize("size", [2.0 ** -100, 2.0 ** 40, 2.0 ** 100])
def test_flat_groups_of_values(eqat, ratio, size):
    """Groups whose elements are all equal have a step of zero and only a minimum, of any size; with and without others."""
    c = Cache(eqat, 128, 64, 2, 16, [500, 300], [1, 1], seed=5)
    held = c.fill()
    for b, n in enumerate(c.lengths):
        for t in range(n):
            page, at = c.table[b][t // 16], t % 16
            flat = C.bf16((c.rng.standard_normal((2, 2)) * size).astype(np.float32))       # by head and group
            for g in range(2):
                if b == 0 or g == 0:
                    c.params[1][page, :, at, g, 0], c.params[1][page, :, at, g, 1] = 0.0, flat[:, g]
                    held[1][b][t, :, 64 * g:64 * g + 64] = flat[:, g, None]
    c.upload()
    Q, O, _ = run_attention(eqat, c, 2 * ratio)
    want = C.attention(Q.astype(np.float64), held[0], held[1], c.lengths, c.offsets, 128 ** -0.5)[0]
    got = host(O).astype(np.float64)
    check_norms(got[:1], want[:1])
    check_norms(got[1:, :, :64], want[1:, :, :64])
    check_norms(got[1:, :, 64:], want[1:, :, 64:])


@pytest.mark.parametrize("n", [1, 200])
@pytest.mark.parametrize("power,keys,scale", [(-98, 98, 1.0), (100, -100, 1.0), (110, -110, 1.0), (118, -118, 1.0), (124, -118, 2.0 ** -6)])
def test_queries_of_any_size(eqat, n, power, keys, scale):
    """With keys of the inverse size, in the kernel for few rows and in the one for prompts; one such row among ordinary ones."""
    c = Cache(eqat, 128, 64, 4, 16, [300, 290], [n, n], seed=7)
    held, scale = c.fill(), scale * 128 ** -0.5
    assert eqat.eqat_cache_attention_plan(c.desc(), eqat.make_attention_desc(32, n, 0.1))[1] == (n > 1)
    ordinary = [p.copy() for p in c.params], [h.copy() for h in held[0]]
    for b, tokens in enumerate(c.lengths):
        pos = np.arange(tokens)
        c.params[0][c.table[b][pos // 16], :, pos % 16] *= np.float32(2.0 ** keys)
        held[0][b] = held[0][b] * 2.0 ** keys
    c.upload()
    Q = c.rng.standard_normal((c.rows, 32, 128)).astype(np.float32)
    Q[..., 3] = 2.0 + np.abs(Q[..., 3])                         # every row's largest element lies in [2, 8)
    large = C.bf16(Q * np.float32(2.0 ** power))
    assert (np.abs(large).max(-1) >= 2.0 ** (power + 1)).all() and (np.abs(large).max(-1) < 2.0 ** (power + 3)).all()
    _, O, _ = run_attention(eqat, c, 32, Q=large, scale=scale)
    check_norms(host(O).astype(np.float64), C.attention(large.astype(np.float64), held[0], held[1], c.lengths, c.offsets, scale)[0])
    c.params, held[0] = ordinary
    c.upload()
    Q = C.bf16(Q)
    want = C.attention(Q.astype(np.float64), held[0], held[1], c.lengths, c.offsets, 128 ** -0.5)[0]
    Q[0, 1] = large[0, 1]
    _, O, _ = run_attention(eqat, c, 32, Q=Q)
    got = host(O).astype(np.float64)
    got[0, 1] = want[0, 1]
    check_norms(got, want)


@pytest.mark.parametrize("n", [1, 200])
@pytest.mark.parametrize("power", [-90, -70, 60, 110])
def test_values_of_any_size(eqat, n, power):
    c = Cache(eqat, 128, 64, 4, 16, [300, 290], [n, n], seed=9)
    held = c.fill()
    assert eqat.eqat_cache_attention_plan(c.desc(), eqat.make_attention_desc(32, n, 0.1))[1] == (n > 1)
    for b, tokens in enumerate(c.lengths):
        pos = np.arange(tokens)
        c.params[1][c.table[b][pos // 16], :, pos % 16] *= np.float32(2.0 ** power)
        held[1][b] = held[1][b] * 2.0 ** power
    c.upload()
    Q, O, _ = run_attention(eqat, c, 32)
    check_norms(host(O).astype(np.float64), C.attention(Q.astype(np.float64), held[0], held[1], c.lengths, c.offsets, 128 ** -0.5)[0])
