"""The 4-bit key/value cache on the GPU against its oracle: bytes and values exactly, attention within a bound that is derived
element by element.  Pools start full of NaN parameters and stray codes, so whatever a kernel reads beside the tokens that a
row sees shows up."""
import math

import numpy as np
import pytest
import torch

from helpers import TOL, Guarded
from oracle import cache_oracle as C

pytestmark = pytest.mark.gpu
U = torch.finfo(torch.bfloat16).eps / 2


@pytest.fixture(scope="module")
def eqat():
    from paper_2407_11062_b200.build import build_library
    build_library()
    from paper_2407_11062_b200 import binding
    return binding


class Cache:
    """A pool with its page table, on the device, and the same contents for the oracle."""

    def __init__(self, eqat, D, group, kv_heads, page, lengths, news, seed=0, pad_rows=0, spare_pages=2, max_pages=None):
        rng = np.random.default_rng(seed)
        self.eqat, self.D, self.group, self.H, self.page, self.rng = eqat, D, group, kv_heads, page, rng
        self.lengths, self.news = list(lengths), list(news)
        need = [(n + page - 1) // page for n in lengths]
        self.pages = sum(need) + spare_pages
        self.max_pages = max_pages or max(1, max(need))
        order = list(rng.permutation(self.pages))
        self.table = np.full((len(lengths), self.max_pages), -77, np.int32)
        for b, n in enumerate(need):
            self.table[b, :n] = [order.pop() for _ in range(n)]
        self.offsets = np.concatenate([[0], np.cumsum(news)]).astype(np.int32)
        self.rows = int(self.offsets[-1]) + pad_rows
        G = D // group
        # stray bytes everywhere, parameters NaN
        self.codes = [rng.integers(0, 256, (self.pages, kv_heads, page, D // 2)).astype(np.uint8) for _ in range(2)]
        self.params = [np.full((self.pages, kv_heads, page, G, 2), np.nan, np.float32) for _ in range(2)]
        self.upload()

    def upload(self):
        self.pool = []
        for c, p in zip(self.codes, self.params):
            self.pool += [torch.from_numpy(c).cuda(), torch.from_numpy(p).cuda().to(torch.bfloat16)]
        self.where = [torch.from_numpy(self.offsets).cuda(), torch.tensor(self.lengths, dtype=torch.int32, device="cuda"),
                      torch.from_numpy(self.table).cuda(), tuple(self.pool)]

    def desc(self, rows=None):
        return self.eqat.make_cache_desc(self.group, self.D, self.H, self.page, self.pages, len(self.lengths), self.max_pages,
                                         self.rows if rows is None else rows)

    def tokens(self, rows, spread=1.0, shift=0.7):
        """bf16 keys or values: channels of different size, some far from zero."""
        x = self.rng.standard_normal((rows, self.H, self.D)) * np.exp(0.5 * spread * self.rng.standard_normal((self.H, self.D)))
        return C.bf16((x + shift * self.rng.standard_normal((self.H, self.D))).astype(np.float32))

    def fill(self):
        """Every token of every sequence, quantised by the oracle; returns the values that the cache stands for."""
        held, self.sizes, self.steps = [[], []], [[], []], []
        for i in (0, 1):
            for b, n in enumerate(self.lengths):
                q, s, m = C.quantise(self.tokens(n), self.group)
                pos = np.arange(n)
                page = self.table[b][pos // self.page]
                self.codes[i][page, :, pos % self.page] = C.pack(q)
                self.params[i][page, :, pos % self.page] = np.stack([s, m], -1)
                held[i].append(C.values(q, s, m))
                # what the kernels add up: s q and m
                s, m = (np.repeat(x.astype(np.float64), self.group, -1) for x in (s, m))
                self.sizes[i].append(s * 15 + np.abs(m))
                if i == 1:
                    self.steps.append(s)
        self.upload()
        return held


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).cuda().to(torch.bfloat16)


def host(t):
    return t.detach().float().cpu().numpy()


def same_values(got, want):
    """Equal numbers; NaN where the oracle has NaN (its bits are free)."""
    return np.array_equal(got, want, equal_nan=True)


# --------------------------------------------------------------------------- append and read
GEOMETRIES = [(128, 128, 8, 16), (128, 64, 5, 32), (128, 32, 3, 48), (64, 64, 1, 16), (64, 32, 7, 64), (256, 128, 2, 16),
              (256, 64, 3, 80), (256, 32, 1, 32)]


@pytest.mark.parametrize("D,group,H,page", GEOMETRIES)
@pytest.mark.parametrize("hat", [True, False])
def test_append_writes_the_oracles_bytes_and_nothing_else(eqat, D, group, H, page, hat):
    # sequences without new tokens, one token, more new tokens than the length, a first page, the middle of one
    c = Cache(eqat, D, group, H, page, [1, 0, 70, 33, 3, 200], [1, 0, 70, 1, 5, 0], seed=D + group + H, pad_rows=3)
    rows, wide = c.rows, (H + 2) * D                            # rows of a wider buffer: K and V side by side with others
    X = [c.tokens(rows), c.tokens(rows)]
    X[0][2, 0, :group] = 1.25                                   # a flat group
    X[0][3, 0, :4], X[1][4, 0, 1], X[1][5, 0, 2] = [3e38, -3e38, 0, 1], np.nan, -np.inf
    X[1][6, 0] = C.bf16(X[1][6, 0] * np.float32(1e-38))         # steps below 2^-126
    X[0][7, 0] = C.bf16(X[0][7, 0] * np.float32(1e30))
    src = [torch.full((rows, wide), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    views = []
    for t, x in zip(src, X):
        v = t.as_strided((rows, H, D), (wide, D, 1), D)
        v.copy_(dev(x))
        views.append(v)
    guard = Guarded()
    out = [guard.empty(rows, H, D, dtype=torch.bfloat16, shift_bytes=16) for _ in range(2)] if hat else [None, None]
    before = [o.clone() for o in out] if hat else []
    eqat.eqat_cache_append(c.desc(), *views, *c.where, *out)
    guard.check()
    seq, page_of, at = C.places(c.offsets, c.lengths, c.table, page, c.pages, rows)
    stands = page_of >= 0
    assert stands.sum() == 1 + 70 + 1 + 3 and (seq < 0).sum() == 3
    for i in (0, 1):
        q, s, m = C.quantise(X[i], group)
        codes, params = c.codes[i].copy(), c.params[i].copy()
        codes[page_of[stands], :, at[stands]] = C.pack(q)[stands]
        params[page_of[stands], :, at[stands]] = np.stack([s, m], -1)[stands]
        got_codes, got_params = c.pool[2 * i].cpu().numpy(), host(c.pool[2 * i + 1])
        sound = ~np.isnan(np.repeat(params[..., 0], group // 2, -1))        # codes of a group that stands for NaN are free
        sound |= codes == c.codes[i]
        untouched = np.isnan(c.params[i]).all((-1, -2))
        untouched[page_of[stands], :, at[stands]] = False
        assert np.array_equal(got_codes[untouched], c.codes[i][untouched])
        written = ~untouched
        ok = ~np.isnan(params[..., 0]).repeat(group // 2, -1)
        assert (got_codes == codes)[written][ok[written]].all()
        steps_ok = ~np.isnan(params[..., 0])
        assert same_values(got_params[..., 0], params[..., 0])
        assert np.array_equal(got_params[..., 1][steps_ok], params[..., 1][steps_ok])
        if hat:
            with np.errstate(all="ignore"):
                want = C.bf16(C.values(q, s, m).astype(np.float32))
            want[(seq >= 0) & ~stands] = 0
            assert same_values(host(out[i])[seq >= 0], want[seq >= 0])
            assert torch.equal(out[i][torch.from_numpy(seq < 0).cuda()].view(torch.int16),
                               before[i][torch.from_numpy(seq < 0).cuda()].view(torch.int16))


@pytest.mark.parametrize("D,group,H,page", GEOMETRIES)
def test_read_gives_the_values_of_the_last_tokens(eqat, D, group, H, page):
    c = Cache(eqat, D, group, H, page, [1, 0, 70, 33, 3, 200], [1, 0, 69, 33, 5, 17], seed=D + group + H, pad_rows=2)
    held = c.fill()
    guard = Guarded()
    out = [guard.empty(c.rows, H, D, dtype=torch.bfloat16, shift_bytes=16) for _ in range(2)]
    before = [o.clone() for o in out]
    eqat.eqat_cache_read(c.desc(), *c.where, *out)
    guard.check()
    for i in (0, 1):
        got = host(out[i])
        for b, (n, k) in enumerate(zip(c.lengths, c.news)):
            mine = got[c.offsets[b]:c.offsets[b + 1]]
            have = min(n, k)
            assert (mine[:k - have] == 0).all()                  # positions before the first
            assert np.array_equal(mine[k - have:], C.bf16(held[i][b][n - have:].astype(np.float32)))
        assert torch.equal(out[i][c.offsets[-1]:].view(torch.int16), before[i][c.offsets[-1]:].view(torch.int16))


def test_many_sequences_are_found(eqat):
    """More sequences than one step of the search looks at, most without rows."""
    rng = np.random.default_rng(5)
    news = [int(x) for x in rng.integers(0, 3, 1500)]
    c = Cache(eqat, 64, 64, 1, 16, [n + int(e) for n, e in zip(news, rng.integers(0, 20, 1500))], news, seed=5, pad_rows=1)
    held = c.fill()
    out = [torch.zeros(c.rows, 1, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    eqat.eqat_cache_read(c.desc(), *c.where, *out)
    for i in (0, 1):
        want = np.concatenate([h[len(h) - k:] for h, k in zip(held[i], news)])
        assert np.array_equal(host(out[i])[:-1], C.bf16(want.astype(np.float32)))


# --------------------------------------------------------------------------- attention
def score_error(size, D, group):
    """How far a score may be off: it is a sum in fp32 of terms that add up to `size` without their signs.  A matrix
    instruction adds 16 at a time and may cut where a sum would round (2 units of 2^-23 allowed for each), the groups' sums
    are scaled and added (5 operations each), the step to log2 and back takes 4 more."""
    return size * (2 * D / 16 + 5 * D / group + 4) * 2.0 ** -23


def check_attention(c, O, lse, Q, held, window=0, scale=None, rows=None):
    scale = c.D ** -0.5 if scale is None else scale
    want, want_lse, mass, size = C.attention(Q.astype(np.float64), held[0], held[1], c.lengths, c.offsets, scale, window, *c.sizes)
    delta = score_error(size, c.D, c.group)
    # the output's rounding; scores, in numerator and denominator; exp2, sums and the division in fp32; and each weight times
    # step off by half a unit, of which the largest (a weight of 1 and at least half the largest step of the row) has 2^20 or
    # more: 15 codes' worth a key, over a sum of weights of at least 1
    longest = np.concatenate([np.full(n, k) for n, k in zip(c.news, c.lengths)] + [np.zeros(c.rows - int(c.offsets[-1]))])
    unit = 15 * np.array([0.0 if not len(z) else float(z.max()) for z in c.steps])
    each = np.concatenate([np.full(n, u) for n, u in zip(c.news, unit)] + [np.zeros(c.rows - int(c.offsets[-1]))])
    bound = 1.02 * (U * np.abs(want) + (2 * delta[..., None] + 2.0 ** -16) * mass + (longest * each)[:, None, None] * 2.0 ** -21) + 1e-30
    used = slice(0, int(c.offsets[-1])) if rows is None else rows
    err = np.abs(host(O)[used].astype(np.float64) - want[used])
    bad = ~(err <= bound[used])
    assert not bad.any(), (np.argwhere(bad)[:5].tolist(), err[bad][:5], bound[used][bad][:5])
    if lse is not None:
        got = lse.cpu().numpy().astype(np.float64)[used]
        empty = np.isneginf(want_lse[used])
        assert np.array_equal(empty, np.isneginf(got))
        assert (np.abs(got - want_lse[used])[~empty] <= (delta + 2.0 ** -18 * (1 + np.abs(want_lse)))[used][~empty]).all()


def run_attention(eqat, c, q_heads, window=0, scale=None, max_new=None, Q=None, guard=None, lse=True):
    Q = C.bf16(c.rng.standard_normal((c.rows, q_heads, c.D)).astype(np.float32)) if Q is None else Q
    a = eqat.make_attention_desc(q_heads, max_new or max(max(c.news), 1), c.D ** -0.5 if scale is None else scale, window)
    guard = guard or Guarded()
    O = guard.empty(c.rows, q_heads, c.D, dtype=torch.bfloat16, shift_bytes=16)
    L = guard.empty(c.rows, q_heads, dtype=torch.float32, shift_bytes=16) if lse else None
    need = eqat.cache_workspace_bytes(c.desc(), a)
    ws = guard.empty(max(need, 256), dtype=torch.uint8) if need else None
    before = O.clone()
    eqat.eqat_cache_attention(c.desc(), a, dev(Q), *c.where, O, L, ws)
    guard.check()
    assert eqat.device_status() == (0, 0)
    n = int(c.offsets[-1])
    assert torch.equal(O[n:].view(torch.int16), before[n:].view(torch.int16))
    return Q, O, L


@pytest.mark.parametrize("D,group,H,page", GEOMETRIES)
@pytest.mark.parametrize("ratio", [1, 3, 8, 11])
def test_decoding(eqat, D, group, H, page, ratio):
    """One new token a sequence: lengths of 1, around a piece of 16, a stage, a unit, a page and several of each; none."""
    lengths = [1, 2, 15, 16, 17, 0, 31, 33, 64, 65, 127, 129, 257, 300, 511, 777]
    c = Cache(eqat, D, group, H, page, lengths, [1] * len(lengths), seed=D + ratio, pad_rows=1)
    held = c.fill()
    Q, O, lse = run_attention(eqat, c, H * ratio)
    check_attention(c, O, lse, Q, held)


@pytest.mark.parametrize("D,group,H,page", GEOMETRIES)
@pytest.mark.parametrize("window", [0, 1, 50])
def test_drafts_and_chunks(eqat, D, group, H, page, window):
    """Several new tokens: some sequences have none, some more than they hold, one is a prompt of its own."""
    lengths, news = [9, 40, 300, 3, 129, 75, 0, 500], [5, 0, 7, 5, 1, 75, 2, 16]
    c = Cache(eqat, D, group, H, page, lengths, news, seed=D + group + window, pad_rows=2)
    held = c.fill()
    Q, O, lse = run_attention(eqat, c, H * 2, window=window)
    check_attention(c, O, lse, Q, held, window)


def check_prompt(c, O, lse, Q, held, window=0, rows=None):
    """Values and weights rounded to bf16 (each off by at most U of itself); U bounds the terms of a score too."""
    want, want_lse, mass, size = C.attention(Q.astype(np.float64), held[0], held[1], c.lengths, c.offsets, c.D ** -0.5, window)
    delta = size * (U + 2 * c.D / 16 * 2.0 ** -23 + 2.0 ** -20)
    bound = 1.02 * (U * np.abs(want) + (2 * U + 2 * delta[..., None] + 2.0 ** -14) * mass) + 1e-30
    used = slice(0, int(c.offsets[-1])) if rows is None else rows
    got = host(O)[used].astype(np.float64)
    err = np.abs(got - want[used])
    bad = ~(err <= bound[used])
    assert not bad.any(), (np.argwhere(bad)[:5].tolist(), err[bad][:5], bound[used][bad][:5])
    assert np.linalg.norm(got - want[used]) <= TOL * np.linalg.norm(want[used])
    if lse is not None:
        got = lse.cpu().numpy().astype(np.float64)[used]
        seen = ~np.isneginf(want_lse[used])
        assert np.array_equal(~seen, np.isneginf(got))
        assert (np.abs(got[seen] - want_lse[used][seen]) <= delta[used][seen] + 2.0 ** -18 * (1 + np.abs(want_lse[used][seen]))).all()


@pytest.mark.parametrize("D,group,page", [(128, 128, 16), (128, 64, 48), (128, 32, 64), (64, 64, 16), (64, 32, 32)])
@pytest.mark.parametrize("window", [0, 1, 77])
@pytest.mark.parametrize("short", [0, 200])
def test_prompts(eqat, D, group, page, window, short):
    """Whole prompts, pieces behind a long text, sequences with few rows and none, in one call; with many short sequences both
    kernels take part, else the one for prompts has all."""
    lengths = [260, 300, 61, 5, 700, 1, 1, 33] + [17 + i % 80 for i in range(short)]
    news = [260, 1, 60, 0, 150, 1, 3, 33] + [1] * short
    c = Cache(eqat, D, group, 4, page, lengths, news, seed=D + group + window, pad_rows=2)
    held = c.fill()
    a = eqat.make_attention_desc(32, max(news), D ** -0.5, window)
    assert eqat.eqat_cache_attention_plan(c.desc(), a)[1] == (33 if short else 1)
    Q, O, lse = run_attention(eqat, c, 32, window=window)
    check_prompt(c, O, lse, Q, held, window)
    for _ in range(3):
        _, O2, lse2 = run_attention(eqat, c, 32, window=window, Q=Q)
        assert torch.equal(O.view(torch.int16), O2.view(torch.int16)) and torch.equal(lse, lse2)


@pytest.mark.parametrize("ratio,H", [(1, 32), (5, 8), (7, 6)])
def test_prompts_of_other_head_counts(eqat, ratio, H):
    c = Cache(eqat, 128, 128, H, 16, [190, 401], [190, 130], seed=ratio)
    held = c.fill()
    assert eqat.eqat_cache_attention_plan(c.desc(), eqat.make_attention_desc(H * ratio, 190, 0.1))[1] == 1
    Q, O, lse = run_attention(eqat, c, H * ratio)
    check_prompt(c, O, lse, Q, held)


@pytest.mark.parametrize("scale", [-0.2, 0.0, 0.6])
def test_prompts_with_other_scales(eqat, scale):
    """Maxima that rise along the sequence, by more than 2^8 at once; a negative scale; none."""
    c = Cache(eqat, 128, 128, 8, 16, [300, 520], [300, 90], seed=4)
    held = c.fill()
    Q = C.bf16((c.rng.standard_normal((c.rows, 32, 128)) * 2).astype(np.float32))
    _, O, lse = run_attention(eqat, c, 32, scale=scale, Q=Q)
    want, want_lse, mass, size = C.attention(Q.astype(np.float64), held[0], held[1], c.lengths, c.offsets, scale)
    # scores of some tens are off by up to U of their terms' sum: the error of a weight is bounded by its exponential
    delta = np.expm1(2 * size * (U + 2.0 ** -16))
    assert (np.abs(host(O) - want) <= 1.02 * (U * np.abs(want) + (2 * U + delta[..., None] + 2.0 ** -14) * (mass + np.abs(want)))).all()
    if scale <= 0.0:
        assert np.linalg.norm(host(O) - want) <= 4 * TOL * np.linalg.norm(want)


@pytest.mark.parametrize("D,group", [(128, 128), (128, 32), (64, 64)])
def test_prompts_of_keys_of_every_size(eqat, D, group):
    """Keys far above and below fp16's range, in sequences of their own and among others, with queries of the inverse size."""
    c = Cache(eqat, D, group, 4, 16, [300, 290, 400, 333], [300, 290, 200, 333], seed=D + group)
    held = c.fill()
    sizes = [2.0 ** 40, 2.0 ** -40, None, 1.0]
    for b, n in enumerate(c.lengths):
        by = np.array([1.0, 2.0 ** -16, 2.0 ** -3, 2.0 ** -9])[np.arange(n) // 3 % 4] if sizes[b] is None else np.full(n, sizes[b])
        pos = np.arange(n)
        c.params[0][c.table[b][pos // 16], :, pos % 16] *= by[:, None, None, None].astype(np.float32)
        held[0][b] = held[0][b] * by[:, None, None]
        c.sizes[0][b] = c.sizes[0][b] * by[:, None, None]
    c.upload()
    Q = c.rng.standard_normal((c.rows, 32, D)).astype(np.float32)
    for b, by in enumerate(sizes):
        Q[c.offsets[b]:c.offsets[b + 1]] *= 1.0 if by is None else np.float32(1.0 / by)
    Q = C.bf16(Q)
    assert eqat.eqat_cache_attention_plan(c.desc(), eqat.make_attention_desc(32, 333, D ** -0.5))[1] == 1
    _, O, lse = run_attention(eqat, c, 32, Q=Q)
    check_prompt(c, O, lse, Q, held)
    # a key is rounded to fp16 (2^-11), with 2^-25 of the power of two at most that its largest element is brought to (from
    # 2^-6 on): 2^-19 of the largest; a query is exact to 2^-25 of its own
    _, want_lse, _, size = C.attention(Q.astype(np.float64), held[0], held[1], c.lengths, c.offsets, D ** -0.5)
    most = np.concatenate([np.abs(Q[c.offsets[b]:c.offsets[b + 1]]).sum(-1) * np.abs(np.asarray(held[0][b])).max() for b in range(4)]) * D ** -0.5
    delta = size * (2.0 ** -11 + 2.0 ** -16) + most * 2.0 ** -18
    assert (np.abs(lse.cpu().numpy() - want_lse) <= delta + 2.0 ** -18 * (1 + np.abs(want_lse))).all()


def test_prompts_do_not_see_what_is_masked(eqat):
    """NaN keys and values at two positions: rows before them are untouched, rows behind are NaN; with a window, rows beyond
    it are untouched again.  NaN queries spoil their own rows only."""
    c = Cache(eqat, 128, 64, 8, 16, [300], [300], seed=6)
    held = c.fill()
    for i, pos in ((0, 100), (1, 140)):
        page = c.table[0][pos // 16]
        c.params[i][page, :, pos % 16] = np.nan
        held[i][0][pos] = 0.0
    c.upload()
    Q = C.bf16(c.rng.standard_normal((300, 32, 128)).astype(np.float32))
    Q[50, 3] = np.nan
    Q, O, lse = run_attention(eqat, c, 32, window=64, Q=Q)
    keep = [r for r in range(300) if r != 50 and not (100 <= r < 164 or 140 <= r < 204)]
    check_prompt(c, O, lse, np.where(np.isnan(Q), 0, Q), held, 64, rows=keep)
    got = host(O)
    assert np.isnan(got[100:204]).all() and np.isnan(got[50, 3]).all()
    assert np.isfinite(got[50, :3]).all() and np.isfinite(got[50, 4:]).all()


def test_outputs_of_another_type_or_size_are_refused(eqat):
    """On the host: nothing is launched, the outputs stay."""
    c = Cache(eqat, 128, 128, 2, 16, [40], [1], seed=9)
    c.fill()
    a = eqat.make_attention_desc(4, 1, 0.1)
    Q = torch.zeros(1, 4, 128, dtype=torch.bfloat16, device="cuda")
    O = torch.full_like(Q, 7.0)
    ws = torch.empty(max(256, eqat.cache_workspace_bytes(c.desc(), a)), dtype=torch.uint8, device="cuda")
    for lse, kind in ((torch.zeros(1, 4, dtype=torch.float16, device="cuda"), TypeError), (torch.zeros(3, device="cuda"), ValueError)):
        with pytest.raises(kind):
            eqat.eqat_cache_attention(c.desc(), a, Q, *c.where, O, lse, ws)
    with pytest.raises(TypeError):
        eqat.eqat_cache_attention(c.desc(), a, Q, *c.where, O.float(), None, ws)
    torch.cuda.synchronize()
    assert (O == 7.0).all()


def test_nan_queries_spoil_their_own_rows(eqat):
    c = Cache(eqat, 128, 128, 2, 16, [700, 40], [1, 3], seed=8)
    held = c.fill()
    Q = C.bf16(c.rng.standard_normal((c.rows, 16, 128)).astype(np.float32))
    Q[0, 5], Q[2, 1, 7] = np.nan, np.inf
    Q, O, lse = run_attention(eqat, c, 16, Q=Q)
    got, want = host(O), C.attention(np.where(np.isfinite(Q), Q, 0).astype(np.float64), held[0], held[1], c.lengths, c.offsets, 128 ** -0.5)[0]
    assert not np.isfinite(got[0, 5]).any() and not np.isfinite(got[2, 1]).any()
    got[0, 5], got[2, 1] = want[0, 5], want[2, 1]
    assert np.isfinite(got).all() and np.linalg.norm(got - want) <= TOL * np.linalg.norm(want)


def test_rows_that_see_nothing_are_zero(eqat):
    c = Cache(eqat, 128, 128, 2, 16, [0, 0, 2], [1, 3, 6], seed=1)
    held = c.fill()
    Q, O, lse = run_attention(eqat, c, 4)
    assert (host(O)[:4] == 0).all() and np.isneginf(lse.cpu().numpy()[:8]).all()
    check_attention(c, O, lse, Q, held)


@pytest.mark.parametrize("ratio", [1, 8])
def test_one_long_sequence_is_split_and_joined(eqat, ratio):
    c = Cache(eqat, 128, 128, 1, 64, [20011], [1], seed=3)
    held = c.fill()
    Q, O, lse = run_attention(eqat, c, ratio)
    check_attention(c, O, lse, Q, held)
    for _ in range(5):                                          # the same bits every time
        _, O2, lse2 = run_attention(eqat, c, ratio, Q=Q)
        assert torch.equal(O.view(torch.int16), O2.view(torch.int16)) and torch.equal(lse, lse2)


def test_large_scores(eqat):
    """Softmax weights from 1 down to nothing, maxima that rise along the sequence."""
    c = Cache(eqat, 128, 64, 2, 32, [700, 350], [1, 2], seed=4)
    held = c.fill()
    Q = C.bf16((c.rng.standard_normal((c.rows, 8, 128)) * 4).astype(np.float32))
    for scale in (0.5, -0.3, 0.0):
        _, O, lse = run_attention(eqat, c, 8, scale=scale, Q=Q)
        check_attention(c, O, lse, Q, held, scale=scale)


def test_what_a_row_does_not_see_may_be_nan(eqat):
    """The keys and values of the tokens behind a row, and of those before its window, are NaN or infinite for the other rows."""
    c = Cache(eqat, 128, 32, 2, 16, [90], [4], seed=6)
    held = c.fill()
    for i in (0, 1):
        for pos, bad in ((89, np.nan), (88, np.inf), (20, -np.inf), (21, np.nan)):
            page = c.table[0][pos // 16]
            c.params[i][page, :, pos % 16] = bad
            held[i][0][pos] = 0.0                                # row 1 (position 87) sees none of them within 64 tokens
    c.upload()
    Q, O, lse = run_attention(eqat, c, 4, window=64)
    check_attention(c, O, lse, Q, held, 64, rows=slice(0, 2))
    assert not np.isfinite(host(O)[2:]).any()


def test_one_key_above_many(eqat):
    """A key whose weight is 2^13 to 2^20 times that of each of 20000 others: theirs are few units, and their sum counts."""
    c = Cache(eqat, 128, 128, 1, 64, [20001], [1], seed=12)
    held = c.fill()
    direction = np.sign(c.rng.standard_normal(128)).astype(np.float32)
    Q = np.broadcast_to(direction, (1, 8, 128)) * np.float32([0.5, 0.75, 1, 1.25, 1.5, 1.75, 2, 2.25])[None, :, None]
    q, s, m = C.quantise(direction[None, None] * np.float32(2.0), 128)
    for pos in (0, 1, 9000, 20000):
        c.codes[0][c.table[0][pos // 64], 0, pos % 64] = C.pack(q)[0, 0]
        c.params[0][c.table[0][pos // 64], 0, pos % 64] = np.stack([s, m], -1)[0, 0]
        held[0][0][pos] = C.values(q, s, m)[0]
    c.upload()
    Q = C.bf16(Q * np.float32(0.5))
    _, O, lse = run_attention(eqat, c, 8, Q=Q)
    check_attention(c, O, lse, Q, held)
    want = C.attention(Q.astype(np.float64), held[0], held[1], c.lengths, c.offsets, 128 ** -0.5)[0]
    assert np.linalg.norm(host(O) - want) <= TOL * np.linalg.norm(want)


def test_more_rows_than_announced_are_left_out(eqat):
    c = Cache(eqat, 128, 128, 2, 16, [50, 60], [9, 3], seed=7)
    held = c.fill()
    Q, O, lse = run_attention(eqat, c, 4, max_new=4)
    rows = [0, 1, 2, 3, 9, 10, 11]
    check_attention(c, O, lse, Q, held, rows=rows)
    left = O[4:9].contiguous().view(torch.uint8)
    assert bool((left == 0xA5).all())
    c = Cache(eqat, 128, 128, 8, 16, [300, 90], [300, 70], seed=7)            # the same in the kernel for prompts
    held = c.fill()
    assert eqat.eqat_cache_attention_plan(c.desc(), eqat.make_attention_desc(32, 120, 0.1))[1] == 1
    Q, O, lse = run_attention(eqat, c, 32, max_new=120)
    check_prompt(c, O, lse, Q, held, rows=list(range(120)) + list(range(300, 370)))
    assert bool((O[120:300].contiguous().view(torch.uint8) == 0xA5).all())


def test_arrays_that_say_too_much_stay_inside(eqat):
    """Offsets beyond the rows, lengths beyond the table, pages outside the pool: values are free, accesses are not (the
    guards around every output; the pool is unchanged)."""
    c = Cache(eqat, 128, 128, 2, 16, [100, 40, 64], [1, 2, 1], seed=8)
    held = c.fill()
    c.where[0] = torch.tensor([0, 1, 3, 900], dtype=torch.int32, device="cuda")
    c.where[1] = torch.tensor([100, -5, 1 << 30], dtype=torch.int32, device="cuda")
    c.where[2][2] = torch.tensor([1 << 30, -1, c.pages, 5, -(1 << 31), 0, 1][:c.max_pages], dtype=torch.int32, device="cuda")
    guard = Guarded()
    O = guard.empty(c.rows, 4, 128, dtype=torch.bfloat16)
    K, V = (guard.empty(c.rows, 2, 128, dtype=torch.bfloat16) for _ in range(2))
    a = eqat.make_attention_desc(4, 2, 0.1)
    need = eqat.cache_workspace_bytes(c.desc(), a)
    ws = guard.empty(max(need, 256), dtype=torch.uint8)
    pool = [t.clone() for t in c.pool]
    Q = torch.randn(c.rows, 4, 128, device="cuda").to(torch.bfloat16)
    eqat.eqat_cache_attention(c.desc(), a, Q, *c.where, O, None, ws)
    eqat.eqat_cache_read(c.desc(), *c.where, K, V)
    guard.check()
    assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(pool, c.pool))
    assert bool(torch.isfinite(O[:1].float()).all()) and bool((O[1:3] == 0).all())          # length -5 is 0
    eqat.eqat_cache_append(c.desc(), K, V, *c.where)            # positions 95.. of sequence 0 and what has a page
    torch.cuda.synchronize()
    assert eqat.device_status() == (0, 0)


def test_long_pools(eqat):
    """Codes beyond 2^32 bytes: the last pages of a pool of 4.6 GB of keys."""
    H, D, page, pages = 8, 128, 64, 140000
    kc, vc = (torch.zeros(pages, H, page, D // 2, dtype=torch.uint8, device="cuda") for _ in range(2))
    kp, vp = (torch.zeros(pages, H, page, 1, 2, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    assert kc.numel() > 1 << 32
    n, pool = 150, (kc, kp, vc, vp)
    table = torch.tensor([[pages - 1, 3, pages - 2]], dtype=torch.int32, device="cuda")
    X = [torch.randn(n, H, D, device="cuda").to(torch.bfloat16) for _ in range(2)]
    off, length = torch.tensor([0, n], dtype=torch.int32, device="cuda"), torch.tensor([n], dtype=torch.int32, device="cuda")
    d = eqat.make_cache_desc(128, D, H, page, pages, 1, 3, n)
    hat, back = ([torch.zeros(n, H, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)] for _ in range(2))
    eqat.eqat_cache_append(d, *X, off, length, table, pool, *hat)
    eqat.eqat_cache_read(d, off, length, table, pool, *back)
    for x, h, r in zip(X, hat, back):
        q, s, m = C.quantise(host(x), 128)
        want = C.bf16(C.values(q, s, m).astype(np.float32))
        assert np.array_equal(host(h), want) and np.array_equal(host(r), want)
    d1 = eqat.make_cache_desc(128, D, H, page, pages, 1, 3, 1)
    off1, Q = torch.tensor([0, 1], dtype=torch.int32, device="cuda"), torch.randn(1, 2 * H, D, device="cuda").to(torch.bfloat16)
    a = eqat.make_attention_desc(2 * H, 1, D ** -0.5)
    need = eqat.cache_workspace_bytes(d1, a)
    O = torch.zeros(1, 2 * H, D, dtype=torch.bfloat16, device="cuda")
    eqat.eqat_cache_attention(d1, a, Q, off1, length, table, pool, O, None, torch.empty(max(need, 1), dtype=torch.uint8, device="cuda"))
    want = C.attention(host(Q).astype(np.float64), [host(back[0]).astype(np.float64)], [host(back[1]).astype(np.float64)], [n], [0, 1], D ** -0.5)
    # read rounds the keys and values to bf16 where the attention does not: 2^-8 of each, in the score and in the value
    assert (np.abs(host(O) - want[0]) <= 4 * U * want[2] + 2 * U * want[3][..., None] * want[2]).all()
    assert eqat.device_status() == (0, 0)


def test_streams_and_graphs(eqat):
    """Two batches on two streams with a workspace each, and a captured step replayed after lengths, tables and queries have
    changed in place."""
    c = Cache(eqat, 128, 128, 2, 16, [3000, 50, 900], [1, 1, 1], seed=9, max_pages=200)
    held = c.fill()
    Q, O, lse = run_attention(eqat, c, 16)
    a = eqat.make_attention_desc(16, 1, 128 ** -0.5)
    need = eqat.cache_workspace_bytes(c.desc(), a)
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.zeros_like(O) for _ in range(2)]
    work = [torch.empty(need, dtype=torch.uint8, device="cuda") for _ in range(2)]
    q = dev(Q)
    torch.cuda.synchronize()
    for _ in range(20):
        for s, o, w in zip(streams, outs, work):
            with torch.cuda.stream(s):
                eqat.eqat_cache_attention(c.desc(), a, q, *c.where, o, None, w)
    torch.cuda.synchronize()
    assert all(torch.equal(o.view(torch.int16), O.view(torch.int16)) for o in outs)

    K, V = (dev(c.tokens(c.rows)) for _ in range(2))
    hat = [torch.zeros(c.rows, 2, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    graph, o = torch.cuda.CUDAGraph(), torch.zeros_like(O)
    pool = [t.clone() for t in c.pool]
    with torch.cuda.graph(graph):
        eqat.eqat_cache_append(c.desc(), K, V, *c.where, *hat)
        eqat.eqat_cache_attention(c.desc(), a, q, *c.where, o, None, work[0])
    for lengths in ([3000, 50, 900], [1000, 51, 16], [2, 1, 3000]):
        c2 = Cache(eqat, 128, 128, 2, 16, lengths, [1, 1, 1], seed=sum(lengths), max_pages=200, spare_pages=c.pages - sum((n + 15) // 16 for n in lengths))
        assert c2.pages == c.pages
        held = c2.fill()
        for t, n in zip(c.pool, c2.pool):
            t.copy_(n)
        for i in (1, 2):
            c.where[i].copy_(c2.where[i])
        graph.replay()
        torch.cuda.synchronize()
        for i, x in enumerate((K, V)):
            vals = C.values(*C.quantise(host(x), 128))
            q8, s8, m8 = C.quantise(host(x), 128)
            for b in range(3):
                held[i][b][-1] = vals[b]
                s, m = s8[b].astype(np.float64), m8[b].astype(np.float64)
                c2.sizes[i][b][-1] = s * 15 + np.abs(m)
        check_attention(c2, o, None, Q, held)
    assert eqat.device_status() == (0, 0)


def test_the_wait_that_runs_out_is_reported(eqat):
    assert eqat.device_status() == (0, 0)
    for which in (5, 6):
        eqat.eqat_selftest_wait_expiry(which)
        assert eqat.device_status()[0] == eqat.EQAT_ERR_TIMEOUT and eqat.device_status() == (0, 0)


def test_a_decoding_block(eqat):
    """Prompt and decoding steps of a small attention block on packed weights: projection, cache, attention, projection, each
    on what the call before has left on the device, against the same steps in 64 bits."""
    heads, kv, D, hidden, g = 8, 2, 64, 512, 64
    gen = torch.Generator(device="cuda").manual_seed(11)

    def linear(out, inp):
        W = (torch.randn(out, inp, device="cuda", generator=gen) * inp ** -0.5).to(torch.bfloat16)
        d = eqat.make_desc(4, g, out, inp)
        s, z = (torch.empty(out, inp // g, device="cuda") for _ in range(2))
        P = torch.empty(out, inp // 2, dtype=torch.uint8, device="cuda")
        z8, s16 = torch.empty(out, inp // g, dtype=torch.uint8, device="cuda"), torch.empty(out, inp // g, dtype=torch.float16, device="cuda")
        codes = torch.empty(out, inp, dtype=torch.uint8, device="cuda")
        eqat.eqat_minmax_init(d, W, s, z)
        eqat.eqat_quantize_pack(d, W, s, z, P, z8, s16)
        eqat.eqat_unpack(d, P, codes)
        w64 = (codes.double().view(out, -1, g) - z8.double()[..., None]).mul(s16.double()[..., None]).view(out, inp)
        return (P, s16, z8), w64

    qkv, w_qkv = linear((heads + 2 * kv) * D, hidden)
    proj, w_o = linear(hidden, heads * D)
    page, lens = 16, [23, 1, 40]
    max_pages, pages = 4, 12
    pool = tuple(t for _ in range(2) for t in (torch.zeros(pages, kv, page, D // 2, dtype=torch.uint8, device="cuda"),
                                              torch.full((pages, kv, page, 1, 2), float("nan"), dtype=torch.bfloat16, device="cuda")))
    table = torch.randperm(pages, generator=torch.Generator().manual_seed(1)).int().view(3, max_pages).cuda()
    keys, vals = [[] for _ in lens], [[] for _ in lens]
    have, news = [0, 0, 0], lens
    for step in range(6):
        rows = sum(news)
        have = [h + n for h, n in zip(have, news)]
        off = torch.tensor([0, *np.cumsum(news)], dtype=torch.int32, device="cuda")
        length = torch.tensor(have, dtype=torch.int32, device="cuda")
        X = torch.randn(rows, hidden, device="cuda", generator=gen).to(torch.bfloat16)
        fused = torch.empty(rows, (heads + 2 * kv) * D, dtype=torch.bfloat16, device="cuda")
        eqat.qlinear_packed_fwd(eqat.make_desc(4, g, (heads + 2 * kv) * D, hidden, rows), X, *qkv, fused)
        q, k, v = (fused[:, a * D:b * D].unflatten(1, (-1, D)) for a, b in ((0, heads), (heads, heads + kv), (heads + kv, heads + 2 * kv)))
        d = eqat.make_cache_desc(64, D, kv, page, pages, 3, max_pages, rows)
        a = eqat.make_attention_desc(heads, max(news), D ** -0.5)
        hat = [torch.empty(rows, kv, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        O = torch.empty(rows, heads, D, dtype=torch.bfloat16, device="cuda")
        Y = torch.empty(rows, hidden, dtype=torch.bfloat16, device="cuda")
        need = eqat.cache_workspace_bytes(d, a)
        ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
        eqat.eqat_cache_append(d, k, v, off, length, table, pool, *hat)
        eqat.eqat_cache_attention(d, a, q, off, length, table, pool, O, None, ws)
        eqat.qlinear_packed_fwd(eqat.make_desc(4, g, hidden, heads * D, rows), O.view(rows, -1), *proj, Y)

        # the projection's own output feeds the reference's cache: its error is tested where it belongs
        x64 = X.double() @ w_qkv.T
        assert float((fused.double() - x64).norm() / x64.norm()) < 5e-3
        at = 0
        for b, n in enumerate(news):
            for store, t in ((keys, k), (vals, v)):
                store[b].append(C.values(*C.quantise(host(t[at:at + n]), 64)))
            at += n
        want = C.attention(host(q).astype(np.float64), [np.concatenate(s) for s in keys], [np.concatenate(s) for s in vals], have,
                           off.cpu().numpy(), D ** -0.5)[0]
        y64 = torch.from_numpy(want).cuda().view(rows, -1) @ w_o.T
        # three roundings to bf16 on the way (softmax weights, O, Y) and the weight's in the product: 2^-8 each at most
        assert float((Y.double() - y64).norm() / y64.norm()) < 4 * U
        news = [1, 1, 1] if step % 2 == 0 else [1, 0, 2]
    assert eqat.device_status() == (0, 0)
