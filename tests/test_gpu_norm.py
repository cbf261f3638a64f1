"""Root-mean-square norm against the oracle: residual, bf16 and 8-bit outputs, gradient.

Bounds.  Statistics are sums of at most 32768 terms, of which a thread adds up 64 in a row before they meet in a tree: c is right to
2^-18 of itself, and with it every output before its rounding, except where dx cancels, whose terms' sizes count instead."""
import numpy as np
import pytest
import torch

from helpers import Guarded, assert_elementwise, torch_to_f64
from oracle import between_oracle as B

pytestmark = pytest.mark.gpu
HALF_STEP, STATS = 2.0 ** -8, 2.0 ** -17
EPS = 1e-5


@pytest.fixture(scope="module")
def eqat():
    from paper_2407_11062_b200.build import build_library
    build_library()
    from paper_2407_11062_b200 import binding
    return binding


def rows_of(rows, n, seed, std=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, n, device="cuda", generator=g) * std
    return (x * torch.where(torch.rand(n, device="cuda", generator=g) < 0.02, 15.0, 1.0)).to(torch.bfloat16)


def weight_of(n, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (1 + 0.3 * torch.randn(n, device="cuda", generator=g)).to(torch.bfloat16)


# widths on both sides of each way to share a row out, odd ones among them; rows: one, a few, more than there are blocks
SHAPES = [(1, 8), (3, 64), (1, 256), (9, 264), (5, 512), (4, 520), (1, 4096), (700, 4096), (37, 5120), (2, 8192), (5, 8200), (3, 16384), (2, 16392),
          (2, 32768), (5003, 128), (20000, 40), (1237, 1000)]


@pytest.mark.parametrize("rows,n", SHAPES)
@pytest.mark.parametrize("residual", [True, False])
def test_forward(eqat, rows, n, residual):
    X, R, W, buf = rows_of(rows, n, 1), rows_of(rows, n, 2) if residual else None, weight_of(n, 3), Guarded()
    H, Y = (buf.empty(rows, n, dtype=torch.bfloat16, shift_bytes=s) for s in (0, 16))
    eqat.eqat_rms_norm_fwd(eqat.make_norm_desc(rows, n, EPS), X, R, W, H, Y)
    buf.check()
    want = X if R is None else (X.float() + R.float()).to(torch.bfloat16)
    assert torch.equal(H, want)
    y = B.norm_fwd(torch_to_f64(H), torch_to_f64(W), EPS)
    assert_elementwise(torch_to_f64(Y), y, (HALF_STEP + STATS) * np.abs(y) + 2.0 ** -133, "Y")
    again, Y2 = (X.clone() if R is None else R.clone()), torch.empty_like(Y)      # in place, and without the sum
    eqat.eqat_rms_norm_fwd(eqat.make_norm_desc(rows, n, EPS), again if R is None else X, None if R is None else again, W, again, Y2)
    assert torch.equal(again, H) and torch.equal(Y2, Y)
    eqat.eqat_rms_norm_fwd(eqat.make_norm_desc(rows, n, EPS), X, R, W, None, Y2.zero_())
    assert torch.equal(Y2, Y)


@pytest.mark.parametrize("rows,n,group", [(1, 32, 32), (1, 8, 8), (3, 64, 32), (1, 4096, 128), (700, 4096, 64), (37, 5120, 256), (37, 5120, 32), (2, 8192, 8192),
                                          (3, 16384, 128), (2, 32768, 32768), (2, 32768, 256), (5003, 128, 128), (1237, 1000, 1000), (9, 288, 32), (6, 16640, 256)])
@pytest.mark.parametrize("kind", ["int8", "e4m3"])
def test_codes(eqat, rows, n, group, kind):
    """Codes to the bit: products of bf16 numbers are exact, the quotient and the products with it are rounded once each."""
    code, top = (eqat.EQAT_CODES_INT8, B.INT8_TOP) if kind == "int8" else (eqat.EQAT_CODES_E4M3, B.E4M3_TOP)
    X, R, W, buf = rows_of(rows, n, 4), rows_of(rows, n, 5), weight_of(n, 6), Guarded()
    if rows > 1:
        X[1], R[1] = 0, 0
    H, Y = (buf.empty(rows, n, dtype=torch.bfloat16) for _ in range(2))
    codes = buf.empty(rows, n, dtype=torch.int8 if kind == "int8" else torch.float8_e4m3fn, shift_bytes=16)
    scales = buf.empty(rows, n // group, shift_bytes=48)
    d = eqat.make_norm_desc(rows, n, EPS, code, group)
    eqat.eqat_rms_norm_fwd(d, X, R, W, H, Y, codes, scales)
    buf.check()
    q, s = B.norm_codes(H.float().cpu().numpy(), W.float().cpu().numpy(), EPS, group, top)
    assert np.array_equal(codes.float().cpu().numpy(), q)
    # the scale: c, a product and a constant rounded to 2^-24
    assert_elementwise(torch_to_f64(scales), s, (STATS + 2.0 ** -21) * s, "scales")
    if group >= 32:
        # the largest of a group reaches the top; no step more than half of one away from what it stands for
        y, lost = B.norm_fwd(torch_to_f64(H), torch_to_f64(W), EPS), np.repeat(s, group, -1)
        bound = 0.501 * lost if kind == "int8" else 2.0 ** -4 * np.abs(y) * 1.01 + lost * 2.0 ** -10
        assert_elementwise(q * lost, y, bound + 1e-30, "what codes stand for")
    want = q * np.repeat(torch_to_f64(scales), group, -1)
    assert_elementwise(torch_to_f64(Y), want, (HALF_STEP + 2.0 ** -22) * np.abs(want) + 2.0 ** -133, "Y of codes")
    only, sc = torch.empty_like(codes), torch.empty_like(scales)
    eqat.eqat_rms_norm_fwd(d, H, None, W, None, None, only, sc)
    assert torch.equal(only.view(torch.uint8), codes.view(torch.uint8)) and torch.equal(sc, scales)


def test_codes_at_the_edges(eqat):
    """Ties go to even, groups below 2^-110 hold zeros, large ones do not overflow."""
    n, one = 64, torch.ones(64, device="cuda", dtype=torch.bfloat16)
    rows = torch.zeros(7, n, dtype=torch.bfloat16)
    rows[0, 0], rows[0, 1:9] = 127, torch.tensor([0.5, 1.5, 2.5, -0.5, -1.5, -2.5, 126.5, 3.5])
    rows[1] = 2.0 ** -121
    rows[2, :3] = torch.tensor([2.0 ** -120, 2.0 ** -121, -(2.0 ** -120)])
    rows[3, :2] = torch.tensor([3.0e38, -1.5e38])
    rows[5, :3] = torch.tensor([2.0 ** -110, 2.0 ** -111, -(2.0 ** -110)])
    rows[6] = 2.0 ** -111
    X = rows.cuda()
    for kind, top in ((eqat.EQAT_CODES_INT8, B.INT8_TOP), (eqat.EQAT_CODES_E4M3, B.E4M3_TOP)):
        codes, scales = torch.empty(7, n, dtype=torch.int8 if kind == 1 else torch.float8_e4m3fn, device="cuda"), torch.empty(7, 2, device="cuda")
        eqat.eqat_rms_norm_fwd(eqat.make_norm_desc(7, n, EPS, kind, 32), X, None, one, None, None, codes, scales)
        q, _ = B.norm_codes(rows.float().numpy(), one.float().cpu().numpy(), EPS, 32, top)
        assert np.array_equal(codes.float().cpu().numpy(), q)
        assert (codes[5].float() != 0).sum() == 3 and (scales[[1, 2, 4, 6]] == 0).all() and torch.isfinite(scales).all()
        if kind == 1:
            assert codes[0, :9].tolist() == [127, 0, 2, 2, 0, -2, -2, 126, 4]


@pytest.mark.parametrize("n", [64, 1000, 4096])
def test_values_that_are_no_numbers(eqat, n):
    """A NaN takes its row, an infinity itself and the others of its row to zero; other rows do not hear of it."""
    X, W = rows_of(6, n, 7), weight_of(n, 8)
    X[1, 3], X[3, 5], X[4, 7] = float("nan"), float("inf"), float("-inf")
    d, Y = eqat.make_norm_desc(6, n, EPS), torch.empty_like(X)
    eqat.eqat_rms_norm_fwd(d, X, None, W, None, Y)
    clean = X.clone()
    clean[[1, 3, 4]] = 1
    Z = torch.empty_like(Y)
    eqat.eqat_rms_norm_fwd(d, clean, None, W, None, Z)
    assert torch.equal(Y[[0, 2, 5]], Z[[0, 2, 5]]) and Y[1].isnan().all()
    for row, at in ((3, 5), (4, 7)):
        assert Y[row, at].isnan() and (Y[row] == 0).sum() == n - 1
    codes, scales = torch.empty(6, n, dtype=torch.int8, device="cuda"), torch.empty(6, 1, device="cuda")
    eqat.eqat_rms_norm_fwd(eqat.make_norm_desc(6, n, EPS, eqat.EQAT_CODES_INT8, n), X, None, W, None, Y, codes, scales)
    assert scales[:, 0].isnan().tolist() == [False, True, False, True, True, False] and Y[1].isnan().all()


def test_rows_beyond_the_range(eqat):
    """Squares past binary32: zeros.  No eps and no size: NaN; no eps and a small row: as by the formula."""
    X = torch.ones(4, 128, dtype=torch.bfloat16, device="cuda")
    X[1], X[2], X[3] = 2.0 ** 100, 0, 2.0 ** -30
    W, Y = weight_of(128, 30), torch.empty_like(X)
    eqat.eqat_rms_norm_fwd(eqat.make_norm_desc(4, 128, 0.0), X, None, W, None, Y)
    assert torch.equal(Y[0], W) and (Y[1] == 0).all() and Y[2].isnan().all() and torch.equal(Y[3], W)


@pytest.mark.parametrize("rows,n", SHAPES)
@pytest.mark.parametrize("residual", [True, False])
def test_backward(eqat, rows, n, residual):
    H, dY, W, buf = rows_of(rows, n, 9), rows_of(rows, n, 10, 0.01), weight_of(n, 11), Guarded()
    dR = rows_of(rows, n, 12, 0.01) if residual else None
    d = eqat.make_norm_desc(rows, n, EPS)
    dX, dW = buf.empty(rows, n, dtype=torch.bfloat16, shift_bytes=16), buf.empty(n, shift_bytes=32)
    need = eqat.rms_norm_workspace_bytes(d)
    ws = buf.empty(need, dtype=torch.uint8)
    eqat.eqat_rms_norm_bwd(d, dY, H, W, dR, dX, dW, ws)
    buf.check()
    h, dy, w = (torch_to_f64(t) for t in (H, dY, W))
    dx, dw = B.norm_bwd(dy, h, w, EPS, None if dR is None else torch_to_f64(dR))
    c = B.norm_scale(h, EPS)
    v = np.abs(dy * w)
    terms = c * (v + np.abs(h) * c * c * (v * np.abs(h)).mean(-1, keepdims=True)) + (0 if dR is None else np.abs(torch_to_f64(dR)))
    assert_elementwise(torch_to_f64(dX), dx, HALF_STEP * np.abs(dx) + 1.01 * STATS * terms + 2.0 ** -133, "dX")
    # a column's products are added up in chains of rows / blocks, at most 200 here, then by blocks
    assert_elementwise(torch_to_f64(dW), dw, (STATS + 300 * 2.0 ** -24) * (np.abs(dy * h) * c).sum(0) + 1e-37, "dW")
    first, second = dX.clone(), dW.clone()
    ws.fill_(0xFF)                                                              # in place; the same bits again
    over = dY.clone()
    eqat.eqat_rms_norm_bwd(d, over, H, W, dR, over, dW.zero_(), ws)
    assert torch.equal(over, first) and torch.equal(dW, second)
    if residual:
        over = dR.clone()
        eqat.eqat_rms_norm_bwd(d, dY, H, W, over, over, dW.zero_(), ws)
        assert torch.equal(over, first) and torch.equal(dW, second)
    eqat.eqat_rms_norm_bwd(d, dY, H, W, dR, dX.zero_())
    assert torch.equal(dX, first)


def test_gradient_against_differences(eqat):
    """The forward pass itself, moved along a direction: (L(h + t) - L(h - t)) / 2t against <dx, direction>.  What bf16 does to y is
    taken out by the oracle's forward pass on the same h: the kernel's gradient, rounded at 2^-8, against differences in 64 bits."""
    rows, n = 5, 640
    H, dY, W = rows_of(rows, n, 13), rows_of(rows, n, 14), weight_of(n, 15)
    dX, dW = torch.empty_like(H), torch.empty(n, device="cuda")
    d = eqat.make_norm_desc(rows, n, EPS)
    ws = torch.empty(eqat.rms_norm_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    eqat.eqat_rms_norm_bwd(d, dY, H, W, None, dX, dW, ws)
    h, dy, w = (torch_to_f64(t) for t in (H, dY, W))
    rng = np.random.default_rng(16)
    for _ in range(8):
        a, b, t = rng.standard_normal((rows, n)), rng.standard_normal(n), 2.0 ** -16
        loss = lambda s: (dy * B.norm_fwd(h + s * a, w + s * b, EPS)).sum()  # noqa: E731
        slope = (loss(t) - loss(-t)) / (2 * t)
        got = (torch_to_f64(dX) * a).sum() + (torch_to_f64(dW) * b).sum()
        room = HALF_STEP * np.sqrt((torch_to_f64(dX) ** 2 * a * a).sum()) * 8 + STATS * (np.abs(dy * h).sum(0) * np.abs(b)).sum()
        assert abs(got - slope) <= room + 1e-6 * abs(slope), (got, slope, room)


def test_streams_and_graphs(eqat):
    """Two captured calls on streams of their own, replayed side by side with new inputs, each with its workspace."""
    rows, n = 300, 2048
    W, d = weight_of(n, 17), None
    d = eqat.make_norm_desc(rows, n, EPS)
    sets, graphs = [], []
    for i in range(2):
        s = {k: rows_of(rows, n, 20 + 5 * i + j) for j, k in enumerate(("X", "R", "dY", "dR"))}
        s.update(H=torch.empty_like(s["X"]), Y=torch.empty_like(s["X"]), dX=torch.empty_like(s["X"]), dW=torch.empty(n, device="cuda"),
                 ws=torch.empty(eqat.rms_norm_workspace_bytes(d), dtype=torch.uint8, device="cuda"))
        sets.append(s)

    def call(s):
        eqat.eqat_rms_norm_fwd(d, s["X"], s["R"], W, s["H"], s["Y"])
        eqat.eqat_rms_norm_bwd(d, s["dY"], s["H"], W, s["dR"], s["dX"], s["dW"], s["ws"])

    call(sets[0])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s, stream in zip(sets, streams):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            call(s)
        graphs.append(g)
    for s in sets:
        s["X"].copy_(rows_of(rows, n, 40))
        s["R"].mul_(2)
    torch.cuda.synchronize()
    for _ in range(3):
        for g, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                g.replay()
    torch.cuda.synchronize()
    got = [[s[k].clone() for k in ("H", "Y", "dX", "dW")] for s in sets]
    for s, was in zip(sets, got):
        call(s)
        assert all(torch.equal(s[k], w) for k, w in zip(("H", "Y", "dX", "dW"), was))
