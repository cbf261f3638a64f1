"""Calls between a block's linears that a program may make and a first test does not: tensors past 2^31 elements, two captured calls
at once, weights that start on any 16 bytes, the same weight twice, results in the place of each input that allows it."""
import numpy as np
import pytest
import torch

from helpers import Guarded, assert_elementwise, torch_to_f64
from test_gpu_gated import FUNCTION, GONE, HALF_STEP, both_weights, normal, projected
from test_gpu_norm import rows_of, weight_of
from oracle import between_oracle as B

pytestmark = pytest.mark.gpu
EPS = 1e-5


@pytest.fixture(scope="module")
def eqat():
    from paper_2407_11062_b200.build import build_library
    build_library()
    from paper_2407_11062_b200 import binding
    return binding


def same_all_through(big, part):
    """A tensor whose inputs repeat every len(part) rows repeats with them."""
    n = part.shape[0]
    for at in range(0, big.shape[0], n):
        assert torch.equal(big[at:at + n].view(torch.uint8), part.view(torch.uint8)), at


# ---------------------------------------------------------------------------------------------- more than 2^31 elements
def test_norm_past_31_bits(eqat):
    part, times, n = 1000, 66, 32768
    small = {k: rows_of(part, n, i) for i, k in enumerate(("X", "R", "dY"))}
    big = {k: t.repeat(times, 1) for k, t in small.items()}
    W, rows = weight_of(n, 9), part * times
    assert rows * n > 2 ** 31
    want, got = [], []
    for s, T, out in ((small, part, want), (big, rows, got)):
        d = eqat.make_norm_desc(T, n, EPS, eqat.EQAT_CODES_E4M3, 128)
        codes, scales = torch.empty(T, n, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(T, n // 128, device="cuda")
        eqat.eqat_rms_norm_fwd(d, s["X"], s["R"], W, s["R"], None, codes, scales)                 # the sum in place of R
        Y, dX = torch.empty_like(s["X"]), s["dY"]
        eqat.eqat_rms_norm_fwd(eqat.make_norm_desc(T, n, EPS), s["R"], None, W, None, Y)
        eqat.eqat_rms_norm_bwd(d, s["dY"], s["R"], W, s["X"], dX)
        out.extend([codes, scales, s["R"], Y, dX])
    for a, b in zip(got, want):
        same_all_through(a, b)


def test_rotary_past_31_bits(eqat):
    part, times, q_heads, kv_heads, dim = 997, 68, 128, 128, 128
    Q, K = (normal(part, h, dim, seed=i) for i, h in enumerate((q_heads, kv_heads)))
    pos, turns = torch.arange(part, dtype=torch.int32, device="cuda") * 131, eqat.rotary_turns(dim).cuda()
    rows = part * times
    assert rows * (q_heads + kv_heads) * dim > 2 ** 31
    small = torch.empty(part, q_heads + kv_heads, dim, dtype=torch.bfloat16, device="cuda")
    heads = lambda t: (t[:, :q_heads], t[:, q_heads:])  # noqa: E731
    eqat.eqat_rotary_fwd(eqat.make_rotary_desc(part, q_heads, kv_heads, dim), Q, K, turns, *heads(small), pos)
    both = torch.cat([Q, K], 1).repeat(times, 1, 1)
    eqat.eqat_rotary_fwd(eqat.make_rotary_desc(rows, q_heads, kv_heads, dim), *heads(both), turns, *heads(both), pos.repeat(times))
    same_all_through(both, small)


def test_gated_past_31_bits(eqat):
    """The tiled kernel's rows are the same sums wherever they stand in a tile."""
    part, times, out, width = 2048, 98, 11008, 128
    gate, up = both_weights(out, width, 2, 64, False)
    T = part * times
    assert T * out > 2 ** 31
    X, dH = normal(part, width, seed=1), normal(part, out, seed=2)
    d = eqat.make_desc(2, 64, out, width, T)
    assert eqat.workspace_bytes(d, eqat.EQAT_OP_PACKED_GATED_FWD) == eqat.workspace_bytes(d, eqat.EQAT_OP_PACKED_GATED_BWD) == 0
    H, G, U = (torch.empty(T, out, dtype=torch.bfloat16, device="cuda") for _ in range(3))
    eqat.qlinear_packed_gated_fwd(d, eqat.EQAT_ACT_SILU, X.repeat(times, 1), gate.on, up.on, H, G, U)
    for t, w in ((G, gate), (U, up)):
        want, room = projected(torch_to_f64(X[-64:]), w.value)
        assert_elementwise(torch_to_f64(t[-64:]), want, room, "projection")
    for t in (H, G, U):
        same_all_through(t, t[:part].clone())
    e = eqat.make_gated_desc(T, out)
    H2 = torch.empty_like(H)
    eqat.eqat_gated_fwd(e, G, U, H2)
    same_all_through(H2, H2[:part].clone())
    one = torch.empty(part, out, dtype=torch.bfloat16, device="cuda")
    eqat.eqat_gated_fwd(eqat.make_gated_desc(part, out), G[:part], U[:part], one)
    assert torch.equal(one, H2[-part:])
    del H, H2
    dX, dHs = torch.empty(T, width, dtype=torch.bfloat16, device="cuda"), dH.repeat(times, 1)
    dG, dU = (torch.empty(part, out, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    eqat.eqat_gated_bwd(eqat.make_gated_desc(part, out), dH, G[:part], U[:part], dG, dU)
    eqat.qlinear_packed_gated_bwd(d, eqat.EQAT_ACT_SILU, dHs, G, U, gate.on, up.on, dX, G, dHs)    # dU in the place of dH
    same_all_through(G, dG)
    same_all_through(dHs, dU)
    same_all_through(dX, dX[:part].clone())
    assert eqat.device_status() == (0, 0)


def test_wide_inputs_past_31_bits(eqat):
    part, times, out, width = 2048, 98, 64, 11008
    gate, up = both_weights(out, width, 4, 128, False)
    T = part * times
    X, dH = normal(part, width, seed=3).repeat(times, 1), normal(part, out, seed=4).repeat(times, 1)
    d = eqat.make_desc(4, 128, out, width, T)
    H, G, U = (torch.empty(T, out, dtype=torch.bfloat16, device="cuda") for _ in range(3))
    need = eqat.workspace_bytes(d, eqat.EQAT_OP_PACKED_GATED_BWD)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    eqat.qlinear_packed_gated_fwd(d, eqat.EQAT_ACT_GELU, X, gate.on, up.on, H, G, U)
    for t in (H, G, U):
        same_all_through(t, t[:part].clone())
    eqat.qlinear_packed_gated_bwd(d, eqat.EQAT_ACT_GELU, dH, G, U, gate.on, up.on, X, G, U, ws)
    same_all_through(X, X[:part].clone())
    assert eqat.device_status() == (0, 0)


# ---------------------------------------------------------------------------------------------- places and weights
@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("rows,n,group", [(1500, 4096, 64), (4000, 256, 32), (900, 16384, 16384)])
def test_codes_with_the_sum_in_place(eqat, kind, rows, n, group):
    """The rows that a block has asked for ahead are not those that it writes."""
    code = eqat.EQAT_CODES_INT8 if kind == "int8" else eqat.EQAT_CODES_E4M3
    X, R, W, d = rows_of(rows, n, 1), rows_of(rows, n, 2), weight_of(n, 3), eqat.make_norm_desc(rows, n, EPS, code, group)
    got = []
    for place in (None, "X", "R"):
        x, r = X.clone(), R.clone()
        H = {None: torch.empty_like(X), "X": x, "R": r}[place]
        codes, scales, Y = torch.empty(rows, n, dtype=torch.uint8, device="cuda"), torch.empty(rows, n // group, device="cuda"), torch.empty_like(X)
        eqat.eqat_rms_norm_fwd(d, x, r, W, H, Y, codes, scales)
        got.append((H, Y, codes, scales))
    for other in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(other, got[0]))


def test_a_backward_pass_takes_the_forward_descriptor(eqat):
    rows, n = 40, 512
    H, dY, W = rows_of(rows, n, 4), rows_of(rows, n, 5), weight_of(n, 6)
    got = []
    for d in (eqat.make_norm_desc(rows, n, EPS), eqat.make_norm_desc(rows, n, EPS, eqat.EQAT_CODES_INT8, 64)):
        dX, dW = torch.empty_like(H), torch.empty(n, device="cuda")
        eqat.eqat_rms_norm_bwd(d, dY, H, W, None, dX, dW, torch.empty(eqat.rms_norm_workspace_bytes(d), dtype=torch.uint8, device="cuda"))
        got.append((dX, dW))
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_products_past_the_range(eqat):
    """h w past binary32: NaN there, and 0 in the rest of the row, whose squares pass it as well."""
    X, W = torch.full((2, 64), 2.0 ** 127, dtype=torch.bfloat16, device="cuda"), torch.ones(64, dtype=torch.bfloat16, device="cuda")
    X[1], W[5] = 1, 4
    Y = torch.empty_like(X)
    eqat.eqat_rms_norm_fwd(eqat.make_norm_desc(2, 64, 0.0), X, None, W, None, Y)
    assert Y[0, 5].isnan() and (Y[0] == 0).sum() == 63 and torch.equal(Y[1], W)


def test_gated_gradients_in_every_place(eqat):
    d, rows, n = eqat.make_gated_desc(33, 264), 33, 264
    src = {k: normal(rows, n, seed=i) for i, k in enumerate(("dH", "G", "U"))}
    want = [torch.empty_like(src["G"]) for _ in range(2)]
    eqat.eqat_gated_bwd(d, src["dH"], src["G"], src["U"], *want)
    for a in (None, "dH", "G", "U"):
        for b in (None, "dH", "G", "U"):
            if a is None or a != b:
                t = {k: v.clone() for k, v in src.items()}
                out = [t[k] if k else torch.empty_like(want[0]) for k in (a, b)]
                eqat.eqat_gated_bwd(d, t["dH"], t["G"], t["U"], *out)
                assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1]), (a, b)


@pytest.mark.parametrize("T", [1, 5, 24, 100, 300, 1500])
@pytest.mark.parametrize("bits,group,fp16", [(2, 64, False), (2, 128, True), (3, 32, False), (3, 256, False), (4, 128, False)])
def test_weights_on_any_16_bytes(eqat, T, bits, group, fp16):
    """Where a weight starts decides how it is loaded, never what comes out; one weight may be both."""
    out, width, buf = 320, 1280, Guarded()
    pair = both_weights(out, width, bits, group, fp16)
    d = eqat.make_desc(bits, group, out, width, T, 0, eqat.EQAT_ZP_FP16 if fp16 else eqat.EQAT_ZP_U8)
    X, dH = normal(T, width, seed=5), normal(T, out, seed=6)
    ws = torch.empty(max(256, *(eqat.workspace_bytes(d, op) for op in (eqat.EQAT_OP_PACKED_GATED_FWD, eqat.EQAT_OP_PACKED_GATED_BWD))), dtype=torch.uint8, device="cuda")

    def moved(w, shift):
        copies = tuple(buf.empty(*t.shape, dtype=t.dtype, shift_bytes=shift) for t in w.on)
        for c, t in zip(copies, w.on):
            c.copy_(t)
        return copies

    def run(gate, up):
        H, G, U, dG, dU = (torch.empty(T, out, dtype=torch.bfloat16, device="cuda") for _ in range(5))
        dX = torch.empty_like(X)
        eqat.qlinear_packed_gated_fwd(d, eqat.EQAT_ACT_SILU, X, gate, up, H, G, U)
        eqat.qlinear_packed_gated_bwd(d, eqat.EQAT_ACT_SILU, dH, G, U, gate, up, dX, dG, dU, ws)
        return H, G, U, dX, dG, dU

    want = run(pair[0].on, pair[1].on)
    for shifts in ((16, 0), (0, 16), (48, 112)):
        assert all(torch.equal(a, b) for a, b in zip(run(*(moved(w, s) for w, s in zip(pair, shifts))), want)), shifts
    H, G, U, *_ = run(pair[0].on, pair[0].on)
    assert torch.equal(G, U) and torch.equal(G, want[1])
    buf.check()


# ---------------------------------------------------------------------------------------------- two at once
def test_two_captured_feed_forwards_at_once(eqat):
    """Each with its workspace, on streams of their own, replayed side by side."""
    out, width = 1408, 1024
    gate, up = both_weights(out, width, 2, 64, False)
    for Ts in ((1, 1), (24, 30), (200, 1), (1500, 130), (300, 40)):
        sets, graphs = [], []
        for i, T in enumerate(Ts):
            d = eqat.make_desc(2, 64, out, width, T)
            b = lambda *s: torch.empty(*s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
            s = dict(d=d, T=T, X=normal(T, width, seed=i), dH=normal(T, out, seed=i + 5), H=b(T, out), G=b(T, out), U=b(T, out), H2=b(T, out), dX=b(T, width), dG=b(T, out), dU=b(T, out))
            for k, op in (("w1", eqat.EQAT_OP_PACKED_GATED_FWD), ("w2", eqat.EQAT_OP_PACKED_GATED_BWD)):
                n = eqat.workspace_bytes(d, op)
                s[k] = torch.empty(n, dtype=torch.uint8, device="cuda") if n else None
            sets.append(s)

        def call(s):
            eqat.qlinear_packed_gated_fwd(s["d"], 0, s["X"], gate.on, up.on, s["H"], s["G"], s["U"])
            eqat.qlinear_packed_gated_fwd(s["d"], 0, s["X"], gate.on, up.on, s["H2"], None, None, s["w1"])
            eqat.qlinear_packed_gated_bwd(s["d"], 0, s["dH"], s["G"], s["U"], gate.on, up.on, s["dX"], s["dG"], s["dU"], s["w2"])

        keys = ("H", "G", "U", "H2", "dX", "dG", "dU")
        want = []
        for s in sets:
            call(s)
            want.append([s[k].clone() for k in keys])
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream() for _ in sets]
        for s, stream in zip(sets, streams):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=stream):
                call(s)
            graphs.append(g)
        for s in sets:
            for k in keys:
                s[k].zero_()
        torch.cuda.synchronize()
        for _ in range(20):
            for g, stream in zip(graphs, streams):
                with torch.cuda.stream(stream):
                    g.replay()
        torch.cuda.synchronize()
        assert eqat.device_status() == (0, 0)
        for s, w in zip(sets, want):
            assert all(torch.equal(s[k], v) for k, v in zip(keys, w)), s["T"]
            a = np.abs(B.activation(torch_to_f64(s["G"]), "silu")[0])
            u = np.abs(torch_to_f64(s["U"]))
            # H of the sums before their rounding: G and U half a step off, |act'| at most 1.13
            room = HALF_STEP * (1.13 * np.abs(torch_to_f64(s["G"])) * u + 2 * a * u) * 1.1 + FUNCTION * a * u + GONE
            assert_elementwise(torch_to_f64(s["H"]), B.activation(torch_to_f64(s["G"]), "silu")[0] * torch_to_f64(s["U"]), room, "H")


@pytest.mark.parametrize("T", [3, 20, 90, 1100])
def test_a_padded_batch(eqat, T):
    """Rows of padding that hold anything, NaN and infinities too, do not reach the others."""
    out, width = 256, 512
    gate, up = both_weights(out, width, 3, 64, False)
    d = eqat.make_desc(3, 64, out, width, T)
    X, got = normal(T, width, seed=7), []
    need = eqat.workspace_bytes(d, eqat.EQAT_OP_PACKED_GATED_BWD)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    dH = normal(T, out, seed=8)
    for pad in (0.0, float("nan"), float("inf")):
        X[1], X[-1], dH[1], dH[-1] = pad, -pad, pad, pad
        H, G, U, dG, dU = (torch.empty(T, out, dtype=torch.bfloat16, device="cuda") for _ in range(5))
        dX = torch.empty_like(X)
        eqat.qlinear_packed_gated_fwd(d, eqat.EQAT_ACT_GELU_TANH, X, gate.on, up.on, H, G, U)
        eqat.qlinear_packed_gated_bwd(d, eqat.EQAT_ACT_GELU_TANH, dH, G, U, gate.on, up.on, dX, dG, dU, ws)
        live = [i for i in range(T) if i not in (1, T - 1)]
        got.append([t[live].clone() for t in (H, G, U, dG, dU, dX)])
    for other in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(other, got[0]))
    assert all(torch.isfinite(t.float()).all() for t in got[0])


# ---------------------------------------------------------------------------------------------- parts of a head
@pytest.mark.parametrize("layout", ["halves", "pairs"])
@pytest.mark.parametrize("head_dim,rotary_dim", [(64, 12), (80, 20), (128, 4), (128, 34), (256, 252), (64, 48), (72, 72), (96, 40), (512, 510), (128, 64)])
@pytest.mark.parametrize("rows,q_heads,kv_heads", [(3, 5, 1), (700, 8, 8)])
def test_any_part_of_a_head(eqat, layout, head_dim, rotary_dim, rows, q_heads, kv_heads):
    """Pieces of every size, on any 16 bytes, in place or not: the same bits; what does not turn is handed on as it is, NaN or not."""
    from test_gpu_rotary import check, heads, layout_code
    turns = eqat.rotary_turns(rotary_dim, 10000.0)
    positions = [17 * i - 40 for i in range(rows)]
    pos = torch.tensor(positions, dtype=torch.int32, device="cuda")
    d = eqat.make_rotary_desc(rows, q_heads, kv_heads, head_dim, rotary_dim, layout_code(eqat, layout), 0.5)
    src = [heads(rows, h, head_dim, i) for i, h in enumerate((q_heads, kv_heads))]
    for t in src:
        t[..., rotary_dim:][..., ::3] = float("nan")
        t[..., rotary_dim:][..., 1::3] = float("inf")
    buf, got = Guarded(), []
    for shift in (0, 16, 32):
        given, out = ([buf.empty(*t.shape, dtype=torch.bfloat16, shift_bytes=shift) for t in src] for _ in range(2))
        for a, b in zip(given, src):
            a.copy_(b)
        eqat.eqat_rotary_fwd(d, *given, turns.cuda(), *out, pos)
        for a, b in zip(given, src):
            assert torch.equal(a.view(torch.int16), b.view(torch.int16))
        eqat.eqat_rotary_fwd(d, *given, turns.cuda(), *given, pos)
        mixed = [given[0].clone(), torch.empty_like(src[1])]                 # queries in place, keys not
        mixed[0].copy_(src[0])
        eqat.eqat_rotary_fwd(d, mixed[0], src[1], turns.cuda(), *mixed, pos)
        got += [out, given, mixed]
    buf.check()
    for pair in got:
        for x, y, want in zip(src, pair, got[0]):
            assert torch.equal(y.view(torch.int16), want.view(torch.int16))
            assert torch.equal(y[..., rotary_dim:].reshape(-1).view(torch.int16), x[..., rotary_dim:].reshape(-1).view(torch.int16))
    some = sorted({0, rows // 2, rows - 1})
    for x, y in zip(src, got[0]):
        check(y[some][..., :rotary_dim], x[some][..., :rotary_dim], turns, [positions[i] for i in some], layout, 1, 0.5)


@pytest.mark.parametrize("rows,n", [(3, 1000), (700, 4096), (5, 16), (64, 8208)])
def test_gated_on_any_16_bytes(eqat, rows, n):
    """Pieces of 16 and of 8: the same bits."""
    src, d, buf, got = [normal(rows, n, seed=i, std=1.5) for i in range(3)], eqat.make_gated_desc(rows, n, eqat.EQAT_ACT_GELU), Guarded(), []
    for shift in (0, 16):
        given = [buf.empty(rows, n, dtype=torch.bfloat16, shift_bytes=shift) for _ in src]
        for a, b in zip(given, src):
            a.copy_(b)
        out = [buf.empty(rows, n, dtype=torch.bfloat16, shift_bytes=shift) for _ in range(3)]
        eqat.eqat_gated_fwd(d, given[0], given[1], out[0])
        eqat.eqat_gated_bwd(d, given[2], given[0], given[1], out[1], out[2])
        got.append(out)
    buf.check()
    assert all(torch.equal(a, b) for a, b in zip(*got))


@pytest.mark.parametrize("rows,n,group", [(3, 256, 32), (700, 4096, 128), (33, 5120, 5120), (50, 1040, 1040), (9, 16384, 64), (2, 32768, 256), (11, 384, 128)])
def test_norm_on_any_16_bytes(eqat, rows, n, group):
    """The order of a sum hangs on the shape alone."""
    src, W, buf, got = [rows_of(rows, n, i) for i in range(2)], weight_of(n, 3), Guarded(), []
    for shift in (0, 16):
        x, r, h, y, h2, y2 = (buf.empty(rows, n, dtype=torch.bfloat16, shift_bytes=shift) for _ in range(6))
        x.copy_(src[0])
        r.copy_(src[1])
        eqat.eqat_rms_norm_fwd(eqat.make_norm_desc(rows, n, EPS), x, r, W, h, y)
        codes, scales = buf.empty(rows, n, dtype=torch.int8, shift_bytes=shift), buf.empty(rows, n // group, shift_bytes=shift)
        eqat.eqat_rms_norm_fwd(eqat.make_norm_desc(rows, n, EPS, eqat.EQAT_CODES_INT8, group), x, r, W, h2, y2, codes, scales)
        got.append((h, y, h2, y2, codes, scales))
    buf.check()
    assert all(torch.equal(a, b) for a, b in zip(*got))
