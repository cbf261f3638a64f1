"""The gated product against the oracle: element-wise, and with both projections packed.

Bounds.  An exponential of x is right to (|x| + 4) 2^-24 of itself, x at most 88 in size, erfc's argument enters twice as strongly:
2^-14 of the activation and of each term of its slope is above all of them.  Activations below 2^-110 may be 0."""
import numpy as np
import pytest
import torch

from helpers import Guarded, assert_elementwise, contraction_bound, torch_to_f64
from oracle import between_oracle as B
from oracle import eqat_oracle as O

pytestmark = pytest.mark.gpu
HALF_STEP, FUNCTION, GONE = 2.0 ** -8, 2.0 ** -14, 2.0 ** -109
KINDS = ["silu", "gelu", "gelu_tanh"]


@pytest.fixture(scope="module")
def eqat():
    from paper_2407_11062_b200.build import build_library
    build_library()
    from paper_2407_11062_b200 import binding
    return binding


def act_code(eqat, kind):
    return {"silu": eqat.EQAT_ACT_SILU, "gelu": eqat.EQAT_ACT_GELU, "gelu_tanh": eqat.EQAT_ACT_GELU_TANH}[kind]


def normal(*shape, seed, std=1.0):
    return (torch.randn(*shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)) * std).to(torch.bfloat16)


def check_h(got, g, u, kind):
    a = B.activation(g, kind)[0]
    assert_elementwise(got, a * u, (HALF_STEP + FUNCTION) * np.abs(a * u) + GONE * np.abs(u) + 2.0 ** -133, f"H {kind}")


def check_grads(dg, du, dh, g, u, kind):
    a, slope, terms = B.activation(g, kind)
    e, f = dh * u * slope, dh * a
    assert_elementwise(dg, e, HALF_STEP * np.abs(e) + np.abs(dh * u) * (FUNCTION * terms + GONE) + 2.0 ** -133, f"dG {kind}")
    assert_elementwise(du, f, (HALF_STEP + FUNCTION) * np.abs(f) + GONE * np.abs(dh) + 2.0 ** -133, f"dU {kind}")


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,n", [(1, 8), (1, 11008), (3, 1000), (257, 72), (1000, 1376), (5, 65536)])
def test_elementwise(eqat, kind, rows, n):
    G, U, dH, buf = normal(rows, n, seed=1, std=2.0), normal(rows, n, seed=2), normal(rows, n, seed=3), Guarded()
    d = eqat.make_gated_desc(rows, n, act_code(eqat, kind))
    H, dG, dU = (buf.empty(rows, n, dtype=torch.bfloat16, shift_bytes=16 * i) for i in range(3))
    eqat.eqat_gated_fwd(d, G, U, H)
    eqat.eqat_gated_bwd(d, dH, G, U, dG, dU)
    buf.check()
    g, u, dh = (torch_to_f64(t) for t in (G, U, dH))
    check_h(torch_to_f64(H), g, u, kind)
    check_grads(torch_to_f64(dG), torch_to_f64(dU), dh, g, u, kind)
    # halves of one tensor, gradients in place of them
    both = torch.cat([G, U], 1)
    H2, left, right = torch.empty_like(H), both[:, :n], both[:, n:]
    eqat.eqat_gated_fwd(d, left, right, H2)
    eqat.eqat_gated_bwd(d, dH, left, right, left, right)
    assert torch.equal(H2, H) and torch.equal(left, dG) and torch.equal(right, dU)
    dh2 = dH.clone()
    eqat.eqat_gated_bwd(d, dh2, G, U, dG.zero_(), dh2)
    assert torch.equal(dh2, dU) and torch.equal(dG, left)


@pytest.mark.parametrize("kind", KINDS)
def test_every_bf16_number(eqat, kind):
    """All 65536: tails, infinities and NaN among them."""
    g = torch.arange(65536, dtype=torch.int32).to(torch.uint16).view(torch.bfloat16).cuda().view(1, -1)
    one, d = torch.ones_like(g), eqat.make_gated_desc(1, 65536, act_code(eqat, kind))
    H, dG, dU = (torch.empty_like(g) for _ in range(3))
    eqat.eqat_gated_fwd(d, g, one, H)
    eqat.eqat_gated_bwd(d, one, g, one, dG, dU)
    x = torch_to_f64(g)[0]
    nan, inf = np.isnan(x), np.isinf(x)
    h, dg, du = (torch_to_f64(t)[0] for t in (H, dG, dU))
    assert np.isnan(h[nan]).all() and np.isnan(dg[nan]).all() and np.isnan(du[nan]).all()
    for got, up, down in ((h, np.inf, 0), (du, np.inf, 0), (dg, 1, 0)):
        assert (got[inf & (x > 0)] == up).all() and (got[inf & (x < 0)] == down).all()
    fine = ~nan & ~inf
    # beyond 1e6 the oracle's own polynomials leave the range; the activation is the identity or 0 there
    mid = fine & (np.abs(x) < 1e6)
    check_h(h[mid], x[mid], np.ones(mid.sum()), kind)
    check_grads(dg[mid], du[mid], np.ones(mid.sum()), x[mid], np.ones(mid.sum()), kind)
    far = fine & ~mid
    assert np.array_equal(h[far], np.maximum(x[far], 0)) and np.array_equal(du[far], np.maximum(x[far], 0)) and np.array_equal(dg[far], (x[far] > 0) * 1.0)


# ---------------------------------------------------------------------------------------------- packed projections
class Weight:
    """Codes, steps and zero points on the device, and the oracle's values of them."""

    def __init__(self, out, width, bits, group, fp16, seed):
        rng = np.random.default_rng(seed)
        q = rng.integers(0, 1 << bits, (out, width), dtype=np.uint8)
        ng = width // group
        s = (0.02 + 0.01 * rng.random((out, ng))).astype(np.float16)
        z = rng.integers(0, 1 << bits, (out, ng)).astype(np.uint8)
        if fp16:
            z = (z + 0.3 * rng.standard_normal((out, ng))).astype(np.float16)
        self.value = O.dequantize(q, s.astype(np.float32), z, group, fp16)
        self.on = tuple(torch.from_numpy(x).cuda() for x in (O.pack_rows(q, bits), s, z))


def both_weights(out, width, bits, group, fp16):
    return Weight(out, width, bits, group, fp16, 1), Weight(out, width, bits, group, fp16, 2)


def projected(X, w):
    """X w^T and how far a kernel's may be off (fp32 sums of a weight rounded to bf16, rounded once more)."""
    x, w = torch.from_numpy(X).cuda(), torch.from_numpy(np.asarray(w, np.float64)).cuda()
    ref, size, square = x @ w.T, x.abs() @ w.abs().T, x.square() @ w.square().T
    ref, size, square = (t.cpu().numpy() for t in (ref, size, square))
    return ref, contraction_bound(ref, size, square)


def forward_cases():
    yield from ((T, 128, 256, 2, 64, False, "silu") for T in (1, 2, 8, 9, 33, 129, 300))
    yield from ((T, 192, 384, 3, 128, False, "gelu") for T in (1, 5, 17, 260))
    yield from ((T, 320, 512, 4, 32, True, "gelu_tanh") for T in (1, 8, 64, 513))
    yield from ((T, 64, 128, b, 128, z, "silu") for T in (1, 3, 700) for b in (2, 3, 4) for z in (False, True))
    yield from ((1100, 576, 640, b, 640, False, "gelu") for b in (2, 4))
    yield from ((1029, 1088, 768, b, g, z, "silu") for b in (2, 3, 4) for g, z in ((64, True), (256, False)))
    yield (4099, 4160, 256, 2, 64, False, "silu")                   # pairs of CTAs, ragged in both directions
    yield (2500, 4224, 512, 3, 32, True, "gelu_tanh")
    yield from ((200, 11008, 256, b, 64, z, k) for b, z, k in ((2, False, "silu"), (3, True, "gelu"), (4, False, "gelu_tanh")))   # single CTAs of 256 rows
    yield from ((257, 11008, 128, b, 128, False, "silu") for b in (2, 3, 4))
    yield (1, 11008, 4096, 2, 64, False, "silu")
    yield (7, 4096, 5120, 3, 128, False, "gelu")
    yield (3, 2048, 11008, 4, 128, True, "silu")
    yield from ((T, 11008, 4096, 3, 128, False, "silu") for T in (37, 64, 100, 333))     # rows of either kernel split over clusters
    yield from ((T, 5120, 1024, b, 64, z, "gelu") for T, b, z in ((12, 2, False), (16, 4, True), (48, 3, False), (70, 4, False), (200, 2, True)))


@pytest.mark.parametrize("T,out,width,bits,group,fp16,kind", list(forward_cases()))
def test_packed_forward(eqat, T, out, width, bits, group, fp16, kind):
    gate, up = both_weights(out, width, bits, group, fp16)
    X, buf = normal(T, width, seed=3), Guarded()
    d = eqat.make_desc(bits, group, out, width, T, 0, eqat.EQAT_ZP_FP16 if fp16 else eqat.EQAT_ZP_U8)
    need = eqat.workspace_bytes(d, eqat.EQAT_OP_PACKED_GATED_FWD)
    H, G, U, H2 = (buf.empty(T, out, dtype=torch.bfloat16, shift_bytes=16 * i) for i in range(4))
    act = act_code(eqat, kind)
    eqat.qlinear_packed_gated_fwd(d, act, X, gate.on, up.on, H, G, U)
    eqat.qlinear_packed_gated_fwd(d, act, X, gate.on, up.on, H2, None, None, buf.empty(need, dtype=torch.uint8) if need else None)
    buf.check()
    assert eqat.device_status() == (0, 0)
    assert torch.equal(H, H2)
    x = torch_to_f64(X)
    (g, eg), (u, eu) = projected(x, gate.value), projected(x, up.value)
    assert_elementwise(torch_to_f64(G), g, eg, "G")
    assert_elementwise(torch_to_f64(U), u, eu, "U")
    # |act'| is at most 1.13 for all three
    a = np.abs(B.activation(g, kind)[0])
    room = 1.13 * eg * (np.abs(u) + eu) + a * eu
    assert_elementwise(torch_to_f64(H), B.activation(g, kind)[0] * u, room + (HALF_STEP + FUNCTION) * (a * np.abs(u) + room) + GONE, "H")


@pytest.mark.parametrize("T,out,width,bits,group,fp16,kind", [
    (1, 64, 128, 2, 64, False, "silu"), (5, 128, 256, 3, 32, True, "gelu"), (130, 192, 384, 4, 128, False, "gelu_tanh"), (300, 320, 640, 2, 640, False, "silu"),
    (1029, 1088, 768, 3, 256, True, "silu"), (1029, 1088, 768, 2, 64, False, "gelu"), (3000, 448, 4224, 4, 32, False, "silu"), (2100, 11008, 512, 2, 64, True, "silu"),
    (1, 11008, 4096, 2, 64, False, "silu"), (130, 4096, 2048, 4, 128, False, "silu"), (640, 1088, 4096, 3, 64, True, "gelu"), (70, 2112, 512, 2, 64, False, "silu"),
    (150, 64, 9600, 2, 64, False, "silu"), (150, 128, 9600, 3, 128, True, "silu"), (256, 64, 9600, 4, 32, False, "gelu")])
def test_packed_backward(eqat, T, out, width, bits, group, fp16, kind):
    gate, up = both_weights(out, width, bits, group, fp16)
    dH, G, U, buf = normal(T, out, seed=4, std=0.1), normal(T, out, seed=5, std=1.5), normal(T, out, seed=6), Guarded()
    d = eqat.make_desc(bits, group, out, width, T, 0, eqat.EQAT_ZP_FP16 if fp16 else eqat.EQAT_ZP_U8)
    dX, dG, dU = buf.empty(T, width, dtype=torch.bfloat16), *(buf.empty(T, out, dtype=torch.bfloat16, shift_bytes=16) for _ in range(2))
    act = act_code(eqat, kind)
    need = eqat.workspace_bytes(d, eqat.EQAT_OP_PACKED_GATED_BWD)
    ws = buf.empty(need, dtype=torch.uint8) if need else None
    eqat.qlinear_packed_gated_bwd(d, act, dH, G, U, gate.on, up.on, dX, dG, dU, ws)
    buf.check()
    assert eqat.device_status() == (0, 0)
    check_grads(torch_to_f64(dG), torch_to_f64(dU), torch_to_f64(dH), torch_to_f64(G), torch_to_f64(U), kind)
    dev = [(t.double(), torch.from_numpy(np.asarray(w.value, np.float64)).cuda()) for t, w in ((dG, gate), (dU, up))]
    ref, size, square = (sum(f(y) @ f(w) for y, w in dev).cpu().numpy() for f in (lambda t: t, torch.abs, torch.square))
    assert_elementwise(torch_to_f64(dX), ref, contraction_bound(ref, size, square), "dX")
    # gradients in place of the projections; the same bits
    G2, U2, dX2 = G.clone(), U.clone(), torch.empty_like(dX)
    if need:
        ws.fill_(0xFF)
    eqat.qlinear_packed_gated_bwd(d, act, dH, G2, U2, gate.on, up.on, dX2, G2, U2, ws)
    assert torch.equal(G2, dG) and torch.equal(U2, dU) and torch.equal(dX2, dX)


@pytest.mark.parametrize("T", [1, 6, 20, 300])
def test_zero_points_of_eight_bits(eqat, T):
    """Bytes past 127, which no hand-off produces, in one weight or the other."""
    out, width, rng = 192, 1280, np.random.default_rng(9)
    for which in (0, 1):
        pair = both_weights(out, width, 4, 128, False)
        z = rng.integers(100, 256, (out, width // 128)).astype(np.uint8)
        w = pair[which]
        q = O.unpack_rows(w.on[0].cpu().numpy(), 4, width)
        w.value = O.dequantize(q, w.on[1].cpu().numpy().astype(np.float32) * 2.0 ** -4, z, 128)
        w.on = (w.on[0], (w.on[1].float() * 2.0 ** -4).half(), torch.from_numpy(z).cuda())
        X, d = normal(T, width, seed=10, std=0.1), eqat.make_desc(4, 128, out, width, T)
        H, G, U = (torch.empty(T, out, dtype=torch.bfloat16, device="cuda") for _ in range(3))
        eqat.qlinear_packed_gated_fwd(d, eqat.EQAT_ACT_SILU, X, pair[0].on, pair[1].on, H, G, U)
        for got, weight in ((G, pair[0]), (U, pair[1])):
            want, room = projected(torch_to_f64(X), weight.value)
            assert_elementwise(torch_to_f64(got), want, room, which)


def test_the_weights_are_not_mixed_up(eqat):
    """A gate of ones and an up weight of twos, and the other way round: H = act(n) 2n against act(2n) n."""
    out, width = 128, 128
    for T in (1, 20, 200, 2000):
        d = eqat.make_desc(2, 64, out, width, T)
        X = torch.full((T, width), 2.0 ** -7, dtype=torch.bfloat16, device="cuda")            # n = 1
        codes = [torch.full((out, width // 4), v * 0x55, dtype=torch.uint8, device="cuda") for v in (1, 2)]
        s, z = torch.ones(out, 2, dtype=torch.float16, device="cuda"), torch.zeros(out, 2, dtype=torch.uint8, device="cuda")
        H = torch.empty(T, out, dtype=torch.bfloat16, device="cuda")
        need = eqat.workspace_bytes(d, eqat.EQAT_OP_PACKED_GATED_FWD)
        ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
        for a, b in ((1, 2), (2, 1)):
            eqat.qlinear_packed_gated_fwd(d, eqat.EQAT_ACT_SILU, X, (codes[a - 1], s, z), (codes[b - 1], s, z), H, None, None, ws)
            want = float(B.activation(float(a), "silu")[0]) * b
            assert (H.double() - want).abs().max() <= 2.0 ** -7 * want


def test_captured_on_another_stream(eqat):
    out, width = 256, 512
    gate, up = both_weights(out, width, 2, 64, False)
    for T in (1, 24, 200, 1500):
        d = eqat.make_desc(2, 64, out, width, T)
        need = eqat.workspace_bytes(d, eqat.EQAT_OP_PACKED_GATED_FWD)
        ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
        X, H = normal(T, width, seed=7), torch.empty(T, out, dtype=torch.bfloat16, device="cuda")
        call = lambda: eqat.qlinear_packed_gated_fwd(d, eqat.EQAT_ACT_GELU, X, gate.on, up.on, H, None, None, ws)  # noqa: E731
        call()
        torch.cuda.synchronize()
        g, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        with torch.cuda.graph(g, stream=side):
            call()
        X.copy_(normal(T, width, seed=8))
        call()
        want = H.clone()
        H.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(H, want)
