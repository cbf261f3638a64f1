"""A decoder block as a program runs it: norm, projections, rotary positions, cache, attention, projection, norm with the
residual, gated feed-forward, projection: a prompt, then single tokens by a captured graph; and a training pass through the same
calls.  Every stage is held against the oracle on the inputs that it had, so that bounds do not pile up."""
import numpy as np
import pytest
import torch

from helpers import assert_elementwise, contraction_bound, torch_to_f64
from oracle import between_oracle as B
from oracle import cache_oracle as C
from oracle import eqat_oracle as O

pytestmark = pytest.mark.gpu
HALF_STEP = 2.0 ** -8
E, F, HEADS, KV, D, EPS, BITS, GROUP = 512, 1408, 8, 2, 64, 1e-5, 4, 64
WIDTH = (HEADS + 2 * KV) * D


@pytest.fixture(scope="module")
def eqat():
    from paper_2407_11062_b200.build import build_library
    build_library()
    from paper_2407_11062_b200 import binding
    return binding


def normal(*shape, seed, std=1.0):
    return (torch.randn(*shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)) * std).to(torch.bfloat16)


class Packed:
    def __init__(self, eqat, out, width, seed):
        self.eqat, self.out, self.width = eqat, out, width
        W = normal(out, width, seed=seed, std=width ** -0.5)
        d = eqat.make_desc(BITS, GROUP, out, width)
        s, z = (torch.empty(out, width // GROUP, device="cuda") for _ in range(2))
        eqat.eqat_minmax_init(d, W, s, z)
        P = torch.empty(out, width * BITS // 8, dtype=torch.uint8, device="cuda")
        z8, s16 = torch.empty_like(z, dtype=torch.uint8), torch.empty_like(s, dtype=torch.float16)
        eqat.eqat_quantize_pack(d, W, s, z, P, z8, s16)
        self.on = (P, s16, z8)
        self.value = O.dequantize(O.unpack_rows(P.cpu().numpy(), BITS, width), s16.cpu().numpy().astype(np.float32), z8.cpu().numpy(), GROUP)

    def desc(self, T):
        return self.eqat.make_desc(BITS, GROUP, self.out, self.width, T)

    def __call__(self, X, Y):
        self.eqat.qlinear_packed_fwd(self.desc(X.shape[0]), X, *self.on, Y)

    def check(self, X, Y):
        x, w = torch_to_f64(X), self.value
        assert_elementwise(torch_to_f64(Y), x @ w.T, contraction_bound(x @ w.T, np.abs(x) @ np.abs(w).T, x ** 2 @ (w ** 2).T), "projection")


class Block:
    """Weights, cache and buffers for calls of T rows."""

    def __init__(self, eqat):
        self.eqat = eqat
        self.qkv, self.o, self.gate, self.up, self.down = (Packed(eqat, *s, i) for i, s in enumerate(((WIDTH, E), (E, HEADS * D), (F, E), (F, E), (E, F))))
        self.w1, self.w2 = (1 + normal(E, seed=10 + i, std=0.2).float() for i in range(2))
        self.w1, self.w2 = self.w1.to(torch.bfloat16), self.w2.to(torch.bfloat16)
        self.turns_host = eqat.rotary_turns(D, 10000.0)
        self.turns = self.turns_host.cuda()
        self.pool = tuple(torch.zeros(20, KV, 16, *s, dtype=t, device="cuda") for _ in range(2) for s, t in (((D // 2,), torch.uint8), ((1, 2), torch.bfloat16)))
        self.table = torch.tensor([[3, 1, 4, 15, 9], [2, 6, 5, 0, 8]], dtype=torch.int32, device="cuda")

    def plan(self, T, new):
        eqat, b = self.eqat, {}
        for name, shape in (("x", (T, E)), ("h1", (T, E)), ("y1", (T, E)), ("qkv", (T, WIDTH)), ("q", (T, HEADS, D)), ("k", (T, KV, D)), ("att", (T, HEADS, D)), ("a", (T, E)),
                            ("h2", (T, E)), ("y2", (T, E)), ("f", (T, F)), ("out", (T, E))):
            b[name] = torch.empty(*shape, dtype=torch.bfloat16, device="cuda")
        b["norm"] = eqat.make_norm_desc(T, E, EPS)
        b["rotary"] = eqat.make_rotary_desc(T, HEADS, KV, D, sequences=2)
        b["cache"] = eqat.make_cache_desc(GROUP, D, KV, 16, 20, 2, 5, T)
        b["attn"] = eqat.make_attention_desc(HEADS, new, D ** -0.5)
        b["gated"] = self.gate.desc(T)
        for name, need in (("ws1", eqat.cache_workspace_bytes(b["cache"], b["attn"])), ("ws2", eqat.workspace_bytes(b["gated"], eqat.EQAT_OP_PACKED_GATED_FWD))):
            b[name] = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
        b["off"], b["len"] = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
        return b

    def run(self, b):
        eqat, where = self.eqat, (b["off"], b["len"], self.table, self.pool)
        eqat.eqat_rms_norm_fwd(b["norm"], b["x"], None, self.w1, None, b["y1"])
        self.qkv(b["y1"], b["qkv"])
        heads = b["qkv"].view(-1, HEADS + 2 * KV, D)
        eqat.eqat_rotary_fwd(b["rotary"], heads[:, :HEADS], heads[:, HEADS:HEADS + KV], self.turns, b["q"], b["k"], None, b["off"], b["len"])
        eqat.eqat_cache_append(b["cache"], b["k"], heads[:, HEADS + KV:], *where)
        eqat.eqat_cache_attention(b["cache"], b["attn"], b["q"], *where, b["att"], None, b["ws1"])
        self.o(b["att"].view(-1, HEADS * D), b["a"])
        eqat.eqat_rms_norm_fwd(b["norm"], b["a"], b["x"], self.w2, b["h2"], b["y2"])
        eqat.qlinear_packed_gated_fwd(b["gated"], eqat.EQAT_ACT_SILU, b["y2"], self.gate.on, self.up.on, b["f"], None, None, b["ws2"])
        self.down(b["f"], b["out"])

    def check(self, b, lens, news, keys, values):
        """`keys`, `values`: what each sequence held before, float64 [tokens, KV, D]; appended to."""
        f = {k: torch_to_f64(v) for k, v in b.items() if isinstance(v, torch.Tensor) and v.dtype == torch.bfloat16}
        w1, w2 = torch_to_f64(self.w1), torch_to_f64(self.w2)
        assert_elementwise(f["y1"], B.norm_fwd(f["x"], w1, EPS), (HALF_STEP + 2.0 ** -17) * np.abs(B.norm_fwd(f["x"], w1, EPS)), "first norm")
        self.qkv.check(b["y1"], b["qkv"])
        heads = f["qkv"].reshape(-1, HEADS + 2 * KV, D)
        pos = [n - k + i for n, k in zip(lens, news) for i in range(k)]
        t = np.array([B.turns_at(self.turns_host.tolist(), p) for p in pos])
        for name, x in (("q", heads[:, :HEADS]), ("k", heads[:, HEADS:HEADS + KV])):
            want = B.rotate(x, t, "halves")
            assert_elementwise(f[name], want, HALF_STEP * np.abs(want) + 2.0 ** -19 * np.abs(x).max(-1, keepdims=True), name)
        at = 0
        for s, k in enumerate(news):
            for store, x in ((keys, f["k"]), (values, heads[:, HEADS + KV:])):
                store[s] = np.concatenate([store[s], C.values(*C.quantise(x[at:at + k].astype(np.float32), GROUP))])
            at += k
        want = C.attention(f["q"], keys, values, lens, list(np.concatenate([[0], np.cumsum(news)])), D ** -0.5)[0]
        assert np.linalg.norm(f["att"] - want) <= 5e-3 * np.linalg.norm(want)                   # the attention's tests have its bounds
        self.o.check(b["att"].view(-1, HEADS * D), b["a"])
        assert torch.equal(b["h2"], (b["a"].float() + b["x"].float()).to(torch.bfloat16))
        y2 = B.norm_fwd(f["h2"], w2, EPS)
        assert_elementwise(f["y2"], y2, (HALF_STEP + 2.0 ** -17) * np.abs(y2), "second norm")
        g, u = f["y2"] @ self.gate.value.T, f["y2"] @ self.up.value.T
        eg, eu = (contraction_bound(r, np.abs(f["y2"]) @ np.abs(w.value).T, f["y2"] ** 2 @ (w.value ** 2).T) for r, w in ((g, self.gate), (u, self.up)))
        a = np.abs(B.activation(g, "silu")[0])
        room = 1.13 * eg * (np.abs(u) + eu) + a * eu
        assert_elementwise(f["f"], B.activation(g, "silu")[0] * u, room + 1.02 * HALF_STEP * (a * np.abs(u) + room), "feed-forward")
        self.down.check(b["f"], b["out"])


def test_prompt_and_tokens(eqat):
    block = Block(eqat)
    keys, values = [np.zeros((0, KV, D)) for _ in range(2)], [np.zeros((0, KV, D)) for _ in range(2)]
    lens, news = [37, 20], [37, 20]
    b = block.plan(57, 37)
    b["off"].copy_(torch.tensor([0, 37, 57]))
    b["len"].copy_(torch.tensor(lens))
    b["x"].copy_(normal(57, E, seed=20))
    block.run(b)
    block.check(b, lens, news, keys, values)
    one = block.plan(2, 1)
    one["off"].copy_(torch.tensor([0, 1, 2]))
    one["len"].copy_(torch.tensor([38, 21]))
    one["x"].copy_(normal(2, E, seed=21))
    block.run(one)                                                  # writes what the first replay writes again
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        block.run(one)
    for step in range(3):
        lens = [n + 1 for n in lens]
        one["len"].copy_(torch.tensor(lens, dtype=torch.int32))
        one["x"].copy_(normal(2, E, seed=21 + step))
        graph.replay()
        block.check(one, lens, [1, 1], keys, values)
    assert eqat.device_status() == (0, 0)


def test_training_pass(eqat):
    """The feed-forward half of a block with packed weights, there and back, and the step sizes' gradients: those of the whole against
    differences of the oracle's loss in 64 bits would hang on every rounding, so each stage's is held against its formula."""
    T = 700
    block = Block(eqat)
    x, dout = normal(T, E, seed=30), normal(T, E, seed=31, std=0.01)
    h, y, dy, dh = (torch.empty_like(x) for _ in range(4))
    f, G, U, df, dG, dU = (torch.empty(T, F, dtype=torch.bfloat16, device="cuda") for _ in range(6))
    out, dw = torch.empty_like(x), torch.empty(E, device="cuda")
    norm = eqat.make_norm_desc(T, E, EPS)
    ws = torch.empty(eqat.rms_norm_workspace_bytes(norm), dtype=torch.uint8, device="cuda")
    desc = block.gate.desc(T)
    need = eqat.workspace_bytes(desc, eqat.EQAT_OP_PACKED_GATED_BWD)
    ws_dx = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None

    def step():
        eqat.eqat_rms_norm_fwd(norm, x, dout, block.w1, h, y)
        eqat.qlinear_packed_gated_fwd(desc, eqat.EQAT_ACT_SILU, y, block.gate.on, block.up.on, f, G, U)
        block.down(f, out)
        eqat.qlinear_packed_bwd_dx(block.down.desc(T), dout, *block.down.on, df)
        eqat.qlinear_packed_gated_bwd(desc, eqat.EQAT_ACT_SILU, df, G, U, block.gate.on, block.up.on, dy, dG, dU, ws_dx)
        for w, d, ds in ((block.gate, dG, ds_gate), (block.up, dU, ds_up)):
            eqat.qlinear_packed_bwd_ds(desc, y, d, w.on[0], w.on[2], None, ds)
        eqat.eqat_rms_norm_bwd(norm, dy, h, block.w1, dout, dh, dw, ws)

    ds_gate, ds_up = (torch.empty(F, E // GROUP, device="cuda") for _ in range(2))
    step()
    got = [t.clone() for t in (h, y, f, G, U, out, df, dG, dU, dy, dh, dw, ds_gate, ds_up)]
    n = {k: torch_to_f64(t) for k, t in dict(h=h, y=y, G=G, U=U, df=df, dG=dG, dU=dU, dy=dy, dh=dh, dout=dout, dw=dw, w=block.w1).items()}
    block.gate.check(y, G)
    block.up.check(y, U)
    e, g = B.gated_bwd(n["df"], n["G"], n["U"], "silu")
    terms = B.activation(n["G"], "silu")[2]
    assert_elementwise(n["dG"], e, HALF_STEP * np.abs(e) + 2.0 ** -14 * np.abs(n["df"] * n["U"]) * terms + 1e-35, "dG")
    assert_elementwise(n["dU"], g, (HALF_STEP + 2.0 ** -14) * np.abs(g) + 1e-35, "dU")
    parts = [(n["dG"], block.gate.value), (n["dU"], block.up.value)]
    ref, size, square = (sum(op(a) @ op(b) for a, b in parts) for op in (lambda v: v, np.abs, np.square))
    assert_elementwise(n["dy"], ref, contraction_bound(ref, size, square), "dy")
    dx, dw64 = B.norm_bwd(n["dy"], n["h"], n["w"], EPS, n["dout"])
    c, v = B.norm_scale(n["h"], EPS), np.abs(n["dy"] * n["w"])
    room = c * (v + np.abs(n["h"]) * c * c * (v * np.abs(n["h"])).mean(-1, keepdims=True)) + np.abs(n["dout"])
    assert_elementwise(n["dh"], dx, HALF_STEP * np.abs(dx) + 2.0 ** -16 * room, "dh")
    assert_elementwise(n["dw"], dw64, 2.0 ** -15 * (np.abs(n["dy"] * n["h"]) * c).sum(0), "dw")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for t in (h, y, f, G, U, out, df, dG, dU, dy, dh, dw, ds_gate, ds_up):
        t.zero_()
    graph.replay()
    assert all(torch.equal(a, t) for a, t in zip(got, (h, y, f, G, U, out, df, dG, dU, dy, dh, dw, ds_gate, ds_up)))
