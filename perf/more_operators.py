"""What stands between the linears of a decoder block: the calls and sizes that their performance is judged on.

    norm     root-mean-square norm of the residual stream, with the addition to it, optionally in 8 bits; its gradient
    rotary   rotary positions of queries and keys; its gradient
    gated    activation of one projection times the other; its gradient
    feed     the same with both projections, whose weights are held in 2 to 4 bits; its gradient

norm, for a row of n elements, in 32 bits or more between the roundings named:
    h = bf16(x + r),  c = (mean(h^2) + eps)^(-1/2),  y = bf16(h c w)
or, in 8 bits, for each group with a = max |h w|  (binary32, half to even; 0 where a < 2^-110):
    q = rint(h w * (127/a))  or  e4m3(h w * (448/a)),   scale = a c / 127  or  a c / 448,   y = bf16(q scale)
    gradient, v = dy w:  dx = dr + c (v - h c^2 mean(v h)),   dw = sum over rows of dy h c

rotary, for a pair (a, b) of a head at position p, angle t = p * frequency of the pair:
    (a cos t - b sin t, b cos t + a sin t) * amplitude,  gradient: by -t

gated:  h = act(g) u,   dg = dh u act'(g),   du = dh act(g)
feed:   g = x Wg^T, u = x Wu^T,   dx = dg Wg + du Wu  with dg, du rounded to bf16;   W = (code - zero) * step
    codes of a row: a little-endian stream, code j at bits [N j, N j + N)
"""
import math
import random

import torch

own = False

DEV = "cuda"
BF16 = torch.bfloat16
SMALL = 2.0 ** -110


# ---------------------------------------------------------------------------------------------- cases
def _norm(name, rows, features, residual=True, backward=False, codes="", group=0):
    return _named(name, {"op": "norm", "rows": rows, "features": features, "residual": residual, "backward": backward,
                         "codes": codes, "group": group})


def _rotary(name, seqs, new, length, q_heads, kv_heads, head_dim, rotary_dim, layout, scaling, fused, backward=False):
    """`fused`: queries and keys are slices of one projection's output."""
    return _named(name, {"op": "rotary", "seqs": seqs, "new": new, "length": length, "q_heads": q_heads, "kv_heads": kv_heads,
                         "head_dim": head_dim, "rotary_dim": rotary_dim, "layout": layout, "scaling": scaling, "fused": fused,
                         "backward": backward})


def _gated(name, rows, features, activation, fused, backward):
    """`fused`: the two projections are the halves of one tensor."""
    return _named(name, {"op": "gated", "rows": rows, "features": features, "activation": activation, "fused": fused,
                         "backward": backward})


def _feed(name, tokens, width, inner, bits, group, zeros, activation, keep=False, backward=False):
    """`keep`: the projections are kept for the backward pass."""
    return _named(name, {"op": "feed", "tokens": tokens, "width": width, "inner": inner, "bits": bits, "group": group,
                         "zeros": zeros, "activation": activation, "keep": keep, "backward": backward})


def _named(name, c):
    return {"name": name, **c} if name else c


def listed():
    # widths and heads are those of 7B, 13B and 70B Llama-2 blocks
    return [
        # one decoding step of one user: latency
        _norm("norm_1x4096", 1, 4096),
        # prompts of a batch, 13B
        _norm("norm_8191x5120", 8191, 5120),
        # activations in 8 bits with a scale for every 128, 70B
        _norm("norm_e4m3_2001x8192_g128", 2001, 8192, codes="e4m3", group=128),
        # training, 7B: two sequences of 2048 tokens
        _norm("norm_bwd_4096x4096", 4096, 4096, backward=True),
        # one decoding step of a batch whose texts are long, 70B, out of the fused projection
        _rotary("rotary_64x1_h64_8", 64, 1, 120000, 64, 8, 128, 128, "halves", "ramp", True),
        # training, 13B, a quarter of each head as neighbouring pairs
        _rotary("rotary_bwd_2x2047_h40", 2, 2047, 2047, 40, 40, 128, 32, "pairs", "plain", False, backward=True),
        # training with fake-quantised weights, 7B: between the linears' calls
        _gated("gated_4096x11008", 4096, 11008, "silu", False, False),
        _gated("gated_bwd_4095x13824", 4095, 13824, "gelu_tanh", True, True),
        # one decoding step of one user, 7B in 2 bits
        _feed("feed_1_7b_w2", 1, 4096, 11008, 2, 64, "u8", "silu"),
        # a small batch of drafted tokens, 13B in 3 bits
        _feed("feed_37_13b_w3", 37, 5120, 13824, 3, 128, "u8", "silu"),
        # training, 7B in 2 bits with trained zero points: forward and the gradient of its input
        _feed("feed_4096_7b_w2", 4096, 4096, 11008, 2, 64, "fp16", "silu", keep=True),
        _feed("feed_bwd_4000_7b_w4", 4000, 4096, 11008, 4, 128, "u8", "silu", backward=True),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    top = {}
    for c in listed():
        for k, v in work(c).items():
            top[c["op"], k] = max(v, top.get((c["op"], k), 0))
    while True:
        op = rng.choice(("norm", "norm", "rotary", "gated", "feed", "feed"))
        activation = rng.choice(("silu", "silu", "gelu", "gelu_tanh"))
        if op == "norm":
            kind = rng.choice(("plain", "plain", "codes", "backward", "backward"))
            features = rng.choice((128, 512, 4096, 5120, 8192, 8 * _log(rng, 8, 2048)))
            groups = [g for g in (32, 64, 128, 256) if features % g == 0] + [features]
            c = _norm(None, _log(rng, 1, 40000), features, rng.random() < 0.8, kind == "backward",
                      rng.choice(("int8", "e4m3")) if kind == "codes" else "", rng.choice(groups) if kind == "codes" else 0)
        elif op == "rotary":
            head_dim = rng.choice((64, 96, 128, 128, 256))
            kv_heads = rng.choice((1, 2, 8, 8, 32, 40))
            seqs, kind = _log(rng, 1, 200), rng.choice(("step", "draft", "chunk", "prompt"))
            length = _log(rng, 1, 200000)
            new = min({"step": 1, "draft": rng.randint(2, 16), "chunk": _log(rng, 17, 2000), "prompt": length}[kind], length)
            c = _rotary(None, seqs, new, length, kv_heads * rng.choice((1, 1, 4, 8)), kv_heads, head_dim,
                        rng.choice((head_dim, head_dim, head_dim // 2, head_dim // 4, 2 * rng.randint(1, head_dim // 2))),
                        rng.choice(("halves", "pairs")), rng.choice(("plain", "linear", "base", "ramp")), rng.random() < 0.5,
                        rng.random() < 0.4)
        elif op == "gated":
            c = _gated(None, _log(rng, 1, 16000), rng.choice((11008, 13824, 28672, 8 * _log(rng, 8, 3000))), activation,
                       rng.random() < 0.5, rng.random() < 0.5)
        else:
            width, inner = rng.choice(((4096, 11008), (5120, 13824), (8192, 28672), (128 * rng.randint(2, 48), 64 * rng.randint(4, 200))))
            group = rng.choice([g for g in (32, 64, 64, 128, 128, 256) if width % g == 0] + [width])
            kind = rng.choice(("serve", "serve", "keep", "backward"))
            c = _feed(None, _log(rng, 1, 5000), width, inner, rng.choice((2, 3, 4)), group, rng.choice(("u8", "u8", "fp16")),
                      activation, kind == "keep", kind == "backward")
        w = work(c)
        if all(w[k] <= top[op, k] for k in ("bytes", "flops")):
            return c


def _held(case):
    """Bytes of one weight as it is held."""
    n = case["width"] * case["inner"]
    return n * case["bits"] // 8 + n // case["group"] * (2 + (1 if case["zeros"] == "u8" else 2))


def work(case):
    if case["op"] == "norm":
        n = case["rows"] * case["features"]
        if case["backward"]:
            return {"bytes": n * (6 + 2 * case["residual"]) + case["features"] * 6, "flops": n * 10}
        out = n * 2 if not case["codes"] else n * 3 + n // case["group"] * 4
        return {"bytes": n * (2 + 4 * case["residual"]) + out + case["features"] * 2, "flops": n * (5 + 2 * bool(case["codes"]))}
    if case["op"] == "rotary":
        heads = case["seqs"] * case["new"] * (case["q_heads"] + case["kv_heads"])
        return {"bytes": heads * case["head_dim"] * 4 + case["seqs"] * 8, "flops": heads * case["rotary_dim"] * 3}
    if case["op"] == "gated":
        n = case["rows"] * case["features"]
        return {"bytes": n * (10 if case["backward"] else 6), "flops": n * (16 if case["backward"] else 8)}
    inner = case["tokens"] * case["inner"] * 2
    rows = case["tokens"] * case["width"] * 2
    moved = inner * 5 if case["backward"] else inner * (3 if case["keep"] else 1)
    return {"bytes": 2 * _held(case) + rows + moved, "flops": 4 * case["tokens"] * case["width"] * case["inner"]}


# ---------------------------------------------------------------------------------------------- inputs
def _scaling(case):
    """Frequencies of the pairs: what a model's configuration says."""
    return {"plain": {"base": 10000.0}, "linear": {"base": 10000.0, "factor": 4.0},
            "base": {"base": 10000.0, "factor": 8.0},
            "ramp": {"base": 500000.0, "factor": 16.0, "low": 1.0, "high": 32.0, "length": 8192.0}}[case["scaling"]]


def _amplitude(case):
    return 1.0 + 0.1 * math.log(_scaling(case)["factor"]) if case["scaling"] == "ramp" else 1.0


def _news(case):
    """Rows of each sequence: a prompt's lengths differ, as do the texts before a step."""
    lens, news = [], []
    for b in range(case["seqs"]):
        f = 0.25 + 0.75 * ((b + 1) * 0.6180339887 % 1.0) if case["length"] > case["new"] else 1.0
        n = max(case["new"], round(case["length"] * f))
        lens.append(n)
        news.append(case["new"])
    return lens, news


def _weight(case, gen):
    """Codes [inner, width * bits / 8] u8, steps fp16, zeros u8 or fp16: a normal weight, quantised to its groups' ranges."""
    bits, top = case["bits"], 2 ** case["bits"] - 1
    w = (torch.randn(case["inner"], case["width"], device=DEV, generator=gen) * 0.02).unflatten(-1, (-1, case["group"]))
    low, high = w.amin(-1, keepdim=True), w.amax(-1, keepdim=True)
    step = ((high - low) / top).clamp_min(2.0 ** -14)
    zero = (-low / step).round_().clamp_(0, top)
    q = (w / step).round_().add_(zero).clamp_(0, top).to(torch.int32).view(case["inner"], -1, 8)     # 8 codes: `bits` bytes
    stream = (q << (bits * torch.arange(8, device=DEV, dtype=torch.int32))).sum(-1, keepdim=True, dtype=torch.int32)
    codes = ((stream >> (8 * torch.arange(bits, device=DEV, dtype=torch.int32))) & 255).to(torch.uint8).flatten(1)
    if case["zeros"] == "u8":
        zero = zero.to(torch.uint8)
    else:                                                           # trained: no longer whole
        zero = (zero + 0.1 * torch.randn(zero.shape, device=DEV, generator=gen)).to(torch.float16)
    return codes.contiguous(), step[..., 0].to(torch.float16), zero[..., 0].contiguous()


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)

    def normal(*shape, std=1.0):
        return torch.randn(*shape, device=DEV, generator=gen).mul_(std).to(BF16)

    s = {"case": dict(case)}
    if case["op"] == "norm":
        rows, n = case["rows"], case["features"]
        # the stream has a few channels that are large in every token, and tokens of different size
        spread = torch.exp(0.3 * torch.randn(rows, 1, device=DEV, generator=gen))
        channel = torch.where(torch.rand(n, device=DEV, generator=gen) < 0.01, 20.0, 1.0)
        s["X"] = (torch.randn(rows, n, device=DEV, generator=gen) * spread * channel).to(BF16)
        s["W"] = (1.0 + 0.2 * torch.randn(n, device=DEV, generator=gen)).to(BF16)
        if case["backward"]:
            s["dY"], s["dR"] = normal(rows, n, std=0.01), normal(rows, n, std=0.01) if case["residual"] else None
            s["dX"], s["dW"] = torch.empty_like(s["X"]), torch.empty(n, device=DEV)
        else:
            s["R"] = normal(rows, n) if case["residual"] else None
            s["H"] = torch.empty_like(s["X"]) if case["residual"] else None
            s["Y"] = torch.empty_like(s["X"])
            if case["codes"]:
                s["codes"] = torch.empty(rows, n, dtype=torch.uint8, device=DEV)
                s["scales"] = torch.empty(rows, n // case["group"], device=DEV)
    elif case["op"] == "rotary":
        lens, news = _news(case)
        offsets = [0]
        for k in news:
            offsets.append(offsets[-1] + k)
        rows, Hq, Hk, D = offsets[-1], case["q_heads"], case["kv_heads"], case["head_dim"]
        if case["fused"]:                                           # queries, keys and values side by side
            qkv = normal(rows, Hq + 2 * Hk, D)
            s["Q"], s["K"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hk]
        else:
            s["Q"], s["K"] = normal(rows, Hq, D), normal(rows, Hk, D)
        s["Q_out"], s["K_out"] = (torch.empty(rows, h, D, dtype=BF16, device=DEV) for h in (Hq, Hk))
        s["row_offsets"] = torch.tensor(offsets, dtype=torch.int32, device=DEV)
        s["lengths"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
    elif case["op"] == "gated":
        rows, n = case["rows"], case["features"]
        if case["fused"]:
            both = normal(rows, 2 * n, std=1.3)
            s["G"], s["U"] = both[:, :n], both[:, n:]
        else:
            s["G"], s["U"] = normal(rows, n, std=1.3), normal(rows, n, std=1.3)
        if case["backward"]:
            s["dH"] = normal(rows, n, std=0.01)
            grads = torch.empty(rows, 2 * n, dtype=BF16, device=DEV) if case["fused"] else None
            s["dG"], s["dU"] = (grads[:, :n], grads[:, n:]) if case["fused"] else (torch.empty_like(s["G"]), torch.empty_like(s["U"]))
        else:
            s["H"] = torch.empty(rows, n, dtype=BF16, device=DEV)
    else:
        T, E, F = case["tokens"], case["width"], case["inner"]
        s["gate"], s["up"] = _weight(case, gen), _weight(case, gen)
        if case["backward"]:
            s["dH"], s["G"], s["U"] = normal(T, F, std=0.01), normal(T, F, std=1.3), normal(T, F, std=1.3)
            s["dX"], s["dG"], s["dU"] = torch.empty(T, E, dtype=BF16, device=DEV), torch.empty_like(s["G"]), torch.empty_like(s["U"])
        else:
            s["X"], s["H"] = normal(T, E), torch.empty(T, F, dtype=BF16, device=DEV)
            s["G"], s["U"] = (torch.empty_like(s["H"]), torch.empty_like(s["H"])) if case["keep"] else (None, None)
    return s


# ---------------------------------------------------------------------------------------------- the plain forms
def _plain_norm(s):
    c, w = s["case"], s["W"].float()
    if c["backward"]:
        h, dy = s["X"].float(), s["dY"].float()
        r = torch.rsqrt(h.square().mean(-1, keepdim=True) + 1e-5)
        v = dy * w
        dx = r * (v - h * (r * r * (v * h).mean(-1, keepdim=True)))
        if s["dR"] is not None:
            dx = dx + s["dR"].float()
        return {"dX": dx.to(BF16), "dW": (dy * (h * r)).sum(0)}
    out = {}
    h = s["X"]
    if s["R"] is not None:
        h = out["H"] = (h.float() + s["R"].float()).to(BF16)
    h = h.float()
    r = torch.rsqrt(h.square().mean(-1, keepdim=True) + 1e-5)
    if not c["codes"]:
        out["Y"] = (h * w * r).to(BF16)
        return out
    t = (h * w).unflatten(-1, (-1, c["group"]))
    top = 127.0 if c["codes"] == "int8" else 448.0
    most = t.abs().amax(-1, keepdim=True)
    most = torch.where(most < SMALL, torch.zeros_like(most), most)
    t = torch.where(most > 0, t * (torch.full_like(most, top) / most), torch.zeros_like(t))
    q = t.round().to(torch.int8) if c["codes"] == "int8" else t.to(torch.float8_e4m3fn)
    scale = most * r.unsqueeze(-1) / top
    out["Y"] = (q.float() * scale).to(BF16).flatten(1)
    out["codes"], out["scales"] = q.view(torch.uint8).flatten(1), scale[..., 0]
    return out


def _frequencies(c):
    """Radians a position, 64 bits, by the definitions of the scalings (`factor` times the length that the model was made for)."""
    p, r = _scaling(c), c["rotary_dim"]
    i = torch.arange(r // 2, dtype=torch.float64, device=DEV)
    base = p["base"]
    if c["scaling"] == "base" and r > 2:
        base = base * p["factor"] ** (r / (r - 2))
    f = base ** (-2.0 * i / r)
    if c["scaling"] == "linear":
        f = f / p["factor"]
    if c["scaling"] == "ramp":                                      # by the turns that a pair makes in the original length
        keep = ((p["length"] * f / (2 * math.pi) - p["low"]) / (p["high"] - p["low"])).clamp(0, 1)
        f = f * keep + f / p["factor"] * (1 - keep)
    return f


def _angles(s):
    """[rows, pairs], 64 bits."""
    off = s["row_offsets"].long()
    n = off[1:] - off[:-1]
    row = torch.arange(s["Q"].shape[0], device=DEV)
    seq = torch.searchsorted(off[1:], row, right=True)
    pos = (s["lengths"].long() - n - off[:-1])[seq] + row
    return pos.double()[:, None] * _frequencies(s["case"])


def _plain_rotary(s):
    c, r = s["case"], s["case"]["rotary_dim"]
    t = _angles(s)
    t = -t if c["backward"] else t
    cos, sin = ((f(t) * _amplitude(c)).float()[:, None] for f in (torch.cos, torch.sin))
    for x, out in ((s["Q"], s["Q_out"]), (s["K"], s["K_out"])):
        y = x[..., :r].float()
        a, b = (y[..., :r // 2], y[..., r // 2:]) if c["layout"] == "halves" else (y[..., 0::2], y[..., 1::2])
        a, b = a * cos - b * sin, b * cos + a * sin
        y = torch.cat([a, b], -1) if c["layout"] == "halves" else torch.stack([a, b], -1).flatten(-2)
        out[..., :r], out[..., r:] = y.to(BF16), x[..., r:]
    return [s["Q_out"], s["K_out"]]


def _act(g, kind):
    """act(g) and act'(g)."""
    if kind == "silu":
        e = torch.sigmoid(g)
        return g * e, e * (1 + g * (1 - e))
    if kind == "gelu":
        phi = 0.5 * torch.erfc(g * -math.sqrt(0.5))
        return g * phi, phi + g * torch.exp(g * g * -0.5) * (1 / math.sqrt(2 * math.pi))
    # 0.5 (1 + tanh z) = sigmoid(2 z): nothing cancels
    k = 2 * math.sqrt(2 / math.pi)
    e = torch.sigmoid(k * (g + 0.044715 * g * g * g))
    return g * e, e + g * e * (1 - e) * (k * (1 + 3 * 0.044715 * g * g))


def _plain_gated(s):
    g, u = s["G"].float(), s["U"].float()
    a, da = _act(g, s["case"]["activation"])
    if not s["case"]["backward"]:
        return (a * u).to(BF16)
    dh = s["dH"].float()
    return [(dh * u * da).to(BF16), (dh * a).to(BF16)]


def _dequantised(weight, bits, group, like):
    """(code - zero) * step of a whole weight."""
    codes, step, zero = weight
    rows = codes.shape[0]
    stream = (codes.view(rows, -1, bits).to(torch.int32) << (8 * torch.arange(bits, device=DEV, dtype=torch.int32))).sum(-1, keepdim=True, dtype=torch.int32)
    q = (stream >> (bits * torch.arange(8, device=DEV, dtype=torch.int32))) & (2 ** bits - 1)
    q = q.to(like).view(rows, -1, group)
    return ((q - zero.to(like)[..., None]) * step.to(like)[..., None]).flatten(1)


def _plain_feed(s):
    c = s["case"]
    gate, up = (_dequantised(w, c["bits"], c["group"], torch.float32) for w in (s["gate"], s["up"]))
    if c["backward"]:
        dg, du = _plain_gated(s)
        return [(dg.float() @ gate + du.float() @ up).to(BF16), dg, du]
    x = s["X"].float()
    g, u = x @ gate.T, x @ up.T
    h = (_act(g, c["activation"])[0] * u).to(BF16)
    return [h, g.to(BF16), u.to(BF16)] if c["keep"] else h


# ---------------------------------------------------------------------------------------------- the framework's calls
def _plan(s):
    """Descriptors, tables and scratch, which a program keeps from step to step."""
    from paper_2407_11062_b200 import binding as eqat
    c = s["case"]

    if c["op"] == "norm":
        kind = {"": eqat.EQAT_CODES_NONE, "int8": eqat.EQAT_CODES_INT8, "e4m3": eqat.EQAT_CODES_E4M3}[c["codes"]]
        desc = eqat.make_norm_desc(c["rows"], c["features"], 1e-5, kind, c["group"])
        return eqat, desc, torch.empty(eqat.rms_norm_workspace_bytes(desc), dtype=torch.uint8, device=DEV) if c["backward"] else None
    if c["op"] == "rotary":
        p = _scaling(c)
        kind = {"plain": eqat.EQAT_ROTARY_PLAIN, "linear": eqat.EQAT_ROTARY_LINEAR, "base": eqat.EQAT_ROTARY_BASE,
                "ramp": eqat.EQAT_ROTARY_RAMP}[c["scaling"]]
        layout = eqat.EQAT_ROTARY_HALVES if c["layout"] == "halves" else eqat.EQAT_ROTARY_PAIRS
        desc = eqat.make_rotary_desc(s["Q"].shape[0], c["q_heads"], c["kv_heads"], c["head_dim"], c["rotary_dim"], layout,
                                     _amplitude(c), c["seqs"])
        return eqat, desc, eqat.rotary_turns(c["rotary_dim"], p["base"], kind, p.get("factor", 1.0), p.get("low", 0.0),
                                             p.get("high", 0.0), p.get("length", 0.0)).to(DEV)
    act = {"silu": eqat.EQAT_ACT_SILU, "gelu": eqat.EQAT_ACT_GELU, "gelu_tanh": eqat.EQAT_ACT_GELU_TANH}[c["activation"]]
    if c["op"] == "gated":
        return eqat, eqat.make_gated_desc(c["rows"], c["features"], act), None
    zeros = eqat.EQAT_ZP_U8 if c["zeros"] == "u8" else eqat.EQAT_ZP_FP16
    desc = eqat.make_desc(c["bits"], c["group"], c["inner"], c["width"], c["tokens"], 0, zeros)
    need = 0 if c["keep"] else eqat.workspace_bytes(desc, eqat.EQAT_OP_PACKED_GATED_BWD if c["backward"] else eqat.EQAT_OP_PACKED_GATED_FWD)
    return eqat, desc, (act, torch.empty(need, dtype=torch.uint8, device=DEV) if need else None)


def _call(s):
    if "plan" not in s:
        s["plan"] = _plan(s)
    c, (eqat, desc, more) = s["case"], s["plan"]
    if c["op"] == "norm":
        if c["backward"]:
            eqat.eqat_rms_norm_bwd(desc, s["dY"], s["X"], s["W"], s["dR"], s["dX"], s["dW"], more)
            return {"dX": s["dX"], "dW": s["dW"]}
        eqat.eqat_rms_norm_fwd(desc, s["X"], s["R"], s["W"], s["H"], s["Y"], s.get("codes"), s.get("scales"))
        return {k: s[k] for k in ("H", "Y", "codes", "scales") if s.get(k) is not None}
    if c["op"] == "rotary":
        call = eqat.eqat_rotary_bwd if c["backward"] else eqat.eqat_rotary_fwd
        call(desc, s["Q"], s["K"], more, s["Q_out"], s["K_out"], None, s["row_offsets"], s["lengths"])
        return [s["Q_out"], s["K_out"]]
    if c["op"] == "gated":
        if c["backward"]:
            eqat.eqat_gated_bwd(desc, s["dH"], s["G"], s["U"], s["dG"], s["dU"])
            return [s["dG"], s["dU"]]
        eqat.eqat_gated_fwd(desc, s["G"], s["U"], s["H"])
        return s["H"]
    act, scratch = more
    if c["backward"]:
        eqat.qlinear_packed_gated_bwd(desc, act, s["dH"], s["G"], s["U"], s["gate"], s["up"], s["dX"], s["dG"], s["dU"], scratch)
        return [s["dX"], s["dG"], s["dU"]]
    eqat.qlinear_packed_gated_fwd(desc, act, s["X"], s["gate"], s["up"], s["H"], s["G"], s["U"], scratch)
    return [s["H"], s["G"], s["U"]] if c["keep"] else s["H"]


def run(state):
    if own:
        return _call(state)
    return {"norm": _plain_norm, "rotary": _plain_rotary, "gated": _plain_gated, "feed": _plain_feed}[state["case"]["op"]](state)


# ---------------------------------------------------------------------------------------------- 64 bits
def _exact_act(g, kind):
    """Activation and derivative by their textbook forms; erfc where 1 + erf would cancel."""
    if kind == "silu":
        d = 1 + torch.exp(-g)
        return g / d, 1 / d + g * torch.exp(-g) / d ** 2
    if kind == "gelu":
        cdf = torch.special.erfc(-g / math.sqrt(2)) / 2
        return g * cdf, cdf + g * torch.exp(-g ** 2 / 2) / math.sqrt(2 * math.pi)
    z = math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)
    d = 1 + torch.exp(-2 * z)                                       # 0.5 (1 + tanh z) = 1 / d
    return g / d, 1 / d + g * 2 * torch.exp(-2 * z) / d ** 2 * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * g ** 2)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        w = s["W"].double()
        if case["backward"]:
            h, dy = s["X"].double(), s["dY"].double()
            scale = (h.pow(2).sum(-1, keepdim=True) / h.shape[-1] + 1e-5).pow(-0.5)
            n = h * scale                                           # y = n w; what the mean of squares takes back
            g = dy * w
            dx = scale * (g - n * (g * n).sum(-1, keepdim=True) / h.shape[-1])
            return {"dX": dx if s["dR"] is None else dx + s["dR"].double(), "dW": torch.einsum("rn,rn->n", dy, n)}
        out, h = {}, s["X"].double()
        if s["R"] is not None:
            out["H"] = h + s["R"].double()
            h = out["H"].float().to(BF16).double()                  # the norm is that of the stream as it is held
        scale = (h.pow(2).sum(-1, keepdim=True) / h.shape[-1] + 1e-5).pow(-0.5)
        if not case["codes"]:
            out["Y"] = h * scale * w
            return out
        # which code: decided in binary32, by definition (products of bf16 numbers are exact there)
        parts = (h * w).float().reshape(h.shape[0], -1, case["group"])
        most = parts.abs().max(-1).values
        most[most < SMALL] = 0
        top = 127 if case["codes"] == "int8" else 448
        scaled = parts * torch.nan_to_num(top / most, posinf=0)[..., None]
        code = torch.round(scaled).double() if top == 127 else scaled.to(torch.float8_e4m3fn).double()
        step = most.double() * scale / top
        out.update(Y=(code * step[..., None]).reshape(h.shape), codes=None, scales=step)
        return out
    if case["op"] == "rotary":
        # complex numbers: a pair times amplitude * e^(+-i t)
        lens, news = _news(case)
        pos = torch.cat([torch.arange(n - k, n, device=DEV) for n, k in zip(lens, news)]).double()
        p, r, out = _scaling(case), case["rotary_dim"], []
        f = []
        for i in range(r // 2):
            base = p["base"] * (p["factor"] ** (r / (r - 2)) if case["scaling"] == "base" and r > 2 else 1.0)
            x = math.exp(-2 * i / r * math.log(base))
            if case["scaling"] == "linear":
                x /= p["factor"]
            if case["scaling"] == "ramp":
                turns = p["length"] * x / (2 * math.pi)
                keep = min(1.0, max(0.0, (turns - p["low"]) / (p["high"] - p["low"])))
                x = keep * x + (1 - keep) * x / p["factor"]
            f.append(x)
        t = pos[:, None] * torch.tensor(f, dtype=torch.float64, device=DEV)
        turn = torch.polar(torch.full_like(t, _amplitude(case)), -t if case["backward"] else t)[:, None]
        for x in (s["Q"], s["K"]):
            y = x.double().clone()
            if case["layout"] == "halves":
                z = torch.complex(y[..., :r // 2].contiguous(), y[..., r // 2:r].contiguous()) * turn
                y[..., :r // 2], y[..., r // 2:r] = z.real, z.imag
            else:
                z = torch.complex(y[..., 0:r:2].contiguous(), y[..., 1:r:2].contiguous()) * turn
                y[..., 0:r:2], y[..., 1:r:2] = z.real, z.imag
            out.append(y)
        return out
    kind = case["activation"]
    if case["op"] == "feed":
        def weight(codes, step, zero):                              # bit by bit
            place = torch.arange(8, device=DEV, dtype=torch.uint8)
            bit = ((codes[..., None] >> place) & 1).flatten(1).view(codes.shape[0], -1, case["bits"]).double()
            q = bit @ (2.0 ** torch.arange(case["bits"], device=DEV, dtype=torch.float64))
            g = case["group"]
            return (q - zero.double().repeat_interleave(g, -1)) * step.double().repeat_interleave(g, -1)
        if not case["backward"]:
            x = s["X"].double()
            g, u = x @ weight(*s["gate"]).T, x @ weight(*s["up"]).T
            h = _exact_act(g, kind)[0] * u
            return [h, g, u] if case["keep"] else h
    g, u = s["G"].double(), s["U"].double()
    a, da = _exact_act(g, kind)
    if not case["backward"]:
        return a * u
    dh = s["dH"].double()
    dg, du = dh * u * da, dh * a
    if case["op"] == "gated":
        return [dg, du]
    return [dg @ weight(*s["gate"]) + du @ weight(*s["up"]), dg, du]
