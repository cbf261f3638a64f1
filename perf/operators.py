"""The 4-bit key/value cache and the attention over it: the calls and sizes that their performance is judged on.

A decoder block whose linears are held in 2 to 4 bits spends its memory and its decoding time on the keys and values of
the tokens before.  They are held in 4 bits here, in pages, every group of `group` consecutive elements of a head with a
step and a minimum of its own:

    append     quantises the new tokens' keys and values, writes them behind each sequence and gives back what the cache
               now holds for them (a prompt's own attention wants the values that later tokens will see)
    read       gives back the values of the last tokens of each sequence
    attention  new tokens of each sequence over its cache, causal, optionally within a window

A group x_1 .. x_g of bf16 numbers with minimum m and maximum M is held as
    s = bf16((M - m) * (1/15)),  0 where that is below 2^-126        (binary32, 1/15 rounded to it)
    q_i = clamp(rint((x_i - m) * (1/s)), 0, 15)                      (binary32, half to even; 0 where s = 0)
and stands for q_i * s + m.  Codes: two a byte, the even element low.
"""
import math
import random

import torch

own = False

DEV = "cuda"
STEP_MIN = 2.0 ** -126


# ---------------------------------------------------------------------------------------------- cases
def _case(name, op, seqs, length, new, q_heads, kv_heads, head_dim, group, page, window=0, ragged=False):
    c = {"op": op, "seqs": seqs, "length": length, "new": new, "q_heads": q_heads, "kv_heads": kv_heads,
         "head_dim": head_dim, "group": group, "page": page, "window": window, "ragged": ragged}
    return {"name": name, **c} if name else c


def listed():
    # head counts: 32/32, 40/40 and 64 query heads on 8 are those of 7B, 13B and 70B Llama-2 blocks
    return [
        # one decoding step of one user: latency of a call that moves a few kilobytes
        _case("append_1x1_h8", "append", 1, 200, 1, 64, 8, 128, 128, 16),
        # one decoding step of a batch
        _case("append_64x1_h40_g64", "append", 64, 250, 1, 40, 40, 128, 64, 64, ragged=True),
        # prompts of a batch, written behind one another; odd lengths
        _case("append_prompts_h32_g32", "append", 5, 3001, 3001, 32, 32, 128, 32, 32, ragged=True),
        # what one sequence holds, an odd number of tokens
        _case("read_1x1001_h8", "read", 1, 1001, 1001, 64, 8, 128, 128, 16),
        # a whole batch read back (moved to another pool, or scored again)
        _case("read_16x4096_h32_g64", "read", 16, 4096, 4096, 32, 32, 128, 64, 64, ragged=True),
        # decoding, one user, 7B, a short text: latency
        _case("decode_1x513_h32", "attention", 1, 513, 1, 32, 32, 128, 128, 16),
        # decoding, one user, 70B, a long text: the axis has to be split
        _case("decode_1x32768_h64_8", "attention", 1, 32768, 1, 64, 8, 128, 128, 64),
        # decoding, a batch of 70B with texts of different lengths
        _case("decode_64x4096_h64_8", "attention", 64, 4096, 1, 64, 8, 128, 128, 16, ragged=True),
        # decoding, a batch of 7B, short groups
        _case("decode_32x2048_h32_g32", "attention", 32, 2048, 1, 32, 32, 128, 32, 64, ragged=True),
        # a few drafted tokens a sequence are checked at once, attention within a window
        _case("draft_16x5_w4000_h64_8", "attention", 16, 6001, 5, 64, 8, 128, 64, 32, window=4000, ragged=True),
        # a piece of a long prompt behind what is cached already
        _case("chunk_1000_of_8192_h64_8", "attention", 1, 8192, 1000, 64, 8, 128, 128, 64),
        # whole prompts of a small batch, small heads
        _case("prompts_4x1500_h32_d64", "attention", 4, 1500, 1500, 32, 32, 64, 64, 16, ragged=True),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    top = {op: [work(c) for c in listed() if c["op"] == op] for op in ("append", "read", "attention")}
    while True:
        op = rng.choice(("append", "read", "attention", "attention", "attention"))
        head_dim = rng.choice((64, 128, 128, 128, 256))
        group = rng.choice([g for g in (32, 64, 128) if g <= head_dim])
        kv_heads = rng.choice((1, 2, 4, 8, 8, 16, 32, 40))
        q_heads = kv_heads * rng.choice((1, 1, 2, 4, 5, 8))
        seqs = _log(rng, 1, 128)
        kind = rng.choice(("step", "step", "draft", "chunk"))
        length = _log(rng, 64, 40000) if op == "attention" else _log(rng, 1, 8000)
        new = {"step": 1, "draft": rng.randint(2, 16), "chunk": _log(rng, 17, 2000)}[kind]
        if op == "read":
            new = length
        c = _case(None, op, seqs, length, min(new, length), q_heads, kv_heads, head_dim, group, rng.choice((16, 16, 32, 64, 128)),
                  rng.choice((0, 0, 0, _log(rng, 16, 8000))) if op == "attention" else 0, rng.random() < 0.7)
        w = work(c)
        scores = seqs * q_heads * c["new"] * length                 # what the plain form holds at once
        values = seqs * kv_heads * length * head_dim
        if q_heads <= 64 and scores <= 6e8 and values <= 3e8 and all(w[k] <= max(t[k] for t in top[op]) for k in ("bytes", "flops")):
            return c


def _lens(case):
    """Tokens that each sequence holds after the call, and how many of them are new."""
    lens, news = [], []
    for b in range(case["seqs"]):
        f = 0.25 + 0.75 * ((b + 1) * 0.6180339887 % 1.0) if case["ragged"] else 1.0
        n = max(1, round(case["length"] * f))
        lens.append(n)
        news.append(n if case["new"] == case["length"] else min(case["new"], n))
    return lens, news


def work(case):
    lens, news = _lens(case)
    H, D, G = case["kv_heads"], case["head_dim"], case["head_dim"] // case["group"]
    held = 2 * H * (D // 2 + 4 * G)                                 # a token's keys and values: codes, steps and minima
    plain = 2 * H * D * 2                                           # the same in bf16
    rows = sum(news)
    if case["op"] == "append":                                      # read, write, and what it stands for
        return {"bytes": rows * (plain + held + plain), "flops": rows * 2 * H * D * 5}
    if case["op"] == "read":
        return {"bytes": rows * (held + plain), "flops": rows * 2 * H * D * 2}
    seen = pairs = 0
    for n, k in zip(lens, news):
        w = case["window"] or n
        first = max(0, n - k + 1 - w)                               # the first key that any new token sees
        seen += n - first
        full = max(0, min(k, n - w + 1)) if w < n else 0            # tokens whose window is full
        part = k - full
        last = n - full                                             # context of the last token with a shorter one
        pairs += full * w + part * (last + (last - part + 1)) // 2
    return {"bytes": seen * held + rows * case["q_heads"] * D * 2 * 2, "flops": 4 * pairs * case["q_heads"] * D}


# ---------------------------------------------------------------------------------------------- inputs
def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    H, D, P, g = case["kv_heads"], case["head_dim"], case["page"], case["group"]
    lens, news = _lens(case)
    table_pages = max((n + P - 1) // P for n in lens)
    pages = sum((n + P - 1) // P for n in lens) + 1                 # one page more than is used
    order = list(range(pages))
    random.Random(seed).shuffle(order)
    table = [[-1] * table_pages for _ in lens]
    for b, n in enumerate(lens):
        for j in range((n + P - 1) // P):
            table[b][j] = order.pop()
    offsets = [0]
    for k in news:
        offsets.append(offsets[-1] + k)
    rows = offsets[-1]

    # keys have channels that are large or far from zero, values hardly any
    def channels(spread, shift):
        scale = torch.exp(spread * torch.randn(H, 1, D, device=DEV, generator=gen))
        return scale, shift * scale * torch.randn(H, 1, D, device=DEV, generator=gen)

    kc, vc = channels(0.5, 1.0), channels(0.2, 0.1)
    state = {"case": dict(case), "lens": lens, "news": news, "rows": rows,
             "row_offsets": torch.tensor(offsets, dtype=torch.int32, device=DEV),
             "lengths": torch.tensor(lens, dtype=torch.int32, device=DEV),
             "page_table": torch.tensor(table, dtype=torch.int32, device=DEV)}

    def held(c):
        x = torch.randn(pages, H, P, D, device=DEV, generator=gen).mul_(c[0]).add_(c[1]).to(torch.bfloat16)
        return _quantise(x, g)

    state["cache"] = (*held(kc), *held(vc))
    if case["op"] == "append":
        state["K"] = (torch.randn(rows, H, D, device=DEV, generator=gen) * kc[0][:, 0] + kc[1][:, 0]).to(torch.bfloat16)
        state["V"] = (torch.randn(rows, H, D, device=DEV, generator=gen) * vc[0][:, 0] + vc[1][:, 0]).to(torch.bfloat16)
    if case["op"] != "attention":
        state["K_hat"] = torch.zeros(rows, H, D, dtype=torch.bfloat16, device=DEV)
        state["V_hat"] = torch.zeros(rows, H, D, dtype=torch.bfloat16, device=DEV)
    else:
        state["Q"] = torch.randn(rows, case["q_heads"], D, device=DEV, generator=gen).to(torch.bfloat16)
        state["O"] = torch.zeros(rows, case["q_heads"], D, dtype=torch.bfloat16, device=DEV)
    return state


# ---------------------------------------------------------------------------------------------- the plain forms
def _quantise(x, group):
    """bf16 [..., D] -> codes [..., D/2] u8 and (step, minimum) [..., D/group, 2] bf16."""
    x = x.float().unflatten(-1, (-1, group))
    low, high = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    step = ((high - low) * (1.0 / 15.0)).to(torch.bfloat16).float()
    step = torch.where(step < STEP_MIN, torch.zeros_like(step), step)
    inverse = torch.where(step > 0, 1.0 / step, torch.zeros_like(step))
    q = ((x - low) * inverse).round_().clamp_(0, 15).to(torch.uint8).flatten(-2)
    return q[..., 0::2] | (q[..., 1::2] << 4), torch.cat([step, low], -1).to(torch.bfloat16)


def _values(codes, params):
    """What codes [..., D/2] with (step, minimum) [..., G, 2] stand for, fp32 [..., D]."""
    q = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).float()
    p = params.float()
    return (q.unflatten(-1, (p.shape[-2], -1)) * p[..., :1] + p[..., 1:]).flatten(-2)


def _places(s):
    """Page and place in the page of every new token."""
    P, off = s["case"]["page"], s["row_offsets"].long()
    row = torch.arange(s["rows"], device=DEV)
    seq = torch.searchsorted(off[1:], row, right=True)
    pos = s["lengths"].long()[seq] - (off[1:] - off[:-1])[seq] + row - off[seq]
    return s["page_table"].long()[seq, pos // P], pos % P


def _append(s):
    page, at = _places(s)
    out = []
    for x, codes, params in ((s["K"], *s["cache"][:2]), (s["V"], *s["cache"][2:])):
        q, p = _quantise(x, s["case"]["group"])
        codes[page, :, at], params[page, :, at] = q, p
        out.append(_values(q, p).to(torch.bfloat16))
    return [*out, *s["cache"]]


def _read(s):
    page, at = _places(s)
    return [_values(codes[page, :, at], params[page, :, at]).to(torch.bfloat16) for codes, params in (s["cache"][:2], s["cache"][2:])]


def _attention(s):
    c = s["case"]
    H, D, P, R = c["kv_heads"], c["head_dim"], c["page"], c["q_heads"] // c["kv_heads"]
    table, lens, off = s["page_table"].long().clamp_min(0), s["lengths"].long(), s["row_offsets"].long()
    B, L, T, dev = table.shape[0], table.shape[1] * P, max(s["news"]), DEV
    k, v = (_values(codes[table], params[table]).transpose(1, 2).reshape(B, H, L, D) for codes, params in (s["cache"][:2], s["cache"][2:]))
    n, i = off[1:] - off[:-1], torch.arange(T, device=dev)
    have = i < n[:, None]                                           # [B, T]
    row = (off[:-1, None] + i).clamp_max(s["rows"] - 1)
    q = s["Q"].float()[row].view(B, T, H, R, D).permute(0, 2, 1, 3, 4).reshape(B, H, T * R, D)
    score = (q @ k.transpose(-1, -2)).mul_(D ** -0.5).view(B, H, T, R, L)
    pos = (lens - n)[:, None] + i
    key = torch.arange(L, device=dev)
    hidden = (key > pos[..., None]) | (key <= pos[..., None] - (c["window"] or L + 1)) | ~have[..., None]
    score.masked_fill_(hidden[:, None, :, None], float("-inf"))
    top = score.amax(-1, keepdim=True)
    p = score.sub_(torch.where(top > float("-inf"), top, torch.zeros_like(top))).exp_()
    total = p.sum(-1, keepdim=True)
    o = (p.view(B, H, T * R, L) @ v).view(B, H, T, R, D) / torch.where(total > 0, total, torch.ones_like(total))
    s["O"][row[have]] = o.permute(0, 2, 1, 3, 4).reshape(B, T, H * R, D)[have].to(torch.bfloat16)
    return s["O"]


# ---------------------------------------------------------------------------------------------- the framework's calls
def _plan(s):
    """Descriptors and scratch, which a program keeps from step to step."""
    from paper_2407_11062_b200 import binding as eqat
    c = s["case"]
    desc = eqat.make_cache_desc(c["group"], c["head_dim"], c["kv_heads"], c["page"], s["cache"][0].shape[0], c["seqs"],
                                s["page_table"].shape[1], s["rows"])
    plan = {"desc": desc}
    if c["op"] == "attention":
        attn = eqat.make_attention_desc(c["q_heads"], max(s["news"]), c["head_dim"] ** -0.5, c["window"])
        need = eqat.cache_workspace_bytes(desc, attn)
        plan |= {"attn": attn, "scratch": torch.empty(need, dtype=torch.uint8, device=DEV) if need else None}
    return eqat, plan


def _call(s):
    if "plan" not in s:
        s["eqat"], s["plan"] = _plan(s)
    eqat, plan = s["eqat"], s["plan"]
    where = (s["row_offsets"], s["lengths"], s["page_table"], s["cache"])
    if s["case"]["op"] == "append":
        eqat.eqat_cache_append(plan["desc"], s["K"], s["V"], *where, s["K_hat"], s["V_hat"])
        return [s["K_hat"], s["V_hat"], *s["cache"]]
    if s["case"]["op"] == "read":
        eqat.eqat_cache_read(plan["desc"], *where, s["K_hat"], s["V_hat"])
        return [s["K_hat"], s["V_hat"]]
    eqat.eqat_cache_attention(plan["desc"], plan["attn"], s["Q"], *where, s["O"], None, plan["scratch"])
    return s["O"]


def run(state):
    if own:
        return _call(state)
    return {"append": _append, "read": _read, "attention": _attention}[state["case"]["op"]](state)


# ---------------------------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    H, D, g, P = case["kv_heads"], case["head_dim"], case["group"], case["page"]
    G, half = D // g, torch.tensor([0, 4], device=DEV, dtype=torch.uint8)

    def spread(codes):                                              # [..., D/2] -> [..., D]
        return ((codes[..., None] >> half) & 15).reshape(*codes.shape[:-1], D).double()

    def token_values(codes, params, b, first, last):                # [last - first, H, D] of sequence b
        pages = s["page_table"][b].tolist()[first // P:(last + P - 1) // P]
        lo = first // P * P
        q = torch.cat([spread(codes[p]).transpose(0, 1) for p in pages])[first - lo:last - lo]
        w = torch.cat([params[p].transpose(0, 1) for p in pages])[first - lo:last - lo].double()
        return q * w[..., 0].repeat_interleave(g, -1) + w[..., 1].repeat_interleave(g, -1)

    if case["op"] == "append":
        values, held = [], []
        for x in (s["K"], s["V"]):
            x = x.reshape(-1, H, G, g)
            least, most = x.min(-1).values.double(), x.max(-1).values.double()
            wide = (most.float() - least.float()) * torch.tensor(1 / 15, dtype=torch.float32, device=DEV)
            step = wide.to(torch.bfloat16).double()                 # decisions are taken in binary32
            step[step < STEP_MIN] = 0
            scaled = (x.float() - least.float()[..., None]) * torch.reciprocal(step.float())[..., None]
            q = torch.where(step[..., None] > 0, scaled, torch.zeros_like(scaled)).round().clamp(0, 15).double()
            values.append((q * step[..., None] + least[..., None]).reshape(-1, H, D))
            held.append(torch.stack([(most - least) / 15, least], -1))
        out = [*values, None, s["cache"][1].double(), None, s["cache"][3].double()]
        at = 0
        for b, (n, k) in enumerate(zip(s["lens"], s["news"])):
            pages = s["page_table"][b].long()
            pos = torch.arange(n - k, n, device=DEV)
            for i in (0, 1):
                out[3 + 2 * i][pages[pos // P], :, pos % P] = held[i][at:at + k]
            at += k
        return out
    if case["op"] == "read":
        out = []
        for codes, params in (s["cache"][:2], s["cache"][2:]):
            out.append(torch.cat([token_values(codes, params, b, n - k, n) for b, (n, k) in enumerate(zip(s["lens"], s["news"]))]))
        return out
    R, out, at = case["q_heads"] // H, torch.zeros(s["rows"], case["q_heads"], D, dtype=torch.float64, device=DEV), 0
    for b, (n, k) in enumerate(zip(s["lens"], s["news"])):
        first = max(0, n - k + 1 - case["window"]) if case["window"] else 0
        keys, vals = (token_values(*pair, b, first, n) for pair in (s["cache"][:2], s["cache"][2:]))
        pos = torch.arange(n - k, n, device=DEV)[:, None]
        key = torch.arange(first, n, device=DEV)[None, :]
        sees = (key <= pos) & ((key > pos - case["window"]) if case["window"] else (key >= 0))
        for h in range(case["q_heads"]):
            z = s["Q"][at:at + k, h].double() @ keys[:, h // R].T / math.sqrt(D)
            out[at:at + k, h] = torch.softmax(z.masked_fill(~sees, -math.inf), -1) @ vals[:, h // R]
        at += k
    return out
