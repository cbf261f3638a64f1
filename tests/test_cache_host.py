"""The 4-bit cache without a GPU: pins of its oracle and the refusals of its entry points."""
import ctypes

import numpy as np
import pytest

from oracle import cache_oracle as C


@pytest.fixture(scope="module")
def eqat():
    from paper_2407_11062_b200.build import build_library
    build_library()
    from paper_2407_11062_b200 import binding
    return binding


# --------------------------------------------------------------------------- oracle
def test_one_group_by_hand():
    """Range [-1, 14]: step bf16(15/15) = 1, codes x + 1; the halves 0.5 and 1.5 above a code go to the even one."""
    x = np.array([-1, 14, 0, 3, 3.5, 4.5, -0.5, 0.5] + [2.0] * 24, np.float32)
    q, s, m = C.quantise(x, 32)
    assert s.tolist() == [1.0] and m.tolist() == [-1.0]
    assert q[:8].tolist() == [0, 15, 1, 4, 4, 6, 0, 2]
    assert C.pack(q)[:4].tolist() == [0xF0, 0x41, 0x64, 0x20]
    assert C.values(q, s, m)[:4].tolist() == [-1, 14, 0, 3]


def test_groups_that_do_not_contain_zero_and_flat_groups():
    x = np.concatenate([np.linspace(100, 107.5, 32), np.full(32, -3.25)]).astype(np.float32)
    q, s, m = C.quantise(C.bf16(x), 32)
    assert m.tolist() == [100.0, -3.25] and s.tolist() == [0.5, 0.0]
    assert np.abs(C.values(q, s, m)[:32] - C.bf16(x)[:32]).max() <= 0.25 and (C.values(q, s, m)[32:] == -3.25).all()


def test_a_value_is_at_most_half_a_step_off():
    """Half a step, and at the top what the rounding of the step (2^-8 of it, 15 times) takes away, as far as it is more;
    (x - m) is rounded once, which at these sizes is less than 2^-20 of the step."""
    rng = np.random.default_rng(1)
    x = C.bf16((rng.standard_normal((400, 64)) * np.exp(rng.standard_normal((400, 1)) * 4)).astype(np.float32))
    q, s, m = C.quantise(x, 32)
    err = np.abs(C.values(q, s, m) - x)
    assert (err <= np.repeat(s, 32, -1) * (0.5 + 15 * 2.0 ** -8)).all()
    assert (q.reshape(400, 2, 32).max(-1) == 15).all() and (q.reshape(400, 2, 32).min(-1) == 0).all()


def test_ends_of_the_range():
    big = np.float32(3e38)
    x = np.zeros((5, 32), np.float32)
    x[0, 0], x[1, 0], x[2, :2], x[3, 0], x[4, 0] = np.nan, np.inf, (big, -big), 2.0 ** -130, C.bf16([big])[0]
    q, s, m = C.quantise(C.bf16(x), 32)
    v = C.values(q, s, m)
    assert np.isnan(v[:3]).all()                            # NaN, an infinity, a range beyond binary32
    assert s[3] == 0 and (v[3] == 0).all()                  # a step below 2^-126
    assert np.isfinite(v[4]).all() and abs(v[4, 0] / big - 1) < 2 ** -7


def test_pack_is_the_dense_stream_of_the_weights():
    from oracle import eqat_oracle as O
    codes = np.random.default_rng(2).integers(0, 16, (3, 128)).astype(np.uint8)
    assert np.array_equal(C.pack(codes), O.pack_rows(codes, 4)) and np.array_equal(C.unpack(C.pack(codes)), codes)


def test_attention_of_equal_keys_is_the_mean_and_of_one_key_its_value():
    rng = np.random.default_rng(3)
    k, v, Q = np.ones((7, 1, 4)), rng.standard_normal((7, 1, 4)), rng.standard_normal((3, 2, 4))
    O, lse, _, _ = C.attention(Q, [k], [v], [7], [0, 3], 0.5)
    assert np.allclose(O[2, 0], v.mean(0)[0]) and np.allclose(O[0, 1], v[:5].mean(0)[0])
    assert np.allclose(lse[2], 0.5 * Q[2].sum(-1) + np.log(7))
    O, lse, _, _ = C.attention(Q, [k], [v], [7], [0, 3], 0.5, window=1)
    assert np.allclose(O[:, 0], v[4:, 0])
    O, lse, _, _ = C.attention(Q, [k[:1]], [v[:1]], [1], [0, 3], 0.5)         # two of three rows see nothing
    assert (O[:2] == 0).all() and np.isneginf(lse[:2]).all() and np.allclose(O[2], v[0])


def test_places():
    seq, page, at = C.places([0, 2, 2, 5], [20, 4, 2], [[7, 9], [1, 0], [3, -1]], 16, 8, 7)
    assert seq.tolist() == [0, 0, 2, 2, 2, -1, -1]
    assert page.tolist() == [-1, -1, -1, 3, 3, -1, -1] and at.tolist()[3:5] == [0, 1]     # page 9 is outside, position -1 too


# --------------------------------------------------------------------------- refusals
def desc(eqat, **kw):
    f = dict(group=128, head_dim=128, kv_heads=8, page_size=16, pages=64, sequences=4, max_pages=32, rows=4, bits=4)
    f.update(kw)
    return eqat.make_cache_desc(**f)


OK, ODD = 0x1000, 0x1008


def append(eqat, d, **kw):
    f = dict(K=OK, kp=1024, V=OK, vp=1024, off=OK, len=OK, table=OK, pool=(OK, OK, OK, OK), K_hat=None, V_hat=None)
    f.update(kw)
    pool = None if f["pool"] is None else ctypes.byref(eqat.eqat_cache(*f["pool"]))
    return eqat.lib.eqat_cache_append(d and ctypes.byref(d), f["K"], f["kp"], f["V"], f["vp"], f["off"], f["len"], f["table"],
                                      pool, f["K_hat"], f["V_hat"], None)


def read(eqat, d, **kw):
    f = dict(off=OK, len=OK, table=OK, pool=(OK, OK, OK, OK), K_hat=OK, V_hat=OK)
    f.update(kw)
    return eqat.lib.eqat_cache_read(ctypes.byref(d), f["off"], f["len"], f["table"], ctypes.byref(eqat.eqat_cache(*f["pool"])),
                                    f["K_hat"], f["V_hat"], None)


def attention(eqat, d, a, **kw):
    f = dict(Q=OK, qp=8192, off=OK, len=OK, table=OK, pool=(OK, OK, OK, OK), O=OK, op=8192, lse=None, ws=OK, bytes=1 << 40)
    f.update(kw)
    return eqat.lib.eqat_cache_attention(d and ctypes.byref(d), a and ctypes.byref(a), f["Q"], f["qp"], f["off"], f["len"],
                                         f["table"], ctypes.byref(eqat.eqat_cache(*f["pool"])), f["O"], f["op"], f["lse"],
                                         f["ws"], f["bytes"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(bits=2), -4), (dict(bits=8), -4), (dict(group=16), -4), (dict(group=96), -4), (dict(group=256), -4),
    (dict(head_dim=96), -4), (dict(head_dim=512), -4), (dict(head_dim=64), -2), (dict(kv_heads=0), -2), (dict(kv_heads=-1), -2),
    (dict(page_size=8), -2), (dict(page_size=24), -2), (dict(page_size=0), -2), (dict(pages=0), -2), (dict(sequences=0), -2),
    (dict(max_pages=0), -2), (dict(rows=0), -2), (dict(rows=1 << 31), -2), (dict(page_size=1 << 20, max_pages=1 << 11), -2),
    (dict(pages=1 << 30), -2), (dict(pages=(1 << 31) - 1, kv_heads=65536, page_size=1 << 30, max_pages=1), -2),
    (dict(sequences=1 << 21), -2),
])
def test_bad_cache_descriptors_are_rejected_on_the_host(eqat, kw, status):
    d, a = desc(eqat, **kw), eqat.make_attention_desc(64, 1, 0.1)
    assert append(eqat, d) == status and read(eqat, d) == status and attention(eqat, d, a) == status
    with pytest.raises(eqat.EqatError):
        eqat.cache_workspace_bytes(d, a)


def test_bad_pointers_and_pitches(eqat):
    d, a = desc(eqat), eqat.make_attention_desc(64, 1, 0.1)
    for name in ("K", "V", "off", "len", "table"):
        assert append(eqat, d, **{name: None}) == eqat.EQAT_ERR_NULL
        assert append(eqat, d, **{name: ODD}) == eqat.EQAT_ERR_ALIGN
    for i in range(4):
        for bad, status in ((None, eqat.EQAT_ERR_NULL), (ODD, eqat.EQAT_ERR_ALIGN)):
            pool = tuple(bad if j == i else OK for j in range(4))
            assert append(eqat, d, pool=pool) == status
            assert read(eqat, d, pool=pool) == status
            assert attention(eqat, d, a, pool=pool) == status
    assert append(eqat, d, pool=None) == eqat.EQAT_ERR_NULL and append(eqat, None) == eqat.EQAT_ERR_NULL
    assert append(eqat, d, K_hat=OK) == eqat.EQAT_ERR_NULL and append(eqat, d, V_hat=OK) == eqat.EQAT_ERR_NULL
    assert append(eqat, d, K_hat=OK, V_hat=ODD) == eqat.EQAT_ERR_ALIGN
    assert read(eqat, d, V_hat=None) == eqat.EQAT_ERR_NULL and read(eqat, d, K_hat=ODD) == eqat.EQAT_ERR_ALIGN
    for pitch in (1016, 1028, -1024, 0):                     # shorter than a row, not a multiple of 8
        assert append(eqat, d, kp=pitch) == eqat.EQAT_ERR_SHAPE and append(eqat, d, vp=pitch) == eqat.EQAT_ERR_SHAPE
        assert attention(eqat, d, a, qp=pitch) == eqat.EQAT_ERR_SHAPE and attention(eqat, d, a, op=pitch) == eqat.EQAT_ERR_SHAPE
    for name in ("Q", "O"):
        assert attention(eqat, d, a, **{name: None}) == eqat.EQAT_ERR_NULL
        assert attention(eqat, d, a, **{name: ODD}) == eqat.EQAT_ERR_ALIGN
    assert attention(eqat, d, a, lse=ODD) == eqat.EQAT_ERR_ALIGN
    assert attention(eqat, d, None) == eqat.EQAT_ERR_NULL and attention(eqat, None, a) == eqat.EQAT_ERR_NULL


@pytest.mark.parametrize("kw,status", [
    (dict(q_heads=0), -2), (dict(q_heads=12), -2), (dict(q_heads=4), -2), (dict(max_new=0), -2), (dict(max_new=-3), -2),
    (dict(window=-1), -2), (dict(scale=float("nan")), -4), (dict(scale=float("inf")), -4),
])
def test_bad_attention_descriptors(eqat, kw, status):
    f = dict(q_heads=64, max_new=1, scale=0.1, window=0)
    f.update(kw)
    assert attention(eqat, desc(eqat), eqat.make_attention_desc(**f)) == status


def test_workspace_is_asked_for(eqat):
    d, a = desc(eqat, max_pages=1024), eqat.make_attention_desc(64, 1, 0.1)
    need = eqat.cache_workspace_bytes(d, a)
    assert need > 0
    for kw in (dict(ws=None), dict(bytes=need - 1), dict(ws=0x1010)):
        assert attention(eqat, d, a, **kw) == eqat.EQAT_ERR_WORKSPACE


def test_the_binding_refuses_what_is_no_row_tensor(eqat):
    """Decided before the library is called: tensors that are not on a GPU, no tensors, another descriptor, no cache."""
    import torch
    d, a = desc(eqat), eqat.make_attention_desc(64, 1, 0.1)
    x, i = torch.zeros(4, 8, 128, dtype=torch.bfloat16), torch.zeros(5, dtype=torch.int32)
    with pytest.raises(ValueError):
        eqat.eqat_cache_append(d, x, x, i, i, i, (i, i, i, i))
    with pytest.raises(ValueError):
        eqat.eqat_cache_read(d, i, i, i, (i, i, i, i), x, x)
    with pytest.raises(ValueError):
        eqat.eqat_cache_attention(d, a, x, i, i, i, (i, i, i, i), x)
    for bad in ((a, x, x, i, i, i, (i, i, i, i)), (d, 1, x, i, i, i, (i, i, i, i)), (d, x, None, i, i, i, (i, i, i, i))):
        with pytest.raises((TypeError, ValueError)):
            eqat.eqat_cache_append(*bad)
    for cache in (None, [i, i, i, i], (i, i, i)):
        with pytest.raises((TypeError, ValueError)):
            eqat.eqat_cache_read(d, None, None, None, cache, None, None)


@pytest.mark.parametrize("rows,q_heads,kv_heads,D,group,plan", [
    (1, 64, 8, 128, 128, (8, 0)), (5, 64, 8, 128, 128, (32, 0)), (1000, 64, 8, 128, 128, (32, 1)), (1, 4, 4, 256, 64, (1, 0)),
    (1000, 4, 4, 256, 64, (8, 0))])
def test_how_a_call_is_divided(eqat, rows, q_heads, kv_heads, D, group, plan):
    """One sequence on 148 SMs: few rows, a prompt, heads that the kernel for prompts does not take (tiles of 8 rows at most)."""
    d = eqat.make_cache_desc(group, D, kv_heads, 16, 4096, 1, 2048, rows)
    assert eqat.eqat_cache_attention_plan(d, eqat.make_attention_desc(q_heads, rows, 0.1), 148) == plan


def test_bad_questions_about_a_call(eqat):
    d = eqat.make_cache_desc(64, 128, 4, 16, 64, 1, 8, 1)
    for a, sms in ((eqat.make_attention_desc(3, 1, 0.1), 148), (eqat.make_attention_desc(4, 1, 0.1), -1)):
        with pytest.raises(eqat.EqatError):
            eqat.eqat_cache_attention_plan(d, a, sms)
    many = eqat.make_cache_desc(64, 128, 4, 16, 64, 1, 8, 1 << 28)
    assert eqat.cache_workspace_bytes(many, eqat.make_attention_desc(4, 1, 0.1)) >= 0
    with pytest.raises(eqat.EqatError):
        eqat.cache_workspace_bytes(many, eqat.make_attention_desc(8, 1, 0.1))


def test_tensor_memory_is_taken_before_the_next_launch_may_start():
    """A CTA of the next launch must find what this one holds counted: columns are taken before dependents are let in."""
    import pathlib
    csrc = pathlib.Path(__file__).resolve().parents[1] / "paper_2407_11062_b200" / "csrc"
    for name, kernel in (("attention.cu", "attention_kernel("), ("prompt.cu", "prompt_kernel(")):
        text = (csrc / name).read_text()
        body = text[text.index(kernel, text.index("__global__")):]
        assert 0 < body.index("take_columns(") < body.index("grid_dependents_launch(")


def test_the_binding_refuses_other_types_and_short_tensors(eqat):
    """Each tensor in turn with another type or one element or row less; decided before anything else about it."""
    import torch
    d, a = eqat.make_cache_desc(64, 128, 2, 16, 3, 4, 5, 6), eqat.make_attention_desc(8, 1, 0.1)
    x, q = torch.zeros(6, 2, 128, dtype=torch.bfloat16), torch.zeros(6, 8, 128, dtype=torch.bfloat16)
    for wrong, match, kind in ((x.half(), "BFloat16", TypeError), (x[:5], "shape", ValueError), (x[:, :1], "shape", ValueError), (x, "CUDA", ValueError)):
        with pytest.raises(kind, match=match):
            eqat.eqat_cache_append(d, wrong, x, None, None, None, None)
    for wrong, match, kind in ((q.float(), "BFloat16", TypeError), (q[:5], "shape", ValueError), (x, "shape", ValueError), (q, "CUDA", ValueError)):
        with pytest.raises(kind, match=match):
            eqat.eqat_cache_attention(d, a, wrong, None, None, None, None, q)
    for at, need in ((0, 5), (1, 4), (2, 20)):
        for t, match, kind in ((torch.zeros(need, dtype=torch.int64), "Int", TypeError),
                               (torch.zeros(need - 1, dtype=torch.int32), "fewer", ValueError),
                               (torch.zeros(need, dtype=torch.int32), "CUDA", ValueError)):
            with pytest.raises(kind, match=match):
                eqat.eqat_cache_read(d, *[t if i == at else None for i in range(3)], (None,) * 4, None, None)
    tokens = 3 * 2 * 16
    for at in range(4):
        good = torch.zeros(tokens * 4, dtype=torch.bfloat16) if at & 1 else torch.zeros(tokens * 64, dtype=torch.uint8)
        for t, match, kind in ((good.float(), "expected a tensor of type", TypeError), (good[:-1], "fewer", ValueError), (good, "CUDA", ValueError)):
            with pytest.raises(kind, match=match):
                eqat.eqat_cache_read(d, None, None, None, tuple(t if i == at else None for i in range(4)), None, None)
    for at in range(2):
        for t, match, kind in ((x.half(), "BFloat16", TypeError), (x[:5], "fewer", ValueError), (x, "CUDA", ValueError)):
            with pytest.raises(kind, match=match):
                eqat.eqat_cache_read(d, None, None, None, (None,) * 4, *[t if i == at else None for i in range(2)])
