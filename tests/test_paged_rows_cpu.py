"""Refusals of the entry points that bring rows into a paged cache, and the frequencies of rotary positions: host work only, nothing is launched."""
import ctypes as C
import math

import numpy as np
import pytest

from paper_2605_29727_amd import binding as btv

fake = C.c_void_p(4096)            # never dereferenced: every call below fails on the host


def refused(name, args, text, code=-1):
    lib = btv.lib()
    assert getattr(lib, name)(*args) == code, name
    assert text in lib.btv_last_error().decode(), lib.btv_last_error()


EXTEND = dict(prefix_len=fake, n_new=fake, depth=None, batch=4, total_max=100, n_pages=fake, free_pages=fake, n_free=fake, num_blocks=50, block_table=fake, max_blocks=8,
              q_offset=fake, slot=fake, position=fake, n_pages_out=C.c_void_p(8192), n_free_out=C.c_void_p(8192), ws=None, stream=None)


@pytest.mark.parametrize("change,text", [
    (dict(prefix_len=None), "null"), (dict(n_free_out=None), "null"), (dict(slot=None), "null"), (dict(batch=0), "batch=0"), (dict(batch=4097), "batch=4097"),
    (dict(total_max=-1), "total_max"), (dict(num_blocks=0), "num_blocks"), (dict(num_blocks=1 << 28), "num_blocks"), (dict(max_blocks=0), "max_blocks"),
    (dict(n_pages_out=fake), "may not be"), (dict(n_free_out=fake), "may not be"),
])
def test_extend_refuses(change, text):
    refused("btv_paged_extend", {**EXTEND, **change}.values(), text)


def rope_args(fp8=False, **change):
    a = dict(Q=fake, qs=C.c_longlong(4096), K=fake, ks=C.c_longlong(1024), V=fake, vs=C.c_longlong(1024), dtype=1, total=8, Hq=32, Hkv=8, D=128, position=fake, slot=fake,
             inv_freq=fake, R=128, interleaved=0, factor=C.c_float(1.0), Qout=C.c_void_p(8192), Kc=fake, Vc=fake, k_scale=C.c_float(1.0), v_scale=C.c_float(1.0),
             num_slots=C.c_longlong(64), ws=None, stream=None)
    a.update(change)
    for k in ("dtype",) if fp8 else ("k_scale", "v_scale"):
        del a[k]
    return a.values()


@pytest.mark.parametrize("change,text", [
    (dict(dtype=7), "dtype=7"), (dict(total=-1), "total"), (dict(Hq=0), "heads"), (dict(Hkv=2000), "heads"), (dict(D=96), "D=96"), (dict(R=8), "R=8"), (dict(R=144), "R=144"),
    (dict(interleaved=2), "interleaved"), (dict(factor=C.c_float(math.nan)), "factor"), (dict(num_slots=C.c_longlong(0)), "num_slots"),
    (dict(num_slots=C.c_longlong(1 << 31)), "num_slots"), (dict(Q=None), "null"), (dict(inv_freq=None), "null"), (dict(Vc=None), "null"), (dict(K=C.c_void_p(4104)), "16-byte"),
    (dict(inv_freq=C.c_void_p(4100)), "8-byte"), (dict(qs=C.c_longlong(4100)), "16 bytes apart"), (dict(ks=C.c_longlong(1016)), "overlap"),
    (dict(Qout=fake, qs=C.c_longlong(6144)), "Qout"),
])
def test_rope_append_refuses(change, text):
    refused("btv_rope_append", rope_args(**change), text)


@pytest.mark.parametrize("total", [(1 << 26) - 3, 1 << 30, 2**31 - 1])
def test_rope_append_refuses_more_rows_than_a_launch_has(total):
    refused("btv_rope_append", rope_args(total=total), "total")
    refused("btv_rope_append_fp8kv", rope_args(True, total=total), "total")


@pytest.mark.parametrize("scale", [0.0, -1.0, math.nan, math.inf, 1e-38])
def test_rope_append_fp8_refuses_scales(scale):
    refused("btv_rope_append_fp8kv", rope_args(True, k_scale=C.c_float(scale)), "scales")
    refused("btv_rope_append_fp8kv", rope_args(True, v_scale=C.c_float(scale)), "scales")


def chunk_args(fp8=False, **change):
    a = dict(Q=fake, K=fake, V=fake, k_scale=C.c_float(1.0), v_scale=C.c_float(1.0), num_blocks=100, table=fake, max_blocks=64, q_offset=fake, prefix_len=fake, batch=2, total_M=20,
             M_max=10, L_max=900, Hq=32, Hkv=8, D=128, scale=C.c_float(0.0), O=fake, ws=fake, ws_bytes=C.c_size_t(1 << 40), stream=None)
    a.update(change)
    if not fp8:
        del a["k_scale"], a["v_scale"]
    return a.values()


@pytest.mark.parametrize("change,text,code", [
    (dict(Q=None), "null", -1), (dict(table=None), "null", -1), (dict(O=C.c_void_p(4104)), "16-byte", -1), (dict(batch=0), "batch=0", -1), (dict(batch=5000), "batch=5000", -1),
    (dict(M_max=0), "M_max=0", -1), (dict(M_max=(1 << 20) + 1), "M_max", -1), (dict(L_max=-1), "L_max", -1), (dict(L_max=1 << 30), "L_max", -1), (dict(Hq=30), "heads", -1),
    (dict(Hq=136), "heads", -1), (dict(D=96), "D=96", -1), (dict(total_M=-1), "total_M", -1), (dict(num_blocks=0), "block", -1), (dict(max_blocks=56), "max_blocks", -1),
    (dict(scale=C.c_float(math.nan)), "scale", -1), (dict(scale=C.c_float(math.inf)), "scale", -1), (dict(ws=None), "workspace is NULL", -2),
    (dict(ws=C.c_void_p(4104)), "aligned", -2), (dict(ws_bytes=C.c_size_t(16)), "too small", -2),
])
def test_chunk_attention_refuses(change, text, code):
    refused("btv_chunk_attn_paged", chunk_args(**change), text, code)
    if "D" not in change:
        refused("btv_chunk_attn_paged_fp8kv", chunk_args(True, **change), text, code)


def test_chunk_attention_fp8_refuses():
    refused("btv_chunk_attn_paged_fp8kv", chunk_args(True, D=64), "D=64")
    for s in (0.0, -1.0, math.nan, math.inf):
        refused("btv_chunk_attn_paged_fp8kv", chunk_args(True, k_scale=C.c_float(s)), "scales")
        refused("btv_chunk_attn_paged_fp8kv", chunk_args(True, v_scale=C.c_float(s)), "scales")


def test_chunk_attention_workspace_queries():
    for bad in ((0, 10, 10, 32, 8, 128), (4, 0, 10, 32, 8, 128), (4, 10, -1, 32, 8, 128), (4, 10, 10, 30, 8, 128), (4, 10, 10, 32, 8, 96)):
        assert btv.btv_chunk_attn_paged_workspace(*bad) == 0 and btv.btv_chunk_attn_paged_fp8kv_workspace(*bad) == 0
    assert btv.btv_chunk_attn_paged_workspace(4, 10, 10, 32, 8, 64) >= 256
    assert btv.btv_chunk_attn_paged_fp8kv_workspace(4, 10, 10, 32, 8, 64) == 0
    # one for the largest sizes serves all smaller ones
    for Hq, Hkv, D in ((32, 8, 128), (28, 4, 128), (64, 8, 128), (16, 16, 64)):
        have = btv.btv_chunk_attn_paged_workspace(64, 3000, 20000, Hq, Hkv, D)
        assert all(btv.btv_chunk_attn_paged_workspace(b, m, l, Hq, Hkv, D) <= have
                   for b in (1, 2, 7, 33, 64) for m in (1, 5, 64, 65, 500, 3000) for l in (0, 100, 1000, 9999, 20000))


def test_wrong_tensors_are_refused_ahead_of_the_library():
    import torch
    i = torch.zeros(4, dtype=torch.int32)
    x = torch.zeros((4, 8, 128), dtype=torch.bfloat16)
    with pytest.raises(AssertionError):            # host tensors
        btv.btv_paged_extend(i, i, None, i, i, i, torch.zeros((4, 4), dtype=torch.int32), i, i, i, i, i)
    with pytest.raises(AssertionError):
        btv.btv_rope_append(x, x, x, i, i, torch.zeros(8, dtype=torch.float64), x, x, x)
    with pytest.raises(AssertionError):
        btv.btv_chunk_attn_paged(x, x.view(1, 4, 8, 128), x.view(1, 4, 8, 128), i.view(1, 4), i, i, 1, 1, x, None)


# ---- frequencies ---------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("R", [2, 16, 64, 128])
def test_frequencies_plain_linear_ntk(R):
    i = np.arange(R // 2)
    f, factor = btv.btv_rope_frequencies(R, 10000.0)
    assert np.allclose(f, 10000.0 ** (-2.0 * i / R), rtol=1e-14, atol=0) and factor == 1.0
    f, factor = btv.btv_rope_frequencies(R, 10000.0, btv.BTV_ROPE_LINEAR, 4.0)
    assert np.allclose(f, 10000.0 ** (-2.0 * i / R) / 4.0, rtol=1e-14, atol=0) and factor == 1.0
    if R > 2:   # the highest frequency stays, the lowest is divided by the stretch
        f, factor = btv.btv_rope_frequencies(R, 10000.0, btv.BTV_ROPE_NTK, 4.0)
        assert f[0] == 1.0 and math.isclose(f[-1], 10000.0 ** (-2.0 * (R // 2 - 1) / R) / 4.0, rel_tol=1e-12) and factor == 1.0


def test_frequencies_by_parts():
    R, theta, s, n, low, high = 128, 500000.0, 8.0, 8192.0, 1.0, 4.0
    plain, _ = btv.btv_rope_frequencies(R, theta)
    f, factor = btv.btv_rope_frequencies(R, theta, btv.BTV_ROPE_PARTS, s, n, low, high)
    seen = set()
    for w, x in zip(plain, f):
        turns = n * w / (2 * math.pi)
        if turns >= high:
            assert x == w
            seen.add("kept")
        elif turns <= low:
            assert math.isclose(x, w / s, rel_tol=1e-14)
            seen.add("divided")
        else:
            assert math.isclose(x, w / s + (w - w / s) * (turns - low) / (high - low), rel_tol=1e-12)
            seen.add("between")
    assert seen == {"kept", "divided", "between"} and factor == 1.0
    y, factor = btv.btv_rope_frequencies(R, theta, btv.BTV_ROPE_YARN, s, n, low, high)
    assert y == f and math.isclose(factor, 0.1 * math.log(s) + 1.0, rel_tol=1e-14)


@pytest.mark.parametrize("args", [(3, 1e4), (0, 1e4), (64, 0.0), (64, math.inf), (64, 1e4, 9), (64, 1e4, 1, 0.5), (64, 1e4, 2, math.nan), (2, 1e4, 2, 2.0),
                                  (64, 1e4, 3, 2.0, 0.0), (64, 1e4, 3, 2.0, 8192.0, 4.0, 4.0), (64, 1e4, 4, 2.0, 8192.0, -1.0, 4.0)])
def test_frequencies_refuse(args):
    with pytest.raises(btv.BtvError):
        btv.btv_rope_frequencies(*args)


# ---- the oracles' own pins ----------------------------------------------------------------------------------------------------

def test_oracle_extend_by_hand():
    import oracle
    table = np.full((3, 4), -1, np.int32)
    table[0, :2] = [7, 3]
    table[2, 0] = 5
    r = oracle.paged_extend([17, 0, 16], [15, 20, 1], [2, 0, 1], np.array([9, 8, 6, 4, 0, 0, 0, 0, 0, 0]), 4, table, 38)
    assert r["q_offset"].tolist() == [0, 15, 35, 36] and r["n_pages"].tolist() == [2, 2, 2] and r["n_free"] == 1 and not r["bad"]
    assert r["table"].tolist() == [[7, 3, -1, -1], [4, 6, -1, -1], [5, 8, -1, -1]]
    assert r["slot"][:3].tolist() == [49, 50, 51] and r["slot"][15] == 64 and r["slot"][31] == 96 and r["slot"][35:].tolist() == [128, -1, -1]
    assert r["position"][[0, 14, 15, 35, 36]].tolist() == [17, 31, 0, 16, 0]


def test_oracle_rope_keeps_lengths_and_relative_angles():
    import oracle
    rng = np.random.default_rng(0)
    w = [1.0, 0.1]
    q, k = rng.standard_normal((1, 1, 4)), rng.standard_normal((1, 1, 4))
    for inter in (False, True):
        dots = [float((oracle.rope(q, [n + 5], w, inter) * oracle.rope(k, [n], w, inter)).sum()) for n in (0, 3, 1000)]
        assert np.allclose(dots, dots[0], rtol=1e-10)
        assert np.isclose((oracle.rope(q, [77], w, inter) ** 2).sum(), (q ** 2).sum())
    y = oracle.rope(np.array([[[1.0, 0.0, 0.0, 0.0]]]), [1], [math.pi / 2, 0.0])
    assert np.allclose(y, [[[0, 0, 1, 0]]], atol=1e-15)
    assert np.allclose(oracle.rope(np.array([[[1.0, 0.0, 0.0, 0.0]]]), [1], [math.pi / 2, 0.0], True), [[[0, 1, 0, 0]]], atol=1e-15)
