"""Pages, slots and positions of new rows (btv_paged_extend) and rotary positions with the append (btv_rope_append, btv_rope_append_fp8kv) against the oracle."""
import numpy as np
import pytest

import oracle
from paper_2605_29727_amd import synth

pytestmark = pytest.mark.gpu
PAGE = 16


# ---- paged_extend ---------------------------------------------------------------------------------------------------------------

def extend_case(seed, Ls, Ms, spare=20, kept=True, width_more=0):
    """Inputs of a consistent cache: every request holds the pages of its prefix, some one more."""
    held = [-(-l // PAGE) + (r % 3 == 1 and kept) for r, l in enumerate(Ls)]
    need = [max(h, -(-(l + m) // PAGE)) for h, l, m in zip(held, Ls, Ms)]
    blocks = sum(need) + spare
    order = synth.permutation(seed, "pages", blocks).astype(np.int32)
    width = max(1, max(need)) + width_more
    table = np.full((len(Ls), width), -1, dtype=np.int32)
    at = 0
    for r, h in enumerate(held):
        table[r, :h] = order[at:at + h]
        at += h
    free = np.full(blocks, -9, dtype=np.int32)
    free[:blocks - at] = order[at:]
    return dict(prefix_len=np.array(Ls, np.int32), n_new=np.array(Ms, np.int32), n_pages=np.array(held, np.int32), free_pages=free, n_free=blocks - at, table=table)


def run_extend(c, total_max, depth=None, stream=None):
    import torch
    import gpu_util as G
    from paper_2605_29727_amd import binding as btv
    n = len(c["prefix_len"])
    d = {k: G.dev(c[k]) for k in ("prefix_len", "n_new", "n_pages", "free_pages", "table")}
    out = {k: torch.full((m,), -77, dtype=torch.int32, device="cuda") for k, m in (("q_offset", n + 1), ("slot", total_max), ("position", total_max), ("n_pages", n), ("n_free", 1))}
    ws = btv.alloc_workspace(256)
    btv.btv_paged_extend(d["prefix_len"], d["n_new"], None if depth is None else G.dev(depth), d["n_pages"], d["free_pages"], G.dev(np.array([c["n_free"]], np.int32)), d["table"],
                         out["q_offset"], out["slot"], out["position"], out["n_pages"], out["n_free"], ws)
    got = {k: v.cpu().numpy() for k, v in out.items()}
    got["table"] = d["table"].cpu().numpy()
    got["bad"] = btv.btv_workspace_status(ws) != 0
    assert np.array_equal(d["free_pages"].cpu().numpy(), c["free_pages"])
    return got


def same(got, ref):
    for k in ("q_offset", "slot", "position", "n_pages", "table"):
        assert np.array_equal(got[k], ref[k]), k
    assert int(got["n_free"][0]) == ref["n_free"] and got["bad"] == ref["bad"]


def check_extend(c, total_max=None, depth=None):
    total = int(np.maximum(c["n_new"], 0).sum()) if total_max is None else total_max
    ref = oracle.paged_extend(c["prefix_len"], c["n_new"], c["n_pages"], c["free_pages"], c["n_free"], c["table"], total, depth)
    same(run_extend(c, total, depth), ref)
    return ref


@pytest.mark.parametrize("batch", [1, 2, 63, 64, 65, 255, 256, 257, 1000, 4096])
def test_extend_batches(batch):
    Ls = synth.integers(batch, "L", (batch,), 0, 200 if batch > 300 else 3000).tolist()
    Ms = synth.integers(batch, "M", (batch,), 0, 9 if batch > 300 else 130).tolist()
    ref = check_extend(extend_case(batch, Ls, Ms, width_more=batch % 3))
    assert not ref["bad"]


@pytest.mark.parametrize("L,M,kept", [(0, 1, False), (0, 0, False), (15, 1, False), (16, 1, False), (16, 16, False), (17, 15, True), (31, 1, True), (0, 70000, False), (1000, 300000, True)])
def test_extend_page_borders_and_long_rows(L, M, kept):
    ref = check_extend(extend_case(3, [5, L, 7], [2, M, 1], kept=kept))
    assert not ref["bad"]


def test_extend_positions_of_a_tree_and_padded_rows():
    Ls, Ms = [40, 0, 333], [30, 64, 7]
    depth = synth.integers(1, "depth", (150,), 1, 16).astype(np.int32)
    ref = check_extend(extend_case(8, Ls, Ms), total_max=150, depth=depth)
    assert (ref["slot"][101:] == -1).all() and not ref["bad"]


@pytest.mark.parametrize("n_free", [0, 1, 3, 4, 5, 100])
def test_extend_with_too_few_pages(n_free):
    c = extend_case(5, [16, 3, 32, 8, 0], [20, 5, 10, 8, 33], spare=100, kept=False)       # takes 2, 0, 1, 0, 3
    c["n_free"] = min(n_free, c["n_free"])
    ref = check_extend(c)
    assert ref["bad"] == (n_free < 6)


def test_extend_with_data_out_of_range():
    base = lambda: extend_case(6, [20, 30, 40, 50], [3, 4, 5, 6])  # noqa: E731
    for key, r, v in (("prefix_len", 1, -1), ("n_new", 2, -5), ("n_pages", 0, 1), ("n_pages", 3, -2), ("n_pages", 3, 1000), ("n_new", 1, 4000), ("prefix_len", 2, 2**31 - 1),
                      ("n_new", 0, 2**31 - 1)):
        c = base()
        c[key][r] = v
        assert check_extend(c, total_max=40)["bad"], (key, r, v)
    c = base()
    c["free_pages"][c["n_free"] - 1] = 10**6
    c["n_new"][0] = 30
    assert check_extend(c)["bad"]
    c = base()
    c["table"][2, 2] = -3
    c["prefix_len"][2] = 33
    assert check_extend(c)["bad"]
    for n in (-1, 10**6):
        c = base()
        c["n_free"] = n
        assert check_extend(c)["bad"]
    assert check_extend(base(), total_max=10)["bad"]           # more rows than entries


# ---- rope_append ----------------------------------------------------------------------------------------------------------------

def half_step(bits):
    return 2.0 ** -bits


def run_rope(T, Hq, Hkv, D, R, dtype, cache, interleaved, packed, start, factor, slots, blocks, seed=1, in_place=False, inputs=None):
    """Returns (inputs in fp64, outputs): caches filled with a pattern first."""
    import torch
    import gpu_util as G
    from paper_2605_29727_amd import binding as btv
    dt = torch.float32 if dtype == "fp32" else torch.bfloat16
    if inputs is None:
        x = torch.from_numpy(synth.normal(seed, "qkv", (T, Hq + 2 * Hkv, D))).to(dt)
    else:
        x = inputs.to(dt)
    q, k, v = (y.contiguous() for y in (x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]))
    if packed:
        xd = x.cuda()
        Q, K, V = xd[:, :Hq], xd[:, Hq:Hq + Hkv], xd[:, Hq + Hkv:]
    else:
        Q, K, V = q.cuda(), k.cuda(), v.cuda()
    w = [10000.0 ** (-2.0 * i / R) for i in range(R // 2)]
    position = (start + np.arange(T)).astype(np.int32)
    Qout = Q if in_place else torch.full((T, Hq, D), 7.0, dtype=dt, device="cuda")
    if cache == "fp8":
        Kc, Vc = (torch.full((blocks, PAGE, Hkv, D), 0x5A, dtype=torch.uint8, device="cuda") for _ in range(2))
    else:
        Kc, Vc = (torch.full((blocks, PAGE, Hkv, D), 7.0, dtype=dt, device="cuda") for _ in range(2))
    ws = btv.alloc_workspace(256)
    args = (Q, K, V, G.dev(position), G.dev(np.asarray(slots, np.int32)), torch.tensor(w, dtype=torch.float64, device="cuda"), Qout, Kc, Vc)
    if cache == "fp8":
        btv.btv_rope_append_fp8kv(*args, 0.013, 0.021, interleaved=interleaved, factor=factor, ws=ws)
    else:
        btv.btv_rope_append(*args, interleaved=interleaved, factor=factor, ws=ws)
    torch.cuda.synchronize()
    back = lambda t: t.double().cpu().numpy()  # noqa: E731
    ref = [oracle.rope(back(q), position, w, interleaved, factor), oracle.rope(back(k), position, w, interleaved, factor), back(v)]
    mag = []                # |a| + |b| of every channel's pair, 0 where nothing turns
    for y in (q, k):
        a = np.abs(back(y))
        m = np.zeros_like(a)
        i, j = (slice(0, R, 2), slice(1, R, 2)) if interleaved else (slice(0, R // 2), slice(R // 2, R))
        m[..., i] = m[..., j] = (a[..., i] + a[..., j]) * abs(factor)
        mag.append(m)
    return ref, mag, Qout, Kc, Vc, btv.btv_workspace_status(ws)


def check_rope(dtype, cache, ref, mag, Qout, Kc, Vc, slots, num_slots):
    import torch
    # Sine and cosine: the fraction of a turn in fp32 is off by 2^-26 turns (2 pi times that in radians, under 1.6 steps of 2^-24), the functions by 2 steps, the factor's
    # product by one; then two products and a sum of one step each at most.  8 steps of 2^-24 cover them, of |a| + |b|.  Then one rounding to the type that is stored.
    step = half_step(24) if dtype == "fp32" else half_step(8)
    turn = lambda m: 8 * half_step(24) * m  # noqa: E731
    got = Qout.double().cpu().numpy()
    assert (np.abs(got - ref[0]) <= turn(mag[0]) + step * (np.abs(ref[0]) + turn(mag[0]))).all()
    written = np.zeros(num_slots, bool)
    for t, s in enumerate(slots):
        if 0 <= s < num_slots:
            written[s] = True
    for pool, r, m, scale in ((Kc, ref[1], mag[1], 0.013), (Vc, ref[2], np.zeros_like(ref[2]), 0.021)):
        if cache == "fp8":
            flat = pool.view(torch.float8_e4m3fn).double().cpu().numpy().reshape(num_slots, *r.shape[1:])
            raw = pool.cpu().numpy().reshape(num_slots, *r.shape[1:])
            assert (raw[~written] == 0x5A).all()
            for t, s in enumerate(slots):
                if 0 <= s < num_slots:
                    x = np.clip(r[t] / scale, -448, 448)
                    # half a step of the code (2^-4 relative, 2^-10 among the subnormals), and the fp32 value ahead of it: the rotation's, the scale's reciprocal and the product
                    slack = turn(m[t]) / scale + 3 * half_step(24) * np.abs(x)
                    assert (np.abs(flat[s] - x) <= np.maximum(half_step(4) * (np.abs(x) + slack), half_step(10)) + slack).all()
        else:
            flat = pool.double().cpu().numpy().reshape(num_slots, *r.shape[1:])
            assert (flat[~written] == 7.0).all()
            for t, s in enumerate(slots):
                if 0 <= s < num_slots:
                    assert (np.abs(flat[s] - r[t]) <= turn(m[t]) + np.where(m[t] > 0, step * (np.abs(r[t]) + turn(m[t])), 0)).all()


@pytest.mark.parametrize("dtype,cache", [("fp32", "fp32"), ("bf16", "bf16"), ("bf16", "fp8")])
@pytest.mark.parametrize("interleaved", [False, True], ids=["half", "interleaved"])
@pytest.mark.parametrize("T,Hq,Hkv,D,R", [(1, 8, 2, 128, 128), (5, 32, 8, 128, 64), (33, 28, 4, 128, 16), (17, 1, 1, 64, 64), (64, 7, 7, 64, 48), (3, 64, 8, 128, 112), (200, 16, 2, 64, 32),
                                          (9, 5, 1, 128, 96)])
def test_rope_append(dtype, cache, interleaved, T, Hq, Hkv, D, R):
    blocks = -(-T // PAGE) + 2
    slots = synth.permutation(T, "slots", blocks * PAGE)[:T]
    ref, mag, *out, status = run_rope(T, Hq, Hkv, D, R, dtype, cache, interleaved, T % 2 == 1, 4000, 1.0 if T % 3 else 1.2079, slots, blocks)
    check_rope(dtype, cache, ref, mag, *out, slots, blocks * PAGE)
    assert status == 0


@pytest.mark.parametrize("dtype,cache", [("fp32", "fp32"), ("bf16", "bf16"), ("bf16", "fp8")])
def test_rope_append_many_rows(dtype, cache):
    T, blocks = 3001, 190
    slots = synth.permutation(2, "slots", blocks * PAGE)[:T]
    ref, mag, *out, status = run_rope(T, 8, 2, 128, 128, dtype, cache, False, True, 100, 1.0, slots, blocks)
    check_rope(dtype, cache, ref, mag, *out, slots, blocks * PAGE)


@pytest.mark.parametrize("start", [0, 2**20 - 3, 2**31 - 8])
def test_rope_append_far_positions(start):
    slots = np.arange(7)
    ref, mag, *out, _ = run_rope(7, 4, 2, 128, 128, "fp32", "fp32", False, False, start, 1.0, slots, 1)
    # fp64: the frequency times 1 / 2 pi and the position, each off by 2^-53 of what may be 2^31 / 6.3 turns: 2^-23 turns, 13 steps of 2^-24 radians more
    mag = [m * (1 if start < 2**21 else 3) for m in mag]
    check_rope("fp32", "fp32", ref, mag, *out, slots, PAGE)


def test_rope_append_passes_rows_over():
    slots = [3, -1, 5, -7, 100, 0]
    ref, mag, *out, status = run_rope(6, 4, 2, 128, 128, "bf16", "bf16", False, False, 9, 1.0, slots, 1)
    check_rope("bf16", "bf16", ref, mag, *out, slots, PAGE)
    assert status != 0                                 # slot 100 of 16
    ref, mag, *out, status = run_rope(6, 4, 2, 128, 128, "bf16", "fp8", True, False, 9, 1.0, [3, -1, 5, -7, 2, 0], 1)
    check_rope("bf16", "fp8", ref, mag, *out, [3, -1, 5, -7, 2, 0], PAGE)
    assert status == 0


def test_rope_append_in_place():
    slots = np.arange(20)
    for dtype in ("fp32", "bf16"):
        ref, mag, *out, _ = run_rope(20, 8, 2, 64, 32, dtype, dtype, False, False, 9, 1.0, slots, 2, in_place=True)
        check_rope(dtype, dtype, ref, mag, *out, slots, 2 * PAGE)


def test_rope_append_without_rotation_and_without_rows():
    import torch
    from paper_2605_29727_amd import binding as btv
    i = torch.arange(4, dtype=torch.int32, device="cuda")
    none = torch.empty(0, dtype=torch.float64, device="cuda")
    x = torch.randn((4, 3, 64), device="cuda")
    Kc, Vc, Qo = torch.zeros((4, 3, 64), device="cuda"), torch.zeros((4, 3, 64), device="cuda"), torch.zeros_like(x)
    btv.btv_rope_append(x, x + 1, x + 2, i, i, none, Qo, Kc, Vc)
    assert torch.equal(Qo, x) and torch.equal(Kc, x + 1) and torch.equal(Vc, x + 2)
    e = x[:0]
    btv.btv_rope_append(e, e, e, i[:0], i[:0], none, Qo[:0], Kc, Vc)


def test_rope_append_special_values():
    """E4M3: beyond the largest number, infinities and NaN; their neighbours are not touched."""
    import torch
    x = torch.zeros((2, 3, 64))
    x[:, :, :] = 1.0
    x[0, 1, 40], x[0, 1, 41], x[0, 1, 42], x[0, 2, 5], x[0, 2, 6], x[0, 2, 7] = 1e4, -1e4, float("nan"), float("inf"), float("-inf"), float("nan")
    _, _, Qo, Kc, Vc, _ = run_rope(2, 1, 1, 64, 16, "bf16", "fp8", False, False, 0, 1.0, [0, 1], 1, inputs=x)
    K, V = Kc.cpu().numpy().reshape(PAGE, 64), Vc.cpu().numpy().reshape(PAGE, 64)
    assert K[0, 40] == 0x7E and K[0, 41] == 0xFE and K[0, 42] & 0x7F == 0x7F and K[0, 39] == K[0, 43] == K[1, 40]
    assert V[0, 5] == 0x7E and V[0, 6] == 0xFE and V[0, 7] & 0x7F == 0x7F and V[0, 4] == V[0, 8] == V[1, 5]


def test_rope_append_cache_beyond_4_gib():
    """Slots whose rows lie more than 2^32 bytes into the pool."""
    import torch
    from paper_2605_29727_amd import binding as btv
    Hkv, D, blocks = 8, 128, 133000                      # 4.36 GB a pool
    n = blocks * PAGE
    Kc = torch.empty((blocks, PAGE, Hkv, D), dtype=torch.bfloat16, device="cuda")
    Vc = torch.empty_like(Kc)
    low = (n - 3) * Hkv * D * 2 - 2**32                  # where the last slots' rows would fall, taken modulo 2^32 bytes
    Kc.view(torch.uint8).view(-1)[low:low + 3 * Hkv * D * 2] = 0
    x = torch.randn((3, Hkv, D), device="cuda").to(torch.bfloat16)
    slot = torch.tensor([n - 3, n - 1, n - 2], dtype=torch.int32, device="cuda")
    pos = torch.zeros(3, dtype=torch.int32, device="cuda")
    btv.btv_rope_append(x, x, x, pos, slot, torch.ones(8, dtype=torch.float64, device="cuda"), torch.empty_like(x), Kc, Vc)
    for c in (Kc, Vc):
        assert torch.equal(c.view(n, Hkv, D)[slot.long()], x)
    assert int(Kc.view(torch.uint8).view(-1)[low:low + 3 * Hkv * D * 2].count_nonzero()) == 0


def test_on_another_stream_and_in_a_graph():
    """Both calls recorded on a side stream: replays with other lengths give what eager calls give."""
    import torch
    import gpu_util as G
    from paper_2605_29727_amd import binding as btv
    T, Hq, Hkv, D = 60, 8, 2, 128
    rounds = [extend_case(20 + i, Ls, Ms, width_more=30 - max(1, max(-(-(l + m) // PAGE) + 1 for l, m in zip(Ls, Ms))) + 5) for i, (Ls, Ms) in
              enumerate([([0, 100, 37], [20, 1, 30]), ([16, 15, 300], [0, 17, 43]), ([5, 5, 5], [1, 1, 1])])]
    width, blocks = 40, 200
    dev = dict(device="cuda", dtype=torch.int32)
    st = {"prefix_len": torch.zeros(3, **dev), "n_new": torch.zeros(3, **dev), "n_pages": torch.zeros(3, **dev), "free_pages": torch.zeros(blocks, **dev),
          "n_free": torch.zeros(1, **dev), "table": torch.zeros((3, width), **dev)}
    out = {k: torch.zeros(n, **dev) for k, n in (("q_offset", 4), ("slot", T), ("position", T), ("n_pages", 3), ("n_free", 1))}
    x = torch.zeros((T, Hq + 2 * Hkv, D), dtype=torch.bfloat16, device="cuda")
    Qo = torch.zeros((T, Hq, D), dtype=torch.bfloat16, device="cuda")
    Kc, Vc = (torch.zeros((blocks, PAGE, Hkv, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    w = torch.tensor(btv.btv_rope_frequencies(128, 10000.0)[0], dtype=torch.float64, device="cuda")

    def step():
        btv.btv_paged_extend(st["prefix_len"], st["n_new"], None, st["n_pages"], st["free_pages"], st["n_free"], st["table"], out["q_offset"], out["slot"], out["position"],
                             out["n_pages"], out["n_free"])
        btv.btv_rope_append(x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], out["position"], out["slot"], w, Qo, Kc, Vc)

    def load(i):
        c = rounds[i]
        for k in ("prefix_len", "n_new", "n_pages"):
            st[k].copy_(G.dev(c[k]))
        st["free_pages"].fill_(-1)
        st["free_pages"][:len(c["free_pages"])] = G.dev(c["free_pages"])
        st["n_free"].fill_(c["n_free"])
        st["table"].fill_(-1)
        st["table"][:, :c["table"].shape[1]] = G.dev(c["table"])[:, :width]
        x.copy_(torch.from_numpy(synth.normal(i, "graph", tuple(x.shape))))
        Kc.zero_(); Vc.zero_()

    def shown():
        torch.cuda.synchronize()
        return [t.clone() for t in (*out.values(), st["table"], Qo, Kc, Vc)]

    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    load(0)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step()
        with torch.cuda.graph(graph, stream=side):
            step()
    torch.cuda.synchronize()
    for i in (0, 1, 2, 1, 0):
        load(i)
        graph.replay()
        got = shown()
        load(i)
        step()
        assert all(torch.equal(a, b) for a, b in zip(got, shown())), i


@pytest.mark.parametrize("batch", [2, 5, 300])
@pytest.mark.parametrize("new", [2**31 - 1, 2**30 + 7])
def test_extend_pages_of_requests_behind_a_length_out_of_range(batch, new):
    """The rows of a request out of range count, so that later requests' rows begin past 2^31 - 1; they get their pages all the same."""
    Ls = synth.integers(batch, "L", (batch,), 0, 300).tolist()
    Ms = synth.integers(batch, "M", (batch,), 17, 130).tolist()
    for far in ([0], [0, batch // 2], [batch - 1]):
        c = extend_case(batch, Ls, Ms)
        c["n_new"][far] = new
        ref = check_extend(c, total_max=60)
        taken = (ref["table"] != c["table"]).any(1)
        assert ref["bad"] and not taken[far].any() and taken[[r for r in range(batch) if ref["n_pages"][r] > c["n_pages"][r]]].all()


@pytest.mark.parametrize("Hkv,D", [(0, 128), (1, 0), (0, 0), (2, 0)])
@pytest.mark.parametrize("T", [3, 0])
def test_rope_append_refuses_caches_without_heads_or_channels(T, Hkv, D):
    import torch
    from paper_2605_29727_amd import binding as btv
    i = torch.zeros(T, dtype=torch.int32, device="cuda")
    f = torch.ones(8, dtype=torch.float64, device="cuda")
    for dt, append, more in ((torch.bfloat16, btv.btv_rope_append, ()), (torch.uint8, btv.btv_rope_append_fp8kv, (1.0, 1.0))):
        q, kv = torch.zeros((T, 1, D), dtype=torch.bfloat16, device="cuda"), torch.zeros((T, Hkv, D), dtype=torch.bfloat16, device="cuda")
        cache = torch.zeros((2, PAGE, Hkv, D), dtype=dt, device="cuda")
        with pytest.raises((btv.BtvError, AssertionError)):       # (the library's refusal, or that such heads do not lie side by side)
            append(q, kv, kv, i, i, f, torch.zeros_like(q), cache, cache.clone(), *more)


@pytest.mark.parametrize("scale", [7 / 512, 15 / 1024, 13 / 1024, 1.0, 0.013, 3e-5, 1234.567, 1e-37, 1e37])
def test_rope_append_fp8_rounds_the_quotient(scale):
    """Every bf16 number, without rotation: the code nearest to x / scale, ties to even; a product with 1 / scale takes a neighbour of some ties."""
    import torch
    from paper_2605_29727_amd import binding as btv
    x = torch.arange(2**16, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).view(-1, 4, 64)
    n = x.shape[0]
    f = torch.tensor(scale, dtype=torch.float32)
    want = (x.float() / f).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    i = torch.arange(n, dtype=torch.int32, device="cuda")
    X = x.cuda()
    Kc, Vc = (torch.zeros((n, 4, 64), dtype=torch.uint8, device="cuda") for _ in range(2))
    btv.btv_rope_append_fp8kv(X, X, X, i, i, torch.empty(0, dtype=torch.float64, device="cuda"), torch.empty_like(X), Kc, Vc, scale, scale)
    number = ~torch.isnan(x)
    for c in (Kc.cpu(), Vc.cpu()):
        assert torch.equal(c[number], want[number]) and bool((c[~number] & 0x7F == 0x7F).all())
