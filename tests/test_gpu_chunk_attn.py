"""Causal attention of chunks over a paged cache (btv_chunk_attn_paged, btv_chunk_attn_paged_fp8kv) against the definition in 64 bits."""
import math

import numpy as np
import pytest

from paper_2605_29727_amd import synth

pytestmark = pytest.mark.gpu
PAGE = 16
KS, VS = 0.0121, 0.0093


def make(seed, Ls, Ms, Hq, Hkv, D, kv, grow=0.0, sharp=1.0, pad=0):
    """A batch on the device: pages in a random order, the unused entries of the table out of range, everything that no request owns NaN.  grow: keys get longer along the
    sequence, so that the running maximum has to follow."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    S = [l + m for l, m in zip(Ls, Ms)]
    table, blocks = synth.paged_layout(seed, S)
    table = np.where(table < 0, np.where(np.arange(table.shape[1]) % 2, -5, 10**9), table).astype(np.int32)
    offsets = np.concatenate([[0], np.cumsum(Ms)]).astype(np.int32)
    total = int(offsets[-1])
    Q = torch.randn((total + pad, Hq, D), generator=g, device="cuda").mul_(sharp).to(torch.bfloat16)
    if kv == "fp8":
        K, V = (torch.full((blocks, PAGE, Hkv, D), 0x7F, dtype=torch.uint8, device="cuda") for _ in range(2))
    else:
        K, V = (torch.full((blocks, PAGE, Hkv, D), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    rows = []
    for r, s in enumerate(S):
        k, v = (torch.randn((s, Hkv, D), generator=g, device="cuda") for _ in range(2))
        k *= 1 + grow * torch.arange(s, device="cuda")[:, None, None] / max(s, 1)
        if kv == "fp8":
            k, v = ((x.clamp(-5, 5) / f).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8) for x, f in ((k, KS), (v, VS)))
        else:
            k, v = k.to(torch.bfloat16), v.to(torch.bfloat16)
        at = torch.arange(s, device="cuda")
        page = torch.from_numpy(table[r]).cuda().long()[at // PAGE]
        K[page, at % PAGE], V[page, at % PAGE] = k, v
        rows.append((k, v))
    return dict(Q=Q, K=K, V=V, table=torch.from_numpy(table).cuda(), q_offset=torch.from_numpy(offsets).cuda(), prefix=torch.tensor(Ls, dtype=torch.int32, device="cuda"), rows=rows,
                Ls=Ls, Ms=Ms, off=offsets, kv=kv, M_max=max(max(Ms), 1), L_max=max(Ls), heads=(Hq, Hkv, D))


def workspace(b, M_max=None, L_max=None):
    from paper_2605_29727_amd import binding as btv
    size = btv.btv_chunk_attn_paged_fp8kv_workspace if b["kv"] == "fp8" else btv.btv_chunk_attn_paged_workspace
    return btv.alloc_workspace(size(len(b["Ls"]), M_max or b["M_max"], b["L_max"] if L_max is None else L_max, *b["heads"]))


def call(b, O, ws, scale=0.0, M_max=None, L_max=None):
    from paper_2605_29727_amd import binding as btv
    M_max, L_max = M_max or b["M_max"], b["L_max"] if L_max is None else L_max
    if b["kv"] == "fp8":
        btv.btv_chunk_attn_paged_fp8kv(b["Q"], b["K"], b["V"], KS, VS, b["table"], b["q_offset"], b["prefix"], M_max, L_max, O, ws, scale)
    else:
        btv.btv_chunk_attn_paged(b["Q"], b["K"], b["V"], b["table"], b["q_offset"], b["prefix"], M_max, L_max, O, ws, scale)


def run(b, scale=0.0, M_max=None, L_max=None):
    import torch
    from paper_2605_29727_amd import binding as btv
    O = torch.full_like(b["Q"], 123.0)
    ws = workspace(b, M_max, L_max)
    call(b, O, ws, scale, M_max, L_max)
    torch.cuda.synchronize()
    assert btv.btv_workspace_status(ws) == 0
    return O


def check(b, O, scale=0.0, only=None):
    """Every output element against the definition, request by request and head by head, to what its roundings allow."""
    import torch
    Hq, Hkv, D = b["heads"]
    scale = scale if scale > 0 else D ** -0.5
    G = Hq // Hkv
    worst = 0.0
    for r, (l, m) in enumerate(zip(b["Ls"], b["Ms"])):
        if m == 0 or (only is not None and r not in only):
            continue
        k, v = b["rows"][r]
        if b["kv"] == "fp8":
            k, v = k.view(torch.float8_e4m3fn).double() * KS, v.view(torch.float8_e4m3fn).double() * VS
        k, v = k.double(), v.double()
        o0 = int(b["off"][r])
        hidden = torch.arange(l + m, device="cuda") > l + torch.arange(m, device="cuda")[:, None]
        for h in range(Hq):
            q, kh, vh = b["Q"][o0:o0 + m, h].double(), k[:, h // G], v[:, h // G]
            w = torch.softmax((q @ kh.T * scale).masked_fill(hidden, -math.inf), -1)
            ref, mass = w @ vh, w @ vh.abs()
            # A probability is rounded to bf16 (half a step: 2^-8) in the numerator and in the row's sum alike: 2 * 2^-8 of sum w |v| at most.  Scores: D products summed in
            # fp32, half a step each of the largest sum of magnitudes, and the exponent's own roundings (fp32 at up to that score times 1.45: 4 steps more), in numerator and sum.
            # A part of a row travels in fp16 beside its magnitude: half a step 2^-11 relative to numbers up to the row's largest, of which a row's parts add up to
            # twice at most.  The result's own rounding: 2^-8.
            mags = float((q.abs().amax(0) @ kh.abs().amax(0)) * scale)
            scores = 2 * (D + 4) * 2.0 ** -24 * mags * mass
            tol = 2.0 ** -7 * mass + scores + 2.0 ** -10 * mass.amax(-1, keepdim=True) + 2.0 ** -8 * ref.abs()
            off = (O[o0:o0 + m, h].double() - ref).abs()
            assert bool((off <= tol).all()), (r, h, float((off / tol.clamp(min=1e-30)).max()), int((off > tol).sum()))
            worst = max(worst, float((off / tol.clamp(min=1e-30)).max()))
    return worst


SHAPES = [("bf16", 32, 8, 128), ("bf16", 8, 2, 64), ("fp8", 8, 2, 128)]
SHAPE_IDS = ["bf16_d128", "bf16_d64", "fp8"]


@pytest.mark.parametrize("kv,Hq,Hkv,D", SHAPES, ids=SHAPE_IDS)
@pytest.mark.parametrize("Ls,Ms", [([0], [1]), ([37], [1]), ([15], [1]), ([16], [1]), ([31], [1]), ([32], [2]), ([0], [16]), ([0], [33]), ([63], [65]), ([5], [200]), ([1000], [64]),
                                   ([96], [97]), ([100], [1]), ([159], [1]), ([190], [4]), ([223], [1]), ([255], [1]), ([256], [1]), ([290], [3]), ([0], [256]), ([0], [257]), ([60], [229]),
                                   ([3000], [1]), ([20000], [1]), ([9000], [17]), ([700], [100]), ([1500], [150]), ([2500], [300]), ([0], [1030]), ([129], [511])],
                         ids=lambda x: "-".join(map(str, x)))
def test_one_request(kv, Hq, Hkv, D, Ls, Ms):
    b = make(sum(Ls) + sum(Ms), Ls, Ms, Hq, Hkv, D, kv)
    check(b, run(b))


@pytest.mark.parametrize("kv,Hq,Hkv,D", [("bf16", 32, 8, 128), ("bf16", 32, 8, 64), ("fp8", 32, 8, 128), ("bf16", 28, 4, 128)], ids=["bf16_d128", "bf16_d64", "fp8", "bf16_7_heads"])
@pytest.mark.parametrize("Ls,Ms", [([8192], [300]), ([0], [2048]), ([4099], [2047]), ([100, 6000, 0, 2222], [900, 1, 1500, 63]), ([30000] * 3, [1] * 3), ([12000], [60])],
                         ids=lambda x: "-".join(map(str, x)))
def test_work_for_all_workgroups(kv, Hq, Hkv, D, Ls, Ms):
    b = make(sum(Ls) + 7 * sum(Ms), Ls, Ms, Hq, Hkv, D, kv)
    check(b, run(b))


# More row blocks than workgroups, by little and by up to eight times, of lengths that whole blocks share out evenly and of others; head counts that do and do not divide the chip.
@pytest.mark.parametrize("kv,Hq,Hkv,D", [("bf16", 16, 8, 128), ("bf16", 32, 8, 64), ("fp8", 8, 8, 128), ("bf16", 24, 6, 128), ("bf16", 12, 12, 64), ("fp8", 7, 7, 128)])
@pytest.mark.parametrize("Ls,Ms", [([0], [4300]), ([3000], [4096]), ([0, 0, 0, 0], [1600, 2000, 1, 1111]), ([5, 900, 0, 0, 77, 3, 40, 2000], [1800, 0, 700, 129, 1000, 65, 1500, 333]),
                                   ([20000, 0], [700, 3500]),
                                   ([0, 9, 64] * 20, [400, 33, 170] * 20), ([0] * 30, [128, 1, 97] * 10), ([0] * 70, [5 * i + 3 for i in range(70)])], ids=lambda x: "-".join(map(str, x[:8])))
def test_more_blocks_than_workgroups(kv, Hq, Hkv, D, Ls, Ms):
    b = make(3 * sum(Ls) + sum(Ms), Ls, Ms, Hq, Hkv, D, kv)
    check(b, run(b))


@pytest.mark.parametrize("kv,Hq,Hkv,D", SHAPES, ids=SHAPE_IDS)
@pytest.mark.parametrize("Ls,Ms", [([10, 0, 700, 33], [1, 1, 1, 1]), ([0, 100, 50], [40, 0, 7]), ([0, 4000, 17, 900], [500, 1, 64, 130]), ([0, 0, 0], [300, 1, 77]),
                                   ([7, 12000, 3], [0, 3, 0]), ([40, 6000, 1, 300, 2000], [33, 1, 257, 16, 65])], ids=lambda x: "-".join(map(str, x)))
def test_ragged_batches(kv, Hq, Hkv, D, Ls, Ms):
    b = make(sum(Ls) + len(Ms), Ls, Ms, Hq, Hkv, D, kv)
    check(b, run(b))


@pytest.mark.parametrize("kv,Hq,Hkv,D", [("bf16", 28, 4, 128), ("bf16", 3, 3, 64), ("bf16", 16, 1, 128), ("bf16", 5, 1, 64), ("fp8", 7, 1, 128), ("fp8", 12, 12, 128), ("bf16", 12, 4, 128)])
def test_head_groups(kv, Hq, Hkv, D):
    b = make(Hq, [100, 0, 1500], [70, 310, 1], Hq, Hkv, D, kv)
    check(b, run(b))


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
@pytest.mark.parametrize("n,lo,hi", [(70, 1, 1), (130, 0, 9), (300, 1, 3)])
def test_many_requests(kv, n, lo, hi):
    Ls = synth.integers(n, "L", (n,), 0, 400).tolist()
    Ms = synth.integers(n, "M", (n,), lo, hi).tolist()
    b = make(n, Ls, Ms, 8, 2, 128, kv)
    check(b, run(b))


@pytest.mark.parametrize("kv,Hq,Hkv,D", SHAPES, ids=SHAPE_IDS)
def test_maxima_that_grow_and_sharp_rows(kv, Hq, Hkv, D):
    b = make(3, [700, 0], [200, 600], Hq, Hkv, D, kv, grow=6.0, sharp=4.0)
    check(b, run(b))
    b = make(4, [2100], [1], Hq, Hkv, D, kv, grow=3.0, sharp=20.0)
    check(b, run(b))


@pytest.mark.parametrize("kv,Hq,Hkv,D", SHAPES, ids=SHAPE_IDS)
def test_other_scales_and_bounds_above_the_lengths(kv, Hq, Hkv, D):
    b = make(5, [300, 20], [40, 130], Hq, Hkv, D, kv)
    check(b, run(b, scale=0.3), scale=0.3)
    check(b, run(b, scale=0.001, M_max=1000, L_max=320), scale=0.001)


# Bounds far above the lengths, as a captured call has them, ask for the most rows per workgroup whatever the requests are.
@pytest.mark.parametrize("kv,Hq,Hkv,D", SHAPES, ids=SHAPE_IDS)
@pytest.mark.parametrize("Ls,Ms", [([0], [1]), ([37], [1]), ([15], [2]), ([31], [40]), ([0], [64]), ([63], [65]), ([5], [200]), ([96], [97]), ([159], [1]), ([255], [9]), ([290], [3]),
                                   ([0], [257]), ([60], [229]), ([3000], [1]), ([9000], [17]), ([2500], [300]), ([10, 0, 700, 33], [1, 1, 1, 1]), ([0, 4000, 17, 900], [500, 1, 64, 130]),
                                   ([7, 12000, 3], [0, 3, 0]), ([40, 6000, 1, 300, 2000], [33, 1, 257, 16, 65])], ids=lambda x: "-".join(map(str, x)))
def test_bounds_for_the_most_rows(kv, Hq, Hkv, D, Ls, Ms):
    import torch
    b = make(sum(Ls) + 5 * sum(Ms), Ls, Ms, Hq, Hkv, D, kv)
    b["table"] = torch.nn.functional.pad(b["table"], (0, 1_000_016 // PAGE - b["table"].shape[1]), value=-5)
    check(b, run(b, M_max=2000, L_max=1_000_000))


@pytest.mark.parametrize("Ms", [[3, 40], [200, 300]], ids=["few", "many"])
def test_rows_that_nobody_owns_stay(Ms):
    b = make(6, [100, 0], Ms, 8, 2, 128, "bf16", pad=9)
    O = run(b)
    check(b, O)
    assert bool((O[sum(Ms):] == 123.0).all())


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
@pytest.mark.parametrize("L,M,at", [(40, 30, 45), (0, 300, 299), (0, 300, 5), (500, 1, 500), (3, 700, 650), (640, 257, 800)])
def test_nan_in_hidden_places(kv, L, M, at):
    """A value (or a key) that is not a number reaches the rows that see it, and no other."""
    import torch
    for what in ("K", "V"):
        b = make(7, [L, 64], [M, 20], 8, 2, 128, kv)
        page = int(b["table"][0, at // PAGE])
        bad = [0x7F] if kv == "fp8" else [float("nan"), float("inf"), float("-inf")] if what == "V" else [float("nan")]
        for x in bad:
            c = {k: v.clone() if k in ("K", "V") else v for k, v in b.items()}
            c[what][page, at % PAGE, 1, 77] = x
            O = run(c)
            clean = run(b)
            sees = torch.zeros(M + 20, dtype=torch.bool, device="cuda")
            sees[max(at - L, 0):M] = True
            assert torch.equal(O[~sees], clean[~sees]) and torch.equal(O[sees][:, :4], clean[sees][:, :4])
            hit, was = O[sees][:, 4:].double(), clean[sees][:, 4:].double()
            if what == "V":
                # The other channels of a row in several parts may move: a part travels in fp16 beside its largest magnitude, which that channel no longer takes part in, so
                # both results are off by a half step 2^-11 of the row's parts (of up to twice its largest number), and then by a half step 2^-8 of their own.
                other = torch.arange(128, device="cuda") != 77
                limit = 2 * (2.0 ** -10 * was.abs().amax(-1, keepdim=True) * 2 + 2.0 ** -8 * was.abs())
                assert bool((~torch.isfinite(hit[..., 77])).all()) and bool(((hit - was).abs() <= limit)[..., other].all())
            else:
                assert bool(torch.isnan(hit).all())


def test_requests_out_of_range_are_passed_over():
    import torch
    from paper_2605_29727_amd import binding as btv
    for change in ({"prefix": (1, -4)}, {"prefix": (1, 10**6)}, {"q_offset": (3, 10**6)}, {"bounds": (16, 700)}):
        b = make(8, [100, 600, 30], [20, 16, 17], 8, 2, 128, "bf16")
        M_max = L_max = None
        skipped = {1}
        if "bounds" in change:
            M_max, L_max = 16, 600
            skipped = {0, 2}
        else:
            (name, (i, v)), = change.items()
            b[name] = b[name].clone()
            b[name][i] = v
            skipped = {2} if name == "q_offset" else {1}
        O = torch.full_like(b["Q"], 123.0)
        ws = workspace(b)
        call(b, O, ws, M_max=M_max, L_max=L_max)
        torch.cuda.synchronize()
        assert btv.btv_workspace_status(ws) == btv.BTV_EDATA
        check(b, O, only={0, 1, 2} - skipped)
        for r in skipped:
            assert bool((O[b["off"][r]:b["off"][r + 1]] == 123.0).all())
        # the workspace serves the next call all the same
        b = make(9, [900], [33], 8, 2, 128, "bf16")
        O = torch.full_like(b["Q"], 123.0)
        need = workspace(b)
        call(b, O, ws if ws.numel() >= need.numel() else need)
        torch.cuda.synchronize()
        check(b, O)


def test_one_workspace_for_calls_of_all_sizes():
    import torch
    ws = None
    for i, (Ls, Ms) in enumerate([([3000, 900], [700, 300]), ([2900], [1]), ([10, 20], [1, 2]), ([2999, 0], [1, 690])]):
        b = make(30 + i, Ls, Ms, 8, 2, 128, "bf16")
        ws = workspace(b) if ws is None else ws
        O = torch.full_like(b["Q"], 123.0)
        call(b, O, ws)
        torch.cuda.synchronize()
        check(b, O)


def test_pool_beyond_4_gib():
    import torch
    Hq, Hkv, D, blocks = 16, 8, 128, 133000
    for L, M in ((90, 3), (200, 130)):
        b = make(10, [L], [M], Hq, Hkv, D, "bf16")
        K = torch.empty((blocks, PAGE, Hkv, D), dtype=torch.bfloat16, device="cuda")
        V = torch.empty_like(K)
        n = -(-(L + M) // PAGE)
        old = b["table"][0, :n].long()
        new = blocks - 1 - torch.arange(n, device="cuda")
        K[new], V[new] = b["K"][old], b["V"][old]
        b["K"], b["V"], b["table"] = K, V, new.to(torch.int32).view(1, n)
        check(b, run(b))


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
@pytest.mark.parametrize("sizes", ["tokens", "chunks"])
def test_graph_replays_with_other_lengths(kv, sizes):
    """Recorded once on a side stream with bounds above the lengths; every replay, and every run of it, gives the eager bits."""
    import torch
    rounds = [([100, 4000, 0], [1, 1, 1]), ([9, 17, 3000], [1, 0, 1]), ([4099, 1, 300], [1, 1, 1])] if sizes == "tokens" else \
             [([100, 4000, 0], [300, 1, 77]), ([9, 17, 3000], [1, 350, 0]), ([4000, 1, 300], [90, 200, 16])]
    batches = [make(40 + i, Ls, Ms, 8, 2, 128, kv) for i, (Ls, Ms) in enumerate(rounds)]
    M_max, L_max = max(b["M_max"] for b in batches), 4200
    blocks, width, rows = max(b["K"].shape[0] for b in batches), -(-(L_max + M_max) // PAGE), max(b["Q"].shape[0] for b in batches)
    s = dict(batches[0], Q=torch.zeros((rows, 8, 128), dtype=torch.bfloat16, device="cuda"), K=torch.zeros((blocks, *batches[0]["K"].shape[1:]), dtype=batches[0]["K"].dtype, device="cuda"),
             table=torch.zeros((3, width), dtype=torch.int32, device="cuda"), q_offset=batches[0]["q_offset"].clone(), prefix=batches[0]["prefix"].clone())
    s["V"] = torch.zeros_like(s["K"])
    O = torch.zeros_like(s["Q"])
    ws = workspace(s, M_max, L_max)

    def load(b):
        s["Q"][:b["Q"].shape[0]] = b["Q"]
        s["K"][:b["K"].shape[0]], s["V"][:b["V"].shape[0]] = b["K"], b["V"]
        s["table"][:, :b["table"].shape[1]] = b["table"]
        s["q_offset"].copy_(b["q_offset"]); s["prefix"].copy_(b["prefix"])
        O.fill_(123.0)

    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    load(batches[0])
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        call(s, O, ws, M_max=M_max, L_max=L_max)
        with torch.cuda.graph(graph, stream=side):
            call(s, O, ws, M_max=M_max, L_max=L_max)
    torch.cuda.synchronize()
    for i in (0, 1, 2, 1, 0):
        load(batches[i])
        graph.replay()
        torch.cuda.synchronize()
        got = O.clone()
        check(batches[i], got)
        load(batches[i])
        call(s, O, ws, M_max=M_max, L_max=L_max)
        torch.cuda.synchronize()
        assert torch.equal(O, got)


def test_two_streams_with_workspaces_of_their_own():
    import torch
    bs = [make(50, [3000, 100], [400, 90], 8, 2, 128, "bf16"), make(51, [2000, 900], [1, 700], 8, 2, 128, "fp8")]
    alone = [run(b) for b in bs]
    streams, wss, Os = [torch.cuda.Stream() for _ in bs], [workspace(b) for b in bs], [torch.full_like(b["Q"], 123.0) for b in bs]
    torch.cuda.synchronize()
    for _ in range(5):
        for b, st, ws, O in zip(bs, streams, wss, Os):
            with torch.cuda.stream(st):
                call(b, O, ws)
    torch.cuda.synchronize()
    assert all(torch.equal(O, a) for O, a in zip(Os, alone))


def test_two_graphs_take_turns_with_one_workspace():
    """Calls of other shapes on one workspace, recorded apart and replayed in turn: single tokens in parts, shares with cuts, whole blocks, small row blocks."""
    import torch
    bs = [make(70, [5000, 30], [1, 1], 8, 2, 128, "bf16"), make(71, [3000, 0, 50], [900, 1500, 70], 8, 2, 128, "bf16"), make(72, [0] * 9, [700, 65, 300] * 3, 8, 2, 128, "bf16"),
          make(73, [2500], [100], 8, 2, 128, "bf16")]
    ws = max((workspace(b) for b in bs), key=lambda w: w.numel())
    Os, graphs, side = [torch.full_like(b["Q"], 123.0) for b in bs], [torch.cuda.CUDAGraph() for _ in bs], torch.cuda.Stream()
    alone = [run(b) for b in bs]
    with torch.cuda.stream(side):
        for b, O, g in zip(bs, Os, graphs):
            with torch.cuda.graph(g, stream=side):
                call(b, O, ws)
    torch.cuda.synchronize()
    for turn in ([0, 1, 2, 3], [3, 1, 0, 2], [1, 1, 3, 0], [2, 0, 2, 1]):
        for i in turn:
            Os[i].fill_(123.0)
            graphs[i].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(Os[i], alone[i]) for i in turn)


def test_the_most_requests_and_heads():
    rng = np.random.default_rng(74)
    b = make(74, rng.integers(0, 70, 4096).tolist(), rng.integers(0, 3, 4096).tolist(), 2, 1, 64, "bf16")
    check(b, run(b), only=set(rng.choice(4096, 200, replace=False).tolist()) | {0, 4095})
    b = make(75, [50, 300, 0], [3, 1, 40], 1024, 1024, 64, "bf16")
    check(b, run(b))
    b = make(76, [50, 300, 0], [3, 1, 40], 1024, 64, 128, "fp8")
    check(b, run(b))


def test_no_rows_at_all():
    import torch
    b = make(60, [40, 8], [0, 0], 8, 2, 128, "bf16")
    run(b)
    b = make(60, [40, 8], [0, 0], 8, 2, 128, "bf16", pad=3)
    assert bool((run(b) == 123.0).all())


# ---- the operators together -----------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("fp8", [False, True], ids=["bf16_cache", "fp8_cache"])
def test_a_prompt_and_a_tree_through_one_cache(oracle, fp8):
    """Two prompts in two chunks each (extend, rotate and append, attend), then a draft tree per request over the same cache (extend with depths, rotate and append, the tree
    attention, acceptance, commit): every step fed by the one before on the device, every attention compared with the oracle's over rows that were rotated on the host."""
    import torch
    import gpu_util as Gu
    from paper_2605_29727_amd import binding as btv
    Hq, Hkv, D, B, V, batch, blocks, width = 8, 2, 128, 6, 500, 2, 40, 20
    chunks, Ns = [[50, 70], [33, 100]], [24, 17]
    dev = dict(dtype=torch.int32, device="cuda")
    table, free, n_free = torch.full((batch, width), -1, **dev), Gu.dev(synth.permutation(3, "free", blocks).astype(np.int32)), torch.full((1,), blocks, **dev)
    n_pages, L = torch.zeros(batch, **dev), torch.zeros(batch, **dev)
    Kc = torch.zeros((blocks, PAGE, Hkv, D), dtype=torch.uint8 if fp8 else torch.bfloat16, device="cuda")
    Vc = torch.zeros_like(Kc)
    freq, factor = btv.btv_rope_frequencies(D, 10000.0, btv.BTV_ROPE_YARN, 4.0, 64.0, 1.0, 32.0)
    inv = torch.tensor(freq, dtype=torch.float64, device="cuda")
    ks = vs = 0.02
    pos_of, keys, values = [[] for _ in range(batch)], [[] for _ in range(batch)], [[] for _ in range(batch)]
    ws_rows = btv.alloc_workspace(256)
    ws_attn = btv.alloc_workspace(max(btv.btv_chunk_attn_paged_workspace(batch, 128, 256, Hq, Hkv, D), btv.btv_chunk_attn_paged_fp8kv_workspace(batch, 128, 256, Hq, Hkv, D),
                                      btv.btv_tree_verify_attn_paged_workspace(batch, 32, 256, Hq, Hkv, D), btv.btv_tree_verify_attn_paged_fp8kv_workspace(batch, 32, 256, Hq, Hkv, D)))

    def rows_in(Ms, depth, seed):
        """extend, rotate, append; returns the device's Q and what the oracle needs."""
        nonlocal n_pages, n_free
        total = sum(Ms)
        qo, slot, position, np_out, nf_out = (torch.zeros(n, **dev) for n in (batch + 1, total, total, batch, 1))
        btv.btv_paged_extend(L, torch.tensor(Ms, **dev), depth, n_pages, free, n_free, table, qo, slot, position, np_out, nf_out, ws_rows)
        n_pages, n_free = np_out, nf_out
        x = torch.from_numpy(synth.normal(seed, "together", (total, Hq + 2 * Hkv, D))).to(torch.bfloat16).cuda()
        Q = torch.zeros((total, Hq, D), dtype=torch.bfloat16, device="cuda")
        args = (x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], position, slot, inv, Q, Kc, Vc)
        if fp8:
            btv.btv_rope_append_fp8kv(*args, ks, vs, factor=factor, ws=ws_rows)
        else:
            btv.btv_rope_append(*args, factor=factor, ws=ws_rows)
        return qo, Q, x.double().cpu().numpy(), position.cpu().numpy()

    def remember(Ms, x, position):
        at = 0
        for r, m in enumerate(Ms):
            keys[r].append(oracle.rope(x[at:at + m, Hq:Hq + Hkv], position[at:at + m], freq, False, factor))
            values[r].append(x[at:at + m, Hq + Hkv:])
            at += m

    def compare(O, Ms, x, position, parents, Lh):
        at, got = 0, O.double().cpu().numpy()
        for r, m in enumerate(Ms):
            q = oracle.rope(x[at:at + m, :Hq], position[at:at + m], freq, False, factor)
            ref = oracle.tree_attn(q.astype(np.float32), np.concatenate(keys[r]).astype(np.float32), np.concatenate(values[r]).astype(np.float32), parents[r], Lh[r])
            # bf16 queries, keys (2^-8 each of scores of up to about 6: the weights move by 5 %), or E4M3 ones (2^-4, on average over 128 channels): what the caches hold is not
            # what the oracle was given
            off = np.sqrt(np.mean((got[at:at + m] - ref) ** 2)) / np.sqrt(np.mean(ref ** 2))
            assert off < (0.08 if fp8 else 0.02), (r, off)
            at += m

    for step in range(2):
        Ms = [c[step] for c in chunks]
        Lh = L.cpu().numpy().tolist()
        qo, Q, x, position = rows_in(Ms, None, 70 + step)
        assert position.tolist() == [l + i for l, m in zip(Lh, Ms) for i in range(m)]
        remember(Ms, x, position)
        O = torch.zeros_like(Q)
        if fp8:
            btv.btv_chunk_attn_paged_fp8kv(Q, Kc, Vc, ks, vs, table, qo, L, 128, 256, O, ws_attn)
        else:
            btv.btv_chunk_attn_paged(Q, Kc, Vc, table, qo, L, 128, 256, O, ws_attn)
        compare(O, Ms, x, position, [np.arange(-1, m - 1, dtype=np.int32) for m in Ms], Lh)
        L = L + torch.tensor(Ms, **dev)

    # ---- a draft tree per request ----
    marg = np.stack([synth.marginals(80 + r, B, V, 3.0) for r in range(batch)])
    trees = [oracle.tree_build(marg[r], Ns[r]) for r in range(batch)]
    total, offs = sum(Ns), np.concatenate([[0], np.cumsum(Ns)]).astype(np.int32)
    parent, token, depth = (torch.zeros(total, **dev) for _ in range(3))
    n_out, ahat = torch.zeros(batch, **dev), torch.zeros(batch, device="cuda")
    btv.btv_tree_build_batch(torch.from_numpy(marg.astype(np.float32)).cuda(), torch.tensor(Ns, **dev), Gu.dev(offs), max(Ns), parent, token, depth,
                             torch.zeros(total, device="cuda"), n_out, ahat, btv.alloc_workspace(btv.btv_tree_build_batch_workspace(batch, B, V, max(Ns))))
    Lh = L.cpu().numpy().tolist()
    qo, Q, x, position = rows_in(Ns, depth, 75)
    assert qo.cpu().numpy().tolist() == offs.tolist()
    assert position.tolist() == [l + int(d) - 1 for l, t in zip(Lh, trees) for d in t["depth"]]
    remember(Ns, x, position)
    O = torch.zeros_like(Q)
    if fp8:
        btv.btv_tree_verify_attn_paged_fp8kv(Q, Kc, Vc, ks, vs, table, qo, L, parent, 32, 256, O, ws_attn)
    else:
        btv.btv_tree_verify_attn_paged(Q, Kc, Vc, table, qo, L, parent, 32, 256, O, ws_attn)
    compare(O, Ns, x, position, [t["parent"] for t in trees], Lh)
    logits = torch.from_numpy(synth.normal(90, "logits", (total + batch, V))).to(torch.bfloat16).cuda()
    row = 0
    for t, n in zip(trees, Ns):            # the target follows the first child of the root, and its first child
        kids = [i for i in range(n) if t["parent"][i] == -1]
        logits[row, int(t["token"][kids[0]])] = 50.0
        for i in range(n):
            if t["parent"][i] == kids[0]:
                logits[row + 1 + kids[0], int(t["token"][i])] = 50.0
                break
        row += n + 1
    path, n_acc, bonus, new_len = torch.zeros(total, **dev), torch.zeros(batch, **dev), torch.zeros(batch, **dev), torch.zeros(batch, **dev)
    btv.btv_tree_accept_greedy_batch(logits, parent, token, qo, max(Ns), path, n_acc, bonus, None, btv.alloc_workspace(btv.btv_tree_accept_batch_workspace(batch, total, V)))
    btv.btv_kv_commit_paged(Kc.unsqueeze(0), Vc.unsqueeze(0), table, L, path, n_acc, new_len, None, q_offset=qo, M_max=max(Ns))
    assert int(n_acc.min()) >= 1 and new_len.cpu().numpy().tolist() == (L + n_acc).cpu().numpy().tolist()
    # the next token of each request, behind what was accepted
    hp, ha = path.cpu().numpy(), n_acc.cpu().numpy()
    for r in range(batch):
        p = hp[offs[r]:offs[r] + ha[r]]
        keys[r][-1], values[r][-1] = keys[r][-1][p], values[r][-1][p]
    L = new_len
    Lh = L.cpu().numpy().tolist()
    qo, Q, x, position = rows_in([1, 1], None, 76)
    remember([1, 1], x, position)
    O = torch.zeros_like(Q)
    if fp8:
        btv.btv_chunk_attn_paged_fp8kv(Q, Kc, Vc, ks, vs, table, qo, L, 1, 256, O, ws_attn)
    else:
        btv.btv_chunk_attn_paged(Q, Kc, Vc, table, qo, L, 1, 256, O, ws_attn)
    compare(O, [1, 1], x, position, [np.array([-1], np.int32)] * 2, Lh)
    assert btv.btv_workspace_status(ws_rows) == 0 and btv.btv_workspace_status(ws_attn) == 0
    assert int(n_free[0]) == blocks - int(n_pages.sum())


@pytest.mark.parametrize("kv,Hq,Hkv,D", [("fp8", 32, 8, 128), ("bf16", 32, 8, 64)], ids=["fp8", "bf16_d64"])
def test_many_single_tokens_of_unequal_requests_are_shared_evenly(kv, Hq, Hkv, D):
    """128 tokens over 100 to 4000 keys, against as many over equal lengths that come to as many keys: no workgroup has much more than its share."""
    import torch
    Ls = [int(100 * 40 ** (r / 127)) for r in range(128)]
    Ls = [Ls[37 * r % 128] for r in range(128)]
    batches = [make(80, lengths, [1] * 128, Hq, Hkv, D, kv) for lengths in (Ls, [sum(Ls) // 128] * 128)]
    wss, Os = [workspace(b) for b in batches], [torch.empty_like(b["Q"]) for b in batches]

    def us(i):
        marks = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
        for k in range(30):
            if k == 5:
                marks[0].record()
            call(batches[i], Os[i], wss[i])
        marks[1].record()
        torch.cuda.synchronize()
        return marks[0].elapsed_time(marks[1]) * 1e3 / 25

    ratios = []
    for _ in range(5):                       # (1.19 and 1.21; 1.37 and 1.31 where a block counted as 60 tiles besides its keys)
        ratios.append(us(0) / us(1))
        if ratios[-1] < 1.27:
            break
    assert min(ratios) < 1.27, ratios
