"""Chunk attention (btv_chunk_attn_paged, btv_chunk_attn_paged_fp8kv) with keys, values and scales at the ends of their types."""
import math

import pytest

from test_gpu_chunk_attn import PAGE, check, make, run

pytestmark = pytest.mark.gpu


def put(b, name, r, keys, channel, value):
    """Sets a channel of the keys (or values) of request r, all heads."""
    import torch
    at = torch.as_tensor(keys, device="cuda")
    b[name][b["table"][r].long()[at // PAGE], at % PAGE, :, channel] = value


# Tiles of 32 keys whose scores all are -infinity: the first of a sequence, of a wavefront, of a part or anywhere, and all but a few.  low: what the other scores
# come to besides (-3200 before the scale: a reference of 0 would leave nothing of their exponentials).
@pytest.mark.parametrize("low", [0.0, -400.0])
@pytest.mark.parametrize("Hq,Hkv,D", [(8, 2, 128), (8, 2, 64), (32, 8, 128), (4, 4, 64)])
@pytest.mark.parametrize("L,M,tiles", [(300, 1, [0]), (300, 1, [1]), (300, 1, [0, 1]), (300, 1, [0, 1, 2, 3, 4]), (300, 40, [0]), (300, 40, [1, 2, 3]), (3000, 1, "some"), (3000, 1, "most"),
                                       (9000, 17, "some"), (700, 100, [0, 1, 2]), (2500, 300, "some"), (2500, 300, "most"), (0, 700, [1, 2]), (0, 700, [0, 1]), (4099, 2047, "some"),
                                       (4099, 2047, "most"), (0, 2048, [0, 2, 3])], ids=lambda x: str(x).replace(" ", ""))
def test_infinite_keys(Hq, Hkv, D, L, M, tiles, low):
    import torch
    b = make(L + M + D, [L], [M], Hq, Hkv, D, "bf16")
    n = (L + M) // 32
    if isinstance(tiles, str):
        g = torch.Generator().manual_seed(n)
        tiles = torch.nonzero(torch.rand(n, generator=g) < (0.4 if tiles == "some" else 0.95)).flatten().tolist()
    keys = [32 * t + j for t in tiles for j in range(32)]
    assert keys[-1] < L + M
    b["Q"][..., 33], b["Q"][..., 34] = -1.0, 8.0
    everything = list(range(L + M))
    put(b, "K", 0, everything, 34, low)
    k, v = (x.double() for x in b["rows"][0])
    k[:, :, 34] = low
    put(b, "K", 0, keys, 33, math.inf)
    gone = torch.zeros(L + M, dtype=torch.bool, device="cuda")
    gone[keys] = True
    O = run(b).double()
    G = Hq // Hkv
    for h in range(Hq):
        q, kh, vh = b["Q"][:, h].double(), k[:, h // G], v[:, h // G]
        hidden = gone | (torch.arange(L + M, device="cuda") > L + torch.arange(M, device="cuda")[:, None])
        none = hidden.all(1)
        w = torch.softmax((q @ kh.T * D ** -0.5).masked_fill(hidden, -math.inf), -1)
        ref, mass = w @ vh, w @ vh.abs()
        # Probabilities in bf16 in numerator and sum, parts in fp16, the result's rounding; scores: D products summed in fp32, half a step each of the largest sum of
        # magnitudes, and the exponent's roundings.  While a row has no finite score its reference may be 2^14: D / 16 sums of that size more, half a step 2^-10 each.
        mags = float((q.abs().amax(0) @ kh.abs().amax(0)) * D ** -0.5)
        scores = 2 * ((D + 4) * 2.0 ** -24 * mags + D / 16 * 2.0 ** -10 * D ** -0.5) * mass
        tol = 2.0 ** -7 * mass + scores + 2.0 ** -10 * mass.amax(-1, keepdim=True) + 2.0 ** -8 * ref.abs()
        off = (O[:, h] - ref).abs()
        assert bool((off <= tol)[~none].all()), (h, float((off / tol)[~none].nan_to_num(1e9).max()))
        assert bool(torch.isnan(O[none, h]).all())


@pytest.mark.parametrize("kv,Hq,Hkv,D", [("bf16", 8, 2, 128), ("bf16", 8, 2, 64), ("fp8", 8, 2, 128), ("bf16", 32, 8, 128)], ids=["bf16_d128", "bf16_d64", "fp8", "bf16_32_heads"])
@pytest.mark.parametrize("L,M,strong,at", [(9000, 1, 100, 8000), (9000, 1, 8000, 100), (30000, 1, 15000, 29999), (9000, 17, 50, 8990), (9000, 17, 8000, 3), (3000, 100, 2900, 60), (12000, 60, 60, 11000),
                                           (8192, 300, 8000, 77), (8192, 300, 77, 8100), (20, 2000, 3, 15)])
def test_a_value_that_is_no_number_behind_a_weight_that_vanishes(kv, Hq, Hkv, D, L, M, strong, at):
    """One key takes all of the weight; a value that is no number still reaches every row that sees it, in whatever part of the keys it lies, and no other channel."""
    import torch
    b = make(L + M, [L], [M], Hq, Hkv, D, kv)
    q = b["Q"][0, 0].clone()
    b["Q"][:] = q
    page, row = int(b["table"][0, strong // PAGE]), strong % PAGE
    # scores: 2^-x of the strong key's for all others with x above 200, past the smallest number of fp32
    if kv == "fp8":
        b["K"][page, row] = (q.float().sign() * 448).to(torch.float8_e4m3fn).view(torch.uint8)
        b["Q"][:] *= 8
    else:
        b["K"][page, row] = (24 * q.float()).to(torch.bfloat16)
    clean = run(b).double()
    assert bool(torch.isfinite(clean).all())
    put(b, "V", 0, [at], 5, 0x7F if kv == "fp8" else math.inf)
    O = run(b).double()
    other = torch.arange(D, device="cuda") != 5
    sees = torch.arange(M, device="cuda") + L >= at
    assert bool((~torch.isfinite(O[sees][..., 5])).all())
    # (parts in fp16 beside their largest magnitude, which channel 5 no longer takes part in: as for values in hidden places)
    limit = 2 * (2.0 ** -9 * clean.abs().amax(-1, keepdim=True) + 2.0 ** -8 * clean.abs())
    assert bool(((O - clean).abs() <= limit)[..., other].all()) and torch.equal(O[~sees], clean[~sees])


@pytest.mark.parametrize("scale", [1e10, 1e25])
@pytest.mark.parametrize("kv,Hq,Hkv,D", [("fp8", 8, 8, 128), ("bf16", 8, 8, 128), ("bf16", 8, 8, 64), ("bf16", 8, 2, 128)], ids=["fp8", "bf16_d128", "bf16_d64", "bf16_groups"])
@pytest.mark.parametrize("Ls,Ms", [([5, 900, 0, 0, 77, 3, 40, 2000], [1800, 0, 700, 129, 1000, 65, 1500, 333]), ([20000, 0], [700, 3500]), ([700], [100]), ([40, 6000, 1, 300, 2000], [33, 1, 257, 16, 65]),
                                   ([113 * i % 900 for i in range(70)], [130 + 37 * i % 200 for i in range(70)])], ids=lambda x: "-".join(map(str, x[:5])))
def test_small_queries_and_a_large_scale(kv, Hq, Hkv, D, Ls, Ms, scale):
    """Scores are as ever; what stands for a row without a score, times the scale, is past the range of fp32, and some parts have rows that see none of their keys."""
    b = make(sum(Ms), Ls, Ms, Hq, Hkv, D, kv, sharp=D ** -0.5 / scale)
    check(b, run(b, scale=scale), scale=scale)
