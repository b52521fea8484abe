"""Chunk attention with values that make every tile of keys count: a tile that a cut or a merge loses, or takes twice, is an error that the tolerance does not cover
(test_chunk_attn_tiles_cpu.py counts it out)."""
import pytest

from test_gpu_chunk_attn import PAGE, check, make, run

pytestmark = pytest.mark.gpu


def tile_channels(b):
    """V: 1 in channel (tile of 32 keys) modulo D, 0 elsewhere, so that a channel of the result is the softmax mass of a few tiles."""
    import torch
    D = b["heads"][2]
    one = 96 if b["kv"] == "fp8" else 1.0
    for r, (l, m) in enumerate(zip(b["Ls"], b["Ms"])):
        at = torch.arange(l + m, device="cuda")
        k, v = b["rows"][r]
        v = torch.zeros(v.shape, device="cuda")
        v[at, :, at // 32 % D] = one
        v = v.to(torch.float8_e4m3fn).view(torch.uint8) if b["kv"] == "fp8" else v.to(torch.bfloat16)
        b["V"][b["table"][r].long()[at // PAGE], at % PAGE] = v
        b["rows"][r] = (k, v)
    return b


@pytest.mark.parametrize("kv,Hq,Hkv,D", [("bf16", 32, 8, 128), ("bf16", 8, 2, 64), ("bf16", 32, 8, 64), ("bf16", 8, 8, 128), ("fp8", 8, 2, 128), ("fp8", 8, 8, 128)],
                         ids=["bf16_d128", "bf16_d64", "bf16_d64_32_heads", "bf16_8_heads", "fp8", "fp8_8_heads"])
@pytest.mark.parametrize("Ls,Ms", [([20000], [1]), ([30000] * 3, [1] * 3), ([3000, 20000, 77, 9000], [1] * 4), ([9000], [17]), ([12000], [60]), ([8192], [300]), ([3000], [1]), ([3000], [4096]),
                                   ([20000, 0], [700, 3500]), ([40, 6000, 1, 300, 2000], [33, 1, 257, 16, 65]), ([5, 900, 0, 0, 77, 3, 40, 2000], [1800, 0, 700, 129, 1000, 65, 1500, 333]),
                                   ([50 * r for r in range(80)], [1] * 80), ([113 * r % 1500 for r in range(70)], [130 + 37 * r % 200 for r in range(70)])],
                         ids=lambda x: "-".join(map(str, x[:5])))
def test_every_tile_counts(kv, Hq, Hkv, D, Ls, Ms):
    b = tile_channels(make(sum(Ls) + sum(Ms), Ls, Ms, Hq, Hkv, D, kv))
    check(b, run(b))


@pytest.mark.parametrize("Ls,Ms", [([20000], [1]), ([3000, 900], [1, 1]), ([9000], [17]), ([2500], [300]), ([40, 6000, 1, 300, 2000], [33, 1, 257, 16, 65])], ids=lambda x: "-".join(map(str, x)))
@pytest.mark.parametrize("kv,Hq,Hkv,D", [("bf16", 32, 8, 128), ("bf16", 8, 2, 64), ("fp8", 8, 2, 128)], ids=["bf16_d128", "bf16_d64", "fp8"])
def test_every_tile_counts_with_bounds_above_the_lengths(kv, Hq, Hkv, D, Ls, Ms):
    import torch
    b = tile_channels(make(sum(Ls) + sum(Ms), Ls, Ms, Hq, Hkv, D, kv))
    b["table"] = torch.nn.functional.pad(b["table"], (0, 1_000_016 // PAGE - b["table"].shape[1]), value=-5)
    check(b, run(b, M_max=2000, L_max=1_000_000))


def test_hundreds_of_prompts_that_are_not_worth_a_cut():
    """Blocks of 256 rows of 64 channels, all of up to 8 tiles: the form without a merge."""
    Ms = [200 + 29 * r % 57 for r in range(450)]
    b = tile_channels(make(81, [0] * 450, Ms, 32, 8, 64, "bf16"))
    check(b, run(b), only=set(range(0, 450, 11)) | {449})
