"""What the tests of chunk attention over long ranges can see: one tile of 32 keys that is lost or taken twice, by the tolerance's own formula, for every tile of a sequence."""
import math

import pytest
import torch


def error_of_one_tile(q, k, M, L, D, lost, channels):
    """For every row and tile: the error of the tile's channel (channels: V is 1 in channel tile % D; else random V, and the largest over the channels) over what the check allows."""
    g = torch.Generator().manual_seed(L + M)
    S, scale = L + M, D ** -0.5
    tiles = -(-S // 32)
    if channels:
        v = torch.zeros((S, D), dtype=torch.float64)
        v[torch.arange(S), torch.arange(S) // 32 % D] = 1.0
    else:
        v = torch.randn((S, D), generator=g).to(torch.bfloat16).double()
    hidden = torch.arange(S) > L + torch.arange(M)[:, None]
    w = torch.softmax((q @ k.T * scale).masked_fill(hidden, -math.inf), -1)
    ref, mass = w @ v, w @ v.abs()
    # (as in test_gpu_chunk_attn.py's check)
    scores = 2 * (D + 4) * 2.0 ** -24 * float((q.abs().amax(0) @ k.abs().amax(0)) * scale) * mass
    tol = 2.0 ** -7 * mass + scores + 2.0 ** -10 * mass.amax(-1, keepdim=True) + 2.0 ** -8 * ref.abs()
    out = torch.empty((M, tiles), dtype=torch.float64)
    sign = -1.0 if lost else 1.0
    for t in range(tiles):
        part = w[:, 32 * t:32 * t + 32]
        there = (ref + sign * (part @ v[32 * t:32 * t + 32])) / (1 + sign * part.sum(-1, keepdim=True))
        out[:, t] = ((there - ref).abs() / tol).amax(-1)
    return out


@pytest.mark.parametrize("lost", [True, False], ids=["lost", "twice"])
@pytest.mark.parametrize("D,L,M", [(128, 20000, 1), (64, 20000, 1), (128, 30000, 1), (64, 30000, 1), (128, 9000, 17), (64, 9000, 17), (64, 12000, 60), (128, 3000, 1), (64, 300, 40)])
def test_one_tile_is_seen(D, L, M, lost):
    g = torch.Generator().manual_seed(D + L)
    q, k = torch.randn((M, D), generator=g).to(torch.bfloat16).double(), torch.randn((L + M, D), generator=g).to(torch.bfloat16).double()
    off = error_of_one_tile(q, k, M, L, D, lost, True)
    whole = (L + 1) // 32                                  # (tiles that all rows see all keys of)
    assert float(off[:, :whole].min()) > 1.0, float(off[:, :whole].min())


def test_random_values_do_not_show_a_tile_of_a_long_sequence():
    """Why those tests have values of their own."""
    g = torch.Generator().manual_seed(1)
    q, k = torch.randn((1, 128), generator=g).to(torch.bfloat16).double(), torch.randn((20001, 128), generator=g).to(torch.bfloat16).double()
    assert float(error_of_one_tile(q, k, 1, 20000, 128, True, False).max()) < 1.0
