"""Workloads of the operators that bring rows into a paged KV cache, for timing: their plain forms in elementary torch operations, and, where `own` is
true, the calls of the library.

Kinds of a case
    extend   pages, slots and positions of the rows that come next, from the requests' lengths (btv_paged_extend)
    rope     rotary positions of queries and keys, and the append of keys and values to the cache (btv_rope_append, btv_rope_append_fp8kv)
    attn     attention of the requests' new rows over their pages: prompts, chunks of them, single tokens (btv_chunk_attn_paged, btv_chunk_attn_paged_fp8kv)

Lengths are part of a case (drawn from its `mix`), values and pages come from the seed.
"""
import math
import random

import torch

own = False

I32, F32, F64, BF16, U8 = torch.int32, torch.float32, torch.float64, torch.bfloat16, torch.uint8
E4M3 = torch.float8_e4m3fn
PAGE = 16
FP8_SCALE = 4.5 / 448.0          # the codes cover |x| <= 4.5 of N(0,1) values


def _case(kind, name=None, **sizes):
    c = {"kind": kind, **sizes}
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # The step of a ragged batch of eight draft trees: a few pages, some hundred rows.  All latency.
        _case("extend", "extend_trees8", requests=8, L_lo=1024, L_hi=16384, M_lo=32, M_hi=128, tree=True, mix=5),
        # A full server: most requests give one token, some a piece of their prompt.
        _case("extend", "extend_server700", requests=700, L_lo=1, L_hi=8000, M_lo=1, M_hi=500, tree=False, mix=9),
        # The smallest append: 16 nodes of one head in fp32, a part of the channels rotated.
        _case("rope", "rope_fp32_tiny", dtype="fp32", cache="fp32", rows=16, Hq=1, Hkv=1, D=64, R=32, pairs="interleaved", scaled=False, packed=False),
        # The trees of a batch into an E4M3 cache, straight from one projection's output; positions far out, frequencies scaled for them.
        _case("rope", "rope_fp8_rows490", dtype="bf16", cache="fp8", rows=490, Hq=32, Hkv=8, D=128, R=128, pairs="half", scaled=True, packed=True),
        # A long prompt's chunk into a bf16 cache.
        _case("rope", "rope_bf16_rows8191", dtype="bf16", cache="bf16", rows=8191, Hq=32, Hkv=8, D=128, R=128, pairs="half", scaled=False, packed=True),
        # The smallest call: one new token behind a few, 64-channel heads.
        _case("attn", "attn_token_L37_d64", kv="bf16", requests=1, L_lo=37, L_hi=37, M_lo=1, M_hi=1, Hq=8, Hkv=2, D=64, mix=1),
        # A decoding step of 32 conversations over an E4M3 cache.
        _case("attn", "attn_tokens32_fp8", kv="fp8", requests=32, L_lo=100, L_hi=4000, M_lo=1, M_hi=1, Hq=32, Hkv=8, D=128, mix=7),
        # Single tokens and pieces of prompts in one batch.
        _case("attn", "attn_mixed8", kv="bf16", requests=8, L_lo=64, L_hi=16384, M_lo=1, M_hi=600, Hq=32, Hkv=8, D=128, mix=4),
        # Four prompts from their first token on, 64-channel heads.
        _case("attn", "attn_prompts4_d64", kv="bf16", requests=4, L_lo=0, L_hi=0, M_lo=300, M_hi=1999, Hq=32, Hkv=8, D=64, mix=3),
        # A chunk of a long prompt on the 8B shape.
        _case("attn", "attn_chunk2048_L8192", kv="bf16", requests=1, L_lo=8192, L_hi=8192, M_lo=2048, M_hi=2048, Hq=32, Hkv=8, D=128, mix=1),
        # Two of them over an E4M3 cache, odd lengths.
        _case("attn", "attn_chunks2_fp8", kv="fp8", requests=2, L_lo=9000, L_hi=12003, M_lo=701, M_hi=1000, Hq=32, Hkv=8, D=128, mix=2),
        # The largest call: a 70B-shaped target at a 32k context.
        _case("attn", "attn_70b_chunk2048_L30720", kv="bf16", requests=1, L_lo=30720, L_hi=30720, M_lo=2048, M_hi=2048, Hq=64, Hkv=8, D=128, mix=1),
    ]


# ----------------------------------------------------------------------------------------------------------------------
# drawn cases
# ----------------------------------------------------------------------------------------------------------------------

HEADS = [(32, 8, 128), (64, 8, 128), (32, 8, 64), (16, 4, 64), (8, 2, 128), (8, 8, 64), (16, 2, 128), (28, 4, 128)]
MOST_FLOPS = 4 * 64 * 128 * 2048 * 30720        # a quarter of a percent below the largest listed case
MOST_SCORES = 64 * 2048 * 32768                 # of the padded batch, in the plain form


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["extend", "rope", "attn", "attn"])
    mix = rng.randint(1, 1 << 20)
    if kind == "extend":
        requests = _log(rng, 1, 1000)
        tree = rng.random() < 0.5
        M_hi = _log(rng, 1, 256 if tree else min(8000, 130000 // requests))
        L_hi = _log(rng, 1, min(32768, 4000000 // requests))
        return _case("extend", requests=requests, L_lo=max(0, L_hi // 32), L_hi=L_hi, M_lo=max(1, M_hi // 32), M_hi=M_hi, tree=tree, mix=mix)
    Hq, Hkv, D = rng.choice(HEADS)
    if kind == "rope":
        dtype = rng.choice(["fp32", "bf16", "bf16", "bf16"])
        cache = "fp32" if dtype == "fp32" else rng.choice(["bf16", "fp8"])
        rows = _log(rng, 1, 8191 if Hq <= 32 and dtype == "bf16" else 3000)
        return _case("rope", dtype=dtype, cache=cache, rows=rows, Hq=Hq, Hkv=Hkv, D=D, R=16 * rng.randint(1, D // 16), pairs=rng.choice(["half", "interleaved"]),
                     scaled=rng.random() < 0.5, packed=rng.random() < 0.5)
    kv = "fp8" if D == 128 and rng.random() < 0.4 else "bf16"
    while True:
        requests = _log(rng, 1, 64)
        M_hi = rng.choice([1, _log(rng, 2, 64), _log(rng, 64, 4096)])
        L_hi = rng.choice([0, _log(rng, 16, 32768), _log(rng, 256, 32768)])
        if requests * Hq * M_hi * (L_hi + M_hi) <= MOST_SCORES // 2 and 4 * requests * Hq * D * M_hi * (L_hi + M_hi) <= MOST_FLOPS and requests * (L_hi + M_hi) <= 400000:
            return _case("attn", kv=kv, requests=requests, L_lo=L_hi // 16, L_hi=L_hi, M_lo=max(1, M_hi // 16), M_hi=M_hi, Hq=Hq, Hkv=Hkv, D=D, mix=mix)


# ----------------------------------------------------------------------------------------------------------------------
# inputs
# ----------------------------------------------------------------------------------------------------------------------

def _between(r, lo, hi):
    """Spread over its logarithm, 0 where that is the upper end."""
    return 0 if hi == 0 else min(hi, max(lo, int(round(math.exp(r.uniform(math.log(max(lo, 1)), math.log(hi)))))))


def _lengths(c):
    r = random.Random(c["mix"])
    n = c["requests"]
    Ls = [_between(r, c["L_lo"], c["L_hi"]) for _ in range(n)]
    Ms = [_between(r, c["M_lo"], c["M_hi"]) for _ in range(n)]
    return Ls, Ms


def _ints(values):
    return torch.tensor(values, dtype=I32, device="cuda")


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _randn(g, shape, dtype):
    return torch.randn(shape, generator=g, dtype=F32, device="cuda").to(dtype)


def _codes(g, shape):
    """N(0,1) values as E4M3 codes of one scale."""
    return torch.randn(shape, generator=g, dtype=F32, device="cuda").clamp_(-4.5, 4.5).div_(FP8_SCALE).to(E4M3).view(U8)


def _cache(g, shape, kind):
    return _codes(g, shape) if kind == "fp8" else _randn(g, shape, F32 if kind == "fp32" else BF16)


def _table(g, pages, width):
    """Block table [len(pages), width] of a pool in which every page belongs to one request, in an order drawn from the seed; -1 past a request's pages."""
    total = sum(pages)
    order = torch.randperm(total, generator=g, device="cuda").to(I32)
    table = torch.full((len(pages), width), -1, dtype=I32, device="cuda")
    n = torch.tensor(pages, device="cuda")
    first = torch.cumsum(n, 0) - n
    k = torch.arange(width, device="cuda")
    mine = k < n[:, None]
    table[mine] = order[(first[:, None] + k)[mine]]
    return table


def _workspace(nbytes):
    return torch.zeros(max(int(nbytes), 256), dtype=U8, device="cuda")


def _prepare_extend(c, g):
    Ls, Ms = _lengths(c)
    held = [-(-l // PAGE) for l in Ls]
    need = [-(-(l + m) // PAGE) for l, m in zip(Ls, Ms)]
    r = random.Random(c["mix"] + 1)
    held = [min(n, h + r.randint(0, 1)) for h, n in zip(held, need)]        # some keep a page from rows that were not accepted
    take, width = sum(need) - sum(held), max(need)
    blocks = sum(held) + take + 16 + take // 4
    table = torch.full((len(Ls), width), -1, dtype=I32, device="cuda")
    order = torch.randperm(blocks, generator=g, device="cuda").to(I32)
    k, n = torch.arange(width, device="cuda"), torch.tensor(held, device="cuda")
    mine = k < n[:, None]
    table[mine] = order[((torch.cumsum(n, 0) - n)[:, None] + k)[mine]]
    free = torch.full((blocks,), -1, dtype=I32, device="cuda")
    n_free = blocks - sum(held)
    free[:n_free] = order[sum(held):]
    total = sum(Ms)
    depth = None
    if c["tree"]:       # depths that grow along a request's rows, as a best-first tree's do on the whole
        i = torch.cat([torch.arange(m, device="cuda") for m in Ms])
        depth = (1 + torch.log2(1.0 + i * torch.rand(total, generator=g, device="cuda"))).floor().clamp(max=16).to(I32)
    zeros = lambda n: torch.zeros(n, dtype=I32, device="cuda")  # noqa: E731
    return {"c": c, "prefix": _ints(Ls), "n_new": _ints(Ms), "depth": depth, "n_pages": _ints(held), "free": free, "n_free": _ints([n_free]), "table": table,
            "total": total, "out": {"q_offset": zeros(len(Ls) + 1), "slot": zeros(total), "position": zeros(total), "n_pages": zeros(len(Ls)), "n_free": zeros(1), "table": table}}


def _run_extend(s):
    o = s["out"]
    if own:
        from paper_2605_29727_amd import binding as btv
        btv.btv_paged_extend(s["prefix"], s["n_new"], s["depth"], s["n_pages"], s["free"], s["n_free"], s["table"], o["q_offset"], o["slot"], o["position"],
                             o["n_pages"], o["n_free"])
        return o
    L, M, P, table, total = s["prefix"].long(), s["n_new"].long(), s["n_pages"].long(), s["table"], s["total"]
    width = table.shape[1]
    need = (L + M + PAGE - 1) // PAGE
    take = (need - P).clamp(min=0)
    upto = torch.cumsum(take, 0)
    granted = upto <= s["n_free"]
    # every place of the table that gets a page: the k-th of them the k-th from the end of the free list
    k = torch.arange(width, device="cuda")
    nth = (upto - take)[:, None] + k - P[:, None]
    fresh = (k >= P[:, None]) & (k < need[:, None]) & granted[:, None]
    new = torch.where(fresh, s["free"][(s["n_free"] - 1 - nth).clamp(0, s["free"].numel() - 1)], table)
    q_offset = torch.cat([torch.zeros(1, dtype=torch.long, device="cuda"), torch.cumsum(M, 0)])
    row = torch.arange(total, device="cuda")
    r = torch.searchsorted(q_offset, row, right=True) - 1
    i = row - q_offset[r]
    at = L[r] + i
    slot = torch.where(granted[r], new[r, (at // PAGE).clamp(max=width - 1)].long() * PAGE + at % PAGE, -1)
    position = at if s["depth"] is None else L[r] + s["depth"] - 1
    return {"q_offset": q_offset.to(I32), "slot": slot.to(I32), "position": position.to(I32), "n_pages": torch.where(granted, torch.maximum(P, need), P).to(I32),
            "n_free": (s["n_free"] - (take * granted).sum()).to(I32), "table": new}


def _frequencies(R, scaled):
    """Radians per position.  Scaled: a context of 8192 stretched by 8, low frequencies divided, high ones kept, a ramp between 1 and 4 turns."""
    f = [500000.0 ** (-2.0 * i / R) for i in range(R // 2)]
    if scaled:
        turns = [8192.0 * x / (2.0 * math.pi) for x in f]
        keep = [min(1.0, max(0.0, (t - 1.0) / 3.0)) for t in turns]
        f = [x * k + x / 8.0 * (1.0 - k) for x, k in zip(f, keep)]
    return f


def _prepare_rope(c, g):
    T, Hq, Hkv, D = (c[k] for k in ("rows", "Hq", "Hkv", "D"))
    dt = F32 if c["dtype"] == "fp32" else BF16
    if c["packed"]:     # as one projection writes them: a row's queries, keys and values one behind the other
        x = _randn(g, (T, Hq + 2 * Hkv, D), dt)
        Q, K, V = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    else:
        Q, K, V = _randn(g, (T, Hq, D), dt), _randn(g, (T, Hkv, D), dt), _randn(g, (T, Hkv, D), dt)
    blocks = -(-T // PAGE) + 4
    slot = torch.randperm(blocks * PAGE, generator=g, device="cuda")[:T].to(I32)
    start = torch.randint(0, 100000 if c["scaled"] else 8192, (1,), generator=g, device="cuda")
    Kc, Vc = _cache(g, (blocks, PAGE, Hkv, D), c["cache"]), _cache(g, (blocks, PAGE, Hkv, D), c["cache"])
    shown = (lambda t: t.view(E4M3)) if c["cache"] == "fp8" else (lambda t: t)
    s = {"c": c, "Q": Q, "K": K, "V": V, "position": (start + torch.arange(T, device="cuda")).to(I32), "slot": slot, "Kc": Kc, "Vc": Vc,
         "inv_freq": torch.tensor(_frequencies(c["R"], c["scaled"]), dtype=F64, device="cuda"), "factor": 0.1 * math.log(8.0) + 1.0 if c["scaled"] else 1.0,
         "Qout": torch.zeros((T, Hq, D), dtype=dt, device="cuda")}
    s["out"] = {"Q": s["Qout"], "K": shown(Kc), "V": shown(Vc)}
    return s


def _rotate(x, cos, sin, R, pairs):
    """The pairs of the first R channels of x [T, H, D], each by its angle [T, 1, R/2]."""
    y = x.clone()
    a, b = (x[..., :R // 2], x[..., R // 2:R]) if pairs == "half" else (x[..., 0:R:2], x[..., 1:R:2])
    u, v = a * cos - b * sin, a * sin + b * cos
    if pairs == "half":
        y[..., :R // 2], y[..., R // 2:R] = u, v
    else:
        y[..., 0:R:2], y[..., 1:R:2] = u, v
    return y


def _run_rope(s):
    c = s["c"]
    fp8 = c["cache"] == "fp8"
    if own:
        from paper_2605_29727_amd import binding as btv
        if fp8:
            btv.btv_rope_append_fp8kv(s["Q"], s["K"], s["V"], s["position"], s["slot"], s["inv_freq"], s["Qout"], s["Kc"], s["Vc"], FP8_SCALE, FP8_SCALE,
                                      interleaved=c["pairs"] == "interleaved", factor=s["factor"])
        else:
            btv.btv_rope_append(s["Q"], s["K"], s["V"], s["position"], s["slot"], s["inv_freq"], s["Qout"], s["Kc"], s["Vc"],
                                interleaved=c["pairs"] == "interleaved", factor=s["factor"])
        return s["out"]
    angle = s["position"][:, None, None].to(F64) * s["inv_freq"]
    cos, sin = (angle.cos() * s["factor"]).to(F32), (angle.sin() * s["factor"]).to(F32)
    q, k = _rotate(s["Q"].to(F32), cos, sin, c["R"], c["pairs"]), _rotate(s["K"].to(F32), cos, sin, c["R"], c["pairs"])
    v, slot = s["V"].to(F32), s["slot"].long()
    s["Qout"].copy_(q)
    Kc, Vc = s["Kc"].view(-1, c["Hkv"], c["D"]), s["Vc"].view(-1, c["Hkv"], c["D"])
    if fp8:
        k, v = ((x / FP8_SCALE).clamp(-448.0, 448.0).to(E4M3).view(U8) for x in (k, v))
    Kc[slot], Vc[slot] = k.to(Kc.dtype), v.to(Vc.dtype)
    return s["out"]


def _prepare_attn(c, g):
    Ls, Ms = _lengths(c)
    Hq, Hkv, D = (c[k] for k in ("Hq", "Hkv", "D"))
    pages = [-(-(l + m) // PAGE) for l, m in zip(Ls, Ms)]
    offsets = [0]
    for m in Ms:
        offsets.append(offsets[-1] + m)
    shape = (sum(pages), PAGE, Hkv, D)
    s = {"c": c, "Q": _randn(g, (offsets[-1], Hq, D), BF16), "K": _cache(g, shape, c["kv"]), "V": _cache(g, shape, c["kv"]), "table": _table(g, pages, max(pages)),
         "q_offset": _ints(offsets), "prefix": _ints(Ls), "M_max": max(Ms), "L_max": max(Ls), "total": offsets[-1]}
    s["O"] = torch.zeros_like(s["Q"])
    if own:             # what a serving loop keeps between calls
        from paper_2605_29727_amd import binding as btv
        size = btv.btv_chunk_attn_paged_fp8kv_workspace if c["kv"] == "fp8" else btv.btv_chunk_attn_paged_workspace
        s["ws"] = _workspace(size(len(Ls), max(Ms), max(Ls), Hq, Hkv, D))
    return s


def _run_attn(s):
    c = s["c"]
    if own:
        from paper_2605_29727_amd import binding as btv
        if c["kv"] == "fp8":
            btv.btv_chunk_attn_paged_fp8kv(s["Q"], s["K"], s["V"], FP8_SCALE, FP8_SCALE, s["table"], s["q_offset"], s["prefix"], s["M_max"], s["L_max"], s["O"], s["ws"])
        else:
            btv.btv_chunk_attn_paged(s["Q"], s["K"], s["V"], s["table"], s["q_offset"], s["prefix"], s["M_max"], s["L_max"], s["O"], s["ws"])
        return s["O"]
    # every request padded to the longest: its pages in order, its rows in a block of their own
    Hq, Hkv, D, M, total = c["Hq"], c["Hkv"], c["D"], s["M_max"], s["total"]
    G, n = Hq // Hkv, s["table"].shape[0]
    row = torch.arange(total, device="cuda")
    r = torch.searchsorted(s["q_offset"], row, right=True) - 1
    i = row - s["q_offset"][r]
    q = torch.zeros((n, M, Hkv, G, D), dtype=F32, device="cuda")
    q[r, i] = s["Q"].view(total, Hkv, G, D).to(F32)
    pages = s["table"].clamp(min=0).long()
    value = (lambda x: x.view(E4M3).to(F32) * FP8_SCALE) if c["kv"] == "fp8" else (lambda x: x.to(F32))
    k = value(s["K"][pages]).view(n, -1, Hkv, D).permute(0, 2, 3, 1).contiguous()
    v = value(s["V"][pages]).view(n, -1, Hkv, D).transpose(1, 2).contiguous()
    x = torch.matmul(q.permute(0, 2, 1, 3, 4).reshape(n, Hkv, M * G, D), k).mul_(D ** -0.5).view(n, Hkv, M, G, -1)
    last = s["prefix"][:, None] + torch.arange(M, device="cuda")                # a row's last visible key
    hidden = torch.arange(x.shape[-1], device="cuda") > last[..., None]
    x.masked_fill_(hidden[:, None, :, None], -math.inf)
    x.sub_(x.amax(-1, keepdim=True)).exp_()
    weight = x.sum(-1, keepdim=True)
    o = torch.matmul(x.view(n, Hkv, M * G, -1), v).view(n, Hkv, M, G, D).div_(weight)
    s["O"].copy_(o.permute(0, 2, 1, 3, 4).reshape(n, M, Hq, D)[r, i])
    return s["O"]


_PREPARE = {"extend": _prepare_extend, "rope": _prepare_rope, "attn": _prepare_attn}
_RUN = {"extend": _run_extend, "rope": _run_rope, "attn": _run_attn}


def prepare(case, seed):
    return _PREPARE[case["kind"]](case, _generator(seed))


def run(state):
    return _RUN[state["c"]["kind"]](state)


# ----------------------------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ----------------------------------------------------------------------------------------------------------------------

def work(case):
    c = case
    if c["kind"] == "rope":
        e, ec = 4 if c["dtype"] == "fp32" else 2, {"fp32": 4, "bf16": 2, "fp8": 1}[c["cache"]]
        per_row = e * c["D"] * (2 * c["Hq"] + 2 * c["Hkv"]) + ec * c["D"] * 2 * c["Hkv"] + 8
        return {"bytes": c["rows"] * per_row + 4 * c["R"], "flops": 6 * c["rows"] * (c["Hq"] + c["Hkv"]) * c["R"] // 2}
    Ls, Ms = _lengths(c)
    if c["kind"] == "extend":
        pages = sum(-(-(l + m) // PAGE) - l // PAGE for l, m in zip(Ls, Ms))    # those that a row lies in
        return {"bytes": 4 * (5 * len(Ls) + 1 + 2 * pages + (3 if c["tree"] else 2) * sum(Ms)), "flops": 0}
    e = 1 if c["kv"] == "fp8" else 2
    keys = sum(m * l + m * (m + 1) // 2 for l, m in zip(Ls, Ms))
    return {"bytes": 2 * (sum(Ls) + sum(Ms)) * c["Hkv"] * c["D"] * e + 4 * sum(Ms) * c["Hq"] * c["D"], "flops": 4 * c["Hq"] * c["D"] * keys}


# ----------------------------------------------------------------------------------------------------------------------
# the same from the definitions, in 64 bits: request by request and head by head
# ----------------------------------------------------------------------------------------------------------------------

def exact(case, seed):
    c = case
    if c["kind"] == "extend":       # whole numbers only
        return None
    s = prepare(case, seed)
    if c["kind"] == "rope":
        turn = torch.polar(torch.full((), s["factor"], dtype=F64, device="cuda"), torch.outer(s["position"].double(), s["inv_freq"]))       # f e^{i t}

        def rotated(x):
            y = x.double().clone()
            R = c["R"]
            first = torch.arange(R // 2, device="cuda")
            a, b = (first, first + R // 2) if c["pairs"] == "half" else (2 * first, 2 * first + 1)
            z = torch.complex(y[..., a], y[..., b]) * turn[:, None, :]
            y[..., a], y[..., b] = z.real, z.imag
            return y

        out = {"Q": rotated(s["Q"])}
        for name, rows, cache in (("K", rotated(s["K"]), s["Kc"]), ("V", s["V"].double(), s["Vc"])):
            full = (cache.view(E4M3) if c["cache"] == "fp8" else cache).double().view(-1, c["Hkv"], c["D"])
            full[s["slot"].long()] = (rows / FP8_SCALE).clamp(-448, 448) if c["cache"] == "fp8" else rows
            out[name] = full.view(s["Kc"].shape)
        return out
    Ls, Ms = _lengths(c)
    Hq, Hkv, D = c["Hq"], c["Hkv"], c["D"]
    O = torch.empty((s["total"], Hq, D), dtype=F64, device="cuda")
    at = 0
    for r, (l, m) in enumerate(zip(Ls, Ms)):
        pos = torch.arange(l + m, device="cuda")
        page = s["table"][r, :-(-(l + m) // PAGE)].long()[pos // PAGE]
        seen = pos <= l + torch.arange(m, device="cuda")[:, None]
        for g in range(Hkv):
            k, v = (x[page, pos % PAGE, g] for x in (s["K"], s["V"]))
            k, v = ((x.view(E4M3).double() * FP8_SCALE if c["kv"] == "fp8" else x.double()) for x in (k, v))
            for h in range(g * (Hq // Hkv), (g + 1) * (Hq // Hkv)):
                x = (s["Q"][at:at + m, h].double() @ k.T) / math.sqrt(D)
                O[at:at + m, h] = torch.softmax(x.masked_fill(~seen, -math.inf), -1) @ v
        at += m
    return O
