"""Performance cases of the 8-bit cache: writing a step's tokens to it, reading rows back, attention over it.

`listed()` holds the fixed cases, `draw(rng)` gives further ones of the same ranges.  A case is a plain dict; its "kind"
names the entry point:

    write   cache8_write               keys and values of a step's tokens, quantised into a dense or paged cache
    read    cache8_read                rows of the cache, back in 16 bits
    attend  sdpa_kv8, sdpa_paged8      attention of single tokens, drafts and prefill chunks over the cache

A cache holds E4M3 codes [pages, Hkv, block_rows, D] and, for each head and 32 rows, the exponent of a power of two as a byte biased by
127.  `run` computes the operators in elementary torch operations, or with `own` through the library.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
LARGEST = 448.0                  # of the codes
BLOCK = 32                       # rows that share a scale
MOST, BIAS = 62, 127             # exponents are -MOST ... MOST


def listed():
    return [
        # one sequence being decoded, dense cache: latency
        dict(name="write_single", kind="write", B=1, S=1, Hkv=8, D=128, dtype="bf16", cap=8192, block_rows=0),
        # a decoding step of a batch, in pages: a row of a partly filled block for every entry
        dict(name="write_batch", kind="write", B=128, S=1, Hkv=8, D=128, dtype="f16", cap=1024, block_rows=128),
        # prefill chunks of 2048 tokens at most, each entry with a number of its own, into pages
        dict(name="write_chunk", kind="write", B=4, S=2048, Hkv=8, D=128, dtype="bf16", cap=8192, block_rows=64),
        # the accepted tokens of a batch of drafted trees, to be moved to the front of the tree's rows
        dict(name="read_path", kind="read", B=32, n=8, Hkv=8, D=128, dtype="bf16", cap=2048, block_rows=128),
        # two sequences of 16384 rows in pages, for the calls that take 16 bits
        dict(name="read_long", kind="read", B=2, n=16384, Hkv=8, D=128, dtype="f16", cap=16384, block_rows=128),
        # a decoding step of one sequence with 8192 cached keys: latency
        dict(name="decode_single", kind="attend", B=1, H=32, Hkv=8, Sq=1, Skv=8192, D=128, dtype="bf16", fill=1.0, block_rows=0, causal=True),
        # a decoding step of a batch of sequences of different lengths, in pages
        dict(name="decode_batch_paged", kind="attend", B=32, H=32, Hkv=8, Sq=1, Skv=8192, D=128, dtype="f16", fill=0.25, block_rows=128, causal=True),
        # long contexts, full
        dict(name="decode_long", kind="attend", B=4, H=32, Hkv=8, Sq=1, Skv=65536, D=128, dtype="bf16", fill=1.0, block_rows=0, causal=True),
        # a head for every query head, a head dim and a length that no tile divides
        dict(name="decode_heads_odd", kind="attend", B=3, H=30, Hkv=30, Sq=1, Skv=4001, D=96, dtype="f16", fill=0.5, block_rows=0, causal=True),
        # four drafted tokens in a chain for each sequence of a batch
        dict(name="drafts", kind="attend", B=8, H=32, Hkv=8, Sq=4, Skv=4096, D=64, dtype="bf16", fill=0.5, block_rows=64, causal=True),
        # prefill chunks of 500 tokens behind cached prefixes, in pages
        dict(name="chunk_paged", kind="attend", B=4, H=32, Hkv=8, Sq=500, Skv=4096, D=128, dtype="f16", fill=0.25, block_rows=64, causal=True),
        # a long prefill chunk of one sequence
        dict(name="chunk_long", kind="attend", B=1, H=32, Hkv=8, Sq=2048, Skv=16384, D=128, dtype="bf16", fill=1.0, block_rows=0, causal=True),
    ]


# what one drawn case may cost at most: the largest listed ones
MOST_BYTES = 5.4e8
MOST_FLOPS = 5.2e11


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    while True:
        kind = rng.choice(["write", "read", "attend", "attend", "attend"])
        D, dtype = rng.choice([64, 96, 128, 160]), rng.choice(["f16", "bf16"])
        if kind == "attend":
            group = rng.choice([1, 4, 8])
            hkv = _log_int(rng, 1, 32 // group)
            case = dict(kind=kind, B=_log_int(rng, 1, 64), H=hkv * group, Hkv=hkv, Sq=rng.choice([1, 1, _log_int(rng, 1, 2048)]), Skv=_log_int(rng, 64, 65536),
                        D=D, dtype=dtype, fill=rng.choice([1.0, 0.5, 0.1]), block_rows=rng.choice([0, 0, 64, 128, 256]), causal=rng.random() < 0.8)
            # (the plain form holds the scores, and the cache in 32 bits)
            if case["Sq"] > case["Skv"] or case["B"] * case["H"] * case["Sq"] * case["Skv"] > 1 << 30 or case["B"] * hkv * case["Skv"] * D > 1 << 28:
                continue
        else:
            case = dict(kind=kind, B=_log_int(rng, 1, 128), Hkv=_log_int(rng, 1, 32), D=D, dtype=dtype, cap=-(-_log_int(rng, 256, 16384) // 256) * 256,
                        block_rows=rng.choice([0, 64, 128, 256]))
            case["S" if kind == "write" else "n"] = _log_int(rng, 1, case["cap"])
            if case["B"] * case["Hkv"] * case["cap"] * D > 1 << 27:
                continue
        w = work(case)
        if w["flops"] <= MOST_FLOPS and w["bytes"] <= MOST_BYTES:
            return case


# ---- inputs

def _lengths(case):
    """Cached rows of each entry, the new ones included: spread evenly from fill * Skv to Skv."""
    B, Skv, fill = case["B"], case["Skv"], case["fill"]
    return [min(Skv, max(case["Sq"], int(Skv * (fill + (1.0 - fill) * (b + 0.5) / B)))) for b in range(B)]


def _power(e):
    """2^e in 32 bits, to the bit (exp2 of whole numbers is not, everywhere)."""
    return (e.to(torch.int32) + BIAS << 23).view(torch.float32)


def _fields(values):
    """Codes and exponent bytes of rows [..., heads, rows, D] in 32 bits."""
    rows = values.shape[-2]
    blocks = -(-rows // BLOCK)
    padded = torch.nn.functional.pad(values.abs().amax(-1), (0, blocks * BLOCK - rows))
    e = _needed(padded.view(*padded.shape[:-1], blocks, BLOCK).amax(-1))
    codes = (values * _power(-e).repeat_interleave(BLOCK, -1)[..., :rows, None]).to(torch.float8_e4m3fn)
    return codes, (e + BIAS).to(torch.uint8)


def _cache(case, g, pages, rows):
    """An 8-bit cache that has been written to: columns and heads of different magnitude, as projections have them."""
    out = []
    for _ in range(2):
        shape = (pages, case["Hkv"], rows, case["D"])
        codes, scales = torch.empty(shape, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(shape[:2] + (-(-rows // BLOCK),), dtype=torch.uint8, device="cuda")
        size = torch.exp(0.5 * torch.randn((case["Hkv"], 1, case["D"]), device="cuda", generator=g))
        some = max(1, (1 << 26) // (case["Hkv"] * rows * case["D"]))
        for p in range(0, pages, some):
            codes[p:p + some], scales[p:p + some] = _fields(torch.randn((min(some, pages - p),) + shape[1:], device="cuda", generator=g) * size)
        out += [codes, scales]
    return dict(k_cache=out[0], k_scales=out[1], v_cache=out[2], v_scales=out[3])


def prepare(case, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    B, Hkv, D, dtype = case["B"], case["Hkv"], case["D"], DTYPES[case["dtype"]]
    cap, R = case["Skv"] if case["kind"] == "attend" else case["cap"], case["block_rows"]
    state = dict(case=case, table=None)
    if R == 0:
        state.update(_cache(case, g, B, cap))
    else:
        M = -(-cap // R)
        state.update(_cache(case, g, B * M, R))
        state.update(table=torch.randperm(B * M, device="cuda", generator=g).to(torch.int32).view(B, M).contiguous())     # as a pool hands pages out
    if case["kind"] == "attend":
        lens = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda")
        state.update(lens=lens[torch.randperm(B, device="cuda", generator=g)].contiguous(),
                     q=torch.randn((B, case["H"], case["Sq"], D), device="cuda", generator=g).to(dtype))
        return state
    if case["kind"] == "read":
        n = case["n"]
        first = torch.randint(0, cap - n + 1, (B, 1), device="cuda", generator=g)
        row = first + torch.arange(n, device="cuda")
        page = torch.arange(B, device="cuda")[:, None].expand(B, n) if R == 0 else state["table"].long().gather(1, row // R)
        state.update(slots=(page * (R or cap) + row % (R or cap)).to(torch.int32).contiguous())
        return state
    S = case["S"]
    counts = torch.full((B,), S, device="cuda")
    if S > 1:
        counts = torch.randint(max(1, S // 2), S + 1, (B,), device="cuda", generator=g)        # entries with fewer tokens, the last of their row
    old = (torch.rand((B,), device="cuda", generator=g) * (cap - counts + 1)).long()
    # keys and values as views into the output of one projection
    size = torch.exp(0.5 * torch.randn((2 * Hkv * D,), device="cuda", generator=g))
    kv = (torch.randn((B, S, 2 * Hkv * D), device="cuda", generator=g) * size).to(dtype)
    k, v = kv.split([Hkv * D, Hkv * D], dim=-1)
    state.update(k=k.view(B, S, Hkv, D), v=v.view(B, S, Hkv, D), old=old.to(torch.int32), new=(old + counts).to(torch.int32))
    return state


# ---- the operators in elementary operations

def _needed(largest):
    """The least exponent with which `largest` is at most the largest code."""
    mantissa, exponent = torch.frexp(largest)              # largest = mantissa * 2^exponent, 448 = 0.875 * 2^9
    e = exponent - 9 + (mantissa > 0.875)
    return torch.where(largest > 0, e, -MOST).clamp(-MOST, MOST)


def _plain_places(s, row):
    """Page and row in it of rows [B, n] of the entries' sequences."""
    R = s["k_cache"].shape[2]
    if s["table"] is None:
        return torch.arange(row.shape[0], device=row.device)[:, None].expand_as(row), row
    return s["table"].long().gather(1, row // R), row % R


def _plain_write(s, x, cache, scales):
    """Rows x [B, S, Hkv, D] behind the entries' rows (every entry appends one at least)."""
    P, Hkv, R, D = cache.shape
    B, S = x.shape[:2]
    old, new = s["old"].long(), s["new"].long()
    i = torch.arange(S, device=x.device)
    # (a token that is not written takes the place of the entry's last)
    token = torch.where(i >= S - (new - old)[:, None], i, S - 1)
    x = x.gather(1, token[:, :, None, None].expand(x.shape)).float()
    page, row = _plain_places(s, new[:, None] - S + token)
    blocks = scales.shape[2]
    block = page * blocks + row // BLOCK
    size = torch.where(x.isfinite(), x.abs(), 0.0).amax(-1)
    largest = torch.zeros((P * blocks, Hkv), device=x.device).scatter_reduce(0, block.reshape(-1, 1).expand(-1, Hkv), size.view(-1, Hkv), "amax")
    # the block that holds the entry's last row and room: its rows keep their values
    lane = torch.arange(BLOCK, device=x.device)
    start = old // BLOCK * BLOCK
    held = start[:, None] + torch.where(lane < (old - start)[:, None], lane, 0)
    held_page, held_row = _plain_places(s, held)
    partial = held_page[:, 0] * blocks + held_row[:, 0] // BLOCK
    flat = scales.permute(0, 2, 1).reshape(P * blocks, Hkv)
    before = flat[partial].int() - BIAS
    need = _needed(largest)
    grown = torch.where((old > start)[:, None], torch.maximum(before, need[partial]), need[partial])
    need[partial] = grown
    held_page, held_row = held_page.reshape(-1), held_row.reshape(-1)
    codes = cache[held_page, :, held_row].view(B, BLOCK, Hkv, D)
    moved = (codes.float() * _power(before - grown)[:, None, :, None]).to(torch.float8_e4m3fn)
    codes = torch.where((old > start)[:, None, None, None], moved.view(torch.uint8), codes.view(torch.uint8))
    raw = cache.view(torch.uint8)
    raw[held_page, :, held_row] = codes.view(-1, Hkv, D)
    # the new rows
    e = need[block.reshape(-1)]
    y = x.view(-1, Hkv, D) * _power(-e)[:, :, None]
    y = torch.where(y.isfinite(), y.clamp(-LARGEST, LARGEST), math.nan).to(torch.float8_e4m3fn)
    raw[page.reshape(-1), :, row.reshape(-1)] = y.view(torch.uint8)
    scales[page.reshape(-1), :, row.reshape(-1) // BLOCK] = (e + BIAS).to(torch.uint8)


def _plain_values(s, cache, scales, page, row):
    """Rows [B, n] of the cache as the values that they stand for, [B, Hkv, n, D]."""
    B, n = page.shape
    Hkv, D = cache.shape[1], cache.shape[3]
    page, row = page.reshape(-1), row.reshape(-1)
    e = scales[page, :, row // BLOCK].int() - BIAS
    x = cache.view(torch.uint8)[page, :, row].view(torch.float8_e4m3fn).float() * _power(e)[:, :, None]
    return x.view(B, n, Hkv, D).transpose(1, 2).contiguous()


def _plain_read(s, cache, scales):
    R = cache.shape[2]
    slot = s["slots"].long()
    inside = (slot >= 0) & (slot < cache.shape[0] * R)
    place = torch.where(inside, slot, 0)
    x = _plain_values(s, cache, scales, place // R, place % R)
    return torch.where(inside[:, None, :, None], x, 0.0).to(DTYPES[s["case"]["dtype"]])


def _plain_attend(s):
    q, lens, n = s["q"], s["lens"].long(), s["case"]["Skv"]
    B, H, Sq, D = q.shape
    Hkv = s["k_cache"].shape[1]
    page, row = _plain_places(s, torch.arange(n, device=q.device).expand(B, n))
    k, v = _plain_values(s, s["k_cache"], s["k_scales"], page, row), _plain_values(s, s["v_cache"], s["v_scales"], page, row)
    scores = torch.matmul(q.float().view(B, Hkv, H // Hkv * Sq, D), k.transpose(-1, -2).contiguous()).view(B, H, Sq, n)
    scores *= 1.0 / math.sqrt(D)
    key, i = torch.arange(n, device=q.device), torch.arange(Sq, device=q.device)
    last = lens[:, None] - Sq + i if s["case"]["causal"] else (lens - 1)[:, None].expand(B, Sq)
    scores.masked_fill_((key > last[:, :, None])[:, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, Hkv, H // Hkv * Sq, n), v).view(B, H, Sq, D)
    return (o / torch.where(total > 0, total, 1.0)).to(q.dtype)


def _run_plain(s):
    kind = s["case"]["kind"]
    if kind == "attend":
        return _plain_attend(s)
    if kind == "read":
        return _plain_read(s, s["k_cache"], s["k_scales"]), _plain_read(s, s["v_cache"], s["v_scales"])
    _plain_write(s, s["k"], s["k_cache"], s["k_scales"])
    _plain_write(s, s["v"], s["v_cache"], s["v_scales"])
    return s["k_cache"], s["v_cache"], s["k_scales"], s["v_scales"]


# ---- the library's

def _run_own(s):
    from paper_2603_01960_amd import binding as lib

    case = s["case"]
    cache = s["k_cache"], s["v_cache"], s["k_scales"], s["v_scales"]
    if case["kind"] == "attend":
        if s["table"] is None:
            return lib.sdpa_kv8(s["q"], *cache, causal=case["causal"], kv_lens=s["lens"])
        return lib.sdpa_paged8(s["q"], *cache, s["lens"], s["table"], causal=case["causal"])
    if case["kind"] == "read":
        return lib.cache8_read(*cache, s["slots"], DTYPES[case["dtype"]])
    lib.cache8_write(s["k"], s["v"], *cache, s["old"], s["new"], block_table=s["table"])
    return cache


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- what a pass cannot do without

def work(case):
    B, Hkv, D = case["B"], case["Hkv"], case["D"]
    if case["kind"] == "attend":
        lens, Sq, H = _lengths(case), case["Sq"], case["H"]
        keys = sum(n * Sq - (Sq * (Sq - 1) // 2 if case["causal"] else 0) for n in lens)
        return {"bytes": 2 * Hkv * sum(lens) * (D + 1 / BLOCK) + 4 * B * H * Sq * D, "flops": 4 * D * H * keys}
    rows = B * (case["S"] if case["kind"] == "write" else case["n"]) * 2 * Hkv
    if case["kind"] == "write" and case["S"] > 1:
        rows = rows * 3 // 4                              # (an entry's count is S / 2 ... S)
    return {"bytes": rows * (3 * D + 1 / BLOCK), "flops": 2 * rows * D}


# ---- the same from the definitions, in 64 bits

def _two_to(e):
    """2^e in 64 bits, of whole numbers."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_codes():
    """The finite codes that are not negative, in order: three bits of mantissa, exponents from -6, the first eight below."""
    return [m / 8 * 2.0 ** -6 for m in range(8)] + [(1 + m / 8) * 2.0 ** e for e in range(-6, 9) for m in range(8) if (e, m) != (8, 7)]


def _exact_round(y):
    """The nearest code of each value, of two equally near ones that with the even mantissa; NaN for what is not finite."""
    codes = torch.tensor(_exact_codes(), dtype=torch.float64, device=y.device)
    middle = (codes[1:] + codes[:-1]) / 2
    size = y.abs()
    at = torch.searchsorted(middle, size.contiguous())     # codes[at] is nearest; at a middle the lower one
    tie = (at < len(middle)) & (size == middle[at.clamp(max=len(middle) - 1)]) & (at % 2 == 1)
    out = torch.copysign(codes[at + tie.long()], y)
    return torch.where(y.isfinite(), out, math.nan)


def _exact_write(s, x, cache, scales):
    R, D = cache.shape[2], cache.shape[3]
    codes, bytes_ = cache.double(), scales.clone()
    old, new = s["old"].tolist(), s["new"].tolist()
    S = x.shape[1]
    tokens = x.double()
    table = None if s["table"] is None else s["table"].tolist()
    for b, (n0, n1) in enumerate(zip(old, new)):
        at = n0
        while at < n1:
            first = at - at % BLOCK
            end = min(n1, first + BLOCK)
            page, r = (b, first) if table is None else (table[b][first // R], first % R)
            rows = tokens[b, S - n1 + at:S - n1 + end].transpose(0, 1)                   # [Hkv, end - at, D]
            size = torch.where(rows.isfinite(), rows.abs(), 0.0).flatten(1).amax(-1)
            e = torch.full_like(size, -float(MOST))
            for _ in range(2 * MOST):
                e = torch.where((size > LARGEST * _two_to(e)) & (e < MOST), e + 1, e)
            if at > first:
                was = bytes_[page, :, r // BLOCK].double() - BIAS
                e = torch.maximum(e, was)
                codes[page, :, r:r + at - first] = _exact_round(codes[page, :, r:r + at - first] * _two_to(was - e)[:, None, None])
            y = rows / _two_to(e)[:, None, None]
            codes[page, :, r + at - first:r + end - first] = _exact_round(torch.where(y.isfinite(), y.clamp(-LARGEST, LARGEST), y))
            bytes_[page, :, r // BLOCK] = (e + BIAS).to(torch.uint8)
            at = end
    return codes, bytes_


def _exact_values(s, cache, scales):
    """All rows of all pages, as the values that they stand for."""
    out = cache.double()
    for x in range(scales.shape[2]):
        out[:, :, x * BLOCK:(x + 1) * BLOCK] *= _two_to(scales[:, :, x].long() - BIAS)[:, :, None, None]
    return out


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "write":
        (k, ks), (v, vs) = _exact_write(s, s["k"], s["k_cache"], s["k_scales"]), _exact_write(s, s["v"], s["v_cache"], s["v_scales"])
        return k, v, ks, vs
    if kind == "read":
        flat = s["slots"].long()
        out = []
        for name in ("k", "v"):
            values = _exact_values(s, s[name + "_cache"], s[name + "_scales"]).transpose(1, 2).flatten(0, 1)       # [slots, Hkv, D]
            out.append(values[flat].transpose(1, 2))
        return tuple(out)
    q, lens = s["q"].double(), s["lens"].tolist()
    B, H, Sq, D = q.shape
    Hkv = s["k_cache"].shape[1]
    out = torch.zeros(B, H, Sq, D, dtype=torch.float64, device="cuda")
    for b, n in enumerate(lens):
        pages = [b] if s["table"] is None else s["table"][b, :-(-n // s["k_cache"].shape[2])].tolist()
        k, v = (torch.cat([x for x in _exact_values(s, s[y + "_cache"][pages], s[y + "_scales"][pages])], dim=1)[:, :n] for y in ("k", "v"))
        hidden = torch.arange(n, device="cuda") > n - Sq + torch.arange(Sq, device="cuda")[:, None]
        for h in range(H):
            scores = (q[b, h] @ k[h // (H // Hkv)].T) / math.sqrt(D)
            if case["causal"]:
                scores[hidden] = -math.inf
            out[b, h] = torch.softmax(scores, dim=-1) @ v[h // (H // Hkv)]
    return out
