"""Performance cases of the operators around attention: trees of drafted tokens over a cache, the index tensors of a
serving step, and the normalisation and rotation of queries and keys.

`listed()` holds the fixed cases, `draw(rng)` gives further ones of the same ranges.  A case is a plain dict; its "kind"
names the entry point:

    mask    tree_mask               ancestor masks and depths of trees of drafted tokens
    step    cache_step              pages, slots and positions of the new tokens of every request
    rope    qk_norm_rope            queries and keys of a projection, normalised per head, rotated, in attention's layout
    bwd     qk_norm_rope_backward   their gradients, and the weights'
    write   qk_norm_rope_cache      the same for a serving step: keys and values go into the cache
    tree    sdpa_tree, sdpa_tree_paged   attention of a tree of drafted tokens over a dense or paged cache

`run` computes the operators in elementary torch operations, or with `own` through the library.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-6
THETA = 10000.0


def listed():
    return [
        # one sequence, a small tree of drafted tokens: host time and one launch
        dict(name="mask_single", kind="mask", B=1, T=15),
        # a batch of sequences with the widest trees that a serving step verifies
        dict(name="mask_batch", kind="mask", B=64, T=255),
        # one sequence being decoded: one token, one page at most; host time and one launch
        dict(name="step_single", kind="step", B=1, S=1, max_blocks=128, block_rows=64, tree=False),
        # a batch of requests, each with a tree of drafted tokens, or with fewer tokens of its own
        dict(name="step_batch", kind="step", B=256, S=60, max_blocks=64, block_rows=128, tree=True),
        # the vision regime of the benchmark trained: 196 patches on two axes (rows, columns) and a class token
        dict(name="rope_vision", kind="rope", B=64, S=197, H=12, Hkv=12, D=64, dtype="f16", rot=64, axes=2, interleaved=False, norm=True),
        # its long-context regime with grouped heads
        dict(name="rope_long", kind="rope", B=2, S=8192, H=32, Hkv=8, D=128, dtype="bf16", rot=128, axes=1, interleaved=False, norm=True),
        # a point of its S x D grid: the widest heads, part of each rotated, neighbouring values as pairs
        dict(name="bwd_grid_wide", kind="bwd", B=4, S=2048, H=16, Hkv=4, D=160, dtype="f16", rot=96, axes=1, interleaved=True, norm=True),
        # the long-context regime's backward
        dict(name="bwd_long", kind="bwd", B=2, S=8192, H=32, Hkv=8, D=128, dtype="bf16", rot=128, axes=1, interleaved=False, norm=True),
        # a decoding step of one sequence into a dense cache: latency
        dict(name="write_single", kind="write", B=1, S=1, H=32, Hkv=8, D=128, dtype="f16", rot=128, axes=1, interleaved=False, norm=True,
             cap=8192, block_rows=0),
        # prefill chunks of 512 tokens at most, each entry with a number of its own, into pages
        dict(name="write_chunk", kind="write", B=4, S=512, H=32, Hkv=8, D=128, dtype="bf16", rot=128, axes=1, interleaved=False, norm=True,
             cap=2048, block_rows=128),
        # one sequence, a tree of 64 drafted tokens, 8192 cached keys
        dict(name="tree_single", kind="tree", B=1, H=32, Hkv=8, T=64, Skv=8192, D=128, dtype="bf16", fill=1.0, block_rows=0),
        # a batch of sequences of different lengths, paged, with smaller trees, which is what a serving step verifies
        dict(name="tree_batch_paged", kind="tree", B=32, H=32, Hkv=8, T=15, Skv=8192, D=128, dtype="f16", fill=0.25, block_rows=128),
    ]


# what one drawn case may cost at most: the largest listed ones
MOST_BYTES = 1.0e9
MOST_FLOPS = 1.2e11


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    while True:
        kind = rng.choice(["mask", "step", "rope", "bwd", "write", "tree", "tree", "tree"])
        if kind == "mask":
            case = dict(kind=kind, B=_log_int(rng, 1, 256), T=_log_int(rng, 1, 512))
            if case["B"] * case["T"] > 1 << 14:
                continue
        elif kind == "step":
            case = dict(kind=kind, B=_log_int(rng, 1, 1024), S=_log_int(rng, 1, 1024), max_blocks=_log_int(rng, 8, 512),
                        block_rows=rng.choice([64, 128, 256]), tree=rng.random() < 0.4)
            if case["S"] * 2 > case["max_blocks"] * case["block_rows"] or case["B"] * case["max_blocks"] > 1 << 17:
                continue
        elif kind == "tree":
            group = rng.choice([1, 4, 8])
            hkv = _log_int(rng, 1, 32 // group)
            case = dict(kind=kind, B=_log_int(rng, 1, 64), H=hkv * group, Hkv=hkv, T=_log_int(rng, 1, 200), Skv=_log_int(rng, 256, 32768),
                        D=rng.choice([64, 96, 128, 160]), dtype=rng.choice(["f16", "bf16"]), fill=rng.choice([1.0, 0.5, 0.1]),
                        block_rows=rng.choice([0, 0, 64, 128, 256]))
            # (the plain form holds the scores, and the cache in 32 bits)
            if case["B"] * case["H"] * case["T"] * case["Skv"] > 1 << 28 or case["B"] * hkv * case["Skv"] * case["D"] > 1 << 28:
                continue
        else:
            group = rng.choice([1, 1, 4, 8])
            hkv = _log_int(rng, 1, 32 // group)
            D = rng.choice([64, 96, 128, 160])
            case = dict(kind=kind, B=_log_int(rng, 1, 64), S=_log_int(rng, 1, 16384), H=hkv * group, Hkv=hkv, D=D,
                        dtype=rng.choice(["f16", "bf16"]), rot=rng.choice([D, D, D, D // 2 // 16 * 16]), axes=rng.choice([1, 1, 2, 3]),
                        interleaved=rng.random() < 0.3, norm=rng.random() < 0.85)
            if kind == "write":
                rows = rng.choice([0, 64, 128, 256])
                case.update(S=_log_int(rng, 1, 1024), block_rows=rows, cap=-(-_log_int(rng, 1024, 8192) // 256) * 256)
                if case["B"] * hkv * case["cap"] * D > 1 << 25:
                    continue
        w = work(case)
        if w["flops"] <= MOST_FLOPS and w["bytes"] <= MOST_BYTES:
            return case


# ---- inputs

def _lengths(case):
    """Cached rows of each entry, the new ones included: spread evenly from fill * Skv to Skv."""
    B, Skv, fill = case["B"], case["Skv"], case["fill"]
    return [min(Skv, max(case["T"], int(Skv * (fill + (1.0 - fill) * (b + 0.5) / B)))) for b in range(B)]


def _parents(B, T, seed):
    """Trees of drafted tokens: a token follows one of the few before it, or the cached sequence."""
    rng = np.random.default_rng([seed, B, T])
    i = np.arange(T)
    back = rng.integers(1, 9, size=(B, T))
    return np.where(back > i, -1, i - back).astype(np.int32)


def _mask_words(parents):
    """Bit masks of _parents' trees on the host."""
    B, T = parents.shape
    reach = np.zeros((B, T, -(-T // 64) * 64), dtype=bool)
    for i in range(T):
        p = parents[:, i]
        reach[:, i] = np.where((p >= 0)[:, None], reach[np.arange(B), np.maximum(p, 0)], False)
        reach[:, i, i] = True
    return np.packbits(reach, axis=-1, bitorder="little").view(np.int64).reshape(B, T, -1)


def _rotation(case, g):
    """Inverse frequencies of the pairs, and which axis each of them turns with."""
    pairs, A = case["rot"] // 2, case["axes"]
    axis = torch.arange(pairs) * A // pairs
    first = torch.tensor([int((axis < a).sum()) for a in range(A)])
    count = torch.tensor([max(1, int((axis == a).sum())) for a in range(A)])
    within = torch.arange(pairs) - first[axis]
    inv_freq = (THETA ** (-within.double() / count[axis].double())).float()
    return inv_freq.cuda(), (axis.to(torch.int32).cuda() if A > 1 else None)


def prepare(case, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    kind = case["kind"]
    state = dict(case=case)
    if kind == "mask":
        state.update(parents=torch.from_numpy(_parents(case["B"], case["T"], seed)).cuda())
        return state
    if kind == "step":
        B, S, M, R = case["B"], case["S"], case["max_blocks"], case["block_rows"]
        rng = np.random.default_rng([seed, B, S])
        lens = rng.integers(0, M * R - S + 1, size=B)
        if B > 1:
            lens[0] = 0                                   # a new request
        counts = np.full(B, S)
        if B > 3:
            counts[rng.permutation(B)[:B // 4]] = rng.integers(0, S + 1, size=B // 4)      # requests with fewer tokens, or none
        held = -(-lens // R)
        order = rng.permutation(B * M).astype(np.int32)                                    # in no order, as a pool hands them out
        table = np.full((B, M), -1, dtype=np.int32)
        at = 0
        for b in range(B):
            table[b, :held[b]] = order[at:at + held[b]]
            at += held[b]
        free = np.full(B * M, -1, dtype=np.int32)
        free[:B * M - at] = order[at:]
        i32 = lambda x: torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()
        state.update(lens=i32(lens), counts=i32(counts), back=i32(-counts), table=i32(table), free=i32(free), pool=i32([B * M - at, 0]),
                     depths=None)
        if case["tree"]:
            parents, depth = _parents(B, S, seed), np.zeros((B, S), dtype=np.int32)
            for i in range(S):
                p = parents[:, i]
                depth[:, i] = np.where(p >= 0, depth[np.arange(B), np.maximum(p, 0)] + 1, 0)
            state.update(depths=i32(depth))
        return state

    dtype = DTYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(shape, dtype=torch.float32, device="cuda", generator=g).to(dtype)

    B, H, Hkv, D = case["B"], case["H"], case["Hkv"], case["D"]
    if kind == "tree":
        T, Skv, R = case["T"], case["Skv"], case["block_rows"]
        lens = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda")
        state.update(q=normal(B, H, T, D), lens=lens[torch.randperm(B, device="cuda", generator=g)].contiguous(),
                     mask=torch.from_numpy(_mask_words(_parents(B, T, seed))).cuda())
        if R == 0:
            state.update(k=normal(B, Hkv, Skv, D), v=normal(B, Hkv, Skv, D), table=None)
        else:
            M = -(-Skv // R)
            state.update(k=normal(B * M, Hkv, R, D), v=normal(B * M, Hkv, R, D),
                         table=torch.randperm(B * M, device="cuda", generator=g).to(torch.int32).view(B, M).contiguous())
        return state

    # q, k, v as views into the output of one projection
    S, A = case["S"], case["axes"]
    qkv = normal(B, S, (H + 2 * Hkv) * D)
    q, k, v = qkv.split([H * D, Hkv * D, Hkv * D], dim=-1)
    inv_freq, axes = _rotation(case, g)
    weights = [None, None]
    if case["norm"]:
        weights = [(1.0 + 0.1 * torch.randn(D, device="cuda", generator=g)).to(dtype) for _ in range(2)]
    state.update(q=q.view(B, S, H, D), k=k.view(B, S, Hkv, D), v=v.view(B, S, Hkv, D), qw=weights[0], kw=weights[1], inv_freq=inv_freq, axes=axes)
    if kind == "write":
        cap, R = case["cap"], case["block_rows"]
        new = torch.randint(S, cap + 1, (B,), device="cuda", generator=g) if S < cap else torch.full((B,), cap, device="cuda")
        count = torch.full((B,), S, device="cuda")
        if S > 1:
            count = torch.randint(max(1, S // 2), S + 1, (B,), device="cuda", generator=g)
        i = torch.arange(S, device="cuda")
        row = new[:, None] - S + i
        if R == 0:
            slots = torch.arange(B, device="cuda")[:, None] * cap + row
            P, R = B, cap
        else:
            M = cap // R
            P = B * M
            table = torch.randperm(P, device="cuda", generator=g).view(B, M)
            slots = table.gather(1, row // R) * R + row % R
        slots = torch.where(i >= S - count[:, None], slots, -1)
        state.update(slots=slots.to(torch.int32), k_cache=normal(P, Hkv, R, D), v_cache=normal(P, Hkv, R, D))
    else:
        row = torch.arange(S, device="cuda").expand(B, S)
    if A == 1:
        positions = row
    elif A == 2:
        side = max(1, math.isqrt(S))
        patch = (row - 1).clamp(min=0)                    # token 0 is the class token
        positions = torch.stack([patch // side, patch % side])
    else:
        positions = torch.stack([row // 64, row // 8 % 8, row % 8])      # time, height, width
    state.update(positions=positions.to(torch.int32).contiguous())
    if kind == "bwd":
        state.update(dq=normal(B, H, S, D), dk=normal(B, Hkv, S, D))
    return state


# ---- the operators in elementary operations

def _plain_mask(parents):
    B, T = parents.shape
    i = torch.arange(T, device=parents.device)
    above = torch.where((parents >= 0) & (parents < i), parents.long(), T)         # row T: no one
    above = torch.cat([above, torch.full((B, 1), T, dtype=torch.long, device=parents.device)], dim=1)
    reach = torch.zeros((B, T + 1, T), dtype=torch.bool, device=parents.device)
    reach[:, i, i] = True
    step = 1
    while step < T:                                       # after this reach holds the nearest 2 * step ancestors
        reach = reach | torch.gather(reach, 1, above[:, :, None].expand(-1, -1, T))
        above = torch.gather(above, 1, above)
        step *= 2
    reach = reach[:, :T]
    W = -(-T // 64)
    bits = torch.zeros((B, T, W * 64), dtype=torch.int64, device=parents.device)
    bits[:, :, :T] = reach
    words = (bits.view(B, T, W, 64) << torch.arange(64, device=parents.device)).sum(-1)
    return words, (reach.sum(-1) - 1).to(torch.int32)


def _plain_step(lens, counts, S, R, table, free, pool, depths):
    B, M = table.shape
    device = lens.device
    new = lens + counts
    held, need = -(-lens // R), -(-new // R)
    grow, drop = (need - held).clamp(min=0), (held - need).clamp(min=0)
    taken, dropped = grow.sum(), drop.sum()
    ok = (need <= M).all() & (taken - dropped <= pool[0]) & (new >= 0).all() & (counts <= S).all()
    missing = (taken - dropped - pool[0]).clamp(min=0) + (need - M).clamp(min=0).sum()
    column = torch.arange(M, device=device)[None]
    # pages that are given up, numbered in the order of their entries
    given = (column >= need[:, None]) & (column < held[:, None]) & ok
    number = (drop.cumsum(0) - drop)[:, None] + column - need[:, None]
    released = torch.zeros(B * M + 1, dtype=torch.int32, device=device)
    released[torch.where(given, number, B * M).view(-1)] = table.view(-1)
    # pages that are needed: released ones first, then the pool's, from its end
    wanted = (column >= held[:, None]) & (column < need[:, None]) & ok
    x = (grow.cumsum(0) - grow)[:, None] + column - held[:, None]
    from_pool = free[(pool[0] - 1 - (x - dropped)).clamp(0, free.numel() - 1)]
    page = torch.where(x < dropped, released[x.clamp(0, B * M)], from_pool)
    # what is left of the released ones goes back, the first of them on top
    back = given & (number >= taken)
    at = torch.where(back, pool[0] + dropped - 1 - number, free.numel()).view(-1)
    grown = torch.cat([free, free[:1]])
    grown[at] = torch.where(back, table, 0).view(-1)
    free.copy_(grown[:-1])
    table.copy_(torch.where(wanted, page, table))
    new = torch.where(ok, new, lens)
    row = new[:, None] - S + torch.arange(S, device=device)
    mine = (row >= lens[:, None]) & ok
    place = row.clamp(min=0)
    slots = torch.where(mine, table.gather(1, (place // R).clamp(max=M - 1).long()) * R + place % R, -1)
    positions = torch.where(mine, row if depths is None else new[:, None] - S + depths, 0)
    pool = torch.stack([torch.where(ok, pool[0] + dropped - taken, pool[0]), torch.where(ok, 0, missing)])
    return new.to(torch.int32), slots.to(torch.int32), positions.to(torch.int32), pool.to(torch.int32)


def _plain_angles(s):
    """cos and sin of every token's pairs, [B, S, 1, rot / 2]; angles in 64 bits."""
    f, p = s["inv_freq"].double(), s["positions"].double()
    if s["axes"] is None:
        phi = p[..., None] * f
    else:
        phi = p[s["axes"].long()].movedim(0, -1) * f
    return phi.cos().float()[:, :, None], phi.sin().float()[:, :, None]


def _pairs(x, rot, interleaved):
    """The two members of each pair, and what is not rotated."""
    if interleaved:
        return x[..., 0:rot:2], x[..., 1:rot:2], x[..., rot:]
    return x[..., :rot // 2], x[..., rot // 2:rot], x[..., rot:]


def _joined(a, b, rest, interleaved):
    both = torch.stack([a, b], dim=-1).flatten(-2) if interleaved else torch.cat([a, b], dim=-1)
    return torch.cat([both, rest], dim=-1)


def _plain_rope(s, x, w):
    case = s["case"]
    y = x.float()
    if w is not None:
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * w.float()
    cos, sin = _plain_angles(s)
    a, b, rest = _pairs(y, case["rot"], case["interleaved"])
    y = _joined(a * cos - b * sin, b * cos + a * sin, rest, case["interleaved"])
    return y.to(x.dtype).transpose(1, 2).contiguous()


def _plain_rope_backward(s, dy, x, w):
    case = s["case"]
    cos, sin = _plain_angles(s)
    a, b, rest = _pairs(dy.transpose(1, 2).float(), case["rot"], case["interleaved"])
    g = _joined(a * cos + b * sin, b * cos - a * sin, rest, case["interleaved"])
    if w is None:
        return g.to(x.dtype), None
    x32 = x.float()
    r = torch.rsqrt((x32 * x32).mean(-1, keepdim=True) + EPS)
    unit = x32 * r
    dw = (g * unit).sum((0, 1, 2))
    g = g * w.float()
    return ((g - unit * (g * unit).mean(-1, keepdim=True)) * r).to(x.dtype), dw.to(w.dtype)


def _plain_write(s, cache, x):
    """Rows x [B, S, Hkv, D] to the cache [P, Hkv, R, D] at their slots; rows without one go nowhere."""
    P, Hkv, R, D = cache.shape
    slot = s["slots"].view(-1).long()
    page, row = torch.where(slot >= 0, slot // R, 0), torch.where(slot >= 0, slot % R, 0)
    x = x.reshape(-1, Hkv, D)
    keep = (slot >= 0)[:, None, None]
    # (a row without a slot takes the place of another's first: written once more with what is there then)
    first = torch.argmax((slot >= 0).int())
    page, row = torch.where(slot >= 0, page, page[first]), torch.where(slot >= 0, row, row[first])
    cache[page, :, row] = torch.where(keep, x, x[first])


def _plain_tree(s):
    case = s["case"]
    q, k, v, lens = s["q"], s["k"], s["v"], s["lens"]
    B, H, T, D = q.shape
    if s["table"] is not None:
        Hkv, R = k.shape[1], k.shape[2]
        M = s["table"].shape[1]
        k = k[s["table"].long()].transpose(1, 2).reshape(B, Hkv, M * R, D)
        v = v[s["table"].long()].transpose(1, 2).reshape(B, Hkv, M * R, D)
    Hkv, n = k.shape[1], k.shape[2]
    scores = torch.matmul(q.float().view(B, Hkv, H // Hkv * T, D), k.float().transpose(-1, -2).contiguous()).view(B, H, T, n)
    scores *= 1.0 / math.sqrt(D)
    key = torch.arange(n, device=q.device)
    node = key[None] - (lens[:, None] - T)                # [B, n]: index of the drafted token, negative in the sequence before them
    words = torch.gather(s["mask"], 2, (node.clamp(0, T - 1) // 64)[:, None].expand(B, T, n))
    bit = (words >> (node.clamp(0, T - 1) % 64)[:, None]) & 1
    sees = ((node < 0)[:, None] | (bit != 0)) & (node < T)[:, None]
    scores.masked_fill_(~sees[:, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, Hkv, H // Hkv * T, n), v.float()).view(B, H, T, D)
    return (o / torch.where(total > 0, total, 1.0)).to(q.dtype)


def _run_plain(s):
    kind = s["case"]["kind"]
    if kind == "mask":
        return _plain_mask(s["parents"])
    if kind == "step":
        S, R = s["case"]["S"], s["case"]["block_rows"]
        new, slots, positions, pool = _plain_step(s["lens"], s["counts"], S, R, s["table"], s["free"], s["pool"], s["depths"])
        lens, _, _, left = _plain_step(new, s["back"], S, R, s["table"], s["free"], pool, None)
        return new, slots, positions, pool, lens, left, s["table"], s["free"]
    if kind == "tree":
        return _plain_tree(s)
    if kind == "rope":
        return _plain_rope(s, s["q"], s["qw"]), _plain_rope(s, s["k"], s["kw"])
    if kind == "bwd":
        (dq, dqw), (dk, dkw) = _plain_rope_backward(s, s["dq"], s["q"], s["qw"]), _plain_rope_backward(s, s["dk"], s["k"], s["kw"])
        return (dq, dk) if dqw is None else (dq, dk, dqw, dkw)
    q = _plain_rope(s, s["q"], s["qw"])
    _plain_write(s, s["k_cache"], _plain_rope(s, s["k"], s["kw"]).transpose(1, 2))
    _plain_write(s, s["v_cache"], s["v"])
    return q, s["k_cache"], s["v_cache"]


# ---- the library's

def _run_own(s):
    from paper_2603_01960_amd import binding as lib

    case = s["case"]
    kind = case["kind"]
    if kind == "mask":
        return lib.tree_mask(s["parents"])
    if kind == "step":
        S, R = case["S"], case["block_rows"]
        # a step's tokens are appended, then all of them dropped again, as rejected drafts are
        new, slots, positions, pool = lib.cache_step(s["lens"], s["counts"], S, R, pages=(s["table"], s["free"], s["pool"]), depths=s["depths"])
        lens, _, _, left = lib.cache_step(new, s["back"], S, R, pages=(s["table"], s["free"], pool))
        return new, slots, positions, pool, lens, left, s["table"], s["free"]
    if kind == "tree":
        if s["table"] is None:
            return lib.sdpa_tree(s["q"], s["k"], s["v"], s["mask"], kv_lens=s["lens"])
        return lib.sdpa_tree_paged(s["q"], s["k"], s["v"], s["lens"], s["table"], s["mask"])
    turn = dict(axes=s["axes"], eps=EPS, interleaved=case["interleaved"])
    if kind == "rope":
        return lib.qk_norm_rope(s["q"], s["k"], s["qw"], s["kw"], s["positions"], s["inv_freq"], **turn)
    if kind == "bwd":
        grads = lib.qk_norm_rope_backward(s["dq"], s["dk"], s["q"], s["k"], s["qw"], s["kw"], s["positions"], s["inv_freq"], **turn)
        return grads if case["norm"] else grads[:2]
    q = lib.qk_norm_rope_cache(s["q"], s["k"], s["v"], s["qw"], s["kw"], s["positions"], s["inv_freq"], s["k_cache"], s["v_cache"], s["slots"], **turn)
    return q, s["k_cache"], s["v_cache"]


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- what a pass cannot do without

def work(case):
    kind, B = case["kind"], case["B"]
    if kind == "mask":
        T = case["T"]
        return {"bytes": B * T * (4 + 4 + 8 * -(-T // 64)), "flops": B * T * -(-T // 64)}
    if kind == "step":
        S = case["S"]
        moved = B * (S // case["block_rows"] + 1)         # pages, about: read from the pool, written to the table, and back
        # both calls: lengths and counts in, lengths out, slots and positions out; depths in where there are some
        return {"bytes": 2 * (12 * B + 8 * B * S + 8 * moved) + (4 * B * S if case["tree"] else 0), "flops": 4 * B * S}
    H, Hkv, D = case["H"], case["Hkv"], case["D"]
    if kind == "tree":
        lens, T = _lengths(case), case["T"]
        keys = sum(n * T for n in lens)                   # (the few drafted tokens that a row does not see among them)
        return {"bytes": 2 * D * (2 * Hkv * sum(lens) + 2 * B * H * T) + 8 * B * T * -(-T // 64), "flops": 4 * D * H * keys}
    rows = B * case["S"] * (H + Hkv)
    turned = 3 * case["rot"] * rows
    if kind == "rope":
        return {"bytes": 4 * rows * D + 4 * B * case["S"] * case["axes"], "flops": 4 * D * rows + turned}
    if kind == "bwd":
        return {"bytes": 6 * rows * D + 4 * B * case["S"] * case["axes"], "flops": 10 * D * rows + turned}
    return {"bytes": 4 * (rows + B * case["S"] * Hkv) * D + 8 * B * case["S"], "flops": 4 * D * rows + turned}


# ---- the same from the definitions, in 64 bits

def _exact_step(s):
    case = s["case"]
    S, R, M = case["S"], case["block_rows"], case["max_blocks"]
    lens, counts = s["lens"].tolist(), s["counts"].tolist()
    table, stack = s["table"].tolist(), s["free"].tolist()
    top = int(s["pool"][0])
    depths = None if s["depths"] is None else s["depths"].tolist()
    news, slots, positions = [], [], []
    pages_of = lambda rows: (rows + R - 1) // R
    for b, (n, c) in enumerate(zip(lens, counts)):
        for x in range(pages_of(n), pages_of(n + c)):
            top -= 1
            table[b][x] = stack[top]
        news.append(n + c)
        at, where = [-1] * S, [0] * S
        for i in range(c):
            row = n + i
            at[S - c + i] = table[b][row // R] * R + row % R
            where[S - c + i] = row if depths is None else n + c - S + depths[b][S - c + i]
        slots.append(at)
        positions.append(where)
    # dropping the same tokens again puts the pages back where they were, so the pool is as before
    as_tensor = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    return (as_tensor(news), as_tensor(slots), as_tensor(positions), as_tensor([top, 0]), s["lens"], s["pool"], as_tensor(table), s["free"])


def _exact_mask(s):
    parents = s["parents"].tolist()
    B, T = s["parents"].shape
    W = -(-T // 64)
    words, depths = np.zeros((B, T, W), dtype=np.uint64), np.zeros((B, T), dtype=np.int32)
    for b in range(B):
        for i in range(T):
            j, n = i, 0
            while True:                                   # up to the root
                words[b, i, j // 64] |= np.uint64(1) << np.uint64(j % 64)
                above = parents[b][j]
                if not 0 <= above < j:
                    break
                j, n = above, n + 1
            depths[b, i] = n
    return torch.from_numpy(words.view(np.int64)).cuda(), torch.from_numpy(depths).cuda()


def _exact_turned(s, x, sign):
    """Complex numbers times e^(i phi): pairs as real and imaginary part."""
    case = s["case"]
    rot, half = case["rot"], case["rot"] // 2
    f = s["inv_freq"].double()
    phi = torch.empty(case["B"], case["S"], half, dtype=torch.float64, device="cuda")
    for i in range(half):
        p = s["positions"] if s["axes"] is None else s["positions"][int(s["axes"][i])]
        phi[..., i] = p.double() * f[i]
    turn = torch.polar(torch.ones_like(phi), sign * phi)[:, :, None]
    out = x.clone()
    first, second = (slice(0, rot, 2), slice(1, rot, 2)) if case["interleaved"] else (slice(0, half), slice(half, rot))
    z = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * turn
    out[..., first], out[..., second] = z.real, z.imag
    return out


def _exact_rope(s, x, w):
    y = x.double()
    if w is not None:
        y = w.double() * y / torch.sqrt(y.square().sum(-1, keepdim=True) / y.shape[-1] + EPS)
    return _exact_turned(s, y, 1.0).permute(0, 2, 1, 3).contiguous()


def _exact_backward(s, dy, x, w):
    g = _exact_turned(s, dy.double().permute(0, 2, 1, 3), -1.0)
    if w is None:
        return g, None
    x, w, D = x.double(), w.double(), x.shape[-1]
    root = torch.sqrt(x.square().sum(-1, keepdim=True) / D + EPS)
    # y = w x / root: dx_j = w_j g_j / root - x_j (sum_i g_i w_i x_i) / (D root^3)
    dx = w * g / root - x * (g * w * x).sum(-1, keepdim=True) / (D * root ** 3)
    return dx, (g * x / root).flatten(0, 2).sum(0)


def _exact_tree(s):
    q, lens = s["q"].double(), s["lens"].tolist()
    B, H, T, D = q.shape
    Hkv = s["k"].shape[1]
    words = s["mask"].cpu().numpy().view(np.uint64)
    out = torch.zeros(B, H, T, D, dtype=torch.float64, device="cuda")
    for b, n in enumerate(lens):
        if s["table"] is None:
            k, v = s["k"][b, :, :n].double(), s["v"][b, :, :n].double()
        else:
            R = s["k"].shape[2]
            pages = s["table"][b, :-(-n // R)].tolist()
            k = torch.cat([s["k"][p] for p in pages], dim=1)[:, :n].double()
            v = torch.cat([s["v"][p] for p in pages], dim=1)[:, :n].double()
        hidden = np.zeros((T, n), dtype=bool)
        for j in range(max(0, n - T), n):
            node = j - (n - T)
            hidden[:, j] = (words[b, :, node // 64] >> np.uint64(node % 64)) & np.uint64(1) == 0
        hidden = torch.from_numpy(hidden).cuda()
        for h in range(H):
            group = h // (H // Hkv)
            scores = (q[b, h] @ k[group].T) / math.sqrt(D)
            scores[hidden] = -math.inf
            out[b, h] = torch.softmax(scores, dim=-1) @ v[group]
    return out


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "mask":
        return _exact_mask(s)
    if kind == "step":
        return _exact_step(s)
    if kind == "tree":
        return _exact_tree(s)
    if kind == "rope":
        return _exact_rope(s, s["q"], s["qw"]), _exact_rope(s, s["k"], s["kw"])
    if kind == "bwd":
        (dq, dqw), (dk, dkw) = _exact_backward(s, s["dq"], s["q"], s["qw"]), _exact_backward(s, s["dk"], s["k"], s["kw"])
        return (dq, dk) if dqw is None else (dq, dk, dqw, dkw)
    k, v = _exact_rope(s, s["k"], s["kw"]), s["v"].double()
    k_cache, v_cache = s["k_cache"].double(), s["v_cache"].double()
    R = k_cache.shape[2]
    b, i = torch.nonzero(s["slots"] >= 0, as_tuple=True)
    slot = s["slots"][b, i].long()
    k_cache[slot // R, :, slot % R] = k[b, :, i]
    v_cache[slot // R, :, slot % R] = v[b, i]
    return _exact_rope(s, s["q"], s["qw"]), k_cache, v_cache
