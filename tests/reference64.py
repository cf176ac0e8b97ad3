"""The operators around attention from their definitions, in 64 bits and without the library: what their GPU tests compare with."""
import math

import torch

U = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}       # half a step, relative


def ancestors(parents):
    """For each token of a tree (a list of parents) the set of itself and those it follows, and how many these are."""
    sets = []
    for i, p in enumerate(parents):
        sets.append({i} | (sets[p] if 0 <= p < i else set()))
    return sets, [len(s) - 1 for s in sets]


def words_of(sets, T):
    """Sets of tokens as rows of 64-bit words."""
    out = torch.zeros(len(sets), (T + 63) // 64, dtype=torch.int64)
    for i, s in enumerate(sets):
        for j in s:
            out[i, j // 64] |= torch.tensor(-(1 << 63) if j % 64 == 63 else 1 << (j % 64))
    return out


def tree_attention(q, k, v, lens, sees, scale=None):
    """(o, lse): q [B, H, T, D] over the first lens[b] rows of k, v [B, Hkv, n, D]; sees[b][i]: the tokens that token i sees."""
    B, H, T, D = q.shape
    Hkv = k.shape[1]
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    o, lse = torch.zeros(B, H, T, D, dtype=torch.float64), torch.full((B, H, T), -math.inf, dtype=torch.float64)
    for b in range(B):
        n = min(max(int(lens[b]), 0), k.shape[2])
        seen = torch.zeros(T, n, dtype=torch.bool)
        seen[:, :max(0, n - T)] = True
        for i in range(T):
            for j in sees[b][i]:
                if j < T and n - T + j >= 0:
                    seen[i, n - T + j] = True
        for h in range(H):
            kk, vv = k[b, h // (H // Hkv), :n].double().cpu(), v[b, h // (H // Hkv), :n].double().cpu()
            x = (q[b, h].double().cpu() @ kk.T) * scale
            for i in range(T):
                m = seen[i]
                if m.any():
                    xi = x[i, m]
                    lse[b, h, i] = torch.logsumexp(xi, 0)
                    o[b, h, i] = torch.softmax(xi, 0) @ vv[m]
    return o, lse


def step(lens, counts, S, R, table=None, free=None, have=0, depths=None, capacity=None):
    """A cache step on lists; table and free are changed in place.  (new_lens, slots, positions, [have, missing])"""
    B = len(lens)
    pages = lambda n: -(-n // R)
    most = R if table is None else len(table[0]) * R if B else 0
    nothing = [[-1] * S for _ in range(B)], [[0] * S for _ in range(B)]
    if any(n < 0 or n > most or n + c < 0 or c > S for n, c in zip(lens, counts)) or (table is not None and not 0 <= have <= len(free)):
        return list(lens), *nothing, [have, -1]
    new = [n + c for n, c in zip(lens, counts)]
    over = sum(max(0, (n - most if table is None else pages(n) - most // R)) for n in new)
    if table is not None:
        kept = [min(n, most) for n in new]
        lack = max(0, sum(max(0, pages(b) - pages(a)) - max(0, pages(a) - pages(b)) for a, b in zip(lens, kept)) - have)
        if over or lack:
            return list(lens), *nothing, [have, over + lack]
        given = [table[b][x] for b in range(B) for x in range(pages(new[b]), pages(lens[b]))]
        stack = free[:have]
        wanted = [(b, x) for b in range(B) for x in range(pages(lens[b]), pages(new[b]))]
        for i, (b, x) in enumerate(wanted):
            table[b][x] = given[i] if i < len(given) else stack.pop()
        stack += reversed(given[len(wanted):])
        free[:len(stack)] = stack
        have = len(stack)
    elif over:
        return list(lens), *nothing, [have, over]
    slots, positions = nothing
    for b in range(B):
        for i in range(S):
            row = new[b] - S + i
            if row >= lens[b]:
                slots[b][i] = (b if table is None else table[b][row // R]) * R + row % R
                positions[b][i] = row if depths is None else new[b] - S + depths[b][i]
    return new, slots, positions, [have, 0]


def angles(positions, inv_freq, axes, B, S):
    """[B, S, rot / 2]"""
    p, f = positions.cpu().double(), inv_freq.cpu().double()
    if axes is None:
        return p.expand(B, S)[..., None] * f
    p = p if p.dim() == 3 else p[:, None].expand(-1, B, -1)
    return torch.stack([p[int(a)] for a in axes], dim=-1) * f if len(axes) else torch.zeros(B, S, 0, dtype=torch.float64)


def rotate(x, phi, interleaved):
    """x [B, S, H, D] turned by phi [B, S, rot / 2]."""
    rot = 2 * phi.shape[-1]
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    c, s = phi.cos()[:, :, None], phi.sin()[:, :, None]
    out = x.clone()
    first, second = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    out[..., first], out[..., second] = a * c - b * s, b * c + a * s
    return out


def norm_rope(x, w, phi, eps, interleaved):
    """[B, heads, S, D] of x [B, S, heads, D] in 64 bits."""
    y = x.double().cpu()
    if w is not None:
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps) * w.double().cpu()
    return rotate(y, phi, interleaved).transpose(1, 2)


def norm_rope_backward(dy, x, w, phi, eps, interleaved):
    """(dx, dw, sizes of the terms of dx row by row, of those of dw)"""
    g = rotate(dy.double().cpu().transpose(1, 2), -phi, interleaved)
    if w is None:
        return g, None, g.abs().amax(-1, keepdim=True), None
    x, w = x.double().cpu(), w.double().cpu()
    r = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    u, gw = x * r, g * w
    dx = r * (gw - u * (gw * u).mean(-1, keepdim=True))
    size = r * (gw.abs().amax(-1, keepdim=True) + u.abs().amax(-1, keepdim=True) * (gw * u).abs().mean(-1, keepdim=True))
    # A term of dw is g * u with g = a cos - b sin: the error of g is one of |a| + |b|, which cancel (a = b = 1, an angle of 45 degrees:
    # g = 0, computed with an error of 2^-24 and more), so that it is bounded by the gradients of the row, not by g.
    return dx, (g * u).sum((0, 1, 2)), size, (2 * g.abs().amax(-1, keepdim=True) * u.abs()).sum((0, 1, 2))
