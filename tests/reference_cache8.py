"""The 8-bit cache from its definition, in 64 bits and without the library: what its GPU tests compare with.  Everything is on the CPU."""
import math

import torch

ROWS, MOST, BIAS, LARGEST = 32, 62, 127, 448.0
POSITIVE = [m / 8 * 2.0 ** -6 for m in range(8)] + [(1 + m / 8) * 2.0 ** e for e in range(-6, 9) for m in range(8) if (e, m) != (8, 7)]
VALUES = torch.tensor(POSITIVE + [math.nan] + [-x for x in POSITIVE] + [math.nan], dtype=torch.float64)       # by code


def nearest(x):
    """Codes (uint8) of numbers: the nearest value, of two equally near ones that with the even mantissa; NaN for NaN.  |x| <= 448."""
    table = torch.tensor(POSITIVE, dtype=torch.float64)
    size = x.double().abs()
    at = torch.searchsorted((table[1:] + table[:-1]) / 2, size.contiguous())
    low, high = table[at], table[(at + 1).clamp(max=len(table) - 1)]
    at = torch.where((size * 2 == low + high) & (at % 2 == 1), at + 1, at)
    codes = at + 128 * torch.signbit(x.double())
    return torch.where(x.isnan(), 127, codes).to(torch.uint8)


def exponent(rows):
    """The least E with max |x| <= 448 * 2^E over the finite values of rows [..., n, D]."""
    x = rows.double()
    size = torch.where(x.isfinite(), x.abs(), 0.0).flatten(-2).amax(-1)
    e = torch.full_like(size, -MOST)
    for _ in range(2 * MOST):
        e = torch.where((size > LARGEST * 2.0 ** e) & (e < MOST), e + 1, e)
    return e


def scale_of(bytes_):
    """2^E of scale bytes."""
    return 2.0 ** (bytes_.double() - BIAS).clamp(-MOST, MOST)


def place(b, row, R, table):
    """(page, row in it) of an entry's row."""
    return (b, row) if table is None else (int(table[b][row // R]), row % R)


def write(x, codes, scales, old, new, table=None):
    """Writes x [B, S, Hkv, D] to codes uint8 [P, Hkv, R, D] and scales uint8 [P, Hkv, blocks], in place."""
    B, S = x.shape[:2]
    P, _, R, _ = codes.shape
    capacity = R if table is None else table.shape[1] * R
    for b in range(B):
        n0, n1 = max(int(old[b]), int(new[b]) - S, 0), min(int(new[b]), capacity)
        at = n0
        while at < n1:
            first = at // ROWS * ROWS
            end = min(n1, first + ROWS)
            page, r = place(b, first, R, table)
            if 0 <= page < P:
                rows = x[b, at - (int(new[b]) - S):end - (int(new[b]) - S)].transpose(0, 1).double()        # [Hkv, n, D]
                e = exponent(rows)
                held = min(int(old[b]), at) - first
                if held > 0:
                    was = (scales[page, :, r // ROWS].double() - BIAS).clamp(-MOST, MOST)
                    e = torch.maximum(e, was)
                    moved = nearest(VALUES[codes[page, :, r:r + held].long()] * (2.0 ** (was - e))[:, None, None])
                    grown = (e > was)[:, None, None]
                    codes[page, :, r:r + held] = torch.where(grown, moved, codes[page, :, r:r + held])
                y = rows / (2.0 ** e)[:, None, None]
                y = torch.where(y.isfinite(), y.clamp(-LARGEST, LARGEST), math.nan)
                codes[page, :, r + at - first:r + end - first] = nearest(y)
                scales[page, :, r // ROWS] = (e + BIAS).to(torch.uint8)
            at = end


def values(codes, scales):
    """What codes [P, Hkv, R, D] (uint8) stand for."""
    R = codes.shape[2]
    return VALUES[codes.long()] * scale_of(scales).repeat_interleave(ROWS, -1)[..., :R, None]


def gathered(codes, scales, lens, table, capacity):
    """(values, codes without scale) of each entry, [B] lists of [Hkv, n, D]."""
    v, c = values(codes, scales), VALUES[codes.long()]
    P, _, R, _ = codes.shape
    out = []
    for b, n in enumerate(lens):
        n = min(max(int(n), 0), capacity)
        if table is None:
            out.append((v[b, :, :n], c[b, :, :n]))
        else:
            pages = [min(max(int(p), 0), P - 1) for p in table[b, :-(-n // R)]]
            pick = lambda x: torch.cat([x[p] for p in pages] or [x[0, :, :0]], dim=1)[:, :n]
            out.append((pick(v), pick(c)))
    return out


def attention(q, k, v, u, causal=False, scale=None):
    """(o, lse, bound of o's error, of lse's) of q [B, H, Sq, D] over k, v: lists of (values, codes) [Hkv, n, D]; u: half a step of the result.

    The bound, for each value of the result.  A weight p_j that enters the product is off by: the FP32 error of its score, D + 8 roundings of a
    sum of |q k| (ds); its rounding to FP16, 2^-11 of it, or 2^-25 of the greatest product of weight and scale in the row where that
    is more; the sums over n keys add n + 16 roundings to FP32 of a sum of sizes A = sum p |v|; the normaliser has the first and the last of
    these too.  Then the result's own rounding.  (FP16's least step, where results are subnormal: 2^-25.)"""
    B, H, Sq, D = q.shape
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    o, lse = torch.zeros(B, H, Sq, D, dtype=torch.float64), torch.full((B, H, Sq), -math.inf, dtype=torch.float64)
    eo, el = torch.zeros_like(o), torch.zeros_like(lse)
    for b in range(B):
        Hkv, n = k[b][0].shape[:2]
        seen = torch.ones(Sq, n, dtype=torch.bool)
        if causal:
            seen = torch.arange(n) <= n - Sq + torch.arange(Sq)[:, None]
        for h in range(H):
            g = h // (H // Hkv)
            kk, vv, cc = k[b][0][g], v[b][0][g], v[b][1][g]
            x = q[b, h].double().cpu()
            s = scale * (x @ kk.T)
            ds = (D + 8) * 2.0 ** -24 * abs(scale) * (x.abs() @ kk.abs().T)
            s = s.masked_fill(~seen, -math.inf)
            some = seen.any(-1)
            if not some.any():
                continue
            m = s[some]
            p = torch.softmax(m, -1)
            # (0 * NaN of what a row does not see is nothing)
            clean = lambda w, y: torch.stack([w[i, seen[some][i]] @ y[seen[some][i]] for i in range(len(w))])
            A = clean(p, vv.abs())
            off = (torch.where(seen[some], ds[some], 0.0).amax(-1) + (n + 16) * 2.0 ** -24 + 2.0 ** -21)[:, None]
            size = torch.where(cc == 0, 0.0, (vv / torch.where(cc == 0, 1.0, cc)).abs())        # 2^E of each value
            top = (p[:, :, None] * torch.where(seen[some][:, :, None], torch.nan_to_num(size), 0.0)).flatten(1).amax(-1)
            small = top[:, None] * 2.0 ** -25 * clean(seen[some].double(), cc.abs())
            o[b, h, some] = clean(p, vv)
            lse[b, h, some] = torch.logsumexp(m, -1)
            eo[b, h, some] = u * o[b, h, some].abs() + (1 + u) * (A * (2.0 ** -11 + 2 * off) + small) + 2.0 ** -25
            el[b, h, some] = off[:, 0] + 2.0 ** -22 * lse[b, h, some].abs()
    return o, lse, eo, el
