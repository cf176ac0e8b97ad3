"""The 8-bit cache against its definition (tests/reference_cache8.py): writing bit for bit, reading exactly, attention within bounds that the
reference derives from the roundings."""
import math

import pytest
import torch

import reference_cache8 as ref
from paper_2603_01960_amd import binding as lib

pytestmark = pytest.mark.gpu

U = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
DTYPES = [torch.float16, torch.bfloat16]


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def new_cache(pages, Hkv, R, D, seed=0):
    """Codes and scales of all kinds, NaN among them: what a cache's memory may hold before anything is written."""
    g = torch.Generator().manual_seed(seed)
    out = [torch.randint(0, 256, (pages, Hkv, R, D), dtype=torch.uint8, generator=g) for _ in range(2)]
    out += [torch.randint(0, 256, (pages, Hkv, -(-R // 32)), dtype=torch.uint8, generator=g) for _ in range(2)]
    return out


def on_gpu(host):
    k, v, ks, vs = (x.cuda() for x in host)
    return k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn), ks, vs


def same_bytes(dev, host):
    for got, want, name in zip(dev, host, ("k_cache", "v_cache", "k_scales", "v_scales")):
        got = got.view(torch.uint8).cpu()
        if got.dim() == 4:                                # (any NaN is one)
            nan = lambda x: (x & 127) == 127
            assert torch.equal(nan(got), nan(want)), name
            got, want = got.masked_fill(nan(got), 0), want.masked_fill(nan(want), 0)
        bad = (got != want).nonzero()
        assert not len(bad), f"{name}: {len(bad)} differ, the first at {bad[0].tolist()}"


def tokens(B, S, Hkv, D, dtype, seed, spread=2.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(B, S, 2 * Hkv, D, generator=g) * torch.exp2(spread * torch.randn(B, S, 2 * Hkv, 1, generator=g))
    return x.to(dtype).cuda().view(B, S, 2 * Hkv * D)


def halves(x, Hkv, D):
    """k, v as views into one projection's output."""
    B, S = x.shape[:2]
    k, v = x.split([Hkv * D, Hkv * D], dim=-1)
    return k.view(B, S, Hkv, D), v.view(B, S, Hkv, D)


def write_both(host, dev, k, v, old, new, table=None):
    lib.cache8_write(k, v, *dev, i32(old), i32(new), block_table=None if table is None else table.cuda())
    for x, codes, scales in ((k, host[0], host[2]), (v, host[1], host[3])):
        ref.write(x.cpu(), codes, scales, old, new, table)


def pages_for(B, blocks, seed=0):
    g = torch.Generator().manual_seed(seed)
    return torch.randperm(B * blocks + 3, generator=g)[:B * blocks].to(torch.int32).view(B, blocks)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [64, 96, 128, 160])
@pytest.mark.parametrize("R", [0, 64])
def test_write_and_append(dtype, D, R):
    """Prefill, single tokens into full and partly filled blocks, drops, tokens that begin and end inside blocks."""
    B, Hkv, cap = 4, 3, 197 if R == 0 else 192
    table = None if R == 0 else pages_for(B, 3)
    host = new_cache(B if R == 0 else B * 3 + 3, Hkv, R or cap, D, seed=D)
    dev = on_gpu(host)
    lens = [0, 0, 0, 0]
    for step, counts in enumerate([[33, 1, 0, 90], [1, 1, 1, 1], [1, 31, 5, 0], [-40, -3, 1, 2], [30, 30, 30, 30], [1, 1, 1, 1], [64, 2, 64, 40]]):
        new = [n + c for n, c in zip(lens, counts)]
        S = max(1, max(counts))
        k, v = halves(tokens(B, S, Hkv, D, dtype, 100 * D + step), Hkv, D)
        write_both(host, dev, k, v, lens, new, table)
        same_bytes(dev, host)
        lens = [max(0, n) for n in new]


@pytest.mark.parametrize("dtype", DTYPES)
def test_write_values(dtype):
    """Ties, the largest code, zeros of both signs, the least and greatest magnitudes of the type, infinities, NaN."""
    Hkv, D, cap = 1, 64, 320
    top, least = torch.finfo(dtype).max, torch.finfo(dtype).smallest_normal
    x = torch.zeros(1, cap, 2 * Hkv, D)
    x[0, 0:32] = torch.linspace(-448, 448, 32 * 2 * D).view(32, 2, D)                       # a scale of 1: near and on ties
    x[0, 32:64] = 0.0
    x[0, 64:96] = -0.0
    x[0, 96] = 449.0                                                                         # a scale of 2
    x[0, 97:128] = torch.arange(31 * 2 * D).view(31, 2, D) / 64.0
    x[0, 128] = top
    x[0, 129:160] = least
    x[0, 160:192] = least * torch.arange(1, 33).view(32, 1, 1) / 32                          # subnormals
    x[0, 192] = math.inf
    x[0, 193] = -math.inf
    x[0, 194] = math.nan
    x[0, 195:224] = 3.0
    x[0, 224:256] = math.inf                                                                 # nothing finite
    x[0, 256, :, 0] = 448.0
    x[0, 256, :, 1:] = 2.0 ** -10 * torch.arange(D - 1)                                      # below the normal codes: ties among them
    x[0, 288] = 1e-12 if dtype == torch.bfloat16 else 2.0 ** -20
    k, v = halves(x.to(dtype).cuda().view(1, cap, 2 * Hkv * D), Hkv, D)
    host = new_cache(1, Hkv, cap, D)
    dev = on_gpu(host)
    write_both(host, dev, k, v, [0], [cap])
    same_bytes(dev, host)


def test_saturation_and_the_least_scale():
    Hkv, D = 2, 128
    x = torch.full((1, 64, 2 * Hkv, D), 3e38)
    x[0, 1] = 448.0 * 2.0 ** 62
    x[0, 2] = -3e38
    x[0, 32:] = 2.0 ** -71
    x[0, 33] = 2.0 ** -72
    x[0, 34] = 1.5 * 2.0 ** -72
    k, v = halves(x.to(torch.bfloat16).cuda().view(1, 64, -1), Hkv, D)
    host = new_cache(1, Hkv, 64, D)
    dev = on_gpu(host)
    write_both(host, dev, k, v, [0], [64])
    same_bytes(dev, host)
    assert host[2].view(-1).tolist() == [189, 65] * 2


def test_growth_keeps_the_older_rows():
    """A block whose scale grows step by step: the older rows' codes move each time."""
    Hkv, D = 2, 96
    host = new_cache(1, Hkv, 50, D)
    dev = on_gpu(host)
    for i in range(40):
        k, v = halves((tokens(1, 1, Hkv, D, torch.bfloat16, i, spread=0.0).float() * 2.0 ** (i * 1.3)).to(torch.bfloat16), Hkv, D)
        write_both(host, dev, k, v, [i], [i + 1])
    same_bytes(dev, host)
    big = (torch.ones(1, 1, 2 * Hkv * D) * 1e30).to(torch.bfloat16).cuda()                    # everything older vanishes
    write_both(host, dev, *halves(big, Hkv, D), [40], [41])
    same_bytes(dev, host)


@pytest.mark.parametrize("R", [0, 64])
def test_lengths_that_write_nothing_or_less(R):
    """Refused steps, drops, lengths that cannot be, more tokens than fit, fewer lengths than tokens."""
    Hkv, D, cap, B = 2, 64, 128, 8
    table = None if R == 0 else pages_for(B, 2)
    host = new_cache(B if R == 0 else 2 * B + 3, Hkv, R or cap, D)
    dev = on_gpu(host)
    old = [5, 100, 0, 120, -7, 128, 3, 2 ** 31 - 1]
    new = [5, 60, 0, 140, 20, 129, -(2 ** 31), 2 ** 31 - 1]
    k, v = halves(tokens(B, 25, Hkv, D, torch.float16, 1), Hkv, D)
    write_both(host, dev, k, v, old, new, table)
    same_bytes(dev, host)
    # a step whose tokens are fewer than the rows between the lengths: the last of them are written, the block's older rows stay
    write_both(host, dev, k[:, :3].contiguous(), v[:, :3].contiguous(), [3] * B, [20] * B, table)
    same_bytes(dev, host)


def test_pages_that_do_not_exist_are_not_written_to():
    Hkv, D, R, P = 2, 64, 64, 4
    host = new_cache(P, Hkv, R, D)
    dev = on_gpu(host)
    table = torch.tensor([[-1, 2], [P, 0], [2 ** 31 - 1, -2 ** 31]], dtype=torch.int32)
    k, v = halves(tokens(3, 100, Hkv, D, torch.float16, 1), Hkv, D)
    write_both(host, dev, k, v, [0, 0, 0], [100, 100, 100], table)
    same_bytes(dev, host)


@pytest.mark.parametrize("S,Hkv,B", [(1, 1, 1), (1, 8, 130), (700, 5, 2), (33, 1, 3)])
def test_write_sizes_and_strides(S, Hkv, B):
    D, cap = 128, 768
    x = tokens(B, S, Hkv + 1, D, torch.float16, S)
    whole = x.view(B, S, 2 * (Hkv + 1), D)
    k, v = whole[:, :, 1:Hkv + 1], whole.transpose(0, 1).contiguous().transpose(0, 1)[:, :, Hkv + 1:2 * Hkv + 1]
    host = new_cache(B, Hkv, cap, D)
    dev = on_gpu(host)
    old = [(7 * b) % (cap - S) for b in range(B)]
    write_both(host, dev, k, v, old, [n + S for n in old])
    same_bytes(dev, host)
    # as attention's layout has them: [B, Hkv, S, D] seen as [B, S, Hkv, D]; and one row for all tokens
    k, v = k.transpose(1, 2).contiguous().transpose(1, 2), v[:, :1].expand(B, S, Hkv, D)
    write_both(host, dev, k, v, old, [n + S for n in old])
    same_bytes(dev, host)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [64, 96, 128, 160])
def test_read(dtype, D):
    P, Hkv, R = 5, 3, 70
    host = new_cache(P, Hkv, R, D, seed=D)
    dev = on_gpu(host)
    slots = torch.randint(0, P * R, (4, 37), generator=torch.Generator().manual_seed(D)).to(torch.int32)
    slots[0, :5] = torch.tensor([-1, -2 ** 31, P * R, 2 ** 31 - 1, P * R - 1])
    slots[1, 7] = slots[1, 6]
    got = lib.cache8_read(*dev, slots.cuda(), dtype)
    given = tuple(torch.full((4, Hkv, 37, D), 7.0, dtype=dtype, device="cuda") for _ in range(2))
    again = lib.cache8_read(*dev, slots.cuda(), dtype, out=given)
    for t, (codes, scales) in enumerate(((host[0], host[2]), (host[1], host[3]))):
        x = ref.values(codes, scales).transpose(1, 2).reshape(P * R, Hkv, D)
        inside = (slots >= 0) & (slots < P * R)
        want = torch.where(inside[..., None, None], x[slots.long().clamp(0, P * R - 1)], 0.0).transpose(1, 2).to(dtype)
        assert torch.equal(torch.nan_to_num(got[t].cpu().double(), 1e300), torch.nan_to_num(want.double(), 1e300))
        assert torch.equal(got[t].isnan().cpu(), want.isnan())
        assert again[t].data_ptr() == given[t].data_ptr() and torch.equal(again[t].view(torch.int16), got[t].view(torch.int16))


def filled(B, Hkv, cap, D, lens, R=0, seed=0, spread=1.5, dtype=torch.bfloat16):
    """A cache whose rows below lens hold tokens, and all others whatever new_cache gives; (host, dev, table)."""
    blocks = -(-cap // R) if R else 0
    table = pages_for(B, blocks, seed) if R else None
    host = new_cache(B * blocks + 3 if R else B, Hkv, R or cap, D, seed)
    dev = on_gpu(host)
    x = tokens(B, cap, Hkv, D, dtype, seed + 1, spread)
    k, v = halves(x, Hkv, D)
    # (the tokens of an entry are the last of its row)
    lib.cache8_write(k, v, *dev, i32([0] * B), i32(lens), block_table=None if table is None else table.cuda())
    return [x.view(torch.uint8).cpu() for x in dev], dev, table


def check_attention(q, host, dev, lens, table, cap, causal=False, scale=None, u=None, **more):
    lens_gpu = None if lens is None else i32(lens)
    if table is None:
        got = lib.sdpa_kv8(q, *dev, causal=causal, scale=scale, kv_lens=lens_gpu, return_lse=True, **more)
    else:
        got = lib.sdpa_paged8(q, *dev, lens_gpu, table.cuda(), causal=causal, scale=scale, return_lse=True, **more)
    lens = [cap] * q.shape[0] if lens is None else lens
    k, v = ref.gathered(host[0], host[2], lens, table, cap), ref.gathered(host[1], host[3], lens, table, cap)
    o, lse, eo, el = ref.attention(q.cpu(), k, v, U[q.dtype], causal, scale)
    off = (got[0].cpu().double() - o).abs()
    assert torch.equal(got[0].isnan().cpu(), o.isnan())
    fine = ~o.isnan()
    worst = (off - eo)[fine].max().item() if fine.any() else 0.0
    assert worst <= 0, f"off by {worst} more than the bound; worst share {(off / eo)[fine].max().item()}"
    fine = lse.isfinite()
    number = ~lse.isnan()
    assert torch.equal(torch.isneginf(got[1]).cpu()[number], torch.isneginf(lse)[number])
    assert ((got[1].cpu().double() - lse).abs() <= el)[fine].all()
    return got


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [64, 96, 128, 160])
@pytest.mark.parametrize("R", [0, 64, 256])
def test_decoding_steps(dtype, D, R):
    """One token per head; lengths at and around the ends of blocks, tiles and pages."""
    B, H, Hkv, cap = 8, 8, 2, 500 if R == 0 else 512
    lens = [1, 31, 32, 33, 64, 257, 0, 500]
    host, dev, table = filled(B, Hkv, cap, D, lens, R, seed=D + R, dtype=dtype)
    q = torch.randn(B, H, 1, D, generator=torch.Generator().manual_seed(1)).to(dtype).cuda()
    check_attention(q, host, dev, lens, table, cap, causal=True)
    check_attention(q, host, dev, lens, table, cap, causal=False)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [64, 96, 128, 160])
@pytest.mark.parametrize("Sq", [2, 5, 17, 33, 70, 130])
@pytest.mark.parametrize("causal", [False, True])
def test_blocks_of_queries(dtype, D, Sq, causal):
    """Drafts and chunks; entries shorter than the block of queries, whose first rows see no key."""
    for G, R in ((1, 0), (4, 64), (3, 128)):
        B, Hkv, cap = 3, 2, 300 if R == 0 else 384
        lens = [300, max(0, Sq - 2), 197]
        host, dev, table = filled(B, Hkv, cap, D, lens, R, seed=Sq + R, dtype=dtype)
        q = torch.randn(B, G * Hkv, Sq, D, generator=torch.Generator().manual_seed(Sq)).to(dtype).cuda()
        check_attention(q, host, dev, lens, table, cap, causal=causal)


@pytest.mark.parametrize("splits", [1, 2, 3, 7, 64, 128])
@pytest.mark.parametrize("G,Sq", [(1, 1), (4, 1), (4, 5), (8, 3), (2, 40)])
def test_splits(splits, G, Sq):
    B, Hkv, cap, D = 2, 2, 1000, 128
    lens = [1000, 77]
    host, dev, table = filled(B, Hkv, cap, D, lens, 0, seed=splits)
    q = torch.randn(B, G * Hkv, Sq, D, generator=torch.Generator().manual_seed(Sq)).to(torch.bfloat16).cuda()
    a = check_attention(q, host, dev, lens, table, cap, causal=True, splits=splits)
    b = check_attention(q, host, dev, lens, table, cap, causal=True, splits=splits)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("scale", [0.0, -0.3, 2.5])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("Sq", [1, 40])
def test_scales(scale, dtype, Sq):
    host, dev, table = filled(2, 2, 200, 96, [200, 130], 0, seed=3, spread=0.5)
    q = torch.randn(2, 4, Sq, 96, generator=torch.Generator().manual_seed(Sq)).to(dtype).cuda()
    check_attention(q, host, dev, [200, 130], table, 200, causal=True, scale=scale)


@pytest.mark.parametrize("Sq", [1, 6, 50])
@pytest.mark.parametrize("dtype", DTYPES)
def test_blocks_of_very_different_scales(Sq, dtype):
    """Exponents at both ends and between them, in K (with queries that keep the scores small) and in V."""
    B, Hkv, cap, D = 1, 2, 320, 64
    host, dev, table = filled(B, Hkv, cap, D, [cap], 0, seed=9, spread=0.0)
    host[3][...] = torch.tensor([127, 65, 189, 127, 100, 150, 65, 189, 120, 130], dtype=torch.uint8)
    if dtype == torch.float16:
        host[3].clamp_(max=127 + 6)                       # (results in FP16's range)
    host[2][...] = torch.tensor([127, 65, 120, 127, 128, 100, 90, 126, 125, 124], dtype=torch.uint8)
    dev = on_gpu(host)
    q = (0.1 * torch.randn(B, 4, Sq, D, generator=torch.Generator().manual_seed(Sq))).to(dtype).cuda()
    check_attention(q, host, dev, [cap], table, cap, causal=True)


@pytest.mark.parametrize("Sq", [1, 9, 70])
@pytest.mark.parametrize("R", [0, 64])
def test_nan_reaches_the_rows_that_see_it(Sq, R):
    B, Hkv, cap, D = 2, 2, 256, 128
    lens = [256, 150]
    host, dev, table = filled(B, Hkv, cap, D, lens, R, seed=2)
    for codes, row, col in ((1, 255, 3), (1, 252, 77), (0, 254, 5), (1, 149, 9), (0, 148, 127)):
        b = 0 if row > 200 else 1
        page, r = ref.place(b, row, R or cap, table)
        host[codes][page, 1, r, col] = 0x7f if col & 1 else 0xff
    dev = on_gpu(host)
    q = torch.randn(B, 2 * Hkv, Sq, D, generator=torch.Generator().manual_seed(Sq)).to(torch.bfloat16).cuda()
    check_attention(q, host, dev, lens, table, cap, causal=True)
    check_attention(q, host, dev, lens, table, cap, causal=False)


def test_write_up_to_the_last_row_that_can_be_counted():
    """An entry of nearly 2^31 rows, all but the last of whose pages do not exist, and more tokens (one in memory) than it has room for."""
    blocks, D = (2 ** 31 - 1) // 64, 64
    table = torch.full((1, blocks), -1, dtype=torch.int32, device="cuda")
    table[0, -1] = 1
    dev = on_gpu(new_cache(3, 1, 64, D, 1))
    before = [x.clone().view(torch.uint8) for x in dev]
    x = torch.randn(1, 1, 1, D, generator=torch.Generator().manual_seed(1)).half().cuda()
    S = 2 ** 29
    lib.cache8_write(x.expand(1, S, 1, D), (2 * x).expand(1, S, 1, D), *dev, i32([blocks * 64 - 64]), i32([blocks * 64]), block_table=table)
    for got, old in zip(dev, before):
        got = got.view(torch.uint8)
        assert torch.equal(got[0], old[0]) and torch.equal(got[2], old[2])
    k, v = lib.cache8_read(*dev, torch.arange(64, 128, dtype=torch.int32, device="cuda").view(1, 64), torch.float16)
    for got, want in ((k, x), (v, 2 * x)):
        want = want.cpu().double().view(1, 1, 1, D)
        assert ((got.cpu().double() - want).abs() <= want.abs() * 2 ** -4 + 2.0 ** -10 * 2 ** -6).all()


# Large tiles of query rows are taken for many of them and many scores, counted by the capacity: a cache of many heads and a large capacity whose entries are short.
LARGE = 1 << 14


def in_large(dev, table, rows):
    """The cache and block table with a capacity of `rows`; what is added holds NaN codes, pages that do not exist."""
    if table is not None:
        wide = torch.full((table.shape[0], rows // dev[0].shape[2]), 2 ** 31 - 1, dtype=torch.int32)
        wide[:, :table.shape[1]] = table
        return dev, wide
    B, Hkv, cap, D = dev[0].shape
    out = []
    for x, shape in zip(dev, [(B, Hkv, rows, D)] * 2 + [(B, Hkv, rows // 32)] * 2):
        y = torch.full(shape, 0x7f, dtype=torch.uint8, device="cuda")
        y[:, :, :x.shape[2]] = x.view(torch.uint8)
        out.append(y.view(x.dtype))
    return out, None


def check_large(q, host, dev, lens, table, cap, causal, scale=None, **more):
    """Some heads of it: the first two and the last."""
    B, H, Sq, D = q.shape
    Hkv = host[0].shape[1]
    G, small = H // Hkv, -(-H // Hkv * Sq // 32)
    assert B * Hkv * small > 1024 and 2 * small > 7 * -(-small // 4) and B * H * Sq * LARGE > 1 << 28       # (what it takes)
    dev, wide = in_large(dev, table, LARGE)
    lens_gpu = i32(lens)
    if wide is None:
        o, lse = lib.sdpa_kv8(q, *dev, causal=causal, scale=scale, kv_lens=lens_gpu, return_lse=True, **more)
    else:
        o, lse = lib.sdpa_paged8(q, *dev, lens_gpu, wide.cuda(), causal=causal, scale=scale, return_lse=True, **more)
    groups = [0, 1, Hkv - 1]
    heads = [g * G + i for g in groups for i in range(G)]
    some = [x[:, groups] for x in host]
    k, v = ref.gathered(some[0], some[2], lens, table, cap), ref.gathered(some[1], some[3], lens, table, cap)
    want, want_lse, eo, el = ref.attention(q[:, heads].cpu(), k, v, U[q.dtype], causal, scale)
    got, got_lse = o[:, heads].cpu().double(), lse[:, heads].cpu().double()
    assert torch.equal(got.isnan(), want.isnan())
    off, fine = (got - want).abs(), ~want.isnan()
    assert not fine.any() or (off - eo)[fine].max() <= 0
    number, fine = ~want_lse.isnan(), want_lse.isfinite()
    assert torch.equal(torch.isneginf(got_lse)[number], torch.isneginf(want_lse)[number])
    assert ((got_lse - want_lse).abs() <= el)[fine].all()
    return o, lse


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [64, 96, 128, 160])
@pytest.mark.parametrize("Hkv,G,Sq,R", [(129, 1, 125, 0), (129, 3, 42, 64), (8, 2, 1153, 128)])
@pytest.mark.parametrize("causal", [False, True])
def test_large_tiles(dtype, D, Hkv, G, Sq, R, causal):
    B, cap = 2, 384
    lens = [371, 70]
    host, dev, table = filled(B, Hkv, cap, D, lens, R, seed=Sq + R, dtype=dtype)
    q = torch.randn(B, G * Hkv, Sq, D, generator=torch.Generator().manual_seed(Sq)).to(dtype).cuda()
    check_large(q, host, dev, lens, table, cap, causal)
    check_large(q, host, dev, lens, table, cap, causal, splits=1)


@pytest.mark.parametrize("splits", [2, 3, 16])
@pytest.mark.parametrize("R", [0, 64])
@pytest.mark.parametrize("scale", [0.0, -0.3])
def test_large_tiles_in_runs(splits, R, scale):
    B, Hkv, cap, D = 3, 86, 512, 128
    lens = [512, 77, 0]
    host, dev, table = filled(B, Hkv, cap, D, lens, R, seed=splits, spread=0.5)
    q = torch.randn(B, 2 * Hkv, 64, D, generator=torch.Generator().manual_seed(splits)).to(torch.bfloat16).cuda()
    a = check_large(q, host, dev, lens, table, cap, True, scale, splits=splits)
    b = check_large(q, host, dev, lens, table, cap, True, scale, splits=splits)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("Hkv,Sq", [(129, 64), (33, 250)])
@pytest.mark.parametrize("R", [0, 64])
def test_nan_in_large_tiles(Hkv, Sq, R):
    B, cap, D = 2, 256, 128
    lens = [256, 150]
    host, dev, table = filled(B, Hkv, cap, D, lens, R, seed=2)
    for codes, row, col in ((1, 255, 3), (1, 252, 77), (0, 254, 5), (1, 149, 9), (0, 148, 127)):
        b = 0 if row > 200 else 1
        page, r = ref.place(b, row, R or cap, table)
        host[codes][page, 1, r, col] = 0x7f if col & 1 else 0xff
    dev = on_gpu(host)
    q = torch.randn(B, 2 * Hkv, Sq, D, generator=torch.Generator().manual_seed(Sq)).to(torch.bfloat16).cuda()
    check_large(q, host, dev, lens, table, cap, True)
    check_large(q, host, dev, lens, table, cap, False)


@pytest.mark.parametrize("dtype", DTYPES)
def test_large_tiles_of_a_full_cache(dtype):
    """Without lengths, more than 2^27 scores: some rows against the definition."""
    B, Hkv, G, Sq, cap, D = 1, 4, 4, 500, 17000, 64
    host, dev, table = filled(B, Hkv, cap, D, [cap], 0, seed=8, dtype=dtype)
    q = torch.randn(B, G * Hkv, Sq, D, generator=torch.Generator().manual_seed(1)).to(dtype).cuda()
    assert B * Hkv * G * Sq * cap > 1 << 27
    o, lse = lib.sdpa_kv8(q, *dev, causal=True, return_lse=True)
    k, v = ref.gathered(host[0], host[2], [cap], None, cap), ref.gathered(host[1], host[3], [cap], None, cap)
    for i in (0, 127, 128, 333, 499):                     # (the keys that row i sees are those of a step that ends there)
        upto = lambda x: [(a[:, :cap - Sq + i + 1], c[:, :cap - Sq + i + 1]) for a, c in x]
        want, want_lse, eo, el = ref.attention(q[:, :, i:i + 1].cpu(), upto(k), upto(v), U[dtype], False)
        assert ((o[:, :, i:i + 1].cpu().double() - want).abs() <= eo).all()
        assert ((lse[:, :, i:i + 1].cpu().double() - want_lse).abs() <= el).all()


# Tiles of 32 rows: units (heads of all entries times runs) that divide over the XCDs in every way, more and fewer tiles than parts.
@pytest.mark.parametrize("B,Hkv", [(1, 1), (1, 2), (1, 3), (3, 4), (2, 4), (5, 1), (1, 30)])
@pytest.mark.parametrize("Sq", [33, 65, 97, 300])
@pytest.mark.parametrize("splits", [1, 2, 3])
def test_small_tiles_over_the_chip(B, Hkv, Sq, splits):
    cap, D = 400, 64
    lens = [400, 1, 333, 64, 390][:B]
    host, dev, table = filled(B, Hkv, cap, D, lens, 0, seed=Hkv + Sq)
    q = torch.randn(B, Hkv, Sq, D, generator=torch.Generator().manual_seed(Sq)).to(torch.bfloat16).cuda()
    check_attention(q, host, dev, lens, table, cap, causal=True, splits=splits)


@pytest.mark.parametrize("lens", [[128, -7, 50, 0, -1], [1, 2, 128, 2, 128], [-3] * 5, [70, 69, 68, 67, 66]])
def test_small_tiles_longest_entry_first(lens):
    """More workgroups than start at once; entries in any order, lengths that are none."""
    B, Hkv, cap, D, Sq = 5, 8, 128, 64, 412
    have = [max(0, x) for x in lens]
    host, dev, table = filled(B, Hkv, cap, D, have, 0, seed=3)
    q = torch.randn(B, Hkv, Sq, D, generator=torch.Generator().manual_seed(Sq)).to(torch.bfloat16).cuda()
    want, want_lse = check_attention(q, host, dev, have, table, cap, causal=False)
    o, lse = lib.sdpa_kv8(q, *dev, kv_lens=i32(lens), return_lse=True)
    assert torch.equal(o, want) and torch.equal(lse, want_lse)


@pytest.mark.parametrize("Skv,Sq", [(2000, 1), (9000, 1), (2000, 60)])
def test_workspace_and_out(Skv, Sq):
    host, dev, table = filled(1, 2, Skv, 64, [Skv], 0, seed=4)
    q = torch.randn(1, 8, Sq, 64, device="cuda").half()
    want = lib.sdpa_kv8(q, *dev)
    n = lib.cache8_default_splits(1, 8, 2, Sq, Skv, 64, lib.F16)
    assert n > 1 or Skv == 2000
    out = torch.empty_like(q)
    ws = torch.empty(lib.kv_workspace_bytes(1, 8, Sq, 64, max(n, 2)), dtype=torch.uint8, device="cuda")
    assert lib.sdpa_kv8(q, *dev, out=out, workspace=ws) is out and torch.equal(out, want)
    for part in (0, 1, ws.numel() // 2, ws.numel() - 16):  # fewer runs, or one
        check_attention(q, host, dev, None, table, Skv, workspace=ws[:part])
    with pytest.raises(lib.TiledSdpaError):
        lib.sdpa_kv8(q, *dev, splits=max(n, 2), workspace=ws[:-16])


def test_pages_that_do_not_exist_are_read_as_the_nearest():
    host, dev, table = filled(2, 2, 128, 64, [100, 128], 64, seed=5)
    table = table.clone()
    table[0, 0], table[1, 1] = -5, 2 ** 31 - 1
    q = torch.randn(2, 4, 1, 64, device="cuda").half()
    check_attention(q, host, dev, [100, 128], table, 128)


def test_past_2_31_bytes():
    """Pages on both sides of offsets that do not fit 32 bits: written, read and attended to."""
    P, Hkv, R, D = 40000, 4, 128, 128                      # 2.6e9 bytes each
    dev = (torch.zeros(P, Hkv, R, D, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn), torch.zeros(P, Hkv, R, D, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn),
           torch.zeros(P, Hkv, R // 32, dtype=torch.uint8, device="cuda"), torch.zeros(P, Hkv, R // 32, dtype=torch.uint8, device="cuda"))
    pages = [P - 1, 3, 32768, 32767]
    k, v = halves(tokens(2, 200, Hkv, D, torch.bfloat16, 5), Hkv, D)
    lib.cache8_write(k, v, *dev, i32([0, 0]), i32([200, 150]), block_table=i32([pages[:2], pages[2:]]))
    small = new_cache(4, Hkv, R, D)
    host_table = torch.tensor([[0, 1], [2, 3]], dtype=torch.int32)
    for x, c, s in ((k, small[0], small[2]), (v, small[1], small[3])):
        ref.write(x.cpu(), c, s, [0, 0], [200, 150], host_table)
    for got, want in zip(dev, small):
        got = got.view(torch.uint8)[pages].cpu()
        rows = want.shape[2]
        for p, n in enumerate([128, 72, 128, 22]):
            n = n if rows == R else -(-n // 32)
            assert torch.equal(got[p, :, :n], want[p, :, :n])
    slots = torch.tensor([[pages[0] * R + 5, pages[1] * R + 71], [pages[2] * R + 127, pages[3] * R]], dtype=torch.int64).to(torch.int32).cuda()
    got = lib.cache8_read(*dev, slots, torch.bfloat16)
    for t in range(2):
        x = ref.values(small[t], small[2 + t])
        want = torch.stack([torch.stack([x[0, :, 5], x[1, :, 71]], 1), torch.stack([x[2, :, 127], x[3, :, 0]], 1)])
        assert torch.equal(got[t].cpu().double(), want)
    q = torch.randn(2, 8, 1, D, device="cuda").to(torch.bfloat16)
    o = lib.sdpa_paged8(q, *dev, i32([200, 150]), i32([pages[:2], pages[2:]]))
    kk, vv = ref.gathered(small[0], small[2], [200, 150], host_table, 256), ref.gathered(small[1], small[3], [200, 150], host_table, 256)
    want, _, eo, _ = ref.attention(q.cpu(), kk, vv, U[torch.bfloat16])
    assert ((o.cpu().double() - want).abs() <= eo).all()
