"""Seeded random combinations of the 8-bit cache's calls: steps that append to and drop from entries, read back and attended to, against the definition."""
import random

import pytest
import torch

import reference_cache8 as ref
from paper_2603_01960_amd import binding as lib
from test_cache8_gpu import check_attention, filled, halves, new_cache, on_gpu, pages_for, same_bytes, tokens, write_both

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("seed", range(48))
def test_attention(seed):
    r = random.Random(seed)
    dtype, D = r.choice([torch.float16, torch.bfloat16]), r.choice([64, 96, 128, 160])
    B, Hkv, G = r.choice([1, 1, 2, 3, 5, 17]), r.choice([1, 2, 3, 8]), r.choice([1, 1, 2, 4, 7])
    Sq = r.choice([1, 1, 2, 3, 8, 16, 31, 33, 64, 100, 257])
    R = r.choice([0, 0, 64, 128, 512])
    most = max(64, 2_000_000 // (B * Hkv * G * Sq))
    cap = min(r.randint(1, 700) if r.random() < 0.5 else r.randint(700, 3000), most)
    cap = max(cap, Sq)
    if R:
        cap = -(-cap // R) * R
    lens = [r.choice([0, 1, cap, cap, r.randint(0, cap), r.randint(0, cap)]) for _ in range(B)]
    host, dev, table = filled(B, Hkv, cap, D, lens, R, seed=seed, spread=r.choice([0.0, 1.0, 3.0]), dtype=dtype)
    q = torch.randn(B, G * Hkv, Sq, D, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()
    given = [n if r.random() < 0.9 or n not in (0, cap) else (-9 if n == 0 else cap + 77) for n in lens]
    print(f"seed {seed}: {dtype} D={D} B={B} Hkv={Hkv} G={G} Sq={Sq} R={R} cap={cap} lens={given}", flush=True)
    check_attention(q, host, dev, given, table, cap, causal=r.random() < 0.7, scale=r.choice([None, None, 0.05, -0.2]), splits=r.choice([0, 0, 1, 2, 5, 13, 128]))


@pytest.mark.parametrize("seed", range(32))
def test_steps(seed):
    """Lengths go up by what is written and down by what is dropped, an entry now and then to nothing."""
    r = random.Random(1000 + seed)
    dtype, D, B, Hkv = r.choice([torch.float16, torch.bfloat16]), r.choice([64, 96, 128, 160]), r.choice([1, 2, 5]), r.choice([1, 3, 8])
    R = r.choice([0, 64, 128])
    cap = r.randint(40, 400) if R == 0 else R * r.randint(1, 4)
    table = pages_for(B, cap // R, seed) if R else None
    host = new_cache(B * (cap // R) + 3 if R else B, Hkv, R or cap, D, seed)
    dev, lens = on_gpu(host), [0] * B
    for step in range(6):
        S = r.choice([1, 1, 5, 17, 40, 130])
        old = [n if r.random() < 0.7 else r.randint(0, n) for n in lens]
        new = [min(n + r.choice([S, S, r.randint(0, S)]), cap) for n in old]
        x = tokens(B, S, Hkv, D, dtype, 7 * seed + step, r.choice([0.0, 2.0, 6.0]))
        k, v = halves(x, Hkv, D)
        print(f"seed {seed} step {step}: {dtype} D={D} B={B} Hkv={Hkv} R={R} cap={cap} S={S} {old} -> {new}", flush=True)
        write_both(host, dev, k, v, old, new, table)
        same_bytes(dev, host)
        lens = new
    pages, rows = host[0].shape[0], R or cap
    slots = torch.randint(-3, pages * rows + 3, (B, 11), generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    got = lib.cache8_read(*dev, slots.cuda(), dtype)
    inside = (slots >= 0) & (slots < pages * rows)
    for t, (codes, scales) in enumerate(((host[0], host[2]), (host[1], host[3]))):
        x = ref.values(codes, scales).transpose(1, 2).reshape(pages * rows, Hkv, D)
        want = torch.where(inside[..., None, None], x[slots.long().clamp(0, pages * rows - 1)], 0.0).transpose(1, 2).to(dtype)
        assert torch.equal(got[t].isnan().cpu(), want.isnan())
        assert torch.equal(torch.nan_to_num(got[t].cpu().double(), 1e300), torch.nan_to_num(want.double(), 1e300))
