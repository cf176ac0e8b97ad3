"""Weights of an 8-bit cache's attention that are small beside the row's largest: rounded to FP16 with a least step of 2^-31 of the greatest product of weight and
scale, so that many of them together are in O as they are in the normaliser.

The bound is the reference's (tests/reference_cache8.py) but for that step: 2^-32 of the product, half of it, where the reference has 2^-25.  Scores are made as in
tests/test_cache8_exponents_gpu.py."""
import pytest
import torch

import reference_cache8 as ref
from paper_2603_01960_amd import binding as lib
from test_cache8_exponents_gpu import LN2, cache_of, queries
from test_cache8_gpu import LARGE, U, i32, in_large, on_gpu

pytestmark = pytest.mark.gpu

STEP = 2.0 ** -32


def bounded(q, host, table, lens, cap, causal):
    """(o, bound) of the reference with the smaller step.  Its own term for the step, of which it is the only one that does not fall with the weights' sum, is taken out by
    a second look: with results' half step 0 and no roundings of sums it is what is left."""
    k, v = ref.gathered(host[0], host[2], lens, table, cap), ref.gathered(host[1], host[3], lens, table, cap)
    o, _, bound, _ = ref.attention(q.cpu(), k, v, U[q.dtype], causal, LN2)
    B, H, Sq, _ = q.shape
    for b in range(B):
        Hkv, n = k[b][0].shape[:2]
        for h in range(H):
            g = h // (H // Hkv)
            seen = torch.arange(n) <= n - Sq + torch.arange(Sq)[:, None] if causal else torch.ones(Sq, n, dtype=torch.bool)
            p = torch.softmax((LN2 * (q[b, h].double().cpu() @ k[b][0][g].T)).masked_fill(~seen, -float("inf")), -1)
            size = (v[b][0][g] / torch.where(v[b][1][g] == 0, 1.0, v[b][1][g])).abs()
            top = (p[:, :, None] * torch.where(seen[:, :, None], size, 0.0)).flatten(1).amax(-1)
            bound[b, h] -= (1 + U[q.dtype]) * top[:, None] * (2.0 ** -25 - STEP) * (seen.double() @ v[b][1][g].abs())
    return o, bound


def cache_with_small(B, Hkv, rows, D, first, small, exponents=None, seed=0):
    """Key 0 of weight 1 (of the last block, unless `first`) with values of 0 in the lower half of its columns, all others 2^small; values of one sign."""
    blocks = rows // 32
    alone = torch.full((32,), float(small))
    alone[0] = 0.0
    at = 0 if first else blocks - 1
    host, _ = cache_of(B, Hkv, rows, D, exponents or [ref.BIAS] * blocks, [alone if i == at else float(small) for i in range(blocks)], seed=seed)
    host[1][...] = 0x30 + (host[1] & 15)                                                      # 0.5 ... 1.9
    host[1][:, :, at * 32, :D // 2] = 0
    return host


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("first", [True, False])
@pytest.mark.parametrize("Sq,splits", [(1, 1), (1, 3), (4, 16), (20, 1), (40, 1), (40, 3)])
def test_one_large_and_many_small(dtype, first, Sq, splits):
    B, Hkv, rows, D = 1, 1, 4096, 64
    for small in (-18.0, -22.0, -26.0):
        host = cache_with_small(B, Hkv, rows, D, first, small)
        q = queries(B, 2, Sq, D, dtype)
        o = lib.sdpa_kv8(q, *on_gpu(host), scale=LN2, splits=splits).cpu().double()
        want, bound = bounded(q, host, None, [rows], rows, False)
        assert ((o - want).abs() <= bound).all(), (small, ((o - want).abs() / bound).max())
        assert (o[..., :D // 2] > 0).all()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("splits", [1, 2])
def test_large_tiles(dtype, splits):
    B, Hkv, rows, D, Sq = 2, 129, 512, 64, 125
    host = cache_with_small(B, Hkv, rows, D, True, -22.0)
    q = queries(B, Hkv, Sq, D, dtype)
    dev, _ = in_large(on_gpu(host), None, LARGE)
    o = lib.sdpa_kv8(q, *dev, causal=True, scale=LN2, kv_lens=i32([rows, 384]), splits=splits)[:, :2].cpu().double()
    want, bound = bounded(q[:, :2], [x[:, :2] for x in host], None, [rows, 384], rows, True)
    assert ((o - want).abs() <= bound).all(), ((o - want).abs() / bound).max()
    assert (o[..., :D // 2] > 0).all()


@pytest.mark.parametrize("Sq", [1, 40])
@pytest.mark.parametrize("apart", [8, 14, 20])
def test_a_block_of_greater_exponent(Sq, apart):
    """Weights that are equal, one block 2^apart greater than the others but 0 in half of the columns: the others' values there."""
    B, Hkv, rows, D = 1, 2, 1024, 64
    blocks = rows // 32
    exponents = [ref.BIAS - 20] * blocks
    exponents[3] = ref.BIAS - 20 + apart
    host, _ = cache_of(B, Hkv, rows, D, exponents, [0.0] * blocks)
    host[1][...] = 0x30 + (host[1] & 15)
    host[1][:, :, 96:128, :D // 2] = 0
    q = queries(B, 4, Sq, D, torch.bfloat16)
    o = lib.sdpa_kv8(q, *on_gpu(host), scale=LN2).cpu().double()
    want, bound = bounded(q, host, None, [rows], rows, False)
    bound -= 2.0 ** -25                                                                       # (FP16's least step: these are BF16)
    assert ((o - want).abs() <= bound).all(), ((o - want).abs() / bound).max()
