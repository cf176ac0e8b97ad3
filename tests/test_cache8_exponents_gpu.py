"""Attention over 8-bit caches whose blocks of V have exponents at both ends of their range, under scores that let the keys of both count: the
normaliser has the keys whose values are nothing beside the others', in every wavefront, run and combination of these.

Keys have one column that is not 0, and the scale is ln 2: a key's score, in powers of two, is the K that it is given.  Bounds are the reference's.  What it does
not count: m and log2 l in LSE = (m + log2 l) ln 2 are of up to 2^8 here, whose half step is 2^-17 each, 1.1e-5 in all; it allows (n + 16) 2^-24 of n keys, which is more from
n = 256 on."""
import math

import numpy as np
import pytest
import torch

import reference_cache8 as ref
from test_cache8_gpu import check_attention, check_large, on_gpu, pages_for

pytestmark = pytest.mark.gpu

LN2 = float(np.float32(math.log(2.0)))
TOP, LOW = ref.BIAS + ref.MOST, ref.BIAS - ref.MOST


def cache_of(B, Hkv, rows, D, exponents, scores, R=0, empty_top=False, seed=0):
    """(host, table): each block of 32 rows with its exponent byte for V and its keys' scores (a number, or those of 32 keys); codes of V of all sizes.  With
    `empty_top` results are in FP16's range: codes of 0 where the exponent is the greatest, or none above 6 if they are of every size."""
    g = torch.Generator().manual_seed(seed)
    blocks = rows // 32
    if empty_top and (len(set(exponents)) > 2 or min(exponents) > LOW):
        exponents = [min(e, ref.BIAS + 6) for e in exponents]
    assert rows % 32 == 0 and len(exponents) == len(scores) == blocks
    k = torch.zeros(B, Hkv, rows, D, dtype=torch.float64)
    for i, s in enumerate(scores):
        k[:, :, i * 32:(i + 1) * 32, 0] = torch.as_tensor(s, dtype=torch.float64).expand(32)
    codes = ref.nearest(k)
    assert torch.equal(ref.VALUES[codes.long()], k)
    v = torch.randint(0, 255, (B, Hkv, rows, D), generator=g).to(torch.uint8)
    v[(v & 127) == 127] = 8
    vs = torch.tensor(exponents, dtype=torch.uint8).expand(B, Hkv, blocks).clone()
    if empty_top:
        v[(vs == TOP).repeat_interleave(32, -1)] = 0
    host = [codes, v, torch.full((B, Hkv, blocks), ref.BIAS, dtype=torch.uint8), vs]
    if R == 0:
        return host, None
    table, M = pages_for(B, rows // R), rows // R
    paged = []
    for x in host:
        y = torch.zeros(B * M + 3, Hkv, x.shape[2] // M, *x.shape[3:], dtype=torch.uint8)
        for b in range(B):
            for i in range(M):
                y[int(table[b, i])] = x[b, :, i * y.shape[2]:(i + 1) * y.shape[2]]
        paged.append(y)
    return paged, table


def queries(B, H, Sq, D, dtype):
    q = torch.zeros(B, H, Sq, D, dtype=dtype)
    q[..., 0] = 1.0
    return q.cuda()


def patterns(blocks):
    """(exponents, scores): alternating, the low ones first, the high ones first, one high key beside many low ones, and one low block beside many high."""
    half = blocks // 2
    alone = torch.full((32,), -208.0)
    alone[5] = 0.0
    return {
        "by turns": ([TOP if i % 2 == 0 else LOW for i in range(blocks)], [0.0 if i % 2 == 0 else -3.0 for i in range(blocks)]),
        "by tile": ([TOP if i // 2 % 2 else LOW for i in range(blocks)], [0.0 if i // 2 % 2 else -4.0 for i in range(blocks)]),
        "low first": ([LOW] * half + [TOP] * (blocks - half), [-2.0] * half + [0.0] * (blocks - half)),
        "low first, far": ([LOW] * half + [TOP] * (blocks - half), [0.0] * half + [20.0] * (blocks - half)),
        "high first": ([TOP] * half + [LOW] * (blocks - half), [0.0] * half + [5.0] * (blocks - half)),
        "one high key": ([TOP] + [LOW] * (blocks - 1), [alone] + [-3.0] * (blocks - 1)),
        "one low block": ([TOP] * (blocks - 1) + [LOW], [-6.0] * (blocks - 1) + [0.0]),
        **{f"apart by {n}": ([TOP if i % 2 == 0 else TOP - n for i in range(blocks)], [-1.0 if i % 2 == 0 else -3.0 * (i % 4 == 3) for i in range(blocks)])
           for n in (70, 90, 94, 97, 100, 110, 123)},
        "low first, less": ([LOW] * half + [TOP] * (blocks - half), [-6.0] * half + [0.0] * (blocks - half)),
        "low first, equal": ([LOW] * half + [TOP] * (blocks - half), [0.0] * blocks),
        "all between": ([LOW + 124 * i // (blocks - 1) for i in range(blocks)], [-2.0 * (i % 4) for i in range(blocks)]),
    }


NAMES = list(patterns(16))


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("G,Sq", [(4, 1), (4, 5), (1, 40)])
@pytest.mark.parametrize("splits", [1, 2, 16])
def test_few_rows(name, G, Sq, splits):
    """The decoding kernel and tiles of 32 rows, runs combined in the kernel and by both merges."""
    B, Hkv, rows, D = 2, 2, 1024, 64
    host, table = cache_of(B, Hkv, rows, D, *patterns(rows // 32)[name])
    for lens in ([rows, rows], [rows, rows - 300]):
        check_attention(queries(B, G * Hkv, Sq, D, torch.bfloat16), host, on_gpu(host), lens, table, rows, causal=True, scale=LN2, splits=splits)


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("D", [96, 128, 160])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("Sq", [1, 40])
def test_head_dims_types_and_pages(name, D, dtype, Sq):
    B, Hkv, rows, R = 2, 1, 512, 64
    host, table = cache_of(B, Hkv, rows, D, *patterns(rows // 32)[name], R=R, empty_top=dtype == torch.float16)
    for splits in (1, 3):
        check_attention(queries(B, 3 * Hkv, Sq, D, dtype), host, on_gpu(host), [rows, 300], table, rows, causal=True, scale=LN2, splits=splits)


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("dtype,D", [(torch.bfloat16, 64), (torch.bfloat16, 128), (torch.float16, 64)])
@pytest.mark.parametrize("splits", [1, 2, 5])
def test_large_tiles(name, dtype, D, splits):
    B, Hkv, rows = 2, 129, 512
    host, table = cache_of(B, Hkv, rows, D, *patterns(rows // 32)[name], empty_top=dtype == torch.float16)
    check_large(queries(B, Hkv, 125, D, dtype), host, on_gpu(host), [rows, 384], table, rows, True, LN2, splits=splits)


@pytest.mark.parametrize("splits", [0, 1, 3, 64])
def test_many_small_weights_beside_one_value(splits):
    """One key of the greatest exponent beside 65536 of the least, each 2^-12 of its weight: 17 weights in all."""
    rows, D = 65536 + 32, 64
    blocks = rows // 32
    alone = torch.full((32,), -208.0)
    alone[0] = 0.0
    for exponents, scores in (([TOP] + [LOW] * (blocks - 1), [alone] + [-12.0] * (blocks - 1)), ([LOW] * (blocks - 1) + [TOP], [-12.0] * (blocks - 1) + [alone])):
        host, table = cache_of(1, 1, rows, D, exponents, scores)
        check_attention(queries(1, 2, 1, D, torch.bfloat16), host, on_gpu(host), None, table, rows, scale=LN2, splits=splits)


@pytest.mark.parametrize("Sq", [1, 40])
@pytest.mark.parametrize("splits", [1, 3, 16])
def test_what_the_library_writes(Sq, splits):
    """A block of zeros beside large values, written by cache8_write, and no score that tells them apart."""
    from paper_2603_01960_amd import binding as lib
    from test_cache8_gpu import i32, new_cache
    B, Hkv, rows, D = 1, 2, 512, 64
    host = new_cache(B, Hkv, rows, D)
    dev = on_gpu(host)
    k, v = torch.zeros(B, rows, Hkv, D), torch.zeros(B, rows, Hkv, D)
    v[:, 64:96] = 3e20 * (1 + torch.rand(32, Hkv, D, generator=torch.Generator().manual_seed(1)))
    lib.cache8_write(k.bfloat16().cuda(), v.bfloat16().cuda(), *dev, i32([0]), i32([rows]))
    host = [x.view(torch.uint8).cpu() for x in dev]
    assert host[3].min() == LOW and host[3].max() == ref.BIAS + 61
    check_attention(queries(B, 2 * Hkv, Sq, D, torch.bfloat16), host, dev, [rows], None, rows, causal=Sq == 1, splits=splits)
