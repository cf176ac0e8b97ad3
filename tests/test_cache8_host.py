"""Refusals of the 8-bit cache's calls, none of which reaches a GPU: the C-ABI's codes in their order, the exceptions of the tensor functions; the
split counts; and the reference that the GPU tests use, against torch's conversions."""
import ctypes
import math

import pytest
import torch

import reference_cache8 as ref
from paper_2603_01960_amd import binding

OK, NULL, SHAPE, DTYPE, BAD_D, ALIGN, SCALE, WORKSPACE, SPLITS, STRIDE = 0, 1, 2, 3, 4, 5, 7, 9, 10, 13
P = 0x1000  # fake, aligned, never dereferenced: every case below fails validation before launch


@pytest.fixture(scope="module")
def lib():
    if not binding.library_path().exists():
        from paper_2603_01960_amd import build
        build.build(force=True)
    return binding.load_library()


def cache(**kwargs):
    a = dict(k=P, v=P, k_scales=P, v_scales=P, block_table=None, pages=2, Hkv=2, block_rows=256, D=64, max_blocks=0)
    a.update(kwargs)
    return binding.Cache8(**a)


def rows(data=P, batch=3 * 512, row=512, head=64):
    return binding.Rows(data, batch, row, head)


# of the cache, in calls that have a batch of 2
COMMON = [
    (dict(D=80), BAD_D), (dict(pages=-1), SHAPE), (dict(Hkv=-1), SHAPE), (dict(block_rows=-1), SHAPE), (dict(max_blocks=-1), SHAPE),
    (dict(pages=1 << 16, block_rows=1 << 16), SHAPE),
    (dict(k=None), NULL), (dict(v_scales=None), NULL), (dict(k=P + 8), ALIGN), (dict(v=P + 8), ALIGN),
]
PAGES = [
    (dict(pages=3), SHAPE),                                                                  # dense: a page for each entry
    (dict(block_table=P, block_rows=48, max_blocks=4), SHAPE), (dict(block_table=P, block_rows=32, max_blocks=4), SHAPE),
    (dict(block_table=P, block_rows=64, max_blocks=1 << 26), SHAPE), (dict(block_table=P + 2, block_rows=64, max_blocks=4), ALIGN),
]


@pytest.mark.parametrize("of_cache,kwargs,expect", [(a, {}, b) for a, b in COMMON + PAGES] + [
    ({}, dict(dtype=2), DTYPE), ({}, dict(B=-1), SHAPE), ({}, dict(S=-1), SHAPE), (dict(pages=0), dict(B=0), OK), ({}, dict(S=0, lens=None), OK),
    (dict(Hkv=0), dict(lens=None), OK), (dict(pages=1 << 20, block_rows=1 << 10, Hkv=1 << 10), dict(B=1 << 20, S=1 << 10), SHAPE),
    (dict(pages=0, block_table=P, block_rows=64, max_blocks=4), dict(lens=None), OK),       # no pages: nothing to write to
    ({}, dict(lens=None), NULL), ({}, dict(new=None), NULL), ({}, dict(k=rows(data=None)), NULL),
    ({}, dict(lens=P + 2), ALIGN), ({}, dict(v=rows(data=P + 2)), ALIGN),
    ({}, dict(k=rows(row=500)), STRIDE), ({}, dict(v=rows(head=-64)), STRIDE),
])
def test_write(lib, of_cache, kwargs, expect):
    a = dict(k=rows(), v=rows(), lens=P, new=P, B=2, S=3, dtype=0)
    a.update(kwargs)
    c, at = cache(**of_cache), ctypes.byref
    assert lib.tiled_sdpa_cache8_write(at(c), at(a["k"]), at(a["v"]), a["lens"], a["new"], a["B"], a["S"], a["dtype"], None) == expect


def test_null_structs(lib):
    at, c, r = ctypes.byref, cache(), rows()
    assert lib.tiled_sdpa_cache8_write(None, at(r), at(r), P, P, 2, 3, 0, None) == NULL
    assert lib.tiled_sdpa_cache8_write(at(c), None, at(r), P, P, 2, 3, 0, None) == NULL
    assert lib.tiled_sdpa_cache8_read(None, P, P, P, 2, 3, 0, None) == NULL
    assert lib.tiled_sdpa_fwd_cache8(None, P, P, None, None, 2, 4, 1, 0.1, 0, 0, 1, None, 0, None) == NULL
    assert lib.tiled_sdpa_cache8_default_splits(1, 4, 2, 1, 100, 64, 0, 0, None) == NULL


@pytest.mark.parametrize("of_cache,kwargs,expect", [(a, {}, b) for a, b in COMMON] + [
    ({}, dict(dtype=3), DTYPE), ({}, dict(B=-1), SHAPE), ({}, dict(n=-1), SHAPE), ({}, dict(B=1 << 16, n=1 << 16), SHAPE), (dict(Hkv=70000), {}, SHAPE),
    ({}, dict(B=0), OK), ({}, dict(n=0, slots=None), OK), (dict(Hkv=0), dict(slots=None), OK),
    ({}, dict(slots=None), NULL), ({}, dict(k=None), NULL), ({}, dict(v=P + 8), ALIGN), ({}, dict(slots=P + 1), ALIGN),
])
def test_read(lib, of_cache, kwargs, expect):
    a = dict(slots=P, k=P, v=P, B=2, n=3, dtype=1)
    a.update(kwargs)
    c = cache(**of_cache)
    assert lib.tiled_sdpa_cache8_read(ctypes.byref(c), *a.values(), None) == expect


@pytest.mark.parametrize("of_cache,kwargs,expect", [(a, {}, b) for a, b in COMMON + PAGES] + [
    ({}, dict(dtype=2), DTYPE), ({}, dict(B=-1), SHAPE), ({}, dict(H=-1), SHAPE), ({}, dict(Sq=-1), SHAPE), ({}, dict(H=5), SHAPE), (dict(Hkv=0), {}, SHAPE),
    (dict(block_rows=0), {}, SHAPE), (dict(block_rows=1 << 24), {}, SHAPE), ({}, dict(Sq=300, flags=8), SHAPE),
    (dict(block_table=P, block_rows=64, max_blocks=0), {}, SHAPE), (dict(pages=0, block_table=P, block_rows=64, max_blocks=4), dict(lens=P), SHAPE),
    ({}, dict(Sq=0, q=None), OK), (dict(pages=0), dict(B=0), OK),
    ({}, dict(q=None), NULL), ({}, dict(o=None), NULL), (dict(block_table=P, block_rows=64, max_blocks=4), dict(lens=None), NULL),
    ({}, dict(q=P + 8), ALIGN), ({}, dict(o=P + 8), ALIGN), ({}, dict(lse=P + 2), ALIGN), ({}, dict(lens=P + 2), ALIGN),
    ({}, dict(scale=math.inf), SCALE), ({}, dict(splits=-1), SPLITS), ({}, dict(splits=129), SPLITS),
    ({}, dict(splits=2), WORKSPACE), ({}, dict(splits=2, ws=P + 8, ws_bytes=1 << 20), WORKSPACE),
    ({}, dict(splits=2, ws=P, ws_bytes=2 * 4 * 2 * 5 * 66 * 4 - 1), WORKSPACE),
    ({}, dict(dtype=9, B=-1, q=None), DTYPE), (dict(D=7), dict(B=-1, q=None), BAD_D), ({}, dict(B=-1, q=None, scale=math.inf), SHAPE),
])
def test_attention(lib, of_cache, kwargs, expect):
    a = dict(q=P, o=P, lse=None, lens=P, B=2, H=4, Sq=5, scale=0.125, dtype=1, flags=0, splits=1, ws=None, ws_bytes=0)
    a.update(kwargs)
    c = cache(**of_cache)
    assert lib.tiled_sdpa_fwd_cache8(ctypes.byref(c), *a.values(), None) == expect


@pytest.mark.parametrize("kwargs,expect", [
    (dict(dtype=2), DTYPE), (dict(D=72), BAD_D), (dict(B=-1), SHAPE), (dict(Hkv=3), SHAPE), (dict(Skv=0), SHAPE), (dict(Skv=1 << 25), SHAPE), (dict(Sq=200, flags=8), SHAPE),
    (dict(B=1 << 20, H=1 << 12, Hkv=1), SHAPE), (dict(Sq=0), OK), (dict(B=0), OK),
])
def test_default_splits_refuses(lib, kwargs, expect):
    a = dict(B=1, H=4, Hkv=2, Sq=1, Skv=100, D=64, dtype=0, flags=0)
    a.update(kwargs)
    n = ctypes.c_int(0)
    assert lib.tiled_sdpa_cache8_default_splits(*a.values(), ctypes.byref(n)) == expect


def test_more_workgroups_than_a_launch_can_have(lib):
    """A launch's threads are counted in 32 bits: 2^24 - 1 workgroups of 256."""
    c, r, z = cache(block_table=P, block_rows=64, max_blocks=(1 << 25) - 1, pages=4, Hkv=1), rows(batch=0, row=0, head=0), ctypes.byref
    args = [z(c), z(r), z(r), None, P, 1]
    assert lib.tiled_sdpa_cache8_write(*args, (1 << 30) - 96, 0, None) == NULL
    assert lib.tiled_sdpa_cache8_write(*args, (1 << 30), 0, None) == SHAPE
    assert lib.tiled_sdpa_cache8_write(*args, (1 << 31) - 1, 0, None) == SHAPE
    n, c = ctypes.c_int(0), cache(pages=1 << 20, Hkv=1, block_rows=64)
    for Sq, splits, expect in ((1, 7, WORKSPACE), (1, 8, SPLITS), (1, 128, SPLITS), (100, 1, NULL), (112, 1, NULL), (113, 1, SHAPE)):
        o = None if expect == NULL else P
        assert lib.tiled_sdpa_fwd_cache8(z(c), P, o, None, P, 1 << 20, 1, Sq, 0.1, 0, 0, splits, None, 0, None) == expect
        assert lib.tiled_sdpa_cache8_default_splits(1 << 20, 1, 1, Sq, 64, 64, 0, 0, z(n)) == (SHAPE if expect == SHAPE else OK)


def test_default_splits(lib):
    """At least one, at most TSDPA_MAX_SPLITS, one where heads are many (three at most where the cache is long), and never fewer for a longer cache of few rows (a workspace for the capacity)."""
    for D in (64, 96, 128, 160):
        for heads in (1, 3, 8, 30, 64, 100, 127, 128, 300):
            for Sq in (1, 4, 20):
                before = 0
                for Skv in (1, 33, 100, 500, 1000, 1700, 3000, 9000, 40000, 300000):
                    n = binding.cache8_default_splits(1, heads, heads, Sq, Skv, D, 0)
                    assert 1 <= n <= 128 and n >= before and (heads < 128 or n <= (3 if Skv * D >= 1 << 20 else 1))
                    before = n


def test_tensor_functions_refuse_the_host():
    z = torch.zeros(1, 2, 64, 64)
    f8, s8 = z.to(torch.float8_e4m3fn), torch.zeros(1, 2, 2, dtype=torch.uint8)
    lens = torch.zeros(1, dtype=torch.int32)
    for call in (lambda: binding.cache8_write(z, z, f8, f8, s8, s8, lens, lens), lambda: binding.cache8_read(f8, f8, s8, s8, lens[None], torch.float16),
                 lambda: binding.sdpa_kv8(z.half(), f8, f8, s8, s8), lambda: binding.sdpa_paged8(z.half(), f8, f8, s8, s8, lens, lens[None]),
                 lambda: binding.sdpa_kv8(z.half(), None, f8, s8, s8)):
        with pytest.raises(ValueError, match="device tensor"):
            call()
    with pytest.raises(ValueError, match="block_table"):
        binding.sdpa_paged8(z.half(), f8, f8, s8, s8, lens, None)


def test_reference_values_and_rounding_are_those_of_torch():
    codes = torch.arange(256, dtype=torch.uint8)
    mine, theirs = ref.VALUES, codes.view(torch.float8_e4m3fn).double()
    assert torch.equal(mine.isnan(), theirs.isnan()) and torch.equal(mine.nan_to_num(), theirs.nan_to_num())
    g = torch.Generator().manual_seed(0)
    x = (torch.randn(100000, generator=g, dtype=torch.float64) * torch.exp2(torch.randint(-12, 8, (100000,), generator=g).double())).clamp(-448, 448).float()
    between = (theirs[:126] + theirs[1:127]).float() / 2                                      # ties
    for y in (x, between, -between, theirs[~theirs.isnan()].float()):
        assert torch.equal(ref.nearest(y.double()), y.to(torch.float8_e4m3fn).view(torch.uint8))


@pytest.mark.parametrize("size,e", [(0.0, -62), (448.0, 0), (448.5, 1), (224.0, -1), (225.0, 0), (896.0, 1), (1.0, -8), (2.0 ** -80, -62), (3e38, 62)])
def test_reference_exponents(size, e):
    assert ref.exponent(torch.tensor([[size, 0.0], [0.0, -size / 2]])).item() == e


def test_reference_write_keeps_and_grows():
    codes, scales = torch.zeros(1, 1, 40, 64, dtype=torch.uint8), torch.zeros(1, 1, 2, dtype=torch.uint8)
    x = torch.full((1, 1, 1, 64), 1.5)
    ref.write(x, codes, scales, [0], [1])
    assert scales[0, 0, 0] == 127 - 8 and ref.values(codes, scales)[0, 0, 0].eq(1.5).all()
    ref.write(x * 64, codes, scales, [1], [2])
    assert scales[0, 0, 0] == 127 - 2 and ref.values(codes, scales)[0, 0, :2].flatten().tolist() == [1.5] * 64 + [96.0] * 64
    ref.write(x / 64, codes, scales, [2], [3])
    assert scales[0, 0, 0] == 127 - 2 and codes[0, 0, 3:].eq(0).all()
    ref.write(x / 64, codes, scales, [0], [1])                                               # from the first row on: a scale of its own
    assert scales[0, 0, 0] == 127 - 14
