"""Refusals of the operators around attention (trees of drafted tokens, cache steps, norm and rotation), none of which reaches a GPU: the
C-ABI's codes in their order, and the exceptions of the tensor functions."""
import ctypes
import inspect
import math

import pytest
import torch

from paper_2603_01960_amd import binding

OK, NULL, SHAPE, DTYPE, BAD_D, ALIGN, SCALE, WORKSPACE, SPLITS, EPS, STRIDE = 0, 1, 2, 3, 4, 5, 7, 9, 10, 12, 13
P = 0x1000  # fake, aligned, never dereferenced: every case below fails validation before launch


@pytest.fixture(scope="module")
def lib():
    if not binding.library_path().exists():
        from paper_2603_01960_amd import build
        build.build(force=True)
    return binding.load_library()


def test_status_strings(lib):
    seen = {binding.status_string(code) for code in range(14)}
    assert len(seen) == 14 and "unknown status" not in seen


@pytest.mark.parametrize("kwargs,expect", [
    (dict(B=-1), SHAPE), (dict(T=-1), SHAPE), (dict(T=1025), SHAPE), (dict(B=0), OK), (dict(T=0, parents=None, mask=None), OK),
    (dict(parents=None), NULL), (dict(mask=None), NULL), (dict(parents=P + 2), ALIGN), (dict(mask=P + 4), ALIGN), (dict(depths=P + 1), ALIGN),
])
def test_tree_mask(lib, kwargs, expect):
    a = dict(parents=P, mask=P, depths=None, B=2, T=5)
    a.update(kwargs)
    assert lib.tiled_sdpa_tree_mask(a["parents"], a["mask"], a["depths"], a["B"], a["T"], None) == expect


STEP = dict(lens=P, counts=P, depths=None, table=P, free=P, pool=P, new_lens=P, slots=P, positions=P, new_pool=P, B=2, S=3, max_blocks=4,
            block_rows=64, pool_size=8)


@pytest.mark.parametrize("kwargs,expect", [
    (dict(B=-1), SHAPE), (dict(B=8193), SHAPE), (dict(S=-1), SHAPE), (dict(block_rows=0), SHAPE), (dict(max_blocks=-1), SHAPE), (dict(pool_size=-1), SHAPE),
    (dict(max_blocks=1 << 25), SHAPE),                       # rows of an entry past an int
    (dict(pool_size=1 << 25), SHAPE),                        # slots past an int
    (dict(B=8192, S=1 << 18), SHAPE),
    (dict(table=None, B=8192, block_rows=1 << 18), SHAPE),   # the same of a dense cache
    (dict(lens=None), NULL), (dict(counts=None), NULL), (dict(free=None), NULL), (dict(pool=None), NULL), (dict(new_lens=None), NULL),
    (dict(slots=None), NULL), (dict(positions=None), NULL), (dict(new_pool=None), NULL), (dict(new_pool=None, B=0), NULL),
    (dict(lens=P + 2), ALIGN), (dict(table=P + 1), ALIGN), (dict(depths=P + 2), ALIGN), (dict(new_pool=P + 2), ALIGN),
])
def test_cache_step(lib, kwargs, expect):
    a = dict(STEP)
    a.update(kwargs)
    assert lib.tiled_sdpa_cache_step(*a.values(), None) == expect


TREE = dict(q=P, k=P, v=P, o=P, lse=None, lens=None, mask=P, mask_batch=5, B=2, H=4, Hkv=2, T=5, Skv=700, D=64, scale=0.125, dtype=1, stream=None,
            splits=1, ws=None, ws_bytes=0)


@pytest.mark.parametrize("kwargs,expect", [
    (dict(dtype=2), DTYPE), (dict(D=80), BAD_D), (dict(T=-1), SHAPE), (dict(Skv=0), SHAPE), (dict(T=70000), SHAPE), (dict(mask_batch=4), SHAPE),
    (dict(T=65, mask_batch=129), SHAPE), (dict(mask_batch=-5), SHAPE), (dict(Hkv=3), SHAPE), (dict(Hkv=0), SHAPE),
    (dict(T=0, q=None, mask=None), OK), (dict(B=0), OK),
    (dict(mask=None), NULL), (dict(q=None), NULL), (dict(mask=P + 4), ALIGN), (dict(v=P + 4), ALIGN), (dict(lens=P + 2), ALIGN),
    (dict(scale=math.inf), SCALE), (dict(splits=129), SPLITS), (dict(splits=2), WORKSPACE), (dict(splits=2, ws=P, ws_bytes=2 * 4 * 2 * 5 * 66 * 4 - 1), WORKSPACE),
])
def test_tree_attention(lib, kwargs, expect):
    a = dict(TREE)
    a.update(kwargs)
    assert lib.tiled_sdpa_fwd_tree(*a.values()) == expect


@pytest.mark.parametrize("kwargs,expect", [
    (dict(block_rows=48), SHAPE), (dict(block_rows=32), SHAPE), (dict(max_blocks=-1), SHAPE), (dict(max_blocks=1 << 26), SHAPE), (dict(max_blocks=0), SHAPE),
    (dict(mask=None), NULL), (dict(lens=None), NULL), (dict(table=None), NULL), (dict(table=P + 2), ALIGN), (dict(dtype=5), DTYPE), (dict(mask_batch=4), SHAPE),
])
def test_tree_attention_over_pages(lib, kwargs, expect):
    a = dict(q=P, k=P, v=P, o=P, lse=None, lens=P, table=P, mask=P, mask_batch=0, B=2, H=4, Hkv=2, T=5, max_blocks=8, block_rows=64, D=64, scale=0.125,
             dtype=1, stream=None, splits=1, ws=None, ws_bytes=0)
    a.update(kwargs)
    assert lib.tiled_sdpa_fwd_tree_paged(*a.values()) == expect


def rope(**kwargs):
    a = dict(B=2, S=3, H=4, Hkv=2, D=64, dtype=0, rot=64, flags=0, eps=1e-6, weight_dtype=0, q_weight=P, k_weight=P, positions=P, pos_batch=3, pos_axis=6,
             inv_freq=P, axes=None, n_axes=1)
    a.update(kwargs)
    return binding.Rope(**a)


def rows(data=P, batch=3 * 512, row=512, head=64):
    return binding.Rows(data, batch, row, head)


COMMON = [
    (dict(dtype=2), DTYPE), (dict(weight_dtype=1), DTYPE), (dict(D=72), BAD_D), (dict(B=-1), SHAPE), (dict(rot=8), SHAPE), (dict(rot=80), SHAPE),
    (dict(rot=-16), SHAPE), (dict(axes=P, n_axes=0), SHAPE), (dict(B=1 << 16, S=1 << 16), SHAPE), (dict(B=1 << 12, S=1 << 12, H=256), SHAPE),
    (dict(positions=None), NULL), (dict(inv_freq=None), NULL), (dict(q_weight=P + 8), ALIGN), (dict(positions=P + 2), ALIGN), (dict(axes=P + 1), ALIGN),
    (dict(eps=-1.0), EPS), (dict(eps=math.nan), EPS), (dict(eps=math.inf), EPS),
]


@pytest.mark.parametrize("kwargs,expect", COMMON + [(dict(B=0), OK), (dict(S=0, positions=None), OK)])
def test_rope_arguments(lib, kwargs, expect):
    p, r = rope(**kwargs), rows()
    at = ctypes.byref
    assert lib.tiled_sdpa_qk_norm_rope(at(p), at(r), at(r), P, P, None) == expect
    assert lib.tiled_sdpa_qk_norm_rope_cache(at(p), at(r), at(r), at(r), P, P, P, P, 4, 64, None) == expect
    if expect != OK:                             # (without rows the weights' gradients are still to be written)
        assert lib.tiled_sdpa_qk_norm_rope_bwd(at(p), P, P, at(r), at(r), at(r), at(r), P, P, P, 1 << 30, None) == expect


BAD_ROWS = [(dict(data=None), NULL), (dict(data=P + 8), ALIGN), (dict(head=60), STRIDE), (dict(row=-512), STRIDE), (dict(batch=4), STRIDE)]


@pytest.mark.parametrize("kwargs,expect", BAD_ROWS)
def test_rope_rows(lib, kwargs, expect):
    p, good, bad = rope(), rows(), rows(**kwargs)
    at = ctypes.byref
    for i in range(2):
        x = [at(good)] * 2
        x[i] = at(bad)
        assert lib.tiled_sdpa_qk_norm_rope(at(p), *x, P, P, None) == expect
    for i in range(3):
        x = [at(good)] * 3
        x[i] = at(bad)
        assert lib.tiled_sdpa_qk_norm_rope_cache(at(p), *x, P, P, P, P, 4, 64, None) == expect
    for i in range(4):
        x = [at(good)] * 4
        x[i] = at(bad)
        assert lib.tiled_sdpa_qk_norm_rope_bwd(at(p), P, P, *x, P, P, P, 1 << 30, None) == expect


@pytest.mark.parametrize("kwargs", [dict(batch=0), dict(row=0), dict(head=0), dict(head=56), dict(row=248), dict(batch=1528)])
def test_gradients_that_would_overlap(lib, kwargs):
    """Four heads of 64 in rows of 512, three rows per entry: strides with which two rows to be written share elements."""
    p, good, bad = rope(H=4, Hkv=4), rows(batch=3 * 512), rows(**kwargs)
    if kwargs == dict(batch=1528):
        bad = rows(batch=2 * 512 + 248)
    at = ctypes.byref
    call = lambda dq, dk: lib.tiled_sdpa_qk_norm_rope_bwd(at(p), P, P, at(good), at(good), at(dq), at(dk), P, P, None, 0, None)
    assert call(bad, good) == STRIDE and call(good, bad) == STRIDE
    assert call(good, good) == WORKSPACE         # what is checked after the strides


def test_rope_null_and_workspace(lib):
    p, r = rope(), rows()
    at = ctypes.byref
    assert lib.tiled_sdpa_qk_norm_rope(None, at(r), at(r), P, P, None) == NULL
    assert lib.tiled_sdpa_qk_norm_rope(at(p), None, at(r), P, P, None) == NULL
    assert lib.tiled_sdpa_qk_norm_rope(at(p), at(r), at(r), None, P, None) == NULL
    assert lib.tiled_sdpa_qk_norm_rope(at(p), at(r), at(r), P, P + 8, None) == ALIGN
    cache = lambda **kw: lib.tiled_sdpa_qk_norm_rope_cache(at(p), at(r), at(r), at(r), *{**dict(slots=P, q=P, k=P, v=P, pages=4, rows=64), **kw}.values(), None)
    assert cache(slots=None) == NULL and cache(k=None) == NULL and cache(v=None) == NULL and cache(slots=P + 2) == ALIGN and cache(v=P + 2) == ALIGN
    assert cache(pages=-1) == SHAPE and cache(rows=0) == SHAPE and cache(pages=1 << 20, rows=1 << 12) == SHAPE
    bwd = lambda **kw: lib.tiled_sdpa_qk_norm_rope_bwd(at(p), *{**dict(a=P, b=P, c=at(r), d=at(r), e=at(r), f=at(r), qw=P, kw=P, ws=P, n=1 << 30), **kw}.values(), None)
    assert bwd(a=None) == NULL and bwd(b=P + 4) == ALIGN and bwd(qw=None) == NULL and bwd(kw=None) == NULL and bwd(qw=P + 1) == ALIGN and bwd(c=None) == NULL
    need = lib.tiled_sdpa_qk_norm_rope_bwd_workspace_bytes(2, 3, 64)
    assert bwd(ws=None) == WORKSPACE and bwd(ws=P + 8) == WORKSPACE and bwd(n=need - 1) == WORKSPACE
    assert lib.tiled_sdpa_qk_norm_rope_bwd_workspace_bytes(-1, 3, 64) == 0
    # never less for more tokens, so that a workspace for the longest serves all
    sizes = [lib.tiled_sdpa_qk_norm_rope_bwd_workspace_bytes(1, n, 128) for n in range(1, 20000, 7)]
    assert sizes == sorted(sizes)


def test_host_tensors_and_other_objects_are_refused(lib):
    x, i = torch.zeros(1, 2, 8, 64, dtype=torch.float16), torch.zeros(1, dtype=torch.int32)
    b = binding
    for bad in (x, None, 3, [1.0]):
        for call in (lambda: b.sdpa_tree(bad, bad, bad, i), lambda: b.sdpa_tree_paged(bad, bad, bad, i, i, i), lambda: b.tree_mask(bad),
                     lambda: b.cache_step(bad, i, 1, 64), lambda: b.qk_norm_rope(bad, bad, None, None, i, i),
                     lambda: b.qk_norm_rope_cache(bad, bad, bad, None, None, i, i, bad, bad, i),
                     lambda: b.qk_norm_rope_backward(bad, bad, bad, bad, None, None, i, i)):
            with pytest.raises(ValueError, match="device tensor"):
                call()
    with pytest.raises(ValueError, match="block_table"):
        b.sdpa_tree_paged(x, x, x, i, None, i)


def test_keyword_names_and_defaults(lib):
    names = lambda f: [(p.name, p.default) for p in inspect.signature(f).parameters.values() if p.default is not p.empty]
    assert names(binding.sdpa_tree) == [("scale", None), ("kv_lens", None), ("splits", 0), ("return_lse", False), ("out", None), ("workspace", None)]
    assert names(binding.sdpa_tree_paged) == [("scale", None), ("splits", 0), ("return_lse", False), ("out", None), ("workspace", None)]
    assert names(binding.tree_mask) == [("out", None)]
    assert names(binding.cache_step) == [("pages", None), ("depths", None), ("out", None)]
    turn = [("axes", None), ("eps", 1e-6), ("interleaved", False)]
    assert names(binding.qk_norm_rope) == turn + [("out", None)]
    assert names(binding.qk_norm_rope_cache) == turn + [("out", None)]
    assert names(binding.qk_norm_rope_backward) == turn + [("workspace", None), ("grads", None)]
