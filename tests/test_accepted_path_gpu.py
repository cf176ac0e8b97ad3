"""Keeping a path of a drafted tree: a step drops the last rows of an entry, whichever tokens they are, so that the accepted tokens' rows are
moved to the front first, by the slots that the step of their appending returned."""
import random

import pytest
import torch

import reference64 as ref
from test_tree_attention_gpu import TOL, Sequences, a_tree, i32, lib  # noqa: F401  (lib: the fixture)

pytestmark = pytest.mark.gpu


def a_path(parents, rng):
    """A root of the tree and some of what follows, in order."""
    at, path = rng.choice([i for i, p in enumerate(parents) if p < 0]), []
    while at is not None:
        path.append(at)
        after = [i for i, p in enumerate(parents) if p == at]
        at = rng.choice(after) if after and rng.random() < 0.8 else None
    return path


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
def test_verify_accept_and_go_on(lib, dtype):  # noqa: F811
    """Steps over trees that branch, in each of which a path that is no prefix of the tokens is kept; every step's attention against 64 bits over
    the rows of the paths kept so far."""
    s = Sequences(lib, dtype)
    B, T, R = s.B, s.T, s.R
    n = [150, 5, 63]
    S = max(n)
    q, k, v = s.project(S, 1)
    lens, slots, positions, s.pool = lib.cache_step(s.lens, i32(n), S, R, pages=s.pages())
    lib.qk_norm_rope_cache(q, k, v, s.qw, s.kw, positions, s.f, s.kc, s.vc, slots)
    rotated, plain = s.rotated(q, k, positions)[1], v.transpose(1, 2).cpu()
    keys, values = [rotated[b, :, S - n[b]:] for b in range(B)], [plain[b, :, S - n[b]:] for b in range(B)]
    rng = random.Random(7)
    scattered = 0
    for turn in range(4):
        trees = [[-1, -1] + a_tree(T, rng)[2:] for _ in range(B)]
        mask, depths = lib.tree_mask(i32(trees))
        q, k, v = s.project(T, 2 + turn)
        grown, slots, positions, s.pool = lib.cache_step(lens, i32([T] * B), T, R, pages=s.pages(), depths=depths)
        qr = lib.qk_norm_rope_cache(q, k, v, s.qw, s.kw, positions, s.f, s.kc, s.vc, slots)
        o = lib.sdpa_tree_paged(qr, s.kc, s.vc, grown, s.table, mask)
        q64, k64 = s.rotated(q, k, positions)
        v64 = v.transpose(1, 2).cpu()
        full = max(x.shape[1] for x in keys) + T
        kk, vv = (torch.zeros(B, s.Hkv, full, s.D, dtype=dtype) for _ in range(2))
        for b in range(B):
            m = keys[b].shape[1]
            kk[b, :, :m], vv[b, :, :m], kk[b, :, m:m + T], vv[b, :, m:m + T] = keys[b], values[b], k64[b], v64[b]
        want, _ = ref.tree_attention(q64, kk, vv, [x.shape[1] + T for x in keys], [ref.ancestors(p)[0] for p in trees])
        # (twice the tolerance of attention alone: q and k may round the other way than the reference's)
        assert float((o.cpu().double() - want).abs().max()) <= 2 * TOL[dtype]

        paths = [a_path(p, rng) for p in trees]
        scattered += sum(p != list(range(len(p))) for p in paths)
        path = torch.tensor([p + list(range(len(p), T)) for p in paths], device="cuda")
        src, dst = slots.gather(1, path), slots
        for cache in (s.kc, s.vc):
            cache[dst // R, :, dst % R] = cache[src // R, :, src % R]
        lens, _, _, s.pool = lib.cache_step(grown, i32([len(p) - T for p in paths]), T, R, pages=s.pages())
        for b in range(B):
            # a kept token's position, that of its depth, is the one of the row that it moves to
            m = keys[b].shape[1]
            assert [int(positions[b, t]) for t in paths[b]] == list(range(m, m + len(paths[b])))
            keys[b], values[b] = torch.cat([keys[b], k64[b][:, paths[b]]], 1), torch.cat([values[b], v64[b][:, paths[b]]], 1)
        assert lens.tolist() == [x.shape[1] for x in keys] and int(s.pool[1]) == 0
    assert scattered > 6
