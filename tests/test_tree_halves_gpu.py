"""Trees of up to 32 rows per key/value head are as exact as the same rows without one: where one run, or streams, took the place of the decoding
kernel's runs of a tile or two, each weight is multiplied as two 16-bit halves.  The bound and its derivation are those of
test_error_of_few_rows in test_kv_route_gpu.py: the rounding of the exact result, times 1.118 (weights rounded in halves) or 1.315 (D =
160: whole, but in runs of a tile), and 3 % for the spread of a few hundred values.  The tree hides at most 32 keys of several hundred."""
import math
import random

import pytest
import torch

import reference64 as ref
from test_tree_attention_gpu import a_tree, i32, lib, paged  # noqa: F401  (lib: the fixture)

pytestmark = pytest.mark.gpu
HALVES = 1.118


def weights_of(q, k, seen, g):
    """Softmax over the keys that each row sees, in 64 bits: q [H, T, D], k [Hkv, n, D], seen [T, n] -> [H, T, n]"""
    x = torch.stack([q[h].double() @ k[h // g].double().t().contiguous() for h in range(q.shape[0])]) * q.shape[2] ** -0.5
    return x.masked_fill(~seen, -math.inf).softmax(-1)


@pytest.mark.parametrize("pages", [False, True])
@pytest.mark.parametrize("Hkv,group,T,n,D,rounded", [
    (16, 1, 2, 744, 96, HALVES), (2, 1, 8, 1473, 64, HALVES), (7, 4, 4, 760, 128, HALVES), (7, 1, 16, 760, 128, HALVES), (9, 1, 1, 635, 160, HALVES),
    (36, 1, 5, 257, 128, HALVES), (20, 3, 1, 260, 160, HALVES), (72, 1, 20, 512, 128, HALVES), (112, 2, 16, 385, 96, HALVES), (72, 1, 24, 900, 64, HALVES),
    (66, 4, 5, 3000, 128, HALVES), (80, 8, 4, 2000, 96, HALVES), (3, 1, 24, 717, 160, 1.315)])
def test_error_of_small_trees(lib, Hkv, group, T, n, D, rounded, pages):  # noqa: F811
    tree = a_tree(T, random.Random(T))
    sets, _ = ref.ancestors(tree)
    mask, _ = lib.tree_mask(i32([tree]))
    seen = torch.ones(T, n, dtype=torch.bool)
    for i in range(T):
        seen[i, n - T:] = torch.tensor([j in sets[i] for j in range(T)])
    seen = seen.cuda()
    for dtype in (torch.bfloat16, torch.float16):
        g = torch.Generator("cuda").manual_seed(7600 + Hkv)
        q, k, v = (torch.randn(1, heads, rows, D, device="cuda", generator=g).to(dtype) for heads, rows in ((Hkv * group, T), (Hkv, n), (Hkv, n)))
        if pages:
            kp, vp, table = paged(k, v, 64, T)
            o = lib.sdpa_tree_paged(q, kp, vp, i32([n]), table, mask)
        else:
            o = lib.sdpa_tree(q, k, v, mask)
        w = weights_of(q[0], k[0], seen, group)
        want = torch.stack([w[h] @ v[0, h // group].double() for h in range(Hkv * group)])
        err, least = (o[0].double() - want).norm(), (want.to(dtype).double() - want).norm()
        assert err <= 1.03 * rounded * least, f"{dtype} {float(err / least):.3f} times the rounding of the result"


@pytest.mark.parametrize("Hkv,T,n,D", [(3, 4, 600, 96), (70, 20, 600, 64), (66, 24, 1000, 128)])
def test_infinities_and_nan_of_tokens_with_halved_weights(lib, Hkv, T, n, D):  # noqa: F811
    """A token's values reach those that see it, as they are, and nobody else."""
    for dtype in (torch.bfloat16, torch.float16):
        g = torch.Generator("cuda").manual_seed(T)
        q, k, v = (torch.randn(1, Hkv, rows, D, device="cuda", generator=g).to(dtype) for rows in (T, n, n))
        tree = a_tree(T, random.Random(T))
        sets, _ = ref.ancestors(tree)
        mask, _ = lib.tree_mask(i32([tree]))
        bad = T // 2
        row = n - T + bad
        k[0, :, row] = 0
        clean = lib.sdpa_tree(q, k, v, mask)
        blind = torch.tensor([bad not in s for s in sets])
        for what in (math.inf, -math.inf, math.nan):
            v2 = v.clone()
            v2[0, :, row, 3::7] = what
            got = lib.sdpa_tree(q, k, v2, mask)
            assert torch.equal(got[:, :, blind], clean[:, :, blind])
            hit = got[:, :, ~blind].float()[..., 3::7]
            assert bool((torch.isnan(hit) if math.isnan(what) else hit == what).all())
        # of the cached sequence too
        v2 = v.clone()
        v2[0, :, 5, 0] = -math.inf
        assert bool((lib.sdpa_tree(q, k, v2, mask)[..., 0] == -math.inf).all())
