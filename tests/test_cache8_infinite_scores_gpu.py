"""Scores of -infinity over 8-bit caches, which an exponent of K and a query reach together: such keys have weight 0 wherever they lie, and are not
taken for keys whose weight has left FP32's numbers; only a row without any finite score has no value (NaN, LSE = -infinity).

All other columns of K are 0: a row's result is the mean of the values that it gives weight to.  Its bound: weights are powers of two, and exact; what is left are
the result's rounding and (n + 16) roundings to FP32 of a sum of sizes."""
import math

import pytest
import torch

import reference_cache8 as ref
from paper_2603_01960_amd import binding as lib
from test_cache8_gpu import LARGE, U, i32, in_large, new_cache, on_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("low", [range(32, 64), range(0, 32), range(96, 224), range(0, 320), range(320, 640), range(1, 640), range(0, 640)], ids=str)
@pytest.mark.parametrize("Hkv,G,Sq,splits,large", [(2, 4, 1, 1, False), (2, 4, 1, 4, False), (2, 4, 5, 7, False), (2, 1, 40, 1, False), (2, 1, 40, 3, False), (129, 1, 125, 1, True), (129, 1, 125, 2, True)])
def test_keys_of_infinitely_low_score(low, Hkv, G, Sq, splits, large):
    B, n, D = 2, 640, 64
    codes, values, _, vs = new_cache(B, Hkv, n, D, seed=3)
    values[(values & 127) == 127] = 8
    codes[...] = 0
    codes[:, :, low.start:low.stop, 0] = 0xfe                                                # -448
    host = [codes, values, torch.full_like(vs, ref.BIAS + 62), torch.full_like(vs, ref.BIAS)]
    q = torch.zeros(B, Hkv * G, Sq, D)
    row = Sq // 2
    q[1, 1, row, 0] = 1e30
    q = q.to(torch.bfloat16).cuda()
    dev = in_large(on_gpu(host), None, LARGE)[0] if large else on_gpu(host)
    o, lse = lib.sdpa_kv8(q, *dev, kv_lens=i32([n, n]), splits=splits, return_lse=True)
    v = ref.values(host[1], host[3])
    heads = [0, 1, Hkv * G - 1]
    for b in range(B):
        for h in heads:
            x = v[b, h // G]
            for i in range(Sq):
                special = (b, h, i) == (1, 1, row)
                seen = torch.ones(n, dtype=torch.bool)
                if special:
                    seen[low.start:low.stop] = False
                got, got_lse = o[b, h, i].cpu().double(), lse[b, h, i].item()
                if not seen.any():
                    assert got.isnan().all() and got_lse == -math.inf
                    continue
                want = x[seen].mean(0)
                bound = U[torch.bfloat16] * want.abs() + 2 * (n + 16) * 2.0 ** -24 * x[seen].abs().mean(0)
                assert ((got - want).abs() <= bound).all(), (b, h, i)
                assert abs(got_lse - math.log(int(seen.sum()))) <= (n + 16) * 2.0 ** -24 + 2.0 ** -21
