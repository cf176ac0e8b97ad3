"""LSE of rows that see a key of NaN: NaN, whatever the number of runs that the keys are cut into and whoever combines them, and not the -infinity of rows
that no key reaches.  Over 8-bit caches and 16-bit ones."""
import pytest
import torch

import reference_cache8 as ref
from paper_2603_01960_amd import binding as lib
from test_cache8_gpu import check_attention, check_large, filled, i32, on_gpu

pytestmark = pytest.mark.gpu

# (page or entry, head, row, column) of NaN in K; one in V besides, which O sees and LSE does not
PLACES = [(0, 1, 250, 3), (1, 0, 3, 17)]


def poisoned(B, Hkv, cap, D, lens, R, seed):
    host, _, table = filled(B, Hkv, cap, D, lens, R, seed=seed)
    for b, h, row, col in PLACES:
        page, r = ref.place(b, row, R or cap, table)
        host[0][page, h, r, col] = 0x7f
    page, r = ref.place(1, 40, R or cap, table)
    host[1][page, 1, r, 9] = 0xff
    return host, on_gpu(host), table


def same_kind(lse, want):
    assert torch.equal(lse.isnan(), want.isnan())
    assert torch.equal(torch.isneginf(lse), torch.isneginf(want))


def wanted(q, host, lens, table, cap, causal):
    k, v = ref.gathered(host[0], host[2], lens, table, cap), ref.gathered(host[1], host[3], lens, table, cap)
    return ref.attention(q.cpu(), k, v, 2.0 ** -8, causal)[1]


@pytest.mark.parametrize("splits", [1, 2, 3, 8, 16, 64])
@pytest.mark.parametrize("G,Sq", [(1, 1), (4, 2), (4, 5), (2, 40)])
@pytest.mark.parametrize("R", [0, 64])
def test_few_rows(splits, G, Sq, R):
    """Combined in the kernel (up to 8 rows and 32 states), by either merge, or not at all; entries that no key reaches among them."""
    B, Hkv, cap, D = 4, 2, 512, 64
    lens = [256, 90, 0, 1]
    host, dev, table = poisoned(B, Hkv, cap, D, lens, R, 7)
    q = torch.randn(B, G * Hkv, Sq, D, generator=torch.Generator().manual_seed(Sq)).to(torch.bfloat16).cuda()
    for causal in (False, True):
        _, lse = check_attention(q, host, dev, lens, table, cap, causal=causal, splits=splits)
        want = wanted(q, host, lens, table, cap, causal)
        assert want.isnan().any() and torch.isneginf(want).any()
        same_kind(lse.cpu().double(), want)


@pytest.mark.parametrize("splits", [1, 2, 16])
@pytest.mark.parametrize("R", [0, 64])
def test_large_tiles(splits, R):
    B, Hkv, cap, D, Sq = 3, 86, 512, 64, 125
    lens = [256, 90, 0]
    host, dev, table = poisoned(B, Hkv, cap, D, lens, R, 3)
    q = torch.randn(B, Hkv, Sq, D, generator=torch.Generator().manual_seed(Sq)).to(torch.bfloat16).cuda()
    for causal in (False, True):
        _, lse = check_large(q, host, dev, lens, table, cap, causal, splits=splits)
        same_kind(lse[:, :2].cpu().double(), wanted(q[:, :2], [x[:, :2] for x in host], lens, table, cap, causal))


@pytest.mark.parametrize("Sq,splits", [(1, 1), (1, 3), (1, 40), (4, 1), (4, 4), (4, 40), (40, 1), (40, 3), (40, 16), (300, 1), (300, 2)])
@pytest.mark.parametrize("D", [64, 128])
def test_caches_of_16_bits(Sq, splits, D):
    B, H, Skv = 3, 2, 1000
    q, k, v = (torch.randn(B, H, n, D, generator=torch.Generator().manual_seed(n)).to(torch.bfloat16).cuda() for n in (Sq, Skv, Skv))
    k[1, 1, 200, 5] = float("nan")
    lens = i32([Skv, 600, 0])
    o, lse = lib.sdpa_kv(q, k, v, kv_lens=lens, splits=splits, return_lse=True)
    want = torch.full((B, H, Sq), -float("inf"), dtype=torch.float64)
    for b, n in ((0, Skv), (1, 600)):
        want[b] = torch.logsumexp(q[b].double().cpu() @ k[b, :, :n].double().cpu().transpose(-1, -2) * D ** -0.5, -1)
    same_kind(lse.cpu().double(), want)
    assert torch.equal(o.isnan().all(-1).cpu(), want.isnan()) and torch.equal(o.isnan().any(-1).cpu(), want.isnan())
