"""Attention of drafted trees on the GPU against its definition in 64 bits, and a whole verification step.

Tolerances as for the forward pass: 2e-3 (FP16), 1.6e-2 (BF16) on outputs of values from N(0, 1), 1e-4 on the log-sum-exp (P is rounded to 16 bits
before the second product, by at most 2^-11 or 2^-8 of each weight: of outputs below 4 that is 2e-3 and 1.6e-2)."""
import math
import random

import pytest
import torch

import reference64 as ref

pytestmark = pytest.mark.gpu
TOL = {torch.float16: 2e-3, torch.bfloat16: 1.6e-2}


@pytest.fixture(scope="module")
def lib():
    from paper_2603_01960_amd import binding
    binding.load_library()
    return binding


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def a_tree(T, rng):
    return [max(-1, i - rng.randrange(1, 6)) for i in range(T)]


def inputs(B, H, Hkv, T, Skv, D, dtype, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    return [torch.randn(s, device="cuda", generator=g).to(dtype) for s in ((B, H, T, D), (B, Hkv, Skv, D), (B, Hkv, Skv, D))]


def paged(k, v, R, seed):
    """The same rows in pages of R, in no order; what no row fills is NaN."""
    B, Hkv, n, D = k.shape
    M = -(-n // R)
    table = torch.randperm(B * M, generator=torch.Generator().manual_seed(seed)).view(B, M)
    out = []
    for x in (k, v):
        full = torch.full((B, Hkv, M * R, D), math.nan, device="cuda", dtype=x.dtype)
        full[:, :, :n] = x
        pages = torch.empty(B * M, Hkv, R, D, device="cuda", dtype=x.dtype)
        pages[table.flatten().cuda()] = full.view(B, Hkv, M, R, D).transpose(1, 2).reshape(B * M, Hkv, R, D)
        out.append(pages)
    return *out, table.to(torch.int32).cuda()


def check(lib, q, k, v, lens, sees, o, lse=None, scale=None):
    want, want_lse = ref.tree_attention(q, k, v, lens, sees, scale)
    err = (o.cpu().double() - want).abs()
    assert bool(torch.isfinite(o).all()) and float(err.max()) <= TOL[q.dtype], float(err.max())
    if lse is not None:
        empty = torch.isinf(want_lse)
        assert torch.equal(torch.isinf(lse.cpu()), empty)
        assert float((lse.cpu().double() - want_lse)[~empty].abs().max() if bool((~empty).any()) else 0.0) <= 1e-4


# (B, H, Hkv, T, Skv, lens, D): every form: the decoding kernel on 16 and 32 rows, streams, 64 and 128 rows; trees that begin and end inside a
# tile, that are all there is, that lie across a split's ends; entries of no rows, of fewer rows than the tree
CASES = [(1, 1, 1, 1, 1, [1], 64), (2, 4, 4, 7, 40, [40, 7], 96), (3, 8, 2, 8, 700, [700, 3, 0], 128), (1, 8, 1, 4, 3000, [2999], 64), (2, 8, 2, 5, 300, [33, 290], 160),
         (1, 4, 1, 20, 5000, [5000], 128), (2, 16, 2, 64, 1024, [1024, 64], 128), (1, 8, 8, 100, 900, [895], 64), (2, 4, 1, 200, 640, [200, 601], 160),
         (1, 2, 2, 130, 130, [130], 96), (1, 2, 2, 300, 290, [290], 64), (4, 32, 4, 33, 2100, [2100, 1999, 40, 33], 128), (16, 16, 16, 12, 250, [16 * i + 9 for i in range(16)], 96),
         (40, 8, 8, 40, 130, [3 * i + 10 for i in range(40)], 64), (70, 4, 4, 70, 200, [100 + i for i in range(70)], 128), (3, 64, 64, 9, 700, [700, 650, 20], 160)]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
@pytest.mark.parametrize("B,H,Hkv,T,Skv,lens,D", CASES)
def test_dense_and_paged(lib, B, H, Hkv, T, Skv, lens, D, dtype):
    rng = random.Random(T)
    q, k, v = inputs(B, H, Hkv, T, Skv, D, dtype, T + D)
    for b, n in enumerate(lens):                 # nothing past an entry's end is read
        k[b, :, n:], v[b, :, n:] = math.nan, math.nan
    trees = [a_tree(T, rng) for _ in range(B)]
    sees = [ref.ancestors(p)[0] for p in trees]
    mask, _ = lib.tree_mask(i32(trees))
    o, lse = lib.sdpa_tree(q, k, v, mask, kv_lens=i32(lens), return_lse=True)
    check(lib, q, k, v, lens, sees, o, lse)
    for R in (64, 256):
        kp, vp, table = paged(k, v, R, T)
        o2, lse2 = lib.sdpa_tree_paged(q, kp, vp, i32(lens), table, mask, return_lse=True)
        check(lib, q, k, v, lens, sees, o2, lse2)


@pytest.mark.parametrize("H,Hkv,T,D", [(4, 4, 3, 64), (4, 1, 8, 128), (8, 2, 31, 96), (2, 2, 65, 128), (16, 1, 70, 160), (4, 4, 129, 64)])
def test_any_pattern_of_bits(lib, H, Hkv, T, D):
    """Tokens that see nothing, not themselves, later ones; bits past the last token; one mask for all entries; entries shorter than the tree."""
    rng = random.Random(T)
    lens = [T + 300, T + 17, T, max(1, T - 2), 0]
    B, Skv = len(lens), T + 300
    q, k, v = inputs(B, H, Hkv, T, Skv, D, torch.float16, T)
    W = (T + 63) // 64
    sets = [set(j for j in range(64 * W) if rng.random() < 0.3) for _ in range(T)]
    sets[0], sets[T // 2], sets[T - 1] = set(), {T - 1, 64 * W - 1}, set(range(64 * W))
    mask = ref.words_of(sets, 64 * W).cuda()
    o, lse = lib.sdpa_tree(q, k, v, mask, kv_lens=i32(lens), return_lse=True)
    check(lib, q, k, v, lens, [sets] * B, o, lse)
    each = mask[None].expand(B, -1, -1).contiguous()
    assert torch.equal(o, lib.sdpa_tree(q, k, v, each, kv_lens=i32(lens)))
    for splits in (1, 2, 5):
        o, lse = lib.sdpa_tree(q, k, v, mask, kv_lens=i32(lens), splits=splits, return_lse=True)
        check(lib, q, k, v, lens, [sets] * B, o, lse)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
@pytest.mark.parametrize("H,Hkv,T,n,D", [(4, 4, 6, 50, 64), (8, 2, 8, 300, 128), (4, 2, 40, 1000, 96), (2, 2, 64, 2500, 128), (32, 8, 24, 100, 160), (128, 128, 70, 200, 64)])
def test_infinities_and_nan_of_tokens_that_a_token_does_not_see(lib, H, Hkv, T, n, D, dtype):
    """Rows of K and V that a token does not see leave its bits as they are, whatever they hold; of V that it sees, they arrive."""
    rng = random.Random(T)
    q, k, v = inputs(1, H, Hkv, T, n, D, dtype, T)
    tree = a_tree(T, rng)
    sets, _ = ref.ancestors(tree)
    mask, _ = lib.tree_mask(i32([tree]))
    bad = T // 2
    row = n - T + bad
    k[0, :, row], v[0, :, row] = 0, 0
    clean = lib.sdpa_tree(q, k, v, mask)
    blind = torch.tensor([bad not in s for s in sets])
    for what in (math.inf, -math.inf, math.nan):
        v2 = v.clone()
        v2[0, :, row, 3::7] = what
        got = lib.sdpa_tree(q, k, v2, mask)
        assert torch.equal(got[:, :, blind], clean[:, :, blind])
        hit = got[:, :, ~blind].float()
        assert bool((torch.isnan(hit[..., 3::7]) if math.isnan(what) else hit[..., 3::7] == what).all())
        rest = [d for d in range(D) if d % 7 != 3]
        assert torch.equal(got[..., rest], clean[..., rest])
        k2 = k.clone()
        k2[0, :, row] = what
        got = lib.sdpa_tree(q, k2, v2, mask)
        assert torch.equal(got[:, :, blind], clean[:, :, blind])
    v2 = v.clone()
    v2[0, :, row, 0], v2[0, :, n - T - 1 if n > T else row, 0] = math.inf, -math.inf        # one that all see, and both signs
    got = lib.sdpa_tree(q, k, v2, mask)
    if n > T:
        assert bool((got[:, :, blind, 0] == -math.inf).all()) and bool(torch.isnan(got[:, :, ~blind, 0]).all())


@pytest.mark.parametrize("H,Hkv,T,n,D", [(8, 2, 3, 3000, 128), (8, 8, 20, 4000, 64), (16, 2, 30, 6000, 96)])
def test_any_workspace_serves(lib, H, Hkv, T, n, D):
    """The size that is reported, less, and next to nothing; a split count that needs more is refused."""
    q, k, v = inputs(1, H, Hkv, T, n, D, torch.float16, T)
    tree = a_tree(T, random.Random(T))
    mask, _ = lib.tree_mask(i32([tree]))
    want = lib.sdpa_tree(q, k, v, mask)
    for nbytes in (1 << 26, 300000, 16):
        o, lse = lib.sdpa_tree(q, k, v, mask, workspace=torch.full((nbytes,), 255, dtype=torch.uint8, device="cuda"), return_lse=True)
        check(lib, q, k, v, [n], [ref.ancestors(tree)[0]], o, lse)
        if nbytes == 1 << 26:
            assert torch.equal(o, want)
    with pytest.raises(lib.TiledSdpaError):
        lib.sdpa_tree(q, k, v, mask, splits=8, workspace=torch.zeros(16, dtype=torch.uint8, device="cuda"))


def test_a_chain_is_the_causal_mask(lib):
    """A tree that is a chain sees what the last positions of a sequence see."""
    for H, Hkv, T, n, D in ((8, 2, 8, 900, 128), (4, 4, 64, 700, 64), (2, 1, 150, 400, 96)):
        q, k, v = inputs(1, H, Hkv, T, n, D, torch.float16, n)
        mask, _ = lib.tree_mask(i32([i - 1 for i in range(T)]))
        a, b = lib.sdpa_tree(q, k, v, mask), lib.sdpa_kv(q, k, v, True)
        assert float((a - b).abs().max()) <= 2e-3


def test_scales(lib):
    rng = random.Random(0)
    q, k, v = inputs(2, 4, 2, 9, 200, 128, torch.float16, 0)
    trees = [a_tree(9, rng) for _ in range(2)]
    mask, _ = lib.tree_mask(i32(trees))
    for scale in (0.0, -0.1, 0.3):
        check(lib, q, k, v, [200, 200], [ref.ancestors(p)[0] for p in trees], lib.sdpa_tree(q, k, v, mask, scale), scale=scale)


def test_refusals(lib):
    q, k, v = inputs(2, 4, 2, 9, 200, 64, torch.float16, 0)
    mask = torch.zeros(2, 9, 1, dtype=torch.int64, device="cuda")
    for bad in (mask[:1], mask.int(), mask[:, :8], torch.zeros(2, 9, 2, dtype=torch.int64, device="cuda"), mask.cpu(), mask.transpose(0, 1), None):
        with pytest.raises(ValueError, match="mask must be"):
            lib.sdpa_tree(q, k, v, bad)
    with pytest.raises(ValueError, match="kv_lens"):
        lib.sdpa_tree(q, k, v, mask, kv_lens=i32([1]))
    with pytest.raises(ValueError, match="multiple"):
        lib.sdpa_tree(q[:, :3].contiguous(), k, v, mask)
    with pytest.raises(ValueError, match="kv_lens"):
        lib.sdpa_tree_paged(q, k, v, None, i32([[0], [1]]), mask)
    with pytest.raises(lib.TiledSdpaError):
        lib.sdpa_tree_paged(q, k, v, i32([1, 1]), i32([[0], [1]]), mask)          # pages of 200 rows
    with pytest.raises(lib.TiledSdpaError):
        lib.sdpa_tree(q, k, v, mask, splits=200)


class Sequences:
    """Entries of a served batch: a paged cache through the library, and beside it each entry's accepted rows in 64 bits."""

    def __init__(self, lib, dtype, B=3, H=8, Hkv=2, D=64, R=64, M=8, T=12):
        self.__dict__.update(lib=lib, dtype=dtype, B=B, H=H, Hkv=Hkv, D=D, R=R, M=M, T=T)
        self.qw, self.kw = (1 + 0.1 * torch.randn(D, device="cuda")).to(dtype), (1 + 0.1 * torch.randn(D, device="cuda")).to(dtype)
        self.f = (10000.0 ** (-torch.arange(D // 2) / (D // 2))).float().cuda()
        self.kc, self.vc = (torch.full((B * M, Hkv, R, D), math.nan, device="cuda", dtype=dtype) for _ in range(2))
        self.lens, self.pool = i32([0] * B), i32([B * M, 0])
        self.table, self.free = torch.full((B, M), -1, dtype=torch.int32, device="cuda"), torch.randperm(B * M, device="cuda").to(torch.int32)

    def pages(self):
        return self.table, self.free, self.pool

    def project(self, S, seed):
        g = torch.Generator("cuda").manual_seed(seed)
        x = torch.randn(self.B, S, self.H + 2 * self.Hkv, self.D, device="cuda", generator=g).to(self.dtype)
        return x.split([self.H, self.Hkv, self.Hkv], dim=2)

    def rotated(self, q, k, positions):
        phi = ref.angles(positions, self.f, None, self.B, q.shape[1])
        return [ref.norm_rope(x, w, phi, 1e-6, False).to(self.dtype) for x, w in ((q, self.qw), (k, self.kw))]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
def test_a_verification_step_as_it_is_used(lib, dtype):
    """A prefill of different lengths, then trees of drafted tokens: mask, pages and slots, norm and rotation into the cache, attention;
    then all drafts dropped.  Compared with 64 bits on keys that are rotated and rounded apart from the library."""
    s = Sequences(lib, dtype)
    B, T = s.B, s.T
    n = [150, 5, 63]
    S = max(n)
    q, k, v = s.project(S, 1)
    lens, slots, positions, s.pool = lib.cache_step(s.lens, i32(n), S, s.R, pages=s.pages())
    assert s.pool.tolist() == [B * s.M - 5, 0]
    lib.qk_norm_rope_cache(q, k, v, s.qw, s.kw, positions, s.f, s.kc, s.vc, slots)
    rng = random.Random(3)
    keys, values = s.rotated(q, k, positions)[1], v.transpose(1, 2).cpu()
    for turn in range(2):
        trees = [a_tree(T, rng) for _ in range(B)]
        mask, depths = lib.tree_mask(i32(trees))
        q, k, v = s.project(T, 2 + turn)
        grown, slots, positions, s.pool = lib.cache_step(lens, i32([T] * B), T, s.R, pages=s.pages(), depths=depths)
        assert positions.tolist() == [[n[b] + d for d in ref.ancestors(trees[b])[1]] for b in range(B)]
        qr = lib.qk_norm_rope_cache(q, k, v, s.qw, s.kw, positions, s.f, s.kc, s.vc, slots)
        o = lib.sdpa_tree_paged(qr, s.kc, s.vc, grown, s.table, mask)
        q64, k64 = s.rotated(q, k, positions)
        full = max(n) + T
        kk, vv = (torch.zeros(B, s.Hkv, full, s.D, dtype=dtype) for _ in range(2))
        for b in range(B):
            kk[b, :, :n[b]], vv[b, :, :n[b]] = keys[b, :, S - n[b]:], values[b, :, S - n[b]:]
            kk[b, :, n[b]:n[b] + T], vv[b, :, n[b]:n[b] + T] = k64[b], v[b].transpose(0, 1).cpu()
        want, _ = ref.tree_attention(q64, kk, vv, [x + T for x in n], [ref.ancestors(p)[0] for p in trees])
        # (q and k may round the other way than the reference's: one step of each of D products, on scores of size 1, is below their own tolerance)
        assert float((o.cpu().double() - want).abs().max()) <= 2 * TOL[dtype]
        lens, _, _, s.pool = lib.cache_step(grown, i32([-T] * B), T, s.R, pages=s.pages())
        assert lens.tolist() == n


def test_a_captured_verification_step(lib):
    """One graph for all steps: replayed on other tokens, trees and lengths, with eager work between, against the eager calls."""
    s = Sequences(lib, torch.bfloat16)
    B, T = s.B, s.T
    n = [100, 7, 200]
    lens, slots, positions, pool = lib.cache_step(s.lens, i32(n), max(n), s.R, pages=s.pages())
    q, k, v = s.project(max(n), 1)
    lib.qk_norm_rope_cache(q, k, v, s.qw, s.kw, positions, s.f, s.kc, s.vc, slots)
    parents, counts = i32([[-1] * T] * B), i32([T] * B)
    x = torch.zeros(B, T, s.H + 2 * s.Hkv, s.D, device="cuda", dtype=torch.bfloat16)
    q, k, v = x.split([s.H, s.Hkv, s.Hkv], dim=2)

    def work(table, free, kc, vc, lens, pool):
        mask, depths = lib.tree_mask(parents)
        grown, slots, positions, after = lib.cache_step(lens, counts, T, s.R, pages=(table, free, pool), depths=depths)
        qr = lib.qk_norm_rope_cache(q, k, v, s.qw, s.kw, positions, s.f, kc, vc, slots)
        return lib.sdpa_tree_paged(qr, kc, vc, grown, table, mask), grown, after, slots

    mine = [t.clone() for t in (s.table, s.free, s.kc, s.vc, lens, pool)]
    work(*[t.clone() for t in mine])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = work(*mine)
    for turn in range(4):
        rng = random.Random(turn)
        parents.copy_(i32([a_tree(T, rng) for _ in range(B)]))
        x.copy_(torch.randn(x.shape, device="cuda", generator=torch.Generator("cuda").manual_seed(turn)).to(x.dtype))
        theirs = [t.clone() for t in mine]
        graph.replay()
        torch.cuda.synchronize()
        want = work(*theirs)
        assert all(torch.equal(a, b) for a, b in zip(got, want)) and torch.equal(mine[0], theirs[0]) and torch.equal(mine[1], theirs[1])
        # some of the drafts are kept, the others dropped
        kept = i32([-(turn * 3 + b) % (T + 1) - T for b in range(B)])
        after = lib.cache_step(got[1], kept, T, s.R, pages=(mine[0], mine[1], got[2]))
        assert int(after[3][1]) == 0
        mine[4].copy_(after[0])
        mine[5].copy_(after[3])


def test_trees_of_several_sizes_in_one_batch(lib):
    """Smaller trees take the last places behind a chain that stands for cached rows: each entry against its own tree alone."""
    B, H, Hkv, T, cap, D = 5, 8, 2, 20, 400, 128
    had, counts = [300, 40, 3, 64, 200], [20, 7, 2, 1, 0]
    rng = random.Random(5)
    own = [a_tree(c, rng) for c in counts]
    parents = [[i - 1 for i in range(T - c)] + [T - c + p for p in tree] for tree, c in zip(own, counts)]      # (a root follows the chain's end, or nothing)
    mask, depths = lib.tree_mask(i32(parents))
    grown, slots, positions, _ = lib.cache_step(i32(had), i32(counts), T, cap, depths=depths)
    for b, c in enumerate(counts):
        assert positions[b].tolist() == [0] * (T - c) + [had[b] + d for d in ref.ancestors(own[b])[1]]
        assert slots[b].tolist() == [-1] * (T - c) + [b * cap + had[b] + i for i in range(c)]
    q, k, v = inputs(B, H, Hkv, T, cap, D, torch.bfloat16, 7)
    o = lib.sdpa_tree(q, k, v, mask, kv_lens=grown)
    for b, c in enumerate(counts):
        if c > 0:
            check(lib, q[b:b + 1, :, T - c:], k[b:b + 1], v[b:b + 1], [had[b] + c], [ref.ancestors(own[b])[0]], o[b:b + 1, :, T - c:])


def test_caches_past_2_to_the_31(lib):
    """Entries and pages on both sides of 2^31 elements, dense and paged, in every form."""
    B, Hkv, cap, D, R = 3, 2, 4_000_000, 128, 128
    lens = [300, 0, 257]
    cache = [torch.empty(B, Hkv, cap, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    pages = [x.view(B * cap // R, Hkv, R, D) for x in cache]
    last = pages[0].shape[0] - 1
    table = i32([[0, last, 5], [7, 8, 9], [last - 1, 40000, 70000]])
    for T, H in ((4, 4), (15, 4), (40, 4), (90, 4)):
        q, k, v = inputs(B, H, Hkv, T, max(lens), D, torch.bfloat16, T)
        sees = [ref.ancestors(a_tree(T, random.Random(b)))[0] for b in range(B)]
        mask = torch.stack([ref.words_of(s, T) for s in sees]).cuda()
        for x, y in zip(cache, (k, v)):
            for b, n in enumerate(lens):
                x[b, :, :n] = y[b, :, :n]
        check(lib, q, k, v, lens, sees, lib.sdpa_tree(q, *cache, mask, kv_lens=i32(lens)))
        for x, y in zip(pages, (k, v)):
            for b, n in enumerate(lens):
                for i in range(-(-n // R)):
                    part = y[b, :, i * R:min(n, i * R + R)]
                    x[int(table[b, i]), :, :part.shape[1]] = part
        check(lib, q, k, v, lens, sees, lib.sdpa_tree_paged(q, *pages, i32(lens), table, mask))
