"""Masks of drafted trees and cache steps on the GPU against their definitions (whole numbers: equal)."""
import random

import pytest
import torch

import reference64 as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib():
    from paper_2603_01960_amd import binding
    binding.load_library()
    return binding


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def trees(T, seed):
    rng = random.Random(seed)
    return [[i - 1 for i in range(T)],                                   # a chain
            [-1] * T,                                                    # all follow the sequence
            [rng.randrange(-1, i) if i else -1 for i in range(T)],       # any earlier token
            [max(-1, i - rng.randrange(1, 9)) for i in range(T)],        # one of the last few
            [(i - 1) // 2 if i else -1 for i in range(T)],               # two tokens after each
            [rng.choice([i - 1, i, i + 1, T, -7, 2 ** 31 - 1, -2 ** 31]) for i in range(T)]]     # numbers that name no earlier token


@pytest.mark.parametrize("T", [1, 2, 15, 63, 64, 65, 128, 129, 255, 511, 1024])
def test_tree_mask(lib, T):
    parents = trees(T, T)
    mask, depths = lib.tree_mask(i32(parents))
    assert mask.shape == (len(parents), T, (T + 63) // 64) and mask.dtype == torch.int64 and depths.dtype == torch.int32
    for b, p in enumerate(parents):
        sets, depth = ref.ancestors(p)
        assert depths[b].tolist() == depth
        assert torch.equal(mask[b].cpu(), ref.words_of(sets, T))
    one_mask, one_depths = lib.tree_mask(i32(parents[2]))
    assert one_mask.shape == (T, (T + 63) // 64) and torch.equal(one_mask, mask[2]) and torch.equal(one_depths, depths[2])
    out = torch.empty_like(mask), torch.empty_like(depths)
    mask.fill_(-1)                               # (the results of a call do not overlap)
    assert bool((depths == lib.tree_mask(i32(parents))[1]).all())
    mask = lib.tree_mask(i32(parents))[0]
    got = lib.tree_mask(i32(parents), out=out)
    assert got[0] is out[0] and got[1] is out[1] and torch.equal(out[0], mask)


def test_tree_mask_refusals(lib):
    for bad in (torch.zeros(4, dtype=torch.int64, device="cuda"), torch.zeros(2, 2, 2, dtype=torch.int32, device="cuda"), torch.zeros(4, 4, dtype=torch.int32, device="cuda").T):
        with pytest.raises(ValueError, match="parents"):
            lib.tree_mask(bad)
    with pytest.raises(lib.TiledSdpaError) as e:
        lib.tree_mask(torch.zeros(1025, dtype=torch.int32, device="cuda"))
    assert e.value.status == 2
    with pytest.raises(ValueError, match="out must be"):
        lib.tree_mask(i32([[0, 0]]), out=(torch.zeros(1, 2, 1, dtype=torch.int32, device="cuda"), i32([[0, 0]])))
    assert lib.tree_mask(torch.zeros(0, 5, dtype=torch.int32, device="cuda"))[0].shape == (0, 5, 1)


class Pool:
    """A paged cache's state on the GPU and as lists."""

    def __init__(self, lib, B, M, R, lens, extra, seed):
        rng = random.Random(seed)
        self.lib, self.R = lib, R
        held = [-(-n // R) for n in lens]
        pages = list(range(sum(held) + extra))
        rng.shuffle(pages)
        self.lens, self.table = list(lens), [[-9] * M for _ in range(B)]
        for b in range(B):
            for x in range(held[b]):
                self.table[b][x] = pages.pop()
        self.have = len(pages)
        self.free = pages + [-9] * (sum(held) + 3)
        self.gpu = i32(self.lens), i32(self.table).view(B, M), i32(self.free), i32([self.have, 0])

    def step(self, counts, S, depths=None):
        lens, table, free, pool = self.gpu
        got = self.lib.cache_step(lens, i32(counts), S, self.R, pages=(table, free, pool), depths=None if depths is None else i32(depths))
        want = ref.step(self.lens, counts, S, self.R, self.table, self.free, self.have, depths)
        for name, a, b in zip(("new_lens", "slots", "positions", "new_pool"), got, want):
            assert a.cpu().flatten().tolist() == [y for x in b for y in (x if isinstance(x, list) else [x])], name
        assert table.tolist() == self.table and free.tolist()[:want[3][0]] == self.free[:want[3][0]]
        assert free.tolist() == self.free                                # what lies past the pool's count is left alone, or alike
        self.lens, self.have = want[0], want[3][0]
        self.gpu = got[0], table, free, got[3]
        return want[3][1]


# (the second of 64 entries: a pool so small that every step is refused)
@pytest.mark.parametrize("B,M,R,S,spare", [(1, 3, 64, 1, 0), (1, 40, 64, 1500, 0), (5, 7, 64, 33, 0), (300, 9, 128, 17, 0), (64, 33, 64, 1024, 1100), (64, 33, 64, 1024, 0),
                                           (1000, 4, 256, 2, 0), (3, 5, 48, 0, 0)])
def test_steps_of_a_paged_cache(lib, B, M, R, S, spare):
    """Appending, dropping, both at once (pages go from one entry to another), done requests, new ones, and steps that are refused."""
    rng = random.Random(B * 1000 + S)
    lens = [rng.randrange(0, max(1, M * R - S + 1)) for _ in range(B)]
    pool = Pool(lib, B, M, R, lens, extra=B * 2 + S // R + 2 + spare, seed=B)
    refused = 0
    for turn in range(8):
        counts = []
        for n in pool.lens:
            kind = rng.randrange(6)
            c = S if kind < 2 else rng.randrange(0, S + 1) if kind == 2 else -rng.randrange(0, n + 1) if kind == 3 else -n if kind == 4 and turn % 2 else 0
            counts.append(max(-n, min(c, M * R - n)) if turn % 4 != 3 else c)
        depths = [[rng.randrange(0, S) for _ in range(S)] for _ in range(B)] if turn == 5 and S else None
        refused += pool.step(counts, S, depths) != 0
    assert refused < 8 or (S == 1024 and spare == 0)


def test_dropping_what_was_appended_restores_the_pool(lib):
    pool = Pool(lib, 6, 8, 64, [0, 64, 100, 63, 400, 1], extra=12, seed=1)
    free = list(pool.free)
    counts = [70, 64, 1, 66, 0, 63]
    assert pool.step(counts, 70) == 0 and pool.step([-c for c in counts], 70) == 0
    assert pool.free[:pool.have] == free[:pool.have]
    first = pool.gpu[1].clone()
    assert pool.step(counts, 70) == 0 and torch.equal(first, pool.gpu[1])


def test_the_results_of_a_call_do_not_overlap(lib):
    got = lib.cache_step(i32([3, 4, 5]), i32([7, 0, 2]), 7, 64)
    want = [x.clone() for x in got]
    for i, x in enumerate(got):
        x.fill_(77)
        assert all(torch.equal(a, b) for a, b in zip(got[i + 1:], want[i + 1:]))
        assert bool((x == 77).all())


def test_refused_steps_change_nothing(lib):
    base = [10, 64, 128]
    for counts, S, pool_now, missing in (([200, 0, 0], 200, None, 2), ([300, 0, 0], 300, None, 4 + 1), ([5, -65, 0], 5, None, -1), ([6, 0, 0], 5, None, -1),
                                         ([1, 1, 1], 1, -1, -1), ([1, 1, 1], 1, 10 ** 6, -1), ([2 ** 31 - 1, 0, 0], 5, None, -1)):
        p = Pool(lib, 3, 4, 64, base, extra=1, seed=2)
        lens, table, free, pool = p.gpu
        if pool_now is not None:
            pool = i32([pool_now, 0])
        before = table.clone(), free.clone()
        new, slots, positions, after = lib.cache_step(lens, i32(counts), S, 64, pages=(table, free, pool))
        assert new.tolist() == base and bool((slots == -1).all()) and bool((positions == 0).all())
        assert torch.equal(table, before[0]) and torch.equal(free, before[1])
        assert int(after[0]) == int(pool[0]) and (int(after[1]) == missing if missing < 0 else int(after[1]) > 0)
    for lens in ([-1, 0, 0], [64 * 4 + 1, 0, 0]):
        p = Pool(lib, 3, 4, 64, base, extra=1, seed=2)
        got = lib.cache_step(i32(lens), i32([0, 0, 0]), 2, 64, pages=p.gpu[1:])
        assert got[0].tolist() == lens and got[3].tolist() == [p.have, -1] and bool((got[1] == -1).all())


@pytest.mark.parametrize("B,R,S", [(1, 100, 1), (7, 1000, 130), (3, 5000, 2500)])
def test_steps_of_a_dense_cache(lib, B, R, S):
    rng = random.Random(B)
    lens = [rng.randrange(0, R - S + 1) for _ in range(B)]
    for counts in ([S] * B, [-n for n in lens], [rng.randrange(0, S + 1) for _ in range(B)], [R] + [0] * (B - 1)):
        got, want = lib.cache_step(i32(lens), i32(counts), S, R), ref.step(lens, counts, S, R)
        for a, b in zip(got[:3], want[:3]):
            assert a.tolist() == b
        assert got[3].tolist() == want[3]


def test_largest_batch_and_empty_ones(lib):
    B = 8192
    pool = Pool(lib, B, 2, 64, [b % 100 for b in range(B)], extra=B, seed=4)
    assert pool.step([1 if b % 3 else -(b % 100) for b in range(B)], 1) == 0
    empty = torch.zeros(0, dtype=torch.int32, device="cuda")
    table = torch.zeros(0, 4, dtype=torch.int32, device="cuda")
    got = lib.cache_step(empty, empty, 3, 64, pages=(table, i32([5, 6]), i32([2, 0])))
    assert got[3].tolist() == [2, 0] and got[1].shape == (0, 3)
    got = lib.cache_step(i32([0, 0]), i32([0, 1]), 1, 64, pages=(torch.zeros(2, 0, dtype=torch.int32, device="cuda"), i32([5, 6]), i32([2, 0])))
    assert got[0].tolist() == [0, 0] and got[3].tolist() == [2, 1]


def test_cache_step_refusals(lib):
    lens, counts, table, free, pool = i32([3, 4]), i32([1, 1]), i32([[0], [1]]), i32([2, 3]), i32([2, 0])
    for kwargs, text in ((dict(counts=i32([1])), "counts"), (dict(pages=(table, free)), "pages"), (dict(pages=(table, free, i32([2]))), "pages"),
                         (dict(pages=(table[:1], free, pool)), "pages"), (dict(pages=(table.long(), free, pool)), "pages"), (dict(depths=i32([[0]])), "depths"),
                         (dict(out=(lens, i32([[0], [0]]), i32([[0], [0]]), i32([0, 0]))), "other tensors"),
                         (dict(out=(i32([0, 0]), i32([0, 0]), i32([[0], [0]]), i32([0, 0]))), "out must be"),
                         (dict(out=(i32([0, 0]), i32([[0], [0]]), i32([[0], [0]]), pool)), "other tensors")):
        a = dict(counts=counts, pages=(table, free, pool), depths=None, out=None)
        a.update(kwargs)
        with pytest.raises(ValueError, match=text):
            lib.cache_step(lens, a["counts"], 1, 64, pages=a["pages"], depths=a["depths"], out=a["out"])
    with pytest.raises(lib.TiledSdpaError):
        lib.cache_step(lens, counts, 1, 0)
    with pytest.raises(lib.TiledSdpaError):
        lib.cache_step(lens, counts, -1, 64)


def test_outputs_that_overlap_inputs_or_each_other_are_refused(lib):
    both = i32([0] * 8)
    parents, mask, depths = i32([[-1, 0]]), torch.zeros(1, 2, 1, dtype=torch.int64, device="cuda"), i32([[0, 0]])
    for out in ((mask, parents), (mask, mask.view(torch.int32).view(-1)[2:].view(1, 2))):
        with pytest.raises(ValueError, match="overlap"):
            lib.tree_mask(parents, out=out)
    lib.tree_mask(parents, out=(mask, depths))
    lens, counts, table, free, pool = i32([3, 4]), i32([1, 1]), i32([[0], [1]]), i32([2, 3]), i32([2, 0])
    good = [i32([0, 0]), i32([[0], [0]]), i32([[0], [0]]), i32([0, 0])]
    for at, t in ((0, counts), (0, lens), (1, table), (1, both[:2].view(2, 1)), (2, free.view(2, 1)), (3, counts), (3, pool), (3, good[0])):
        out = list(good)
        out[at] = t
        if t.data_ptr() == both.data_ptr():
            out[2] = both[1:3].view(2, 1)
        with pytest.raises(ValueError, match="other tensors"):
            lib.cache_step(lens, counts, 1, 64, pages=(table, free, pool), out=out)
    lib.cache_step(lens, counts, 1, 64, pages=(table, free, pool), out=good)
    assert good[0].tolist() == [4, 5]


def test_what_a_refused_step_lacks(lib):
    """Of an entry that would pass its end the pages up to the end are missing from the pool, those behind it from its row."""
    for lens, counts, R, M, free_now in (([0, 0], [5, 1], 1, 3, 2), ([60, 64], [400, 100], 64, 4, 1), ([0, 100, 7], [10, -100, 300], 64, 2, 0), ([3], [6], 1, 8, 3)):
        p = Pool(lib, len(lens), M, R, lens, extra=free_now, seed=4)
        have = min(p.have, free_now)
        table, free = p.gpu[1].tolist(), p.gpu[2].tolist()
        S = max(counts)
        want = ref.step(lens, counts, S, R, table, free, have)
        assert want[3][1] > 0
        got = lib.cache_step(i32(lens), i32(counts), S, R, pages=(p.gpu[1], p.gpu[2], i32([have, 0])))
        assert [x.tolist() for x in got] == [want[0], want[1], want[2], want[3]]
