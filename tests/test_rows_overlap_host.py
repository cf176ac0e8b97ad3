"""Whether strided rows share memory (csrc/rows_overlap.h), against the sets of their bytes."""
import random
import shutil
import subprocess
from pathlib import Path

import pytest

CSRC = Path(__file__).resolve().parents[1] / "paper_2603_01960_amd" / "csrc"
CXX = shutil.which("g++") or shutil.which("c++")

PROGRAM = r"""
#include <cstdio>
#include "rows_overlap.h"
static bool read(tsdpa::RowSet &r)
{
    long long at, bytes;
    if (std::scanf("%lld %lld %d", &at, &bytes, &r.dims) != 3) return false;
    r.at = at;
    r.bytes = bytes;
    for (int i = 0; i < r.dims; ++i) {
        long long stride, size;
        if (std::scanf("%lld %lld", &stride, &size) != 2) return false;
        r.dim[i] = {stride, size};
    }
    return true;
}
int main()
{
    tsdpa::RowSet a{}, b{};
    while (read(a) && read(b)) std::printf("%d", tsdpa::RowsOverlap()(a, b) ? 1 : 0);
}
"""


@pytest.fixture(scope="module")
def overlap(tmp_path_factory):
    if CXX is None:
        pytest.skip("no host compiler")
    d = tmp_path_factory.mktemp("overlap")
    (d / "overlap.cpp").write_text(PROGRAM)
    subprocess.run([CXX, "-O2", "-std=c++17", "-Wall", "-Werror", f"-I{CSRC}", str(d / "overlap.cpp"), "-o", str(d / "overlap")], check=True)

    def ask(pairs):
        text = "\n".join(f"{at} {n} {len(dims)} " + " ".join(f"{s} {m}" for s, m in dims) for pair in pairs for at, n, dims in pair)
        out = subprocess.run([str(d / "overlap")], input=text, capture_output=True, text=True, check=True).stdout
        assert len(out) == len(pairs)
        return [c == "1" for c in out]

    return ask


def bytes_of(at, n, dims):
    starts = {at}
    for stride, size in dims:
        starts = {s + stride * i for s in starts for i in range(size)}
    return {s + i for s in starts for i in range(n)}


def test_any_small_sets(overlap):
    """Random rows and strides, those of 0 and of rows that overlap themselves among them, dimensions of none and one."""
    rng = random.Random(0)
    pairs = []
    for _ in range(4000):
        sets = []
        for _ in range(2):
            dims = [(rng.choice([0, 1, 3, 8, 8, 16, 24, 40, 64, 100, 128]), rng.choice([0, 1, 2, 3, 5])) for _ in range(rng.randrange(4))]
            sets.append((rng.randrange(0, 200), rng.choice([0, 1, 4, 8, 16, 30]), dims))
        pairs.append(sets)
    want = [bool(bytes_of(*a) & bytes_of(*b)) for a, b in pairs]
    assert 400 < sum(want) < 3600
    assert overlap(pairs) == want


def test_views_of_a_projection(overlap):
    """Heads of Q, K and V in one packed tensor, [B, S, heads, D] of 2 bytes: apart at any size; one head further they are not."""
    pairs, want = [], []
    for B, S, H, Hkv, D in ((1, 1, 1, 1, 64), (2, 8192, 32, 8, 128), (64, 197, 12, 12, 64), (1, 140000, 128, 1, 128), (4, 2048, 16, 4, 160)):
        row = (H + 2 * Hkv) * D * 2
        view = lambda head, heads, n=D * 2: (head * D * 2, n, [(S * row, B), (row, S), (D * 2, heads)])
        pairs += [(view(0, H), view(H, Hkv)), (view(H, Hkv), view(H + Hkv, Hkv)), (view(0, H + 1), view(H, Hkv)), (view(H, Hkv), view(H, Hkv))]
        want += [False, False, True, True]
        # contiguous memory behind, in front of, and over the last element
        end = B * S * row
        pairs += [(view(0, H), (end, 1000, [])), (view(H + Hkv, Hkv), (end - 2, 1000, [])), ((-64, 64, []), view(0, H)), ((end - row + H * D * 2, 2 * D, []), view(0, H))]
        want += [False, True, False, False]
        # the halves of wider rows, and tokens taken in turns
        half = lambda first: (first * 2, D, [(S * row, B), (row, S), (D * 2, H)])
        turns = lambda t: (t * row, D * 2, [(2 * row, B * S), (D * 2, H)])
        pairs += [(half(0), half(D // 2)), (half(0), half(D // 2 - 1)), (turns(0), turns(1)), (turns(0), turns(2))]
        want += [False, True, False, B * S > 1]
    assert overlap(pairs) == want


def test_strides_that_have_nothing_to_do_with_each_other_end(overlap):
    """Large sets that take too many tries come back all the same."""
    a, b = (0, 2, [(1 << 30, 4), (9_999_991 * 4, 1000), (1_000_003 * 4, 1000)]), (2, 2, [(1 << 29, 8), (7_777_777 * 4, 1000), (999_983 * 4, 1000)])
    overlap([(a, b)])
