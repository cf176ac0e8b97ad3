"""Every kernel for trees of drafted tokens on the compiler's own output (no GPU): no registers spilled in the loop over the unmasked tiles, and in
the one over the masked tiles, where what is not finite in V is taken apart, no more than there are.  With weights in halves the streams
count their loads as without (test_tree_kernels_host.py)."""
import re
import subprocess
from concurrent.futures import ThreadPoolExecutor
from pathlib import Path

import pytest

from test_kernel_budget import CSRC, HIPCC, kernels_of
from test_tree_kernels_host import loops_of

# Scratch accesses in the masked loop, by head dim and form (rows of a wavefront's stream, streams): the most of either type, dense or paged.
# Everything else has none.
MASKED = {(128, 32, 4): 10, (128, 64, 2): 5, (128, "halves"): 16, (160, 32, 4): 26, (160, 64, 2): 29, (160, 128, 1): 24}


@pytest.fixture(scope="module")
def listings(tmp_path_factory):
    if not Path(HIPCC).exists():
        pytest.skip("hipcc not available")
    from paper_2603_01960_amd import build as lib_build
    d = tmp_path_factory.mktemp("trees")

    def one(src):
        asm = d / (src.stem + ".s")
        subprocess.run([HIPCC, *lib_build.FLAGS, *lib_build.extra_flags(src), "-S", "--cuda-device-only", str(src), "-o", str(asm)], check=True,
                       capture_output=True, timeout=600)
        return src.stem, kernels_of(asm.read_text())

    with ThreadPoolExecutor(max_workers=8) as ex:
        return dict(ex.map(one, sorted(s for s in CSRC.glob("sdpa_tree_*_d*.hip"))))


def test_all_loops_of_the_trees(listings):
    forms = {}
    for stem, kernels in listings.items():
        for name, lines in kernels.items():
            D, waves, tile, _, kvm = map(int, re.search(r"Li(\d+)ELi(\d+)ELi(\d+)ELi(\d+)ELi(\d+)EEEvPK", name).groups())
            rows, streams = waves * 32, 1 + tile // 1000
            form = (D, "halves") if kvm >= 7 else (D, rows, streams)
            loops = [body for body in loops_of(lines) if any("v_mfma" in line for line in body)]
            assert len(loops) == 2, f"{stem} {name}: {len(loops)} loops with matrix instructions (unmasked tiles, masked tiles)"
            spilled = [sum("scratch_" in line for line in body) for body in loops]
            assert spilled[0] == 0, f"{stem} {name}: {spilled[0]} scratch accesses in the unmasked loop"
            assert spilled[1] <= MASKED.get(form, 0), f"{stem} {name}: {spilled[1]} scratch accesses in the masked loop, {MASKED.get(form, 0)} so far"
            forms[form] = forms.get(form, 0) + 1
            if kvm >= 7:
                body, each = loops[0], 2 * D * 2 * 32 // 1024
                assert sum("buffer_load" in line and " lds" in line for line in body) == 2 * each, name
                waits = [int(w) for line in body for w in re.findall(r"vmcnt\((\d+)\)", line)]
                assert waits.count(each) == 4 and min(waits) == each, f"{name}: waits {waits}"
    wanted = {(D, *form): 4 for D in (64, 96, 128, 160) for form in ((32, 4), (64, 2), (128, 1))}
    assert forms == {**wanted, **{(D, "halves"): 4 for D in (64, 96, 128)}}
