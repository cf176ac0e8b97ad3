"""The attention kernels over 8-bit caches on the compiler's own output (no GPU): no registers spilled where a wavefront spends its time; tiles of codes go
straight to the LDS in the two forms that count their loads, whose waits are the ones written; conversions, not shuffles, between LDS and matrix instructions."""
import re
import subprocess
from concurrent.futures import ThreadPoolExecutor
from pathlib import Path

import pytest

from test_kernel_budget import CSRC, HIPCC
from test_tree_kernels_host import loops_of

# Scratch accesses in the loop over unmasked tiles of the large tiles (two tiles a turn), by head dim: the most of either type, dense or paged.
UNMASKED = {64: 0, 96: 0, 128: 0, 160: 4}


@pytest.fixture(scope="module")
def listings(tmp_path_factory):
    if not Path(HIPCC).exists():
        pytest.skip("hipcc not available")
    from paper_2603_01960_amd import build as lib_build
    d = tmp_path_factory.mktemp("cache8")

    def one(src):
        asm = d / (src.stem + ".s")
        subprocess.run([HIPCC, *lib_build.FLAGS, *lib_build.extra_flags(src), "-S", "--cuda-device-only", str(src), "-o", str(asm)], check=True,
                       capture_output=True, timeout=600)
        kernels, name = {}, None
        for line in asm.read_text().split("\n"):
            m = re.match(r"^(_ZN5tsdpa\d+sdpa_cache8_\w+_kernel\S+):", line)
            if m:
                name = m.group(1)
                kernels[name] = []
            elif name is not None:
                kernels[name].append(line)
                if line.startswith(".Lfunc_end"):
                    name = None
        return src.stem, kernels

    with ThreadPoolExecutor(max_workers=8) as ex:
        return dict(ex.map(one, sorted(CSRC.glob("sdpa_cache8_*.hip"))))


def head_dim(name):
    return int(re.search(r"Li(\d+)E", name).group(1))


@pytest.mark.parametrize("form", ["decode", "rows"])
def test_kernels_that_count_their_loads(listings, form):
    for dtype in ("f16", "bf16"):
        kernels = listings[f"sdpa_cache8_{form}_{dtype}"]
        assert len(kernels) == 8
        for name, lines in kernels.items():
            each = head_dim(name) * 64 // 1024
            assert not any("scratch_" in line for line in lines), name
            loops = [body for body in loops_of(lines) if any("v_mfma" in line for line in body)]
            assert len(loops) == 1, name
            body = loops[0]
            assert sum("buffer_load" in line and " lds" in line for line in body) == 2 * each, name
            assert not any("ds_bpermute" in line or "ds_write" in line for line in body), name
            waits = [int(w) for line in body for w in re.findall(r"vmcnt\((\d+)\)", line)]
            assert waits.count(each) >= 2, f"{name}: waits {waits}"


def test_large_tiles(listings):
    for dtype in ("f16", "bf16"):
        kernels = listings[f"sdpa_cache8_chunk_{dtype}"]
        assert len(kernels) == 8
        for name, lines in kernels.items():
            loops = [body for body in loops_of(lines) if any("v_mfma" in line for line in body)]
            spilled = [sum("scratch_" in line for line in body) for body in loops]
            assert len(loops) == 2 and spilled[0] <= UNMASKED[head_dim(name)], f"{name}: {spilled}"
