"""Registers that the large tiles of attention over 8-bit caches keep in scratch memory, on the compiler's own output (no GPU): none in the loop over unmasked tiles,
some in the loop over masked tiles (the causal mask's, the last ones of an entry; all of a short chunk) from D = 128 on."""
import re
import subprocess
from concurrent.futures import ThreadPoolExecutor
from pathlib import Path

import pytest

from test_cache8_loops_host import head_dim
from test_kernel_budget import CSRC, HIPCC
from test_tree_kernels_host import loops_of

# (unmasked, two tiles a turn; masked, two forms of a tile, one of which runs), by head dim: the most of either type, dense or paged
MOST = {64: (0, 0), 96: (0, 0), 128: (0, 8), 160: (0, 55)}


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    if not Path(HIPCC).exists():
        pytest.skip("hipcc not available")
    from paper_2603_01960_amd import build as lib_build
    d = tmp_path_factory.mktemp("scratch")

    def one(src):
        asm = d / (src.stem + ".s")
        subprocess.run([HIPCC, *lib_build.FLAGS, *lib_build.extra_flags(src), "-S", "--cuda-device-only", str(src), "-o", str(asm)], check=True,
                       capture_output=True, timeout=600)
        found, name = {}, None
        for line in asm.read_text().split("\n"):
            m = re.match(r"^(_ZN5tsdpa\d+sdpa_cache8_chunk_kernel\S+):", line)
            if m:
                name = m.group(1)
                found[name] = []
            elif name is not None:
                found[name].append(line)
                if line.startswith(".Lfunc_end"):
                    name = None
        return found

    with ThreadPoolExecutor(max_workers=2) as ex:
        return {name: lines for found in ex.map(one, sorted(CSRC.glob("sdpa_cache8_chunk_*.hip"))) for name, lines in found.items()}


def test_scratch_accesses_of_large_tiles(kernels):
    assert len(kernels) == 16
    for name, lines in kernels.items():
        loops = [body for body in loops_of(lines) if any("v_mfma" in line for line in body)]
        spilled = tuple(sum("scratch_" in line for line in body) for body in loops)
        print(name, head_dim(name), spilled)
        assert len(spilled) == 2 and all(n <= most for n, most in zip(spilled, MOST[head_dim(name)])), f"{name}: {spilled}"
