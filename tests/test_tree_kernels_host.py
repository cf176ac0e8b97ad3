"""The streams of the tree kernels on the compiler's own output (no GPU): their loop counts its loads to the LDS and reads the LDS in assembly, so
that two tiles are on their way while one is worked on.  A wait for all loads in it (the compiler's, in front of an LDS access that it takes for one
of theirs) or a register spilled there would keep the results and lose that."""
import re
import shutil
import subprocess
from pathlib import Path

import pytest

from test_kernel_budget import CSRC, HIPCC, kernels_of


def loops_of(lines):
    """Lines of the blocks of each depth-1 loop, in the order of their headers (blocks of a loop may stand in front of its header)."""
    loops, order, current = {}, [], None
    for line in lines:
        if re.match(r"^(\.LBB\d+_\d+:|; %bb\.\d+:)", line):
            header, inside = re.match(r"^\.L(BB\d+_\d+):.*Loop Header: Depth=1", line), re.search(r"in Loop: Header=(BB\d+_\d+)", line)
            label = header.group(1) if header else inside.group(1) if inside else None
            if header:
                order.append(label)
            current = loops.setdefault(label, []) if label else None
        elif current is not None:
            current.append(line)
    return [loops[label] for label in order]


@pytest.mark.skipif(not Path(HIPCC).exists(), reason="hipcc not available")
@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("f16", 96), ("bf16", 128), ("f16", 160)])
def test_loops_of_the_streams(dtype, D, tmp_path):
    from paper_2603_01960_amd import build as lib_build

    src, asm = CSRC / f"sdpa_tree_{dtype}_d{D}.hip", tmp_path / "tree.s"
    subprocess.run([HIPCC, *lib_build.FLAGS, *lib_build.extra_flags(src), "-S", "--cuda-device-only", str(src), "-o", str(asm)], check=True,
                   capture_output=True, timeout=600)
    kernels = kernels_of(asm.read_text())
    checked = 0
    for name, lines in kernels.items():
        m = re.search(r"Li%dELi(\d)ELi(\d+)ELi2ELi([56])E" % D, name)
        assert m, name
        waves, loops = int(m.group(1)), [body for body in loops_of(lines) if any("v_mfma" in line for line in body)]
        assert len(loops) == 2, f"{name}: {len(loops)} loops with matrix instructions (unmasked tiles, masked tiles)"
        # the loop over the unmasked tiles: two steps written out
        body = loops[0]
        assert not any("scratch_" in line for line in body), f"{name}: registers spilled in the loop"
        loads = sum("buffer_load" in line and " lds" in line for line in body)
        tile = D * 2 * 32 // 1024                 # load instructions per tile, shared out over the wavefronts
        assert loads == 2 * 2 * tile // waves, f"{name}: {loads} loads of two tiles' K and V"
        waits = [int(w) for line in body for w in re.findall(r"vmcnt\((\d+)\)", line)]
        assert waits.count(2 * tile // waves) == 4 and min(waits) == 2 * tile // waves, f"{name}: waits {waits}"
        assert sum("s_barrier" in line for line in body) == (4 if waves > 1 else 0), name
        checked += 1
    assert checked == 4, f"32 and 64 rows, dense and paged: found {checked}"
