"""The product kernels' assembly on the CPU: their direct-to-LDS loads read bases that scalar instructions have formed (or formed long
enough before), M0 is written a state before its use, and an address that a load's offset takes back never falls below 0."""
import os
import re
import subprocess

import pytest

from paper_2407_20485_amd import build
from test_dma_statements import too_close


@pytest.fixture(scope="module")
def assembly():
    return subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), *build.COMMON, "--cuda-device-only", "-S", "-o", "-",
                          os.path.join(build.CSRC, "matmul.hip")], capture_output=True, text=True, check=True).stdout


def bodies(assembly, name):
    found = {}
    for m in re.finditer(r"^(_ZN\w*%s\w*):(.*?)\.size" % name, assembly, re.S | re.M):
        lines = [ln.split(";")[0].strip().replace("\t", " ") for ln in m[2].splitlines()]
        found[m[1]] = [ln for ln in lines if ln and not ln.startswith(".") and not ln.endswith(":")]
    return found


@pytest.fixture(scope="module")
def kernels(assembly):
    return bodies(assembly, "matmul_tile_kernel")


def test_distances_before_direct_loads(kernels):
    assert len(kernels) >= 4
    for name, lines in kernels.items():
        close, loads = too_close(lines)
        assert loads > 20 and not close, (name, close[:3])


def test_no_spills_and_ordered_products(kernels):
    """Operands stay in registers, and between two barriers of the unrolled group there is not more than one half block's share of
    matrix instructions (the compiler does not gather them at its end)."""
    for name, lines in kernels.items():
        assert not any(ln.startswith("scratch_") for ln in lines), name
        run, most = 0, 0
        for ln in lines:
            run = 0 if ln.startswith("s_barrier") else run + ln.startswith("v_mfma")
            most = max(most, run)
        rows, columns = (int(x) for x in re.search(r"Li(\d+)ELi(\d+)E", name).groups())
        waves = 8 if rows == 256 else 4
        share = (rows // 32) * (columns // 32) // waves * (4 if "IfLi" in name else 1)
        assert most <= 2 * share, (name, most, share)  # (two, where the text of one loop follows another's)


def test_strips(assembly):
    """The same distances where few rows stream through rings, nothing spilled, and the loop's waits leave loads under way."""
    strips = bodies(assembly, "matmul_strip_kernel")
    assert len(strips) >= 8
    for name, lines in strips.items():
        close, loads = too_close(lines)
        assert loads >= 12 and not close, (name, close[:3])
        assert not any(ln.startswith("scratch_") for ln in lines), name
        per_step = 4 + 2 * int(re.search(r"Li(\d+)E", name)[1])
        ahead = [int(n) for ln in lines for n in re.findall(r"s_waitcnt vmcnt\((\d+)\)$", ln)]
        assert any(n > 0 and n % per_step == 0 for n in ahead), (name, ahead)


def test_first_stages_are_written_before_the_first_barrier(kernels):
    """A half block that k ends in is written to LDS by way of registers, also when it is the first (k < 64): those writes have
    arrived before the barrier behind which other waves read them."""
    for name, lines in kernels.items():
        barrier = lines.index("s_barrier")
        writes = [i for i, ln in enumerate(lines[:barrier]) if ln.startswith("ds_write")]
        assert writes, name
        assert any(ln.startswith("s_waitcnt") and "lgkmcnt(0)" in ln for ln in lines[writes[-1]: barrier]), name
