"""The product kernels' assembly on the CPU: their direct-to-LDS loads read bases that scalar instructions have formed (or formed long
enough before), M0 is written a state before its use, and an address that a load's offset takes back never falls below 0."""
import os
import re
import subprocess

import pytest

from paper_2407_20485_amd import build
from test_dma_statements import too_close


@pytest.fixture(scope="module")
def kernels():
    out = subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), *build.COMMON, "--cuda-device-only", "-S", "-o", "-",
                          os.path.join(build.CSRC, "matmul.hip")], capture_output=True, text=True, check=True).stdout
    found = {}
    for m in re.finditer(r"^(_ZN\w*matmul_tile_kernel\w*):(.*?)\.size", out, re.S | re.M):
        lines = [ln.split(";")[0].strip().replace("\t", " ") for ln in m[2].splitlines()]
        found[m[1]] = [ln for ln in lines if ln and not ln.startswith(".") and not ln.endswith(":")]
    return found


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
        edge = int(re.search(r"Li(\d+)E", name)[1])
        waves = 8 if edge == 256 else 4
        share = (edge // 32) ** 2 // waves * (4 if "IfLi" in name else 1)
        assert most <= 2 * share, (name, most, share)  # (two, where the text of one loop follows another's)
