"""What the two-length Pass 1 keeps in registers, read from the built library: its whole blocks at
bf16 d = 64 fit three waves per SIMD (512 registers a lane: 170 each) with a bias as without one,
and those at d = 128 and two waves spill next to nothing in their loop."""
import re
import subprocess

import pytest

from tests.test_wait_states_cpu import code_objects, llvm_tool


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    found = {}
    for obj in code_objects(str(tmp_path_factory.mktemp("objects"))):
        notes = subprocess.run([llvm_tool("llvm-readelf"), "--notes", obj], check=True, capture_output=True,
                               text=True).stdout
        for kernel in notes.split("- .agpr_count")[1:]:
            name = re.search(r"\.symbol:\s+(\S+)\.kd", kernel).group(1)
            found[name] = tuple(int(re.search(rf"\.{what}:\s+(\d+)", kernel).group(1))
                                for what in ("vgpr_count", "vgpr_spill_count"))
    return found


def pass1(kernels, d, shape, bias):
    """(registers, spilled ones) of ext_pass1_kernel<bf16, d, shape..., bias>."""
    args = "".join(f"Li{n}E" for n in (d, *shape)) + f"Lb{int(bias)}E"
    match = [v for k, v in kernels.items() if k.startswith("_ZN2fb16ext_pass1_kernelIDF16b" + args)]
    assert len(match) == 1, (args, len(match))
    return match[0]


@pytest.mark.parametrize("bias", [False, True])
def test_three_waves_per_simd_at_d64(kernels, bias):
    registers, spilled = pass1(kernels, 64, (1, 4, 2, 1, 0), bias)
    assert registers <= 168 and spilled == 0


@pytest.mark.parametrize("bias,most", [(False, 0), (True, 2)])
def test_spills_at_d128(kernels, bias, most):
    registers, spilled = pass1(kernels, 128, (1, 8, 2, 1, 1), bias)
    assert registers <= 256 and spilled <= most
