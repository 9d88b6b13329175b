"""Registers and spilled words of the prompt kernels, from the built code objects: their forms are chosen, and their loops laid out, for two or three waves a
SIMD (512 registers, handed out in eights), and a reload in a loop waits for the rows asked for."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2506_18226_amd import build as B

BIN = "/opt/rocm/llvm/bin"


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """Mangled name -> (registers, spilled words)."""
    if not os.path.exists(f"{BIN}/llvm-objdump"):
        pytest.skip("no llvm-objdump beside hipcc")
    if not os.path.exists(B.LIB_PATH):
        B.build_library()
    tmp = tmp_path_factory.mktemp("lib")
    subprocess.run([f"{BIN}/llvm-objdump", "--offloading", shutil.copy(B.LIB_PATH, tmp)], check=True, capture_output=True, cwd=tmp, timeout=60)
    found = {}
    for name in sorted(os.listdir(tmp)):
        if "gfx950" not in name:
            continue
        notes = subprocess.run([f"{BIN}/llvm-readelf", "--notes", str(tmp / name)], check=True, capture_output=True, text=True, timeout=60).stdout
        for kernel in notes.split("- .agpr_count")[1:]:
            number = lambda key: int(re.search(rf"\.{key}:\s+(\d+)", kernel).group(1))
            found[re.search(r"\.name:\s+(\S+)", kernel).group(1)] = number("vgpr_count"), number("vgpr_spill_count")
    return found


# mangled name and template arguments, waves per SIMD, spilled words at most
@pytest.mark.parametrize("kernel,waves,spilled", [
    (r"k_prompt_manyILi64ELi4ELi[01]ELb0E", 3, 5), (r"k_prompt_manyILi64ELi4ELi([23]ELb0|[0123]ELb1)E", 2, 0), (r"k_prompt_manyILi128ELi4ELi[01]E", 2, 4), (r"k_prompt_manyILi128ELi4ELi[23]ELb0E", 2, 35),
    (r"k_prompt_manyILi128ELi4ELi[23]ELb1E", 2, 109),
    (r"k_promptILi2ELi64ELi4ELb[01]E", 2, 0), (r"k_promptILi2ELi128ELi4ELb0E", 2, 0), (r"k_promptILi2ELi128ELi4ELb1E", 2, 14), (r"k_promptILi4ELi64ELi4ELb[01]E", 2, 6),
    (r"k_promptILi4ELi128ELi2ELb[01]E", 1, 2), (r"k_prompt_massILi2E", 2, 0), (r"k_prompt_massILi4E", 1, 0), (r"k_sharedILi2ELi64ELi4ELi[03]ELb[01]ELb0E", 3, 3),
    (r"k_sharedILi2ELi64ELi4ELi[0123]ELb[01]ELb1E", 2, 0), (r"k_sharedILi2ELi128E", 2, 6), (r"k_sharedILi4ELi64E", 2, 0), (r"k_sharedILi4ELi128E", 1, 0),
    (r"k_rotateILi[24]E", 4, 0), (r"k_prompt_finishI", 8, 0), (r"k_shared_finishI", 4, 0)])
def test_waves_per_simd_and_spills(kernels, kernel, waves, spilled):
    mine = {k: v for k, v in kernels.items() if re.search(kernel, k)}
    assert mine
    for name, (registers, words) in mine.items():
        assert 512 // ((registers + 7) // 8 * 8) >= waves and words <= spilled, (name, registers, words)
