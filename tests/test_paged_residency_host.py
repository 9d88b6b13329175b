"""Registers, spilled words and LDS of the kernels over pages and of sampling, from the built code objects.  The forms over pages keep page numbers beside the dense
forms' registers, and spill more than those where they are held to as many waves a SIMD."""
import re
import subprocess

import pytest

from test_residency_host import BIN, code_objects  # noqa: F401  (a fixture)


@pytest.fixture(scope="module")
def kernels(code_objects):  # noqa: F811
    """Mangled name -> (registers, spilled words, bytes of static LDS)."""
    found = {}
    for path in code_objects:
        notes = subprocess.run([f"{BIN}/llvm-readelf", "--notes", path], check=True, capture_output=True, text=True, timeout=60).stdout
        for kernel in notes.split("- .agpr_count")[1:]:
            number = lambda key: int(re.search(rf"\.{key}:\s+(\d+)", kernel).group(1))
            found[re.search(r"\.name:\s+(\S+)", kernel).group(1)] = number("vgpr_count"), number("vgpr_spill_count"), number("group_segment_fixed_size")
    return found


# mangled name and template arguments, waves per SIMD, spilled words at most
@pytest.mark.parametrize("kernel,waves,spilled", [
    (r"k_paged_prompt_manyILi64ELi4ELi0ELb0E", 3, 40), (r"k_paged_prompt_manyILi64ELi4ELi1ELb0E", 3, 65), (r"k_paged_prompt_manyILi64ELi4ELi([23]ELb0|[0123]ELb1)E", 2, 0),
    (r"k_paged_prompt_manyILi128ELi4ELi[01]ELb0E", 2, 0), (r"k_paged_prompt_manyILi128ELi4ELi[01]ELb1E", 2, 64), (r"k_paged_prompt_manyILi128ELi4ELi2ELb0E", 2, 25),
    (r"k_paged_prompt_manyILi128ELi4ELi(3ELb0|[23]ELb1)E", 2, 133),
    (r"k_paged_promptILi2ELi64ELi4ELb[01]E", 2, 0), (r"k_paged_promptILi2ELi128ELi4ELb0E", 2, 0), (r"k_paged_promptILi2ELi128ELi4ELb1E", 2, 9), (r"k_paged_promptILi4ELi64ELi4ELb[01]E", 2, 0),
    (r"k_paged_promptILi4ELi128ELi2ELb[01]E", 1, 2), (r"k_paged_prompt_massILi2E", 2, 0), (r"k_paged_prompt_massILi4E", 1, 0),
    (r"k_attend_gqaILi(64|128)ELi[48]ELb[01]ELi\dELi1E", 2, 0), (r"k_attend_gqaILi(64|128)ELi[48]ELb[01]ELi\dELi2E", 2, 8), (r"k_attendI\w*Li0ELi0ELi[12]EEEv", 3, 0),
    (r"k_compact_planI\w*ELb1EEEv", 4, 0), (r"k_paged_moveILi(4|8)E", 7, 0), (r"k_paged_moveILi16E", 4, 0), (r"k_paged_moveILi24E", 2, 0), (r"k_rotateI\w*ELb1ELb1EEEv", 6, 0),
    (r"k_sampleILi[24]ELi256ELi1024E", 3, 0), (r"k_sampleILi[24]ELi1024ELi2048E", 4, 0), (r"k_sampleILi[24]ELi1024ELi8192E", 4, 54)])
def test_waves_per_simd_and_spills(kernels, kernel, waves, spilled):
    mine = {k: v for k, v in kernels.items() if re.search(kernel, k)}
    assert mine
    for name, (registers, words, _) in mine.items():
        assert 512 // ((registers + 7) // 8 * 8) >= waves and words <= spilled, (name, registers, words)


@pytest.mark.parametrize("kernel,forms,words", [(r"k_attend_gqaILi\d+ELi[48]ELb[01]ELi\dELi0E", 8, 2048), (r"k_attend_gqaILi\d+ELi4ELb[01]ELi\dELi[12]E", 12, 2576),
                                                (r"k_attend_gqaILi\d+ELi8ELb[01]ELi\dELi[12]E", 4, 3104)])
def test_static_words_of_grouped_lists(kernels, kernel, forms, words):
    """What the rule for two workgroups on a compute unit takes them for: dense, and with a row of the table."""
    mine = [v[2] for k, v in kernels.items() if re.search(kernel, k)]
    assert len(mine) == forms and max(mine) <= words
    assert words == 2048 or min(mine) > 2048                 # (the dense figure would not do)
