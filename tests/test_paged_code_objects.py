"""What the compiler made of the kernels that read pages: facts of the built library that their speed and results rest on."""
import re
import subprocess

import pytest

from test_code_objects import LLVM, code_objects  # noqa: F401  (the fixture)


@pytest.fixture(scope="module")
def paged(code_objects):  # noqa: F811
    """The code object that holds them, and its kernels' resources."""
    for path in code_objects:
        notes = subprocess.run([f"{LLVM}/llvm-readelf", "--notes", path], capture_output=True, text=True, check=True).stdout
        kernels = {re.search(r"\.name:\s+(\S+)", k)[1]: k for k in re.split(r"\n\s+- \.agpr_count", notes)[1:]}
        if any("k_paged_attn" in name for name in kernels):
            return path, kernels
    raise AssertionError("no kernels over pages")


def test_kernels_over_bf16_pages_keep_their_vectors_in_registers(paged):
    seen = 0
    for name, notes in paged[1].items():
        # k_paged_attn<D, NWAVES, KV8, KS, FIND, WHOLE>, k_paged_few<D, KV8>, k_paged_mix<D, KV8, WHOLE>, k_paged_join<D>
        if re.search(r"k_paged_attnILi\d+ELi\d+ELb0|k_paged_(few|mix)ILi\d+ELb0|k_paged_join", name):
            seen += 1
            assert re.search(r"\.vgpr_spill_count:\s+0\b", notes) and re.search(r"\.private_segment_fixed_size:\s+0\b", notes), name
    assert seen == 28           # ten, few and two of mix for both sizes of a head, and two of the join


def test_addresses_in_scalars_are_written_long_before_loads_use_them(paged):
    """A vector instruction's scalar result may be a memory instruction's address five wait states later; the compiler does not see addresses inside inline
    assembly, so the distance is checked in what it made."""
    text = subprocess.run([f"{LLVM}/llvm-objdump", "-d", "--no-show-raw-insn", paged[0]], capture_output=True, text=True, check=True).stdout
    recent, loads, near = [], 0, []             # (wait states so far, first and last register)
    at = 0
    for line in text.splitlines():
        line = line.split("//")[0].strip()
        if not line or line.endswith(":"):
            continue
        m = re.match(r"global_load_lds_dword\w* \w+, s\[(\d+):(\d+)\]", line)
        if m:
            loads += 1
            a, b = int(m[1]), int(m[2])
            near += [line for t, lo, hi in recent if at - t <= 5 and lo <= b and hi >= a]
        at += 1 + (int(line.split()[1], 0) if line.startswith("s_nop") else 0)
        w = re.match(r"v_(?:readfirstlane|readlane)_b32 s(\d+)|v_cmp\w+ s\[(\d+):(\d+)\]", line)
        if w:
            lo = int(w[1] or w[2])
            recent = [r for r in recent if at - r[0] <= 8] + [(at, lo, int(w[3] or lo) if w[3] else lo)]
    assert loads > 100 and near == []
