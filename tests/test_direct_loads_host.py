"""Host check on the AMD assembly of the kernels built here for gfx950 that load
from memory straight into LDS through inline assembly. Such a load takes its LDS
address from M0, which a scalar instruction writes; the hardware asks for one
wait state between the two, and the compiler's own hazard pass does not look into
inline assembly. So every M0 write has to be followed by a wait state and then
its load, every load to LDS has to come right after such a pair, and nothing else
may name M0. The same goes for the load's other scalars: five wait states after a
vector instruction wrote one of them."""
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BUILD = os.path.join(ROOT, "paper_1809_02839_amd", "_build")
LLVM = "/opt/rocm/llvm/bin"


def _instructions(obj, tmp_path):
    fat, co = tmp_path / "fatbin", tmp_path / "gfx950.co"
    subprocess.run([os.path.join(LLVM, "llvm-objcopy"), f"--dump-section=.hip_fatbin={fat}", obj,
                    str(tmp_path / "host.o")], check=True, capture_output=True)
    subprocess.run([os.path.join(LLVM, "clang-offload-bundler"), "--unbundle", "--type=o",
                    "--targets=hipv4-amdgcn-amd-amdhsa--gfx950", f"--input={fat}", f"--output={co}"],
                   check=True, capture_output=True)
    dis = subprocess.run([os.path.join(LLVM, "llvm-objdump"), "-d", "--mcpu=gfx950", str(co)], check=True,
                         capture_output=True, text=True).stdout
    lines = [l.split("//")[0].strip() for l in dis.splitlines()]
    return [l for l in lines if l and not l.endswith(":")]


def _scalars(text):
    out = {int(n) for n in re.findall(r"\bs(\d+)\b", text)}
    for a, b in re.findall(r"\bs\[(\d+):(\d+)\]", text):
        out |= set(range(int(a), int(b) + 1))
    return out


@pytest.mark.parametrize("source", ["attention_masked.hip", "gemm_bf16.hip"])
def test_a_wait_state_lies_between_m0_and_the_load_to_lds(source, tmp_path):
    obj = os.path.join(BUILD, source + ".o")
    if not os.path.exists(obj):
        pytest.skip("the library has not been built here")
    if not os.path.exists(os.path.join(LLVM, "llvm-objdump")):
        pytest.skip("ROCm LLVM tools not available")
    lines = _instructions(obj, tmp_path)
    writes = [i for i, l in enumerate(lines) if re.search(r"\bm0\b", l)]
    loads = [i for i, l in enumerate(lines) if l.startswith(("buffer_load", "global_load", "scratch_load"))
             and re.search(r"\blds\b", l)]
    assert loads, "no direct LDS loads found"
    wrong = [lines[i:i + 3] for i in writes
             if not (lines[i].startswith("s_mov_b32 m0,") and lines[i + 1].startswith("s_nop"))]
    assert not wrong, wrong[:5]
    assert [i + 2 for i in writes] == loads
    for i in loads:
        used, waits, j = _scalars(lines[i]), 0, i - 1
        while j >= 0 and waits < 5:
            if lines[j].startswith("v_"):
                written = _scalars(lines[j].split(None, 1)[1].split(",")[0])
                assert not written & used, lines[j:i + 1]
            nop = re.match(r"s_nop (\d+)", lines[j])
            waits += 1 + (int(nop[1]) if nop else 0)
            j -= 1
