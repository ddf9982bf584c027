"""Host check on the AMD assembly of the masked attention kernels as built here
for gfx950: their direct LDS loads set M0 through inline assembly that declares
it clobbered, which is sound only while nothing else in the kernels keeps a
value in M0. Every M0 write has to be the one immediately before its load, and
no other instruction may name M0."""
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OBJ = os.path.join(ROOT, "paper_1809_02839_amd", "_build", "attention_masked.hip.o")
LLVM = "/opt/rocm/llvm/bin"


@pytest.mark.skipif(not os.path.exists(OBJ), reason="the library has not been built here")
@pytest.mark.skipif(not os.path.exists(os.path.join(LLVM, "llvm-objdump")), reason="ROCm LLVM tools not available")
def test_m0_only_feeds_the_direct_lds_loads(tmp_path):
    fat, co = tmp_path / "fatbin", tmp_path / "gfx950.co"
    subprocess.run([os.path.join(LLVM, "llvm-objcopy"), f"--dump-section=.hip_fatbin={fat}", OBJ,
                    str(tmp_path / "host.o")], check=True, capture_output=True)
    subprocess.run([os.path.join(LLVM, "clang-offload-bundler"), "--unbundle", "--type=o",
                    "--targets=hipv4-amdgcn-amd-amdhsa--gfx950", f"--input={fat}", f"--output={co}"],
                   check=True, capture_output=True)
    dis = subprocess.run([os.path.join(LLVM, "llvm-objdump"), "-d", "--mcpu=gfx950", str(co)], check=True,
                         capture_output=True, text=True).stdout
    lines = [l.split("//")[0].strip() for l in dis.splitlines()]
    lines = [l for l in lines if l and not l.endswith(":")]
    named = [i for i, l in enumerate(lines) if re.search(r"\bm0\b", l)]
    other = [lines[i] for i in named
             if not (lines[i].startswith("s_mov_b32 m0,") and lines[i + 1].startswith("buffer_load_dwordx4")
                     and lines[i + 1].endswith(" lds"))]
    assert named and not other, other[:10]
