"""Host checks on the AMD assembly of the product's kernels, built here for gfx950:
their direct loads keep the wait states that inline assembly has to spell out,
every kernel waits for its loads into LDS before it ends (the memory may be another
block's then), and no K loop spills."""
import os
import re

import pytest

import test_direct_loads_host as loads

OBJ = os.path.join(loads.BUILD, "product.hip.o")


def _lines(tmp_path):
    if not os.path.exists(OBJ):
        pytest.skip("the library has not been built here")
    if not os.path.exists(os.path.join(loads.LLVM, "llvm-objdump")):
        pytest.skip("ROCm LLVM tools not available")
    return loads._instructions(OBJ, tmp_path)


def test_wait_states_around_the_direct_loads(tmp_path):
    loads.test_a_wait_state_lies_between_m0_and_the_load_to_lds("product.hip", tmp_path)


def test_loads_into_lds_are_waited_for_before_a_block_ends(tmp_path):
    """After its last load into LDS a kernel waits for all of them (vmcnt(0)) before any s_endpgm."""
    kernel, seen = [], 0
    for l in _lines(tmp_path):
        kernel.append(l)
        if not l.startswith("s_endpgm"):
            continue
        last = max((i for i, x in enumerate(kernel) if re.search(r"\blds\b", x) and x.startswith("buffer_load")), default=None)
        if last is not None:
            seen += 1
            assert any(x.startswith("s_waitcnt") and "vmcnt(0)" in x for x in kernel[last:]), kernel[last:last + 20]
            kernel = []
    assert seen >= 9


def test_the_loops_of_matrix_instructions_do_not_spill(tmp_path):
    """From the branch before the loop's barrier to the one behind it nothing goes to scratch memory."""
    lines, loops = _lines(tmp_path), 0
    branch = [i for i, l in enumerate(lines) if l.startswith(("s_cbranch", "s_branch", "s_endpgm"))]
    for i, l in enumerate(lines):
        if not l.startswith("s_barrier"):
            continue
        end = next(b for b in branch if b > i)
        behind = lines[i:end]
        if not (any("v_mfma" in x for x in behind) and any("ds_read" in x for x in behind)
                and any(re.search(r"\blds\b", x) for x in behind)):
            continue
        loops += 1
        start = max((b for b in branch if b < i), default=0)
        assert not any(x.startswith("scratch_") for x in lines[start:end])
    assert loops >= 9
