"""The assembly of the kernels around the attention call: wait states in front of written-out loads, no spilled registers, no
arguments read by vector loads, no scalar read that waits as a vector load in the loops over keys."""

import os
import re
import subprocess

import pytest

from paper_2508_10774_amd import build
from tests.test_asm_hazards import Listing, _argument_loads, _functions

SOURCES = ("asa_cache.hip", "asa_norm.hip")


@pytest.fixture(scope="module")
def assembly(tmp_path_factory):
    out = tmp_path_factory.mktemp("asm")
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    running = {src: subprocess.Popen([hipcc, *build.HIPCC_FLAGS, "-S", "--cuda-device-only", os.path.join(build.CSRC, src),
                                      "-o", str(out / src)], stderr=subprocess.DEVNULL) for src in SOURCES}
    for src, p in running.items():
        assert p.wait() == 0, src
    return {src: (out / src).read_text() for src in running}


def test_wait_states_in_front_of_written_out_loads(assembly):
    loads = 0
    for name, lines in _functions(assembly["asa_cache.hip"]):
        found, seen = Listing(lines).faults()
        assert not found, f"{name}: {found[:4]}"
        loads += seen["load"]
    assert loads > 0


@pytest.mark.parametrize("src,kernels", [("asa_cache.hip", 20), ("asa_norm.hip", 25)])
def test_no_registers_are_spilled(assembly, src, kernels):
    spills = re.findall(r"\.name:\s+(\S+)[\s\S]*?\.private_segment_fixed_size:\s+(\d+)[\s\S]*?\.vgpr_spill_count:\s+(\d+)", assembly[src])
    assert len(spills) >= kernels
    assert not [x for x in spills if x[1] != "0" or x[2] != "0"]


def test_kernel_arguments_are_read_by_scalar_loads(assembly):
    for src in SOURCES:
        for name, lines in _functions(assembly[src]):
            assert not _argument_loads(lines), (src, name)


def test_loops_over_keys_have_no_vector_load_but_the_copies(assembly):
    """A vector load of a scale or a list's entry waits for every copy in flight: the blocks that hold matrix instructions
    without a mask have none in the kernel that copies to LDS."""
    seen = 0
    for name, lines in _functions(assembly["asa_cache.hip"]):
        if "cache_attn_tile_kernel" not in name:
            continue
        blocks, now = [], []
        for line in lines:
            code = line.split(";")[0].strip()
            if re.match(r"\.LBB\w+:", code):
                blocks.append(now)
                now = []
            elif code:
                now.append(code)
        blocks.append(now)
        for b in blocks:
            if any(x.startswith("v_mfma") for x in b):
                seen += 1
                assert not [x for x in b if re.match(r"(global|flat|buffer|scratch)_load_(?!lds)", x)], name
    assert seen >= 8
