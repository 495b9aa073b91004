"""What the compiler makes of the training kernels: the assembly for gfx950 of instances of each, compiled here without a GPU."""
import os
import re
import subprocess

import pytest

from paper_1911_11377_amd import build as lib_build

pytestmark = pytest.mark.skipif(not os.path.exists(lib_build.HIPCC), reason="no hipcc")
KERNELS = ["gemm_kernel<__bf16, 256, 256, 128, 64, false, false, EPI_GATE>", "gemm_kernel<float, 128, 128, 64, 64, true, true, EPI_STORE>",
           "gemm_small_kernel<_Float16, 32, 128, 16, 64, 4, false, true, EPI_DHID>", "gemm_small_kernel<float, 32, 128, 16, 64, 1, false, true, EPI_STORE>"]


@pytest.fixture(scope="module")
def instructions(tmp_path_factory):
    """instructions of all instances, in order; indices of the loads to LDS among them"""
    tmp = tmp_path_factory.mktemp("code")
    src, out = tmp / "instances.hip", tmp / "instances.s"
    src.write_text('#include "train_gemm.h"\n' + "".join("template __global__ void %s(GemmArgs);\n" % k for k in KERNELS))
    flags = [f for f in lib_build.FLAGS if f not in ("-shared", "-fPIC", "-Wall")]
    subprocess.check_call([lib_build.HIPCC] + flags + ["--cuda-device-only", "-S", "-I", lib_build.CSRC, str(src), "-o", str(out)], stderr=subprocess.DEVNULL)
    lines = [m.group(1) for m in re.finditer(r"^\s+([a-z]\w+[^;\n]*)", out.read_text(), re.M)]
    loads = [i for i, text in enumerate(lines) if re.match(r"buffer_load_dword\w* .*\blds\b", text)]
    assert len(loads) >= 4 * len(KERNELS)
    return lines, loads


def test_m0_is_set_a_wait_state_before_the_loads_that_use_it(instructions):
    """a load to LDS takes its LDS address from m0 and needs one other instruction (or s_nop) between the write of m0 and itself;
    the compiler sees to that for what it emits itself, not inside an assembly block"""
    lines, loads = instructions
    bad = [lines[i - 1] for i in loads if re.match(r"s_\w+ m0\b", lines[i - 1])]
    assert not bad, (len(bad), len(loads), bad[0])
    before = [lines[i - 2:i] for i in loads]
    assert all(any(re.match(r"s_mov_b32 m0\b", t) for t in b) for b in before), before[0]


def _scalars(text):
    found = {int(n) for n in re.findall(r"\bs(\d+)\b", text)}
    for first, last in re.findall(r"\bs\[(\d+):(\d+)\]", text):
        found |= set(range(int(first), int(last) + 1))
    return found


def test_descriptors_are_not_vector_results_of_the_instructions_before(instructions):
    """a memory instruction that reads a scalar register which a vector instruction has written needs five others in between; inside an
    assembly block the compiler does not count.  The descriptors come from scalar arithmetic"""
    lines, loads = instructions
    for i in loads:
        for text in lines[max(0, i - 6):i]:
            if re.match(r"v_(readfirstlane|readlane)_b32 ", text):
                assert not _scalars(text.split(",")[0]) & _scalars(lines[i]), (text, lines[i])
