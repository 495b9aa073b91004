"""What the compiler makes of the products of directions, 4-bit products and norms: the assembly for gfx950 of instances of each, compiled here without a
GPU.  The rules for loads to LDS are those of the other products; no registers of these go to memory."""
import os
import re
import subprocess

import pytest

from paper_1911_11377_amd import build as lib_build
from test_training_code import (test_descriptors_are_not_vector_results_of_the_instructions_before,  # noqa: F401
                                test_m0_is_set_a_wait_state_before_the_loads_that_use_it)

pytestmark = pytest.mark.skipif(not os.path.exists(lib_build.HIPCC), reason="no hipcc")
SERIES = ["gemm_kernel<_Float16, 256, 256, 128, 64, false, true, EPI_APPLY, SeriesArgs>(SeriesArgs)", "gemm_kernel<_Float16, 128, 128, 64, 64, false, false, EPI_GRAM, SeriesArgs>(SeriesArgs)",
          "gemm_small_kernel<_Float16, 32, 128, 16, 64, 4, false, false, EPI_SQUARE, SeriesArgs>(SeriesArgs)",
          "gemm_small_kernel<_Float16, 32, 128, 16, 64, 1, false, true, EPI_APPLY, SeriesArgs>(SeriesArgs)"]
OTHERS = ["series_small_kernel<float, __bf16, true>(PassArgs, SmallSeries)", "series_join_kernel<EPI_APPLY>(SeriesArgs)",
          "rows4_kernel<__bf16, __bf16, false, 1, true, 1, 8, 4>(Rows4Args)", "rows4_kernel<__bf16, float, true, 3, false, 4, 8, 1>(Rows4Args)",
          "norm_forward_kernel<__bf16, 512, 1, true>(NormArgs)", "norm_backward_kernel<__bf16, 512, true, false>(NormArgs)", "norm_backward_kernel<float, 256, true, true>(NormArgs)",
          "norm_backward_kernel<__bf16, 1024, false, false>(NormArgs)"]


def assembly(tmp, names):
    src, out = tmp / "instances.hip", tmp / "instances.s"
    src.write_text('#include "train_series.h"\n#include "train_rows4.h"\n#include "train_norm.h"\n' + "".join("template __global__ void %s;\n" % k for k in names))
    flags = [f for f in lib_build.FLAGS if f not in ("-shared", "-fPIC", "-Wall")]
    subprocess.check_call([lib_build.HIPCC] + flags + ["--cuda-device-only", "-S", "-I", lib_build.CSRC, str(src), "-o", str(out)], stderr=subprocess.DEVNULL)
    return out.read_text()


@pytest.fixture(scope="module")
def instructions(tmp_path_factory):
    """instructions of the products' instances, in order; indices of the loads to LDS among them"""
    lines = [m.group(1) for m in re.finditer(r"^\s+([a-z]\w+[^;\n]*)", assembly(tmp_path_factory.mktemp("code"), SERIES), re.M)]
    loads = [i for i, text in enumerate(lines) if re.match(r"buffer_load_dword\w* .*\blds\b", text)]
    assert len(loads) >= 4 * len(SERIES)
    return lines, loads


def test_registers_stay_registers(tmp_path):
    """(the kernels of layer norms of the widest rows and of f32 blocks of more than 32 rows say what they keep in memory)"""
    names = SERIES + OTHERS
    sizes = [int(n) for n in re.findall(r"\.amdhsa_private_segment_fixed_size (\d+)", assembly(tmp_path, names))]
    assert len(sizes) == len(names) and not any(sizes), list(zip(names, sizes))
