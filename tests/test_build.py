"""CPU checks of the build: kernels that have to stay in registers are refused where the compiler gave them scratch memory."""
import os
import subprocess

import pytest

from paper_2506_02850_amd import build

KERNEL = """#include <hip/hip_runtime.h>
extern "C" __global__ void in_registers(float* x) { x[threadIdx.x] *= 2.f; }
extern "C" __global__ void in_scratch(float* x, const int* at) {
    volatile float a[64];
    for (int i = 0; i < 64; ++i) a[i] = x[i];
    x[threadIdx.x] = a[at[threadIdx.x] & 63];
}
"""


def compile_(src, obj):
    p = subprocess.run(build.compile_command(str(src), str(obj)), stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    return build.compiled(str(src), p.returncode, p.stdout)


def test_scratch_memory_is_refused_where_it_is_not_allowed(tmp_path):
    try:
        build.hipcc()
    except RuntimeError:
        pytest.skip("no hipcc")
    src = tmp_path / build.NO_SCRATCH[0]
    src.write_text(KERNEL)
    with pytest.raises(RuntimeError, match="scratch memory: in_scratch$"):
        compile_(src, tmp_path / "x.o")
    src.write_text(KERNEL[:KERNEL.index('extern "C" __global__ void in_scratch')])
    assert compile_(src, tmp_path / "x.o") == ""
    other = tmp_path / "other.hip"
    other.write_text(KERNEL)
    assert compile_(other, tmp_path / "x.o") == ""


def test_reports_are_read():
    tail = " [-Rpass-analysis=kernel-resource-usage]"
    lines = lambda name, scratch, spill: [f"x.h:1:1: remark: Function Name: {name}{tail}", f"x.h:1:1: remark:     VGPRs: 90{tail}",
                                          f"x.h:1:1: remark:     ScratchSize [bytes/lane]: {scratch}{tail}", f"x.h:1:1: remark:     SGPRs Spill: 7{tail}",
                                          f"x.h:1:1: remark:     VGPRs Spill: {spill}{tail}"]
    text = "\n".join(lines("a", 0, 0) + lines("b", 52, 0) + lines("c", 0, 3) + lines("d", 8, 8))
    assert build.kernels_with_scratch(text) == ["b", "c", "d"]
    for status, out in ((1, text), (0, ""), (0, text)):
        with pytest.raises(RuntimeError):
            build.compiled(build.NO_SCRATCH[0], status, out)
    assert build.compiled("evict.hip", 0, text) == "" and build.compiled(build.NO_SCRATCH[0], 0, "\n".join(lines("a", 0, 0))) == ""


def test_all_kernels_of_the_rule_are_built_under_it():
    """Every source that includes the rule's header."""
    with_header = [s for s in build.SOURCES if "decode_attention.h" in open(os.path.join(build.CSRC, s)).read()]
    assert sorted(with_header) == sorted(build.NO_SCRATCH)
