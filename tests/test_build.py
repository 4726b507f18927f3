"""The build refuses operators whose kernels do not fit their registers (no GPU needed)."""
import os

import pytest

from paper_2506_09282_amd import build

FITS = """
__global__ void fits(const float* x, float* y) { y[threadIdx.x] = 2.0f * x[threadIdx.x]; }
"""
SPILLS = """
__global__ __launch_bounds__(1024) void spills(const float* x, const int* at, float* y) {
  float v[200];  // (read at a place that is known only as it runs)
  for (int i = 0; i < 200; ++i) v[i] = x[i * 1024 + threadIdx.x];
  float s = 0.0f;
  for (int i = 0; i < 200; ++i) s = s * v[i] + v[at[i] % 200];
  y[threadIdx.x] = s;
}
"""


@pytest.fixture
def as_ops(tmp_path, monkeypatch):
    monkeypatch.setattr(build, "OPS", str(tmp_path))
    monkeypatch.setattr(build, "BUILD", str(tmp_path))
    return tmp_path


@pytest.mark.skipif(not os.path.exists(build.HIPCC), reason="no hipcc")
def test_kernels_in_scratch_are_refused(as_ops):
    for name, text in (("fits", FITS), ("spills", SPILLS)):
        (as_ops / f"{name}.hip").write_text("#include <hip/hip_runtime.h>\n" + text)
    obj = build._compile(str(as_ops / "fits.hip"), False)
    assert os.path.exists(obj)
    with pytest.raises(RuntimeError, match="spills"):
        build._compile(str(as_ops / "spills.hip"), False)
    assert not os.path.exists(as_ops / "spills.hip.o")


def test_remarks():
    def line(what):
        return f"a.hip:3:1: remark: {what} [-Rpass-analysis=kernel-resource-usage]"

    text = "\n".join([line("Function Name: one"), line("    ScratchSize [bytes/lane]: 0"),
                      line("    Dynamic Stack: False"), line("Function Name: two"),
                      line("    ScratchSize [bytes/lane]: 48"), line("Function Name: three"),
                      line("    ScratchSize [bytes/lane]: 0"), line("    Dynamic Stack: True")])
    assert build.spilling(text) == ["two", "three"]
    assert build.spilling("") == []
