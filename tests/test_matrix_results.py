"""No kernel keeps results of matrix instructions in accumulation registers, which this compiler has read too early (a sum one product short)."""
import glob
import os
import re
import subprocess

import pytest

from paper_2502_15779_amd import _build

MATRIX = sorted(s for s in glob.glob(os.path.join(_build.CSRC, "*.hip")) if "__builtin_amdgcn_mfma" in open(s).read())


@pytest.mark.parametrize("source", MATRIX, ids=os.path.basename)
def test_results_stay_in_vector_registers(source, tmp_path):
    out = str(tmp_path / "kernels.s")
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    subprocess.run([hipcc] + _build.COMPILE_FLAGS + ["--cuda-device-only", "-S", "-I", os.path.join(_build.ROOT, "include"), "-I", _build.CSRC, source, "-o", out],
                   check=True, capture_output=True)
    text = open(out).read()
    assert re.search(r"^\s*v_mfma", text, re.M)
    assert not re.findall(r"^\s*v_mfma\w* a\[.*", text, re.M)
