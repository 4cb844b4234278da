"""The waits between matrix products and the instructions that take their registers, in the
compiled kernels of attention over pages: every path on from every product is followed, as for attention
over a shared prompt (test_ops_waits)."""
import os
import subprocess

import pytest
import test_ops_waits as W

from paper_2308_04623_amd import build


def test_results_are_taken_when_they_are_complete(tmp_path, monkeypatch):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not os.path.exists(hipcc):
        pytest.skip("no compiler")
    monkeypatch.setitem(W.STATES, "v_mfma_f32_16x16x32_f16", 8)
    out = str(tmp_path / "attn.s")
    flags = [f for f in build.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    subprocess.run([hipcc, *flags, "-I", os.path.join(build.ROOT, "include"), "--cuda-device-only", "-S",
                    os.path.join(build.HERE, "csrc", "ops_pages_attn.hip"), "-o", out], check=True, capture_output=True)
    kernels = W.functions(open(out).read())
    assert sum(line.startswith("v_mfma") for code in kernels.values() for line in code) > 1000
    for name, code in kernels.items():
        assert not list(W.early(code)), name
