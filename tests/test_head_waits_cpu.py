"""Matrix results of the dense layers' and the weighing kernels are used only after the wait states they
need, on every path (test_mfma_waits_cpu.py says why and how)."""
import os
import subprocess

import pytest

from paper_1906_07155_amd import build as B
from test_mfma_waits_cpu import NEEDS, early_uses


@pytest.mark.parametrize("source", ["gemm_bf16", "gemm_f32", "linear", "weigh"])
def test_products_are_waited_for(source, tmp_path):
    path = os.path.join(os.path.dirname(B.__file__), "csrc", source + ".hip")
    out = tmp_path / (source + ".s")
    subprocess.check_call([B.HIPCC, *B.FLAGS, "--cuda-device-only", "-S", path, "-o", str(out)], stderr=subprocess.DEVNULL)
    text = out.read_text()
    assert any(op in text for op in NEEDS)
    assert early_uses(text) == []
