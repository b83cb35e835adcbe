"""Loads straight into LDS in the assembly of the 8-bit products: one wait state or more behind the scalar instruction that wrote M0."""
import os
import subprocess

import pytest

from paper_2605_24058_amd import binding
from test_m0_wait_states import HIPCC, _too_early


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="needs hipcc")
def test_loads_into_lds_wait_for_m0(tmp_path):
    out = str(tmp_path / "lordba_i8_product.s")
    flags = [f for f in binding.HIPCC_FLAGS if f != "-shared"]
    subprocess.run([HIPCC] + flags + ["-I", os.path.join(binding._ROOT, "include"), "--cuda-device-only", "-S",
                                      os.path.join(binding._CSRC, "lordba_i8_product.hip"), "-o", out], check=True, capture_output=True, timeout=300)
    with open(out) as f:
        early, loads = _too_early(f.read().splitlines())
    assert loads > 0
    assert early == []
