"""Loads straight into LDS in the assembly of the 4-bit products: one wait state or more behind the scalar instruction that wrote M0."""
import os
import subprocess

import pytest

from paper_2605_24058_amd import binding
from test_m0_wait_states import HIPCC, _too_early


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="needs hipcc")
@pytest.mark.parametrize("source", ["lordba_i4_few.hip", "lordba_i4_many.hip"])
def test_loads_into_lds_wait_for_m0(tmp_path, source):
    out = str(tmp_path / "products.s")
    flags = [f for f in binding.HIPCC_FLAGS if f != "-shared"]
    subprocess.run([HIPCC] + flags + ["-I", os.path.join(binding._ROOT, "include"), "--cuda-device-only", "-S", os.path.join(binding._CSRC, source), "-o", out],
                   check=True, capture_output=True, timeout=300)
    with open(out) as f:
        early, loads = _too_early(f.read().splitlines())
    assert loads > 0
    assert early == []
