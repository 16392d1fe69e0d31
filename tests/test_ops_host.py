"""The C ABI layer of the operators around attention, built for the host with its launches replaced by
recorders, plain and under AddressSanitizer and UndefinedBehaviorSanitizer (host code only)."""
import os

import pytest

from test_host_logic import HIPCC, SAN_ENV, SAN_HIPCC, _build_run


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not available")
@pytest.mark.parametrize("sanitize", [False, True])
def test_ops_abi(tmp_path, sanitize):
    out = _build_run(tmp_path, "ops_abi_check.cpp", "ops_abi_check",
                     SAN_HIPCC if sanitize else ["-O2"], env=SAN_ENV if sanitize else None)
    assert out.startswith("ops abi ok")
    assert int(out.split()[-1]) > 5000
