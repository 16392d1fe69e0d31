"""The C ABI layer of attention over spans and of decode over shared prefixes, built for the host with its
launches replaced by recorders, and the cuts of both: plain and under AddressSanitizer and
UndefinedBehaviorSanitizer (host code only)."""
import os

import pytest

from test_host_logic import HIPCC, SAN_ENV, SAN_HIPCC, _build_run


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not available")
@pytest.mark.parametrize("sanitize", [False, True])
def test_span_abi(tmp_path, sanitize):
    out = _build_run(tmp_path, "span_abi_check.cpp", "span_abi_check",
                     SAN_HIPCC if sanitize else ["-O2"], env=SAN_ENV if sanitize else None)
    assert out.startswith("span abi ok")
    assert int(out.split()[-1]) > 50000
