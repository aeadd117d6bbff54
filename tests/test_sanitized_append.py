"""The host side of the entry points that norm, rotate and append heads, built for the CPU with AddressSanitizer and
UndefinedBehaviorSanitizer and called with random arguments, ordinary and hostile.  The launch is a stand-in that checks what the kernel takes for granted."""
import os
import shutil

import pytest

from tests.test_sanitized_host import CSRC, ROOT, SAN, _build, _run

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="no host C++ compiler")


@pytest.fixture(scope="module")
def append_fuzz(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("san") / "append_fuzz")
    _build(out, [os.path.join(CSRC, f) for f in ("append.cpp", "trace.cpp", "es.cpp", "api.cpp")] +
           [os.path.join(SAN, "host_stubs.cpp"), os.path.join(SAN, "append_fuzz.cpp")], [os.path.join(ROOT, "include"), CSRC])
    return out


@pytest.mark.parametrize("seed", [1, 11688, 2 ** 40 + 3])
def test_random_calls_keep_what_the_kernel_relies_on(append_fuzz, seed):
    assert "20000 iterations" in _run([append_fuzz, str(seed), "20000"])
