"""The host side of the cache and attention entry points, built for the CPU with AddressSanitizer and UndefinedBehaviorSanitizer and
called with random arguments, ordinary and hostile.  The launches are stand-ins that check what the kernels take for granted."""
import os
import shutil

import pytest

from tests.test_sanitized_host import CSRC, ROOT, SAN, _build, _run

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="no host C++ compiler")


@pytest.fixture(scope="module")
def attention_fuzz(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("san") / "attention_fuzz")
    _build(out, [os.path.join(CSRC, f) for f in ("attention.cpp", "trace.cpp", "es.cpp", "api.cpp")] +
           [os.path.join(SAN, "host_stubs.cpp"), os.path.join(SAN, "attention_fuzz.cpp")], [os.path.join(ROOT, "include"), CSRC])
    return out


@pytest.mark.parametrize("seed", [1, 11688, 2 ** 40 + 3])
def test_random_calls_keep_what_the_kernels_rely_on(attention_fuzz, seed):
    assert "20000 iterations" in _run([attention_fuzz, str(seed), "20000"])
