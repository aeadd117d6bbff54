"""The host side of the entry points that norm, rotate and append heads, and of attention with sinks, built for the CPU with AddressSanitizer and
UndefinedBehaviorSanitizer and called with random arguments.  The launches are stand-ins that check what the kernels take for granted."""
import os
import shutil

import pytest

from tests.test_sanitized_host import CSRC, ROOT, SAN, _build, _run

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="no host C++ compiler")


def _built(tmp_path_factory, source, name):
    out = str(tmp_path_factory.mktemp("san") / name)
    _build(out, [os.path.join(CSRC, f) for f in (source, "trace.cpp", "es.cpp", "api.cpp")] +
           [os.path.join(SAN, "host_stubs.cpp"), os.path.join(SAN, name + ".cpp")], [os.path.join(ROOT, "include"), CSRC])
    return out


@pytest.fixture(scope="module")
def append_fuzz(tmp_path_factory):
    return _built(tmp_path_factory, "append.cpp", "append_fuzz")


@pytest.fixture(scope="module")
def sinks_fuzz(tmp_path_factory):
    return _built(tmp_path_factory, "attention.cpp", "sinks_fuzz")


@pytest.mark.parametrize("seed", [1, 11688, 2 ** 40 + 3])
def test_random_calls_keep_what_the_kernel_relies_on(append_fuzz, seed):
    assert "20000 iterations" in _run([append_fuzz, str(seed), "20000"])


@pytest.mark.parametrize("seed", [1, 11688, 2 ** 40 + 3])
def test_random_sinks_fit_the_workspace(sinks_fuzz, seed):
    assert "20000 iterations" in _run([sinks_fuzz, str(seed), "20000"])
