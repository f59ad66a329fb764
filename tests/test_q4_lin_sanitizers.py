"""The host code of the 4-bit cache and of linear attention built host-only with g++ under the address and
undefined-behaviour sanitizers, driven over seeded random waves (``tests/native/q4_lin_fuzz.cpp``)."""
import os
import tempfile

from tests.test_host_sanitizers import CSRC, HOST_SOURCES, NATIVE, _build, _run, pytestmark  # noqa: F401


def test_plans_cover_their_waves():
    with tempfile.TemporaryDirectory() as d:
        exe = os.path.join(d, "q4_lin_fuzz")
        _build(exe, HOST_SOURCES + [os.path.join(CSRC, "q4_host.cpp"), os.path.join(NATIVE, "launch_stubs.cpp"),
                                    os.path.join(NATIVE, "q4_lin_fuzz.cpp")], "address,undefined")
        assert "q4_lin_fuzz ok" in _run(exe, [], {"ASAN_OPTIONS": "detect_leaks=1"})
