"""The host code of the 8-bit cache and of rotary positions built host-only with g++ under the address and
undefined-behaviour sanitizers, driven over seeded random waves (``tests/native/q8_rope_fuzz.cpp``)."""
import os
import tempfile

from tests.test_host_sanitizers import CSRC, HOST_SOURCES, NATIVE, _build, _run, pytestmark  # noqa: F401


def test_plans_blocks_and_overlaps():
    with tempfile.TemporaryDirectory() as d:
        exe = os.path.join(d, "q8_rope_fuzz")
        _build(exe, HOST_SOURCES + [os.path.join(CSRC, "q8_host.cpp"), os.path.join(NATIVE, "launch_stubs.cpp"),
                                    os.path.join(NATIVE, "q8_rope_fuzz.cpp")], "address,undefined")
        assert "q8_rope_fuzz ok" in _run(exe, [], {"ASAN_OPTIONS": "detect_leaks=1:alloc_dealloc_mismatch=0"})
