"""Which plans of the 8-bit cache load pages past the caches (``tests/native/q8_shared_pages.cpp``), on the CPU under sanitizers."""
import os
import tempfile

from tests.test_host_sanitizers import CSRC, HOST_SOURCES, NATIVE, _build, _run, pytestmark  # noqa: F401


def test_pages_that_no_query_reads_do_not_count():
    with tempfile.TemporaryDirectory() as d:
        exe = os.path.join(d, "q8_shared_pages")
        _build(exe, HOST_SOURCES + [os.path.join(CSRC, "q8_host.cpp"), os.path.join(NATIVE, "launch_stubs.cpp"),
                                    os.path.join(NATIVE, "q8_shared_pages.cpp")], "address,undefined")
        assert "q8_shared_pages ok" in _run(exe, [], {"ASAN_OPTIONS": "detect_leaks=1:alloc_dealloc_mismatch=0"})
