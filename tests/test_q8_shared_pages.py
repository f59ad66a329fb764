"""Which plans of the 8-bit cache load pages past the caches (``tests/native/q8_shared_pages.cpp``), and the first key that each item
loads (``tests/native/q8_first_keys.cpp``), on the CPU under sanitizers."""
import os
import tempfile

from tests.test_host_sanitizers import CSRC, HOST_SOURCES, NATIVE, _build, _run, pytestmark  # noqa: F401


def run(name):
    with tempfile.TemporaryDirectory() as d:
        exe = os.path.join(d, name)
        _build(exe, HOST_SOURCES + [os.path.join(CSRC, "q8_host.cpp"), os.path.join(NATIVE, "launch_stubs.cpp"),
                                    os.path.join(NATIVE, name + ".cpp")], "address,undefined")
        assert name + " ok" in _run(exe, [], {"ASAN_OPTIONS": "detect_leaks=1:alloc_dealloc_mismatch=0"})


def test_pages_that_no_query_reads_do_not_count():
    run("q8_shared_pages")


def test_items_begin_with_the_first_key_that_a_query_sees():
    run("q8_first_keys")
