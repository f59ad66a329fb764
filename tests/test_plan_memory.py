"""A wave's plan that runs out of host memory is refused, not thrown through the C entry (``tests/native/plan_memory.cpp``)."""
import os
import tempfile

from tests.test_host_sanitizers import CSRC, HOST_SOURCES, NATIVE, _build, _run, pytestmark  # noqa: F401


def test_every_allocation_of_a_plan_may_fail():
    with tempfile.TemporaryDirectory() as d:
        exe = os.path.join(d, "plan_memory")
        _build(exe, HOST_SOURCES + [os.path.join(CSRC, "q4_host.cpp"), os.path.join(CSRC, "lin_host.cpp"),
                                    os.path.join(NATIVE, "launch_stubs.cpp"), os.path.join(NATIVE, "plan_memory.cpp")],
               "address,undefined")
        assert "plan_memory ok" in _run(exe, [], {"ASAN_OPTIONS": "detect_leaks=1:alloc_dealloc_mismatch=0"})
