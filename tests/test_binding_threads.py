"""The binding's first call from several threads at once (no GPU)."""
import sys

import paper_2609_35263_amd as wp


def test_the_runtimes_functions_are_all_there_as_soon_as_one_thread_sees_that_they_are(monkeypatch):
    """Another thread may run between any two lines of the first call: wherever it then finds the functions looked up, it uses
    every one of them."""
    for name in ("_is_initialized", "_get_device", "_current_stream"):
        monkeypatch.setattr(wp, name, None)
    between = []

    def trace(frame, event, arg):
        if frame.f_code is not wp._current_device.__code__:
            return None
        between.append(wp._get_device is None or (wp._is_initialized is not None and wp._current_stream is not None))
        return trace

    held = sys.gettrace()
    sys.settrace(trace)
    try:
        wp._current_device()
    finally:
        sys.settrace(held)
    assert len(between) > 4 and all(between)
    assert None not in (wp._is_initialized, wp._get_device, wp._current_stream)
