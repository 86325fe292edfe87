"""The binding's look-up of the current stream."""
import sys


def test_first_look_up_never_shows_half_of_its_state(monkeypatch):
    """Another thread's call between any two steps of the first one finds nothing looked up yet, or both functions."""
    import torch
    from paper_2605_06665_amd import binding as B
    monkeypatch.setattr(B, "_STREAM_OF", None)
    monkeypatch.setattr(B, "_DEVICE", None)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 100 + device, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 3, raising=False)
    steps = []

    def trace(frame, event, arg):
        if frame.f_code is not B._current_stream.__code__:
            return None
        frame.f_trace_opcodes = True
        steps.append((B._STREAM_OF is not None, B._DEVICE is not None))
        return trace
    before = sys.gettrace()
    sys.settrace(trace)
    try:
        assert B._current_stream() == 103
    finally:
        sys.settrace(before)
    assert steps[0] == (False, False) and steps[-1] == (True, True) and (True, False) not in steps
    assert B._current_stream() == 103
