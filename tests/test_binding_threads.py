"""What the binding looks up once: a second thread that comes in at any step of the first call finds all of it or
none (on the host, with stand-ins for the device's tensors and calls)."""
import sys
import threading
import types

import pytest

from paper_2505_11594_amd import binding as bd


def failure(codes, reset, first, second):
    """Run first() again and again, each time in a fresh state, and let second() run from start to end in another thread
    before one step (of the interpreter's, in these functions' code) of it: the first step, the second, and so on.
    What second() raised, or None."""
    raised, at = [], 0

    def other():
        try:
            second()
        except BaseException as e:                       # noqa: BLE001 (given to the caller)
            raised.append("before step %d: %r" % (at, e))

    while True:
        reset()
        seen = 0

        def trace(frame, event, arg):
            nonlocal seen
            if frame.f_code not in codes:
                return None
            frame.f_trace_opcodes = True
            if event == "opcode":
                if seen == at:
                    t = threading.Thread(target=other)
                    t.start()
                    t.join()
                seen += 1
            return trace

        before = sys.gettrace()
        sys.settrace(trace)
        try:
            first()
        finally:
            sys.settrace(before)
        if raised:
            return raised[0]
        if seen <= at:
            assert at > 20, "the steps were not seen"
            return None
        at += 1


class OnDevice:
    """A host tensor that says it lies on device 0."""
    is_cuda = True

    def __init__(self, t):
        self.t, self.device = t, types.SimpleNamespace(index=0)

    def get_device(self):
        return 0

    def __getattr__(self, name):
        return getattr(self.t, name)


def test_first_calls_of_two_threads(monkeypatch):
    import torch
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(bd, "lib", lambda: types.SimpleNamespace(one=lambda *a: 0, two=lambda *a: 0))
    device = types.SimpleNamespace(index=0)

    def calls(*names):
        def run():
            for name in names:
                bd._call(name, device)
        return run

    for second in (calls("one"), calls("two"), calls("two", "one")):
        assert failure({bd._call.__code__}, lambda: monkeypatch.setattr(bd, "_calls", {}), calls("one"), second) is None


@pytest.mark.parametrize("what", ["q", "pos", "lens"])
def test_first_argument_checks_of_two_threads(monkeypatch, what):
    import torch
    q, k = (OnDevice(torch.zeros((2, h, 5, 64), dtype=torch.bfloat16)) for h in (4, 2))
    w, inv = OnDevice(torch.ones(64)), OnDevice(torch.ones(32))
    i32 = OnDevice(torch.zeros(2, dtype=torch.int32))
    pos, lens = i32 if what != "q" else None, i32 if what == "lens" else None
    if q.t.data_ptr() & 15 or k.t.data_ptr() & 15:
        pytest.skip("a host allocation off 16 bytes")
    check = lambda: bd._check_norm_rope(q, k, w, w, inv, pos, lens, 1e-6, False)

    def reset():
        for name in ("_F32", "_I32"):
            monkeypatch.setattr(bd, name, None, raising=False)
        monkeypatch.setattr(bd, "_in_flags", {})
    reset()
    check()
    assert failure({bd._check_norm_rope.__code__, bd._in_flag.__code__}, reset, check, check) is None
