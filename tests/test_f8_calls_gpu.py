"""The quick calls from Python beside other threads of the interpreter."""
import ctypes
import threading
import time

import pytest
import torch

pytestmark = pytest.mark.gpu


def test_other_threads_run_during_a_call(b2):
    """A launch that has to wait (for room in the stream, say) does not hold the interpreter: here the call is one that sleeps."""
    calls = pytest.importorskip("paper_1611_08035_b200._b2calls")
    real = dict(b2._connected)
    usleep = ctypes.cast(ctypes.CDLL(None).usleep, ctypes.c_void_p).value  # its first argument is the call's first: d microseconds
    x = torch.zeros(4, 128, device="cuda")
    q, s = torch.empty(4, 128, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(4, 1, dtype=torch.float8_e8m0fnu, device="cuda")
    w, f, ws = torch.zeros(128, device="cuda"), torch.zeros(128, device="cuda"), torch.zeros(256, dtype=torch.uint8, device="cuda")
    y = torch.zeros(4, 128, dtype=torch.bfloat16, device="cuda")
    d = 400_000
    arguments = {"b2_quant_f8": (d, 4, 1, x, 128, q, 128, s, 1), "b2_rmsnorm_f8": (d, 4, x, 128, None, 128, w, 1e-5, None, 128, q, 128, s, 1, f),
                 "b2_rmsnorm_backward": (d, 4, x, 128, x, 128, f, w, None, 128, x, 128, f, ws),
                 "b2_wgrad_f8": (d, 4, 4, 1.0, q, 128, s, 1, y, 128, 0.0, x, 128, None)}
    try:
        calls.connect(b2.B2Error, {n: (usleep, full) for n, (_, full) in real.items()})
        for name, args in arguments.items():
            done, ticks = threading.Event(), 0

            def sleep():
                getattr(calls, name)(*args)
                done.set()

            thread = threading.Thread(target=sleep)
            begin = time.monotonic()
            thread.start()
            while not done.is_set():
                ticks += 1
                time.sleep(0.001)
            thread.join()
            assert time.monotonic() - begin >= 0.35, name
            assert ticks >= 50, f"{name}: the interpreter stood still ({ticks} turns in 0.4 s)"
    finally:
        calls.connect(b2.B2Error, real)
    assert b2.b2_quant_f8(128, 4, 1, x, 128, q, 128, s, 1) == 0
