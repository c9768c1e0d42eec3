"""The short way from Python to the library: other threads run while a call does."""
import ctypes
import threading
import time

import pytest
import torch

pytestmark = pytest.mark.gpu

ENTRIES = ("gvq_set_stream", "gvq_i8_scratch_bytes", "gvq_i8_quantize", "gvq_i8_matmul", "gvq_i8_gated", "gvq_gated_workspace_bytes",
           "gvq_gated_forward", "gvq_gated_backward")


@pytest.mark.parametrize("call", ["gvq_i8_quantize", "gvq_i8_matmul", "gvq_i8_gated", "gvq_gated_forward", "gvq_gated_backward"])
def test_other_threads_run_while_a_call_waits(call):
    """A call that takes 0.4 s (the C library's usleep in its place and in that of gvq_set_stream, each of which takes its microseconds
    where the handle is) leaves the interpreter to this thread, which wakes up every millisecond."""
    from paper_1811_03617_b200 import gvq
    L = gvq.lib()
    ctx = gvq.Context(gvq.HostLayout(4, 4, [0], [4]))
    short, q, x = gvq._short, gvq.I8(64, 64), torch.zeros(64, 64, device="cuda", dtype=torch.bfloat16)
    torch.cuda.synchronize()
    real = {name: ctypes.cast(getattr(L, name), ctypes.c_void_p).value for name in ENTRIES}
    slow = ctypes.cast(ctypes.CDLL(None).usleep, ctypes.c_void_p).value
    calls = {"gvq_i8_quantize": lambda: short.i8_quantize(200000, 0, x, True, True, False, 0, 0),
             "gvq_i8_matmul": lambda: short.i8_matmul(200000, 0, q, q, x),
             "gvq_i8_gated": lambda: short.i8_gated(200000, 0, q, q, q, x, 0),
             "gvq_gated_forward": lambda: short.gated_forward(200000, 0, x, x, x, x, 0, None, None),
             "gvq_gated_backward": lambda: short.gated_backward(200000, 0, x, x, x, x, x, x, 0, x, None, None)}
    got = []
    short.bind(*[slow if name in (call, "gvq_set_stream") else real[name] for name in ENTRIES], gvq.I8)
    try:
        t = threading.Thread(target=lambda: got.append(calls[call]()))
        gaps, last = [], time.perf_counter()
        t.start()
        while t.is_alive():
            time.sleep(0.001)
            now = time.perf_counter()
            gaps.append(now - last)
            last = now
        t.join()
    finally:
        short.bind(*real.values(), gvq.I8)
    assert got[0] is not None and got[0] is not False
    assert max(gaps) < 0.15 and len(gaps) > 50
    assert gvq.I8(64, 64).rows == 64 and ctx.i8_quantize(x).rows == 64
    ctx.device_status()


def test_threads_may_share_a_context():
    """Calls of one context take turns, each on its own thread's stream: what a stream has written before a call is what the call reads."""
    from paper_1811_03617_b200 import gvq
    ctx, wrong = gvq.Context(gvq.HostLayout(4, 4, [0], [4])), []
    w = ctx.i8_quantize(torch.eye(512, device="cuda"))
    want = ctx.i8_matmul(ctx.i8_quantize(torch.ones(64, 512, device="cuda")), w, torch.empty(64, 512, device="cuda"))
    torch.cuda.synchronize()

    def work(k):
        with torch.cuda.stream(torch.cuda.Stream()):
            x, y = torch.empty(64, 512, device="cuda"), torch.empty(64, 512, device="cuda")
            for i in range(200):
                x.zero_()
                x.add_(float(2 ** ((i + k) % 7)))
                ctx.i8_matmul(ctx.i8_quantize(x), w, y)
                if not torch.equal(y, want * 2.0 ** ((i + k) % 7)):
                    wrong.append((k, i))
    threads = [threading.Thread(target=work, args=(k,)) for k in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    ctx.device_status()
    assert not wrong
