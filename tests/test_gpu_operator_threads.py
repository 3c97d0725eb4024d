"""The operators around the layer called by several host threads at a time."""
import ctypes
import threading
import time

import pytest
import torch

from paper_2503_21135_b200 import binding
from paper_2503_21135_b200 import operators as ops

pytestmark = pytest.mark.gpu


def test_wide_gradients_side_by_side():
    """The wide gradient with column sums (up to 128 KB of shared memory a CTA) and without any, through the C-ABI (ctypes gives the
    interpreter's lock away for a call): each launch has what it needs whatever another thread asks for."""
    L, rounds = binding.load(), 3000
    failed = []

    def work(d, columns):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            r, y, dn, dr, dy = torch.ones((5, 4, d), dtype=torch.bfloat16, device="cuda")
            stats = torch.ones((4, 2), device="cuda")
            w = torch.ones((2, d), device="cuda")
            dw = torch.empty((2, d), device="cuda")
            D = binding.JoinDesc(d, 0, 0, 0, 1, 0, 1, 1, 1.0, 1.0, 1e-6)
            n = ctypes.c_size_t()
            assert L.dynamo_norm_join_workspace_bytes(ctypes.byref(D), 4, ctypes.byref(n)) == 0
            ws = torch.empty(n.value, dtype=torch.uint8, device="cuda")
            a = [t.data_ptr() for t in (dn, r, y, stats, w[0], w[1], dr, dy, dw[0], dw[1], ws)]
            for _ in range(rounds):
                st = L.dynamo_norm_join_backward(ctypes.byref(D), a[0], None, a[1], a[2], a[3], a[4], None, a[5], 4, a[6], a[7],
                                                 a[8] if columns else None, None, a[9] if columns else None,
                                                 a[10] if columns else None, n.value if columns else 0, stream.cuda_stream)
                if st != 0:
                    failed.append((d, columns, st))
                    return
            stream.synchronize()

    threads = [threading.Thread(target=work, args=a) for a in ((16384, True), (16384, False), (8200, True), (12296, True))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed


@pytest.mark.parametrize("name", ["dispatch", "combine", "combine_backward", "norm_join", "norm_join_backward", "quantize_linear", "linear"])
def test_other_threads_run_while_a_launch_waits(name):
    """Launches behind a kernel of about a second, more than a stream takes: the caller waits in a launch, another thread goes on."""
    idx, x = torch.zeros((8, 1), dtype=torch.int32, device="cuda"), torch.ones((8, 256), dtype=torch.bfloat16, device="cuda")
    s = ops.dispatch(idx, 1, x)
    stats = ops.norm_join(x, want_stats=True)[2]
    codes, params = ops.quantize_linear(x)
    n_out, y = torch.empty_like(x), torch.empty((8, 8), device="cuda")
    d_rows = torch.empty_like(s.rows)
    call = {"dispatch": lambda: ops.dispatch(idx, 1, x, out=tuple(s)), "combine": lambda: ops.combine(s.rows, s.pos, out=n_out),
            "combine_backward": lambda: ops.combine_backward(x, s.rows, s.pos, d_rows=d_rows, want_d_w=False),
            "norm_join": lambda: ops.norm_join(x, n_out=n_out), "norm_join_backward": lambda: ops.norm_join_backward(x, None, x, None, stats),
            "quantize_linear": lambda: ops.quantize_linear(x), "linear": lambda: ops.linear(x, codes, params, out=y)}[name]
    torch.cuda.synchronize()
    gaps, stop = [0.0], threading.Event()

    def watch():
        last = time.perf_counter()
        while not stop.is_set():
            time.sleep(0.001)
            now = time.perf_counter()
            gaps[0], last = max(gaps[0], now - last), now

    watcher = threading.Thread(target=watch)
    watcher.start()
    t0 = time.perf_counter()
    torch.cuda._sleep(2_000_000_000)
    for _ in range(6000):
        call()
    waited = time.perf_counter() - t0
    stop.set()
    watcher.join()
    torch.cuda.synchronize()
    assert waited > 0.5, "the queue was not full: nothing was tested"
    assert gaps[0] < 0.3
