"""The operators around the layer called by several host threads at a time."""
import ctypes
import threading

import pytest
import torch

from paper_2503_21135_b200 import binding

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
