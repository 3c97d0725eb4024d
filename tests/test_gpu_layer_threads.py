"""Layers of different sizes driven by different host threads: contexts are independent of one another, so is what their launches ask for."""
import threading

import pytest
import torch

from helpers import make_gpu_layer, make_inputs
from paper_2503_21135_b200 import binding
from paper_2503_21135_b200 import workloads as wl

pytestmark = pytest.mark.gpu


def test_two_layers_on_two_threads():
    """The wide layer's decode step runs three CTAs an SM with small rings, the narrow one's two with large ones."""
    tiny = wl.CONFIGS["tiny"]
    wide = wl.scaled(tiny, d_ff=8192)
    rounds, failed = 10000, []

    def steps(cfg, gpu, x, logits, want):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            y = torch.empty_like(want)
            for _ in range(rounds):
                st = binding.dynamo_moe_forward(gpu.ctx, x.data_ptr(), logits.data_ptr(), len(x), y.data_ptr(), binding.F32, None,
                                                stream.cuda_stream)
                if st != binding.OK:
                    failed.append((cfg.d_ff, st))
                    return
            if not torch.equal(y, want):
                failed.append((cfg.d_ff, "result"))

    threads = []
    for cfg in (tiny, wide, tiny, wide):
        wg, wu, wd, bits, pool, sets = make_inputs(cfg)
        gpu = make_gpu_layer(cfg, wg, wu, wd, bits, pool, max_tokens=16)
        gpu.set_channel_switch(sets)
        g = torch.Generator(device="cuda").manual_seed(1)
        x = torch.randn((8, cfg.d_model), generator=g, device="cuda").bfloat16()
        logits = torch.randn((8, cfg.n_experts), generator=g, device="cuda")
        want = gpu.forward(x, logits)
        threads.append(threading.Thread(target=steps, args=(cfg, gpu, x, logits, want)))
    torch.cuda.synchronize()
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not failed
