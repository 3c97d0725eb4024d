"""The same call over and over, its inputs out of the caches each time: the same bits.  Loads are then late and uneven, so that the warps of a
kernel run far apart; a place in shared memory that is filled again too early, or read too early, shows in the results."""
import pytest
import torch

from helpers import make_gpu_layer, make_inputs
from paper_2503_21135_b200 import operators as ops
from paper_2503_21135_b200 import workloads as wl

pytestmark = pytest.mark.gpu


def repeated(call, rounds):
    """How many of the rounds differ from the one that most agree with."""
    flush = torch.empty(160 << 20, dtype=torch.uint8, device="cuda")      # more than the L2
    seen = []
    for i in range(rounds):
        flush.fill_(i & 255)
        y = call()
        for s in seen:
            if torch.equal(s[0], y):
                s[1] += 1
                break
        else:
            seen.append([y, 1])
            if len(seen) > 8:
                break
    return sum(n for _, n in seen) - max(n for _, n in seen)


@pytest.mark.parametrize("G", [64, 128])
@pytest.mark.parametrize("T,N,K", [(1, 4096, 4096), (8, 14336, 4096), (12, 1000, 4096), (9, 14393, 4096), (16, 14336, 14336), (32, 14336, 14336),
                                   (64, 14336, 14336), (130, 4099, 4096)])
def test_linear(T, N, K, G):
    g = torch.Generator(device="cuda").manual_seed(T)
    codes, params = ops.quantize_linear((torch.randn((N, K), generator=g, device="cuda") * 0.02).bfloat16(), G)
    x = torch.randn((T, K), generator=g, device="cuda").bfloat16()
    assert repeated(lambda: ops.linear(x, codes, params), 300) == 0
    assert ops.poll_linear_status() == 0


@pytest.fixture(scope="module", params=[("tiny", dict(d_model=2048, d_ff=4096)), ("finegrained", dict(n_experts=16, n_shared=1))],
                ids=["G128", "G64"])
def layer(request):
    name, kw = request.param
    cfg = wl.scaled(wl.CONFIGS[name], **kw)
    wg, wu, wd, bits, pool, sets = make_inputs(cfg)
    gpu = make_gpu_layer(cfg, wg, wu, wd, bits, pool, max_tokens=1024)
    gpu.set_channel_switch(sets)
    return cfg, gpu


@pytest.mark.parametrize("T", [1, 8, 40, 139, 500, 1000])   # streaming, fold and pair kernels
def test_layer(layer, T):
    cfg, gpu = layer
    g = torch.Generator(device="cuda").manual_seed(T)
    x = torch.randn((T, cfg.d_model), generator=g, device="cuda").bfloat16()
    logits = torch.randn((T, cfg.n_experts), generator=g, device="cuda")
    assert repeated(lambda: gpu.forward(x, logits), 300) == 0
    assert gpu.poll_status() == 0
