"""A bounded wait of the 4-bit product that runs out: the results concerned are NaN, the others are right, the status says so, and the
GPU goes on as before."""
import ctypes
import threading

import pytest
import torch

from paper_2503_21135_b200 import binding
from paper_2503_21135_b200 import operators as ops

pytestmark = pytest.mark.gpu
TIMEOUT = binding.STATUS_NAMES.index("ERR_TIMEOUT")


@pytest.fixture(autouse=True)
def status_set_back():
    yield
    ops.clear_linear_status()


def expired(x, codes, params, G):
    """dynamo_debug_expire_linear of these."""
    (T, K), N, L = x.shape, codes.shape[0], binding.load()
    n = ctypes.c_size_t()
    assert L.dynamo_linear_workspace_bytes(T, N, K, G, ctypes.byref(n)) == 0
    ws = torch.empty(n.value, dtype=torch.uint8, device="cuda")
    y = torch.zeros((T, N), device="cuda")
    assert L.dynamo_debug_expire_linear(x.data_ptr(), T, N, K, G, codes.data_ptr(), params.data_ptr(), y.data_ptr(), binding.F32,
                                        ws.data_ptr(), n.value, torch.cuda.current_stream().cuda_stream) == 0
    torch.cuda.synchronize()
    return y


# one CTA's run is part of a block of 256 rows (16, 32 and 64 tokens a tile), or six blocks (three of each of the first two tiles)
@pytest.mark.parametrize("T,N,K,G,lost", [(16, 14336, 4096, 128, (16, 256)), (31, 6401, 4096, 64, (31, 256)), (40, 4352, 4096, 128, (40, 256)),
                                          (20000, 700, 64, 64, (128, 700))])
def test_results_behind_an_expired_wait(T, N, K, G, lost):
    g = torch.Generator(device="cuda").manual_seed(T)
    codes, params = ops.quantize_linear((torch.randn((N, K), generator=g, device="cuda") * 0.02).bfloat16(), G)
    x = torch.randn((T, K), generator=g, device="cuda").bfloat16()
    want = ops.linear(x, codes, params)
    assert ops.poll_linear_status() == 0
    y = expired(x, codes, params, G)
    assert ops.poll_linear_status() == TIMEOUT
    nan = torch.isnan(y)
    assert nan[0, 0] and nan[:lost[0], :lost[1]].all() and int(nan.sum()) == lost[0] * lost[1]
    assert torch.equal(y[~nan], want[~nan])
    assert torch.equal(ops.linear(x, codes, params), want)


def test_every_user_is_told():
    """One user's question does not take the answer from another, in this thread or the next."""
    codes, params = ops.quantize_linear(torch.ones((4352, 4096), dtype=torch.bfloat16, device="cuda"), 128)
    x = torch.ones((40, 4096), dtype=torch.bfloat16, device="cuda")
    expired(x, codes, params, 128)
    answers = [ops.poll_linear_status(), ops.poll_linear_status(), binding.load().dynamo_linear_poll_status(None)]
    other = threading.Thread(target=lambda: answers.append(ops.poll_linear_status()))
    other.start()
    other.join()
    ops.linear(x, codes, params)          # a call that goes well changes nothing
    answers.append(ops.poll_linear_status())
    assert answers == [TIMEOUT] * 5
    ops.clear_linear_status()
    assert ops.poll_linear_status() == 0
