"""Status calls of the operators around the layer: what is refused or reported without a GPU."""
import contextlib
import types

import pytest
import torch

from paper_2503_21135_b200 import binding, build
from paper_2503_21135_b200 import operators as ops


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return binding.load()


def test_expire_linear_refusals(lib):
    """No wait to expire; otherwise what dynamo_linear_forward refuses."""
    P = 1 << 20   # an aligned address, never followed

    def call(T=40, N=8192, K=8192, G=64, ws=P, nb=1 << 30, x=P):
        return binding.STATUS_NAMES[lib.dynamo_debug_expire_linear(x, T, N, K, G, P, P, P, binding.F32, ws, nb, None)]

    assert call(T=8) == "ERR_ARG" and call(N=64) == "ERR_ARG" and call(T=0) == "ERR_ARG"
    assert call(T=-1) == "ERR_TOKENS" and call(G=32) == "ERR_SHAPE" and call(x=None) == "ERR_NULL" and call(nb=8) == "ERR_ARENA_TOO_SMALL"


def test_a_status_that_cannot_be_read_raises(monkeypatch):
    """OK and ERR_TIMEOUT are answers, anything else is no answer; the device that was named is asked."""
    asked = []

    @contextlib.contextmanager
    def on(device):
        asked.append(device)
        yield

    monkeypatch.setattr(torch.cuda, "device", on)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: types.SimpleNamespace(cuda_stream=0))
    for name in binding.STATUS_NAMES:
        code = binding.STATUS_NAMES.index(name)
        monkeypatch.setattr(ops, "load", lambda: types.SimpleNamespace(dynamo_linear_poll_status=lambda s: code,
                                                                       dynamo_linear_clear_status=lambda s: code))
        if name in ("OK", "ERR_TIMEOUT"):
            assert ops.poll_linear_status("cuda:3") == code
        else:
            with pytest.raises(binding.DynamoError):
                ops.poll_linear_status()
        if name == "OK":
            ops.clear_linear_status("cuda:1")
        else:
            with pytest.raises(binding.DynamoError):
                ops.clear_linear_status()
    assert asked[0] == "cuda:3" and asked[1] == "cuda:1" and asked[2] is None
