"""The binding's checks of tensors and arrays, with and without the interpreter's asserts: what is wrong never reaches the library."""
import subprocess
import sys

import pytest

# forward_block on fake CUDA tensors, one argument wrong at a time; the library's call is replaced by one that says that it was reached
PROGRAM = """
import contextlib, types
import numpy as np
import torch
from paper_2503_21135_b200 import binding, build

assert_statements = False
assert (globals().__setitem__("assert_statements", True) or True)
build.build_library()
layer = binding.DynamoLayer(256, 512, 8, 2, 64, 16, 16, 64)

class Fake(torch.Tensor):
    is_cuda = True

def tensor(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype).as_subclass(Fake)

class Reached(Exception):
    pass

def reached(*a):
    raise Reached

torch.cuda.device = lambda d: contextlib.nullcontext()
binding._stream = lambda: 0
real = binding.load()
binding.load = lambda: types.SimpleNamespace(dynamo_moe_block_forward=reached, dynamo_destroy=real.dynamo_destroy)
T, d, f32 = 4, 256, torch.float32
good = dict(r=tensor(T, d), n=tensor(T, d), w_router=tensor(8, d), bias=tensor(8, dtype=f32), w_post=tensor(d), w_pre=tensor(d),
            gate=tensor(T, 1, dtype=f32), y=tensor(T, d, dtype=f32))
try:
    layer.forward_block(**good)
except Reached:
    pass
else:
    raise SystemExit("a call that is right did not reach the library")
wrong = [dict(r=tensor(T, 128)), dict(r=tensor(T, d, dtype=torch.float16)), dict(n=tensor(3, d)), dict(n=tensor(T, d, dtype=f32)),
         dict(w_router=tensor(4, d)), dict(w_router=tensor(8, d, dtype=f32)), dict(bias=tensor(8)), dict(bias=tensor(7, dtype=f32)),
         dict(w_post=tensor(128)), dict(w_pre=tensor(d, dtype=f32)), dict(gate=tensor(3, 1, dtype=f32)), dict(gate=tensor(T, 1)),
         dict(gate=tensor(128)), dict(y=tensor(T, d)), dict(y=tensor(3, d, dtype=f32)), dict(post_norm=False), dict(pre_norm=False),
         dict(y_dtype=5), dict(n=torch.zeros((T, d), dtype=torch.bfloat16)), dict(n=tensor(d, T).t())]
for kw in wrong:
    try:
        layer.forward_block(**{**good, **kw})
    except ValueError as e:
        if not isinstance(e, AssertionError):
            raise SystemExit("not what callers catch so far: %r" % e)
    else:
        raise SystemExit("passed")
for f in (lambda: layer.set_channel_precision([8] * 7), lambda: layer.set_channel_precision_down([8] * 9),
          lambda: binding.assign_bits(np.zeros((5, 2)), [2, 3, 4]), lambda: binding._i32p(np.zeros(3)),
          lambda: layer.forward(tensor(T, d, dtype=f32), tensor(T, 8, dtype=f32)), lambda: layer.forward(tensor(T, d), tensor(T, 8)),
          lambda: layer.forward_router(tensor(T, d), tensor(4, d))):
    try:
        f()
    except ValueError:
        pass
    else:
        raise SystemExit("passed")
print("asserts" if assert_statements else "no asserts")
"""


@pytest.mark.parametrize("flags,says", [([], "asserts"), (["-O"], "no asserts")])
def test_checks_of_arguments(flags, says):
    r = subprocess.run([sys.executable] + flags + ["-c", PROGRAM], capture_output=True, text=True, timeout=600)
    assert r.returncode == 0 and r.stdout.strip() == says, r.stdout + r.stderr
