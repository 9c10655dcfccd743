"""What the binding takes for a tensor: types that it refuses, without a GPU.  In a process of its own, in which torch's queries of the
device and the stream are stood in for, with tensors that are none: they have a shape, a type, strides and an address between two 16-byte
places, at which the library stops (status 3) every call that the binding lets through."""
import os
import subprocess
import sys

import pytest

from paper_2609_09208_b200 import build as sa_build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
COMMON = """
import numpy as np, torch
torch._C._cuda_getDevice = lambda: 0
torch._C._cuda_getCurrentRawStream = lambda device: 0
from paper_2609_09208_b200 import binding as sa

class Stand:
    def __init__(self, dtype, *shape):
        self.dtype, self.shape = dtype, shape
    def stride(self):
        return tuple(int(np.prod(self.shape[i + 1:])) for i in range(len(self.shape)))
    def is_contiguous(self): return True
    def get_device(self): return 0
    def data_ptr(self): return 264

def outcome(call):
    try:
        call()
    except ValueError:
        return "refused"
    except sa.SaError as e:
        return e.status
    return 0

cfg = sa.make_config(64, 4, 2, sa.SA_KV_FP4)
rot = sa.Rotary(cfg, dtype=torch.bfloat16)
rot.handle.rotary_dim, rot.handle.inv_freq = 64, 256
cache = sa.SaCache(256, 256, 256, 2, 4, 8)

def rotate(positions=torch.int32, out=torch.float16):
    q = Stand(torch.bfloat16, 6, 4, 64)
    return outcome(lambda: sa.rotate_qkv(rot, q, None, None, Stand(positions, 1, 6), Stand(out, 6, 4, 64), None, None))

def read(t):
    both = [outcome(lambda: sa.read_kv(cfg, cache, None, np.array([0, 5, 9]), *kv)) for kv in ((Stand(t, 9, 2, 64), None), (None, Stand(t, 9, 2, 64)))]
    assert both[0] == both[1]
    return both[0]
"""


@pytest.fixture(scope="module", autouse=True)
def _built():
    sa_build.build()


def outcomes(expression):
    run = subprocess.run([sys.executable, "-c", COMMON + "print(repr(%s))" % expression], cwd=ROOT, capture_output=True, text=True,
                         env={**os.environ, "CUDA_VISIBLE_DEVICES": ""}, timeout=600)
    assert run.returncode == 0, run.stderr
    return eval(run.stdout.strip().splitlines()[-1])


def test_positions_are_32_bit_integers():
    """A float's bits taken for an integer would turn every head by garbage, with a status of success."""
    got = outcomes("{str(t): rotate(positions=t) for t in (torch.int32, torch.float32, torch.uint32, torch.int64, torch.float16)}")
    assert got.pop("torch.int32") == 3
    assert set(got.values()) == {"refused"}, got


def test_outputs_are_binary16_or_their_bits():
    """A bfloat16 tensor of the right size would come back full of binary16 patterns."""
    got = outcomes("{str(t): (rotate(out=t), read(t)) for t in (torch.float16, torch.int16, torch.uint16, torch.bfloat16, torch.float32, torch.uint8, torch.complex32)}")
    for bits in ("float16", "int16", "uint16"):
        assert got.pop("torch." + bits) == (3, 3), bits
    assert set(got.values()) == {("refused", "refused")}, got
