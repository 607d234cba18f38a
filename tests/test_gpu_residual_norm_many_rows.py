"""mxfp4_residual_norm_fwd / _bwd where workgroups walk many rows, several at a time, for each pair of types: the checks and tolerances of
test_gpu_residual_norm.py."""
import pytest
import torch

import test_gpu_residual_norm as few

pytestmark = pytest.mark.gpu
BF16, FP32 = torch.bfloat16, torch.float32

# (from one wave for a row, and as many rows at a time as there are waves, to sixteen waves for one; a whole number of rounds for none of them)
SIZES = [(5003, 300), (3001, 1000), (2050, 1440), (1601, 2000), (1300, 2500), (777, 4096), (520, 6000), (601, 9000)]


@pytest.mark.parametrize("gate", ["none", "vector", "row"])
@pytest.mark.parametrize("types", [(BF16, BF16), (FP32, BF16), (BF16, FP32), (FP32, FP32)], ids=str)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_forward_and_gradients(size, types, gate):
    few.test_forward_and_gradients(dict(rows=size[0], cols=size[1], stream=types[0], branch=types[1], gate=gate, seed=size[1], alpha=0.9, beta=0.5))


@pytest.mark.parametrize("rows", [511, 512, 513, 767, 769])
@pytest.mark.parametrize("cols", [64, 1440])
def test_around_the_rows_that_get_a_workgroup_each(rows, cols):
    for stream in (BF16, FP32):
        few.test_forward_and_gradients(dict(rows=rows, cols=cols, stream=stream, gate="vector", post=False))


def test_more_rows_than_a_launch_has_places_for():
    few.test_forward_and_gradients(dict(rows=2**22 + 4099, cols=8, gate="row"))
