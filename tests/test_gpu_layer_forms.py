"""Forms of the calls around a linear layer beside the usual ones: each gives what the usual form of the same call gives."""
import pytest
import torch

import paper_2605_09825_amd as mx

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("layout", [mx.ROPE_HALF, mx.ROPE_PAIRS])
@pytest.mark.parametrize("shape", [(1, 5, 64), (7, 1, 64), (1, 1, 64), (1, 5, 80)], ids=str)
def test_rope_in_place_through_two_views_of_one_token_or_head(shape, layout):
    """The stride of an axis of one has no meaning: two views of the same memory may differ in it."""
    T, H, D = shape
    rot = 48 if D == 64 else 24
    table = mx.mxfp4_rope_table(16, rot, mx.make_rope_cfg())
    near = torch.randn(shape, device="cuda").bfloat16()
    want = mx.mxfp4_rope(near, table, layout=layout)
    whole = near.clone().flatten()
    strides = whole.view(shape).stride()
    other = tuple(4096 if n == 1 else s for n, s in zip(shape[:2], strides)) + (1,)
    for x, out in ((whole.view(shape), whole.as_strided(shape, other)), (whole.as_strided(shape, other), whole.view(shape))):
        whole.copy_(near.flatten())
        mx.mxfp4_rope(x, table, layout=layout, out=out)
        assert torch.equal(whole.view(shape), want)
