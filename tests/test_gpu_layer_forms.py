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


@pytest.mark.parametrize("layout", [mx.ROPE_HALF, mx.ROPE_PAIRS])
@pytest.mark.parametrize("factor", [0.0, 1.5])
def test_rope_there_and_back_is_the_square_of_the_attention_factor(factor, layout):
    """cos^2 + sin^2 of table values (2^-23 each) is within 2^-21 of the factor's square, and two turns of fp32 elements within 2^-21 of |u| + |v|."""
    cfg = mx.make_rope_cfg(scaling=mx.ROPE_SCALE_YARN, factor=16.0, attention_factor=factor)
    square = (factor or 0.1 * torch.tensor(16.0, dtype=torch.float64).log().item() + 1.0) ** 2
    table = mx.mxfp4_rope_table(300, 64, cfg)
    x = torch.randn((300, 2, 96), device="cuda")
    back = mx.mxfp4_rope(mx.mxfp4_rope(x, table, layout=layout), table, layout=layout, inverse=True)
    assert torch.equal(back[..., 64:], x[..., 64:])
    pair = x[..., :64].view(300, 2, 2, 32).abs().sum(2).repeat(1, 1, 2) if layout == mx.ROPE_HALF else x[..., :64].view(300, 2, 32, 2).abs().sum(3).repeat_interleave(2, -1)
    assert ((back[..., :64].double() - square * x[..., :64].double()).abs() <= square * 2.0 ** -20 * pair.double()).all()


def test_what_a_call_allocates_belongs_to_its_stream():
    """Else the allocator would hand a workspace that the caller drops to the current stream's next tensor, while the call's stream still works on it."""
    side = torch.cuda.Stream()
    x, o = (torch.randn((600, 4096), device="cuda").bfloat16() for _ in range(2))
    w, g = torch.ones(4096, device="cuda"), torch.randn((300, 4096), device="cuda")
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    side.wait_stream(torch.cuda.current_stream())
    cfg = mx.make_norm_cfg()
    x_out, h, rstd = mx.mxfp4_residual_norm_fwd(x, o, cfg, w_pre=w, stream=side)
    made = [x_out, h, rstd, mx.mxfp4_residual_norm_bwd(x, o, x_out, o, rstd, cfg, w_pre=w, dx=dx, dw_pre=dw, stream=side)]
    made += mx.mxfp4_orthogonalize(g, mx.make_muon_cfg(), stream=side)
    table = mx.mxfp4_rope_table(1 << 15, 128, mx.make_rope_cfg(), stream=side)
    made += [table, mx.mxfp4_rope(x.view(600, 32, 128), table, stream=side)]
    side.synchronize()
    segments = torch.cuda.memory_snapshot()
    for t in made:
        mine = [s for s in segments if s["address"] <= t.data_ptr() < s["address"] + s["total_size"]]
        assert len(mine) == 1 and mine[0]["stream"] == side.cuda_stream, t.shape
    here = mx.mxfp4_orthogonalize(g, mx.make_muon_cfg())[0]
    assert torch.equal(here, made[4])
