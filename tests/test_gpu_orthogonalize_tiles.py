"""mxfp4_orthogonalize on every tile shape with ragged edges, in batches, joined and single, with more steps and with other coefficients.

Tolerances are those of test_gpu_orthogonalize.py, whose derivation counts 6.3e-4 for a step and 1.7e-3 for the output; joined steps round more m x m matrices in place of
X: no more than as many again for white gradients, whose errors no step singles out."""
import pytest
import torch

import paper_2605_09825_amd as mx
from test_gpu_orthogonalize import gradient, near, steps_of

pytestmark = pytest.mark.gpu
BOTH = pytest.mark.parametrize("join", [False, True])


# tiles of P X: 256 x 256 for the first three (the third turned on its way out), 192 x 256 for the next two, 192 x 192, and whole ones that are joined
@BOTH
@pytest.mark.parametrize("shape", [(2880, 4450), (2881, 4452), (4450, 2880), (3000, 3700), (3701, 3001), (2900, 3003), (4096, 14336), (6144, 4096), (1440, 4321)], ids=str)
def test_wide_tiles_with_ragged_edges(shape, join):
    cfg = mx.make_muon_cfg(join_steps=join)
    g = gradient(shape, sum(shape), strong=0.5)
    near(mx.mxfp4_orthogonalize(g, cfg)[0], steps_of(g, cfg))


@BOTH
@pytest.mark.parametrize("shape", [(2880, 4448), (4450, 2880), (3000, 3700), (1024, 4096)], ids=str)
def test_output_rows_at_odd_places(shape, join):
    """Of any distance and alignment; what lies between them stays."""
    N, K = shape
    cfg = mx.make_muon_cfg(join_steps=join)
    g = gradient(shape, 1, torch.bfloat16)
    want = mx.mxfp4_orthogonalize(g, cfg)[0]
    for more, at in ((5, 1), (8, 2), (16, 0)):
        room = torch.full((N + 2, K + more), 7.0, dtype=torch.bfloat16, device="cuda")
        out = room[1:N + 1, at:at + K]
        mx.mxfp4_orthogonalize(g, cfg, out=out)
        assert torch.equal(out, want)
        out.fill_(7.0)
        assert (room == 7.0).all()


@BOTH
@pytest.mark.parametrize("shape", [(2, 1024, 4096), (2, 1440, 4320), (2, 4320, 1440), (2, 2050, 3001), (3, 1440, 2222), (2, 3001, 2050)], ids=str)
def test_batches_on_larger_tiles(shape, join):
    cfg = mx.make_muon_cfg(join_steps=join)
    g, m = gradient(shape, 5, strong=0.5), gradient(shape, 6)
    alone = m.clone()
    out = mx.mxfp4_orthogonalize(g, cfg, momentum=m)[0]
    near(out, steps_of(g.double() + float(torch.tensor(0.95)) * m.double(), cfg))
    for b in range(shape[0]):
        single = mx.mxfp4_orthogonalize(g[b], cfg, momentum=alone[b])[0]
        near(single, steps_of(g[b].double() + float(torch.tensor(0.95)) * m[b].double(), cfg))
    assert torch.equal(alone, m)


@pytest.mark.parametrize("steps", [1, 2, 3, 4, 5])
@pytest.mark.parametrize("shape", [(1024, 4096), (4320, 1440), (600, 8000)], ids=str)
def test_runs_of_joined_steps(shape, steps):
    cfg = mx.make_muon_cfg(steps=steps, join_steps=True, out_scale=2.0)
    g = gradient(shape, steps, strong=0.5)
    near(mx.mxfp4_orthogonalize(g, cfg)[0], steps_of(g, cfg))


@pytest.mark.parametrize("shape", [(1024, 4096), (2, 1440, 4320)], ids=str)
def test_joined_steps_repeated_and_with_other_contents_of_the_workspace(shape):
    cfg = mx.make_muon_cfg(join_steps=True)
    g = gradient(shape, 7)
    first, ws = mx.mxfp4_orthogonalize(g, cfg)
    for fill in (0x00, 0xFF, 0x7C):
        ws.fill_(fill)
        for _ in range(3):
            assert torch.equal(mx.mxfp4_orthogonalize(g, cfg, workspace=ws)[0], first)


@pytest.mark.parametrize("kw", [dict(steps=8), dict(steps=15), dict(steps=15, join_steps=True), dict(steps=12, a=1.5, b=-0.5, c=0.0),
                                dict(steps=14, a=1.875, b=-1.25, c=0.375), dict(steps=9, a=2.0, b=-1.5, c=0.5), dict(steps=12, a=1.5, b=-0.5, c=0.0, join_steps=True),
                                dict(steps=1, a=0.0, b=1.0, c=0.0), dict(steps=1, a=0.0, b=0.0, c=1.0), dict(steps=1, a=-1.0, b=0.5, c=0.25)], ids=str)
@pytest.mark.parametrize("shape", [(128, 700), (512, 2048), (3001, 1024), (1024, 6000)], ids=str)
def test_more_steps_and_other_coefficients(shape, kw):
    """White gradients: every step adds its 6.3e-4, and the output 1.7e-3.  (With a = 0 there is no term with X's two words: the product's operands, three of 2.1e-4
    and A's squared, stay below that.)"""
    cfg = mx.make_muon_cfg(**kw)
    g = gradient(shape, cfg.steps)
    want = steps_of(g, cfg)
    assert float((mx.mxfp4_orthogonalize(g, cfg)[0].double() - want).norm() / want.norm()) <= 6.3e-4 * cfg.steps * (2 if cfg.join_steps else 1) + 1.7e-3
