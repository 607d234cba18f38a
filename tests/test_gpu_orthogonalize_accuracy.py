"""What include/mxfp4.h says of the accuracy of mxfp4_orthogonalize, against Newton-Schulz steps in 64 bits, on the spectra that gradients have.

The result's error before it is rounded to bf16: what is off in all, less (as squares) what rounding the 64-bit result to bf16 would be off.  The two are
independent, since the rounding's place within an ulp is, and there are so many elements that nothing of that is left to chance."""
import pytest
import torch

import paper_2605_09825_amd as mx

pytestmark = pytest.mark.gpu


def steps_of(g, cfg):
    x = g.double()
    tall = x.shape[-2] > x.shape[-1]
    x = x.transpose(-1, -2).contiguous() if tall else x
    x = x / (x.square().sum((-1, -2), keepdim=True).sqrt() + cfg.eps)
    for _ in range(cfg.steps):
        p = x @ x.transpose(-1, -2).contiguous()
        x = cfg.a * x + (cfg.b * p + cfg.c * (p @ p)) @ x
    return x.transpose(-1, -2) if tall else x


def before_rounding(got, want):
    total, own = (float((t.double() - want).norm() / want.norm()) for t in (got, want.bfloat16()))
    return max(0.0, total ** 2 - own ** 2) ** 0.5


def gradient(shape, spectrum, seed=0):
    gen = torch.Generator().manual_seed(seed)
    m, n = min(shape), max(shape)

    def normal(*s):
        return torch.randn(s, generator=gen)

    i = torch.arange(1, m + 1, dtype=torch.float32)
    values = {"1/i": 1 / i, "1/i^2": i ** -2.0, "exponential": torch.exp(-20.0 * i / m)}.get(spectrum)
    if values is not None:
        g = torch.linalg.qr(normal(m, m))[0] * values @ torch.linalg.qr(normal(n, m))[0].T
    else:  # noise, alone or under sixteen directions or one
        g = normal(m, n)
        if spectrum == "sixteen":
            g = 1e-4 * g + 1e-2 * normal(m, 16) @ (2.5e-3 * normal(16, n))
        elif spectrum == "one":
            g = 1e-3 * g + normal(m, 1) @ normal(1, n)
    return (g if shape[0] <= shape[1] else g.T).contiguous().cuda()


SPECTRA = ["white", "sixteen", "one", "1/i", "1/i^2", "exponential"]


@pytest.mark.parametrize("join", [False, True])
@pytest.mark.parametrize("spectrum", SPECTRA)
@pytest.mark.parametrize("shape", [(512, 2048), (1024, 4096), (4320, 1440), (600, 8000)], ids=str)
def test_five_steps(shape, spectrum, join):
    cfg = mx.make_muon_cfg(join_steps=join)
    g = gradient(shape, spectrum)
    assert before_rounding(mx.mxfp4_orthogonalize(g, cfg)[0], steps_of(g, cfg)) <= (5e-3 if join else 1e-3)


def test_steps_are_single_unless_asked_for():
    """Joined steps round otherwise: at a size where they pay, the two settings differ in some bits, and the default is the single steps'."""
    g = gradient((1024, 4096), "1/i")
    single, joined = (mx.mxfp4_orthogonalize(g, mx.make_muon_cfg(join_steps=join))[0] for join in (False, True))
    assert torch.equal(mx.mxfp4_orthogonalize(g, mx.make_muon_cfg())[0], single) and not torch.equal(single, joined)


@pytest.mark.parametrize("join", [False, True])
def test_rows_that_are_nearly_equal(join):
    """Two rows hold nearly all of the gradient, and differ by 1.4e-3 of themselves.  A step makes each of them from its own first word and the other's (rounded by
    at most 2.1e-4 of it in the root mean square): with T the matrix of the step, off by T01 2.1e-4 each, which is 2^.5 as much of their difference, where the
    difference itself becomes a (1.4e-3).  T01 is (0.7 - a) / 2 for one step (0.7: what the polynomial makes of 1), and (0.7 - a^3) / 2 for three: 0.084 and 0.103 of
    the difference, and later steps, in which it is larger, add less than a tenth of that.  (The whole matrix is off by 1e-3 all the same: the bound on it is that of
    a few directions, 5e-3.)"""
    gen = torch.Generator().manual_seed(8)
    g = 1e-6 * torch.randn((1024, 4096), generator=gen)
    g[:2] += 1e-3 * torch.randn((4096,), generator=gen)
    g = g.cuda()
    cfg = mx.make_muon_cfg(join_steps=join)
    got, want = mx.mxfp4_orthogonalize(g, cfg)[0].double(), steps_of(g, cfg)
    assert float((got - want).norm() / want.norm()) <= 5e-3
    apart = (got[0] - got[1]) - (want[0] - want[1])
    assert float(apart.norm() / (want[0] - want[1]).norm()) <= (0.114 if join else 0.093)
