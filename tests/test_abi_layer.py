"""CPU-only checks that the calls around a linear layer refuse on the host what they cannot do."""
import ctypes
import os

import pytest

import paper_2605_09825_amd as mx

P = 0x10000  # an aligned, non-null address that is never followed on the host


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(mx.LIB_PATH):
        from paper_2605_09825_amd.build import build
        build()
    return mx.lib()


def changed(ok, **by):
    return list(dict(ok, **by).values())


def test_residual_norm_forward_refusals(L):
    cfg = mx.make_norm_cfg(post_norm=True)
    ok = dict(x=P, ld_x=64, o=P, ld_o=64, gate=None, ld_gate=0, w_post=P, w_pre=P, rows=4, cols=64, xt=0, bt=0, cfg=ctypes.byref(cfg),
              x_out=P, ld_x_out=64, h=P, ld_h=64, rstd=P, stream=None)

    def call(**by):
        return L.mxfp4_residual_norm_fwd(*changed(ok, **by))

    assert call(rows=0, x=None, o=None, w_post=None, cfg=ctypes.byref(mx.make_norm_cfg())) == mx.OK
    for by in (dict(x=None), dict(x_out=None, h=None, w_pre=None), dict(xt=2), dict(bt=-1), dict(cfg=None), dict(o=None), dict(h=None),
               dict(o=None, w_post=None, gate=P, cfg=ctypes.byref(mx.make_norm_cfg())), dict(cfg=ctypes.byref(mx.make_norm_cfg()))):
        assert call(**by) == mx.EINVAL, by
    for bad in (dict(eps=-1.0), dict(eps=float("nan")), dict(residual_scale=float("inf")), dict(weight_offset=float("nan"))):
        assert call(cfg=ctypes.byref(mx.make_norm_cfg(post_norm=True, **bad))) == mx.EINVAL, bad
    for by in (dict(rows=-1), dict(cols=0), dict(cols=16385, ld_x=16385), dict(ld_x=63), dict(ld_o=63), dict(ld_h=1), dict(ld_x_out=0),
               dict(gate=P, ld_gate=63)):
        assert call(**by) == mx.ESHAPE, by
    for by in (dict(x=P + 1), dict(x=P + 2, xt=1), dict(gate=P + 2), dict(h=P + 1), dict(w_pre=P + 2), dict(rstd=P + 2)):
        assert call(**by) == mx.EALIGN, by


def test_residual_norm_backward_refusals_and_workspace(L):
    cfg = mx.make_norm_cfg(post_norm=True)
    ok = dict(dx_out=P, ld_dxo=64, dh=P, ld_dh=64, x_out=P, ld_x=64, o=P, ld_o=64, gate=P, ld_gate=0, w_post=P, w_pre=P, rstd=P, rows=4,
              cols=64, xt=0, bt=0, cfg=ctypes.byref(cfg), dx=P, ld_dx=64, do=P, ld_do=64, dgate=P, ld_dgate=0, dw_post=P, dw_pre=P,
              ws=P, n=1 << 20, stream=None)

    def call(**by):
        return L.mxfp4_residual_norm_bwd(*changed(ok, **by))

    nothing = dict(dx=None, do=None, dgate=None, dw_post=None, dw_pre=None)
    assert call(**nothing) == mx.OK
    for by in (dict(dx_out=None, dh=None), dict(rstd=None), dict(x_out=None), dict(o=None), dict(gate=None), dict(ws=None), dict(dh=None),
               dict(cfg=ctypes.byref(mx.make_norm_cfg())), dict(cfg=None)):
        assert call(**by) == mx.EINVAL, by
    for by in (dict(ld_dxo=1), dict(ld_dh=63), dict(ld_x=63), dict(ld_dx=63), dict(ld_do=0), dict(cols=20000), dict(rows=-2),
               dict(ld_gate=64, ld_dgate=63)):
        assert call(**by) == mx.ESHAPE, by
    for by in (dict(ws=P + 8), dict(dw_pre=P + 1), dict(dgate=P + 2), dict(do=P + 1)):
        assert call(**by) == mx.EALIGN, by
    need = mx.mxfp4_residual_norm_workspace_bytes(4, 64)
    assert call(n=need - 1) == mx.EWORKSPACE and need >= 2 * 64 * 4
    assert mx.mxfp4_residual_norm_workspace_bytes(0, 64) == 0 and mx.mxfp4_residual_norm_workspace_bytes(1, 16385) == 0
    # grows with the rows up to a limit only
    assert mx.mxfp4_residual_norm_workspace_bytes(1 << 30, 4096) == mx.mxfp4_residual_norm_workspace_bytes(1 << 20, 4096)


def test_rope_refusals(L):
    ok = dict(x=P, xt=6144, xh=128, out=P + 4096, ot=5120, oh=128, tokens=4, heads=40, dim=128, rot=128, dtype=0, layout=0, inverse=0,
              positions=None, first=0, table=P, n=100, stream=None)

    def call(**by):
        return L.mxfp4_rope(*changed(ok, **by))

    assert call(tokens=0, x=None) == mx.OK and call(heads=0, out=None) == mx.OK
    for by in (dict(x=None), dict(out=None), dict(table=None), dict(dtype=2), dict(layout=2), dict(inverse=2), dict(out=P)):
        assert call(**by) == mx.EINVAL, by
    for by in (dict(tokens=-1), dict(heads=-1), dict(dim=1), dict(rot=0), dict(rot=127), dict(rot=130), dict(xt=-1), dict(oh=127), dict(ot=5119),
               dict(oh=0), dict(n=-1)):
        assert call(**by) == mx.ESHAPE, by
    for by in (dict(x=P + 1), dict(out=P + 2, dtype=1), dict(positions=P + 2), dict(table=P + 8)):
        assert call(**by) == mx.EALIGN, by


def test_rope_table_refusals(L):
    def call(table=P, positions=8, rot=64, **kw):
        return L.mxfp4_rope_table(table, positions, rot, ctypes.byref(mx.make_rope_cfg(**kw)), None)

    assert call(positions=0) == mx.OK and L.mxfp4_rope_table(P, 8, 64, None, None) == mx.EINVAL
    yarn = dict(scaling=mx.ROPE_SCALE_YARN, factor=2.0)
    for kw in (dict(table=None), dict(base=1.0), dict(base=float("nan")), dict(scaling=5), dict(scaling=1, factor=0.5), dict(yarn, low=0.0),
               dict(yarn, low=4.0, high=4.0), dict(yarn, original_positions=0.0), dict(attention_factor=-1.0)):
        assert call(**kw) == mx.EINVAL, kw
    assert call(rot=63) == mx.ESHAPE and call(rot=0) == mx.ESHAPE and call(positions=-1) == mx.ESHAPE
    assert call(table=P + 4) == mx.EALIGN


def test_orthogonalize_refusals_and_workspace(L):
    need = mx.mxfp4_orthogonalize_workspace_bytes(2, 100, 200)
    ok = dict(g=P, ld_g=200, gm=20000, m=P, out=P, ld_out=200, om=20000, batch=2, N=100, K=200, dtype=1,
              cfg=ctypes.byref(mx.make_muon_cfg()), ws=P, n=need, stream=None)

    def call(**by):
        return L.mxfp4_orthogonalize(*changed(ok, **by))

    for by in (dict(batch=0), dict(N=0), dict(K=0)):
        assert call(g=None, out=None, ws=None, **by) == mx.OK, by
    for by in (dict(g=None), dict(out=None), dict(ws=None), dict(dtype=2), dict(cfg=None)):
        assert call(**by) == mx.EINVAL, by
    # (the last three take a singular value, or the polynomial, out of the range that the operands' scales allow)
    for bad in (dict(steps=0), dict(steps=65), dict(eps=0.0), dict(eps=float("nan")), dict(momentum=float("inf")), dict(out_scale=float("nan")),
                dict(a=float("nan")), dict(a=4.0, b=0.0, c=0.0), dict(b=-20.0), dict(a=2.0, b=0.0, c=0.0, steps=2)):
        assert call(cfg=ctypes.byref(mx.make_muon_cfg(**bad))) == mx.EINVAL, bad
    assert L.mxfp4_orthogonalize(*changed(ok, cfg=ctypes.byref(mx.MuonCfg(0.9, 2, 5, 1.0, 0.0, 0.0, 1e-7, 1.0)))) == mx.EINVAL
    for by in (dict(batch=-1), dict(N=-1), dict(K=(1 << 20) + 1), dict(ld_g=199), dict(ld_out=199), dict(om=19999), dict(gm=-1),
               dict(batch=65535, N=1 << 14, K=1 << 14, ld_g=1 << 14, ld_out=1 << 14, om=1 << 28, n=1 << 62)):
        assert call(**by) == mx.ESHAPE, by
    for by in (dict(g=P + 2), dict(out=P + 1), dict(ws=P + 128), dict(m=P + 2)):
        assert call(**by) == mx.EALIGN, by
    assert call(n=need - 1) == mx.EWORKSPACE
    assert mx.mxfp4_orthogonalize_workspace_bytes(0, 1, 1) == 0 and mx.mxfp4_orthogonalize_workspace_bytes(1, 1, (1 << 20) + 1) == 0
    # X's first words twice, its second ones, three symmetric matrices, at 2 bytes
    assert mx.mxfp4_orthogonalize_workspace_bytes(1, 128, 256) >= 3 * 2 * 128 * 256 + 3 * 2 * 128 * 128


class Device:
    """What the binding asks of a tensor before it hands its address on, of one that is in CUDA memory by its word alone."""
    is_cuda = True

    def __init__(self, t):
        self.t, self.dtype, self.shape = t, t.dtype, t.shape

    def __getattr__(self, name):
        return getattr(self.t, name)

    def data_ptr(self):
        return P


@pytest.mark.parametrize("branch", ["bfloat16", "float32"])
@pytest.mark.parametrize("what", ["forward", "backward", "dgate"])
def test_a_gate_per_row_that_is_broadcast_over_rows_is_refused(L, monkeypatch, what, branch):
    """Its leading dimension is 0, which the C calls take as one fp32 vector [cols] for all rows: refused with the code of any other operand's 0."""
    import torch
    monkeypatch.setattr(mx, "_stream_ptr", lambda stream: None)
    branch = getattr(torch, branch)
    dense = Device(torch.empty((4, 64), dtype=branch))
    broadcast = Device(torch.empty(64, dtype=branch).expand(4, 64))
    rstd, ws = Device(torch.empty((2, 4))), Device(torch.empty(1 << 20, dtype=torch.uint8))
    cfg = mx.make_norm_cfg()
    reached = []
    for call in ("mxfp4_residual_norm_fwd", "mxfp4_residual_norm_bwd"):
        monkeypatch.setattr(L, call, lambda *args: reached.append(args) or mx.OK)
    with pytest.raises(mx.Mxfp4Error) as e:
        if what == "forward":
            mx.mxfp4_residual_norm_fwd(dense, dense, cfg, gate=broadcast, x_out=dense, h=dense, rstd=rstd)
        else:
            gate, dgate = (broadcast, dense) if what == "backward" else (dense, broadcast)
            mx.mxfp4_residual_norm_bwd(dense, dense, dense, dense, rstd, cfg, gate=gate, dgate=dgate, dx=dense, workspace=ws)
    assert e.value.status == mx.ESHAPE and not reached
    # one row, or rows of their own, are the C call's to check
    for rows in (1, 4):
        t, r = Device(torch.empty((rows, 64), dtype=branch)), Device(torch.empty((2, rows)))
        gate = Device(torch.empty(64, dtype=branch).expand(1, 64)) if rows == 1 else t
        mx.mxfp4_residual_norm_fwd(t, t, cfg, gate=gate, x_out=t, h=t, rstd=r)
        assert reached.pop()[5] == 64


def test_steps_are_joined_on_request_only(L):
    assert mx.make_muon_cfg().join_steps == 0 and mx.make_muon_cfg(join_steps=True).join_steps == 1
    cfg = mx.make_muon_cfg()
    for join, status in ((0, mx.OK), (1, mx.OK), (2, mx.EINVAL), (-1, mx.EINVAL)):
        cfg.join_steps = join
        assert L.mxfp4_orthogonalize(None, 200, 0, None, None, 200, 0, 0, 100, 200, 1, ctypes.byref(cfg), None, 0, None) == status, join


def test_sizes_whose_products_pass_64_bits_are_refused(L):
    """Strides that no allocation has: what is worked out of them on the host, and the kernels' offsets, would wrap around."""
    rope = dict(x=P, xt=6144, xh=128, out=P + 4096, ot=5120, oh=128, tokens=4, heads=40, dim=128, rot=128, dtype=0, layout=0, inverse=0,
                positions=None, first=0, table=P, n=100, stream=None)
    for by in (dict(tokens=2**24 + 1, heads=2, ot=2**40, oh=128, dim=256, rot=256),          # (tokens - 1) ot is 2^64: heads that overlap
               dict(tokens=2**24 + 1, ot=2**40), dict(tokens=2**24 + 1, xt=2**40),             # ... and that do not
               dict(tokens=2**40, heads=2**20, dim=2**16, rot=2, ot=2**36, oh=2**16, xt=0),    # 2^76 elements
               dict(n=2**31 + 1), dict(n=2**62)):
        assert L.mxfp4_rope(*changed(rope, **by)) == mx.ESHAPE, by
    cfg = mx.make_norm_cfg()
    norm = dict(x=P, ld_x=64, o=P, ld_o=64, gate=None, ld_gate=0, w_post=None, w_pre=None, rows=2**24 + 1, cols=64, xt=0, bt=0, cfg=ctypes.byref(cfg),
                x_out=P, ld_x_out=64, h=P, ld_h=64, rstd=None, stream=None)
    for by in (dict(ld_x=2**40), dict(ld_o=2**40), dict(ld_x_out=2**40), dict(ld_h=2**40), dict(gate=P, ld_gate=2**40)):
        assert L.mxfp4_residual_norm_fwd(*changed(norm, **by)) == mx.ESHAPE, by
    norm = dict(dx_out=P, ld_dxo=64, dh=P, ld_dh=64, x_out=P, ld_x=64, o=P, ld_o=64, gate=P, ld_gate=64, w_post=None, w_pre=None, rstd=P, rows=2**24 + 1,
                cols=64, xt=0, bt=0, cfg=ctypes.byref(cfg), dx=P, ld_dx=64, do=P, ld_do=64, dgate=P, ld_dgate=64, dw_post=None, dw_pre=None,
                ws=None, n=0, stream=None)
    for by in ("ld_dxo", "ld_dh", "ld_x", "ld_o", "ld_gate", "ld_dx", "ld_do", "ld_dgate"):
        assert L.mxfp4_residual_norm_bwd(*changed(norm, **{by: 2**40})) == mx.ESHAPE, by


def test_no_workspace_is_named_for_an_update_that_is_refused(L):
    """Sizes within 2^20 each, whose tiles of 64 x 64 are too many for a launch."""
    for batch, N, K, there in ((1, 1 << 18, 1 << 18, False), (1, (1 << 18) - 64, 1 << 18, True), (65535, 1 << 14, 1 << 14, False), (256, 1 << 14, 1 << 14, False),
                               (255, 1 << 14, 1 << 14, True), (1, 1 << 20, 1 << 20, False)):
        need = mx.mxfp4_orthogonalize_workspace_bytes(batch, N, K)
        cfg = mx.make_muon_cfg()
        args = [P, K, N * K, None, P, K, N * K, batch, N, K, 1, ctypes.byref(cfg), P, 0, None]  # (a workspace of 0 bytes: no call gets beyond the checks)
        assert L.mxfp4_orthogonalize(*args) == (mx.EWORKSPACE if there else mx.ESHAPE), (batch, N, K)
        assert (need > 0) == there, (batch, N, K)


def test_range_of_coefficients_that_are_nearly_a_cubic(L):
    """A third coefficient that is nothing beside the others changes nothing of where the polynomial's extremes lie."""
    def call(**kw):
        return L.mxfp4_orthogonalize(None, 1, 0, None, None, 1, 0, 0, 1, 1, 1, ctypes.byref(mx.make_muon_cfg(**kw)), None, 0, None)

    for c in (0.0, 1e-7, 1e-12, 1e-20, -1e-20, 1e-38):
        assert call(steps=2, a=3.4, b=-2.7, c=c) == mx.EINVAL, c  # 1.47 at s^2 = 0.42; from there -3.6
        assert call(steps=1, a=3.4, b=-2.7, c=c) == mx.OK, c
        assert call(steps=64, a=1.5, b=-0.5, c=c) == mx.OK, c
    assert call(steps=64) == mx.OK and call(steps=3, a=0.0, b=1.0, c=0.0) == mx.OK and call(steps=64, a=1.0, b=0.0, c=0.0) == mx.OK
    assert call(steps=1, a=0.0, b=0.0, c=0.0) == mx.OK
