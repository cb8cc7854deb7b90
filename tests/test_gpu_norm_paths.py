"""ntp_block_norm_fwd / _bwd in every kernel that their rules choose between (tests/test_host_norm_paths.py counts them), and the two calls as the pair that a
training step makes of them, on a real MI355X.  Tolerances as in test_gpu_block_norm.py; where the backward call reads rounded rows beside the statistics of
unrounded ones, what that rounding does to the gradient is added, as derived at the test."""
import numpy as np
import pytest

from oracle import block_oracle as B
from tests.test_gpu_block_norm import BF, Case, U, _bwd_inputs, _close, _norm_size, _say, _step, _through_size, check_bwd, check_fwd, f64, run_bwd

pytestmark = pytest.mark.gpu

# Forward: chunks of 8 columns a thread and the residual's type; rows enough that they do not get more threads each.
# M, H, kind, post, pre, gate, bias, fp32, a, b, pad
FORWARD = [
    (700, 512, B.LAYER, True, True, "channel", True, False, 1.0, 0.5, 0),
    (700, 456, B.RMS, True, True, "token", True, True, 1.5, 1.0, 8),
    (4100, 1000, B.RMS, True, True, "channel", False, False, 1.0, 1.0, 8),
    (300, 8192, B.LAYER, True, True, "none", True, True, 1.0, 0.25, 0),
    (300, 12288, B.LAYER, False, True, "none", True, False, 1.0, 1.0, 0),
    (270, 11272, B.RMS, True, True, "token", True, True, 0.5, 1.0, 8),
    (260, 16384, B.RMS, True, True, "channel", False, False, 1.0, 0.25, 0),
    (257, 16384, B.LAYER, True, True, "channel", True, True, 1.0, 1.0, 0),
]

# Backward: chunks a thread and threads a row go by H alone
ROWS = [(700, 200), (531, 1000), (130, 1288), (41, 4104), (13, 12288), (11, 13000), (9, 17000)]
KINDS = [("none", False, False), ("channel", True, False), ("channel", True, True), ("token", True, True)]  # gate, norm behind the block, betas
BACKWARD = [(M, H, kind, fp32) for M, H in ROWS for kind in range(4) for fp32 in (False, True)]


@pytest.mark.parametrize("M,H,kind,post,pre,gate,bias,fp32,a,b,pad", FORWARD)
def test_forward_kernels(M, H, kind, post, pre, gate, bias, fp32, a, b, pad):
    c = Case(M, H, kind, post, pre, gate, bias, fp32, a, b, pad=pad, seed=M)
    _say(f"block norm forward {M} x {H}, fp32 residual {fp32}")
    Xout, Y = c.new(c.rt), c.new()
    Stats = c.torch.full((4, M), 7.0, device="cuda")
    c.N.ntp_block_norm_fwd(c.shape, c.X, c.Z, Xout, Y, Stats, **c.w)
    c.torch.cuda.synchronize()
    check_fwd(c, c.X, c.Z, Xout, Y, Stats)


@pytest.mark.parametrize("M,H,kind,fp32", BACKWARD)
def test_backward_kernels(M, H, kind, fp32):
    gate, post, bias = KINDS[kind]
    c = Case(M, H, (B.RMS, B.LAYER)[(kind + fp32) % 2], post, True, gate, bias, fp32, a=1.5, b=0.5, seed=H)
    _say(f"block norm backward {M} x {H}, gate {gate}, norm behind the block {post}, betas {bias}, fp32 residual {fp32}")
    dXo, dY, Xout, Z, Stats = _bwd_inputs(c)
    h = c.N.ntp_create()
    n = sum(v.dim() == 1 for v in c.w.values())
    # three workgroups: several turns for each, and the second launch
    c.N.ntp_set_workspace(c.torch.full((3 * n * H,), float("nan"), device="cuda"), handle=h)
    dX, dZ, grads = run_bwd(c, dXo, dY, Xout, Z, Stats, handle=h)
    c.torch.cuda.synchronize()
    check_bwd(c, dXo, dY, Xout, Z, Stats, dX, dZ, grads)
    c.N.ntp_destroy(h)


def _behind_norm(e_up, t, st):
    """What an error of at most e_up in the gradient of a norm's values becomes in the gradient of its input."""
    hat = np.abs(B._hat(t, st))
    return st[1][:, None] * (e_up + e_up.mean(1, keepdims=True) + hat * (e_up * hat).mean(1, keepdims=True))


@pytest.mark.parametrize("kind", [B.RMS, B.LAYER])
@pytest.mark.parametrize("fp32", [False, True], ids=["bf16 residual", "fp32 residual"])
@pytest.mark.parametrize("M,H,post,gate,bias", [(33, 1032, True, "channel", True), (70, 4096, False, "token", False), (19, 12288, False, "none", True), (600, 520, True, "token", True)])
def test_gradient_from_what_the_forward_call_kept(M, H, post, gate, bias, fp32, kind):
    """The forward call keeps statistics of the unrounded X', the backward call reads them beside the rounded one.

    First what it makes of these inputs.  Then against the gradient of the unrounded chain: with e = rstd |X' - its rounding| (half a step of X' at most) in hat_x,
    the gradient u - mean(u) - hat mean(u hat) is off by e |mean(u hat)| + |hat| mean(|u| e) + e mean(|u| e), and sum dY hat by sum |dY| e; behind that
    everything is linear in G."""
    c = Case(M, H, kind, post, True, gate, bias, fp32, a=1.0, b=0.5, seed=M)
    torch = c.torch
    Xout, Y, Stats = c.new(c.rt), c.new(), torch.zeros(4, M, device="cuda")
    c.N.ntp_block_norm_fwd(c.shape, c.X, c.Z, Xout, Y, Stats, **c.w)
    dXo, dY = c.rand(0.1, c.rt), c.rand(0.1)
    dX, dZ, grads = run_bwd(c, dXo, dY, Xout, c.Z, Stats)
    torch.cuda.synchronize()
    check_bwd(c, dXo, dY, Xout, c.Z, Stats, dX, dZ, grads)
    # the chain in float64, nothing rounded between the calls
    w, x, z, d0, dy = c.w64(), f64(c.X), f64(c.Z), f64(dXo), f64(dY)
    out, _, st = B.block_norm_fwd(x, z, w, kind, c.eps, c.a, c.b)
    want = B.block_norm_bwd(d0, dy, out, z, st, w, kind, c.a, c.b)
    half = U if fp32 else BF
    size_x = np.abs(c.a * x) + np.abs(c.b * w.get("gate", 1.0)) * (_norm_size(z, st[:2], w["post_gamma"], w.get("post_beta", 0.0)) if post else np.abs(z))
    hat, u = B._hat(out, st[2:]), dy * w["pre_gamma"]
    # the forward call's fp32 arithmetic: rows within 512 U of their sizes, statistics as in check_fwd
    top = size_x.max(1, keepdims=True)
    rs = st[3][:, None]
    e = rs * (half * np.abs(out) + 512 * U * (size_x + size_x.mean(1, keepdims=True))) + 512 * U * (1 + rs * top) * np.abs(hat)
    mean = lambda t: t.mean(1, keepdims=True)  # noqa: E731
    e_G = rs * (e * np.abs(mean(u * hat)) + np.abs(hat) * mean(np.abs(u) * e) + e * mean(np.abs(u) * e))
    e_G = e_G + 512 * U * (1 + rs * top) * rs * _through_size(u, out, st[2:])  # (of the factor rstd)
    G_size = np.abs(d0) + rs * _through_size(u, out, st[2:])
    e_G = e_G + 512 * U * G_size
    _close(dX, want["dX"], _step(want["dX"], dX) * (1 + half) + (1 + half) * abs(c.a) * e_G, "dX")
    _close(grads["pre_gamma"], want["pre_gamma"], (np.abs(dy) * e).sum(0) + (M + 512) * U * (np.abs(dy) * (np.abs(hat) + rs * (np.abs(out) + np.abs(st[2][:, None])) + e)).sum(0),
           "pre_gamma")
    g = np.abs(w.get("gate", 1.0))
    e_r, r_size = abs(c.b) * e_G, abs(c.b) * (G_size + e_G)
    zs = np.abs(z)
    if post:
        zs = np.abs(B._hat(z, st[:2])) + st[1][:, None] * (np.abs(z) + mean(np.abs(z)))
    r = zs * np.abs(w.get("post_gamma", 1.0)) + np.abs(w.get("post_beta", 0.0))
    stat = 512 * U * (1 + st[1][:, None] * np.abs(z).max(1, keepdims=True)) if post else 0.0  # of the kept statistics of Z, relative to sizes
    if "gate" in w:
        e_gate = e_r * r + (512 * U + 2 * stat) * r_size * r
        if gate == "token":
            _close(grads["gate"], want["gate"], _step(want["gate"], grads["gate"]) * (1 + half) + (1 + BF) * e_gate, "gate")
        else:
            _close(grads["gate"], want["gate"], e_gate.sum(0) + (M + 512) * U * (r_size * r).sum(0), "gate")
    e_z, z_size = e_r * g, r_size * g
    if post:
        _close(grads["post_gamma"], want["post_gamma"], (e_z * zs).sum(0) + ((M + 512) * U + 2 * stat.max()) * (z_size * zs).sum(0), "post_gamma")
        up = np.abs(w["post_gamma"])
        e_z = _behind_norm(e_z * up, z, st[:2]) + (512 * U + 4 * stat) * st[1][:, None] * (z_size * up + mean(z_size * up) + zs * mean(z_size * up * zs))
    else:
        e_z = e_z + 512 * U * z_size
    _close(dZ, want["dZ"], _step(want["dZ"], dZ) * (1 + BF) + (1 + BF) * e_z, "dZ")


@pytest.mark.parametrize("fp32", [False, True], ids=["bf16 residual", "fp32 residual"])
@pytest.mark.parametrize("M,H", [(37, 264), (300, 4104), (5, 16392)])
@pytest.mark.parametrize("post,gate", [(False, "none"), (False, "channel"), (False, "token"), (True, "none")])
def test_a_block_without_a_norm_before_the_next(post, gate, M, H, fp32):
    """Residual addition alone, with a gate, or with the norm behind the block: no dY and no X' are read; the gradient without a residual's own is zero."""
    c = Case(M, H, B.LAYER, post, False, gate, True, fp32, a=1.5, b=0.5, seed=H)
    torch = c.torch
    Xout, Stats = c.new(c.rt), torch.full((4, M), 7.0, device="cuda")
    c.N.ntp_block_norm_fwd(c.shape, c.X, c.Z, Xout, None, Stats, **c.w)
    dXo = c.rand(0.1, c.rt)
    dX, dZ, grads = run_bwd(c, dXo, None, None, c.Z, Stats if post else None)
    torch.cuda.synchronize()
    st = check_fwd(c, c.X, c.Z, Xout, None, Stats)
    check_bwd(c, dXo, None, None, c.Z, Stats, dX, dZ, grads)
    assert post or not st.any()
    dX0, dZ0, grads0 = run_bwd(c, None, None, None, c.Z, Stats if post else None)
    torch.cuda.synchronize()
    assert not any(bool(t.any()) for t in (dX0, dZ0, *grads0.values()))
    if gate == "none" and not post:  # Z is not read
        dX2 = c.new(c.rt)
        dZ2 = c.new()
        c.N.ntp_block_norm_bwd(c.shape, dXo, None, None, None, None, dX2, dZ2)
        torch.cuda.synchronize()
        assert torch.equal(dX2, dX) and torch.equal(dZ2, dZ)
