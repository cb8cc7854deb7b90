"""ntp_block_norm_fwd / _bwd against the float64 oracle, on a real MI355X.

Tolerances.  An output is rounded once: half a step of its type (bf16 2^-8 of the value).  Before that the arithmetic is fp32: a row's sums have at
most 32 additions in a thread, 6 in a wavefront, 16 over wavefronts, their relative error is below 64 * 2^-24 of the sum of the terms' sizes; mean, deviation
and the value made from them add less than as much again, and a second norm behind the first doubles that: 512 * 2^-24 of the size of what is
added up.  Sums over M rows: (M + 512) * 2^-24 of the sum of the sizes."""
import sys

import numpy as np
import pytest

from oracle import block_oracle as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BF = 2.0 ** -8


def _say(msg):
    print(f"[gpu-case] {msg}", file=sys.stderr, flush=True)


class Case:
    """Inputs on the device (rows `pad` elements longer than H, the pad poisoned) and in float64."""

    def __init__(self, M, H, kind, post, pre, gate, bias, fp32, a=1.0, b=1.0, eps=1e-5, seed=0, pad=0, scale=2.0):
        import torch
        import paper_2504_06095_amd as N
        self.torch, self.N, self.M, self.H, self.kind, self.a, self.b, self.eps, self.pad = torch, N, M, H, kind, a, b, eps, pad
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        self.bf, self.rt = torch.bfloat16, torch.float32 if fp32 else torch.bfloat16
        self.fp32 = fp32
        self.X, self.Z = self.rand(scale, self.rt), self.rand(1.0)
        self.w = {}
        for at, on in (("post", post), ("pre", pre)):
            if on:
                self.w[at + "_gamma"] = (1 + 0.2 * self.vec()).to(self.bf)
                if bias:
                    self.w[at + "_beta"] = self.vec().to(self.bf)
        if gate == "channel":
            self.w["gate"] = self.vec().to(self.bf)
        if gate == "token":
            self.w["gate"] = self.rand(1.0)
        self.shape = N.block_norm_shape(M, H, kind, {"none": 0, "channel": 1, "token": 2}[gate], fp32, eps, a, b)

    def vec(self):
        return self.torch.randn(self.H, device="cuda", generator=self.g)

    def rand(self, std, dtype=None):
        t = self.new(dtype)
        t.copy_(self.torch.randn(self.M, self.H, device="cuda", generator=self.g) * std)
        return t

    def new(self, dtype=None):
        full = self.torch.full((self.M, self.H + self.pad), float("nan"), dtype=dtype or self.bf, device="cuda")
        return full[:, :self.H]

    def w64(self):
        return {k: f64(v) for k, v in self.w.items()}


def f64(t):
    return t.double().cpu().numpy()


def _close(got, want, tol, name):
    err = np.abs(f64(got) - want)
    assert np.isfinite(f64(got)).all(), f"{name}: not finite"
    over = err - tol
    assert (over <= 0).all(), f"{name}: {err.flat[over.argmax()]} against {np.broadcast_to(tol, err.shape).flat[over.argmax()]} at {np.unravel_index(over.argmax(), err.shape)}"


def _step(want, t):
    return BF * np.abs(want) if t.dtype != __import__("torch").float32 else U * np.abs(want)


def _norm_size(t, stats, gamma, beta):
    """Size of what a norm adds up, per element."""
    rs = stats[1][:, None]
    return rs * (np.abs(t) + np.abs(t).mean(1, keepdims=True)) * np.abs(gamma) + np.abs(beta)


def check_fwd(c, X, Z, Xout, Y, Stats):
    w = c.w64()
    x, z = f64(X), None if Z is None else f64(Z)
    out, y, st = B.block_norm_fwd(x, z, w, c.kind, c.eps, c.a, c.b)
    size = np.abs(x)
    if z is not None:
        r = _norm_size(z, st[:2], w["post_gamma"], w.get("post_beta", 0.0)) if "post_gamma" in w else np.abs(z)
        size = np.abs(c.a * x) + np.abs(c.b * w.get("gate", 1.0)) * r
    if Xout is not None:
        _close(Xout, out, _step(out, Xout) + 512 * U * size, "Xout")
    if y is not None:
        top = size.max(1, keepdims=True)
        _close(Y, y, _step(y, Y) + 512 * U * (st[3][:, None] * 2 * top * np.abs(w["pre_gamma"]) * (1 + np.abs(B._hat(out, st[2:]))) + np.abs(w.get("pre_beta", 0.0))), "Y")
    if Stats is not None:
        got = f64(Stats)
        for i, on, t, s in ((0, "post_gamma" in w, z, None), (2, "pre_gamma" in w, out, size)):
            if on:
                s = np.abs(t) if s is None else s
                mean_err = 512 * U * s.mean(1)
                assert (np.abs(got[i] - st[i]) <= mean_err).all(), f"mean {i}"
                # a row of deviation 1 / rstd whose elements are off by 512 U s
                assert (np.abs(got[i + 1] - st[i + 1]) <= 512 * U * st[i + 1] * (1 + st[i + 1] * s.max(1))).all(), f"rstd {i}"
            else:
                assert (got[i:i + 2] == 7).all()
    return st


FWD = [
    # M, H, kind, post, pre, gate, bias, fp32, a, b, pad
    (1, 8, B.RMS, False, True, "none", False, False, 1.0, 1.0, 0),
    (3, 72, B.LAYER, True, True, "channel", True, False, 1.5, 0.5, 8),
    (5, 1024, B.RMS, True, True, "token", False, True, 1.0, 0.25, 24),
    (257, 1032, B.LAYER, False, True, "none", True, True, 1.0, 1.0, 0),
    (16, 8192, B.RMS, False, True, "none", False, False, 1.0, 1.0, 0),
    (33, 4104, B.RMS, True, False, "channel", True, False, 0.5, 2.0, 16),
    (65, 12288, B.LAYER, False, True, "token", True, False, 1.0, 1.0, 0),
    (7, 16384, B.RMS, True, True, "channel", False, False, 1.0, 0.25, 0),
    (3, 16392, B.LAYER, True, True, "channel", True, True, 1.0, 1.0, 8),
    (2, 32768, B.RMS, True, True, "token", True, False, 1.0, 1.0, 0),
    (1031, 2048, B.LAYER, True, True, "channel", True, False, 1.0, 1.0, 0),
    (5, 16384, B.LAYER, True, True, "channel", True, True, 1.0, 1.0, 0),       # the most registers and LDS that a row of 512 threads has
    (4, 16384, B.RMS, True, True, "token", True, False, 1.0, 0.5, 0),
    (9, 12288, B.LAYER, True, True, "channel", True, False, 1.0, 1.0, 0),
    (70, 8192, B.RMS, True, True, "token", True, True, 1.0, 1.0, 0),
    (2500, 1024, B.RMS, True, True, "channel", False, False, 1.0, 0.25, 0),    # several rows side by side, several turns
    (2100, 512, B.LAYER, True, True, "token", False, True, 2.0, 1.0, 8),
    (300, 6144, B.RMS, True, True, "channel", False, True, 1.0, 0.5, 0),
    (11, 12288, B.LAYER, True, True, "channel", True, True, 1.0, 0.5, 8),      # three chunks that are not loaded ahead
    (530, 5640, B.RMS, True, True, "token", True, True, 1.0, 1.0, 8),
]


@pytest.mark.parametrize("M,H,kind,post,pre,gate,bias,fp32,a,b,pad", FWD)
def test_forward(M, H, kind, post, pre, gate, bias, fp32, a, b, pad):
    c = Case(M, H, kind, post, pre, gate, bias, fp32, a, b, pad=pad)
    _say(f"block norm forward {M} x {H} {kind} {post} {pre} {gate} {bias} {fp32}")
    Xout, Y = c.new(c.rt), c.new() if pre else None
    Stats = c.torch.full((4, M), 7.0, device="cuda")
    c.N.ntp_block_norm_fwd(c.shape, c.X, c.Z, Xout, Y, Stats, **c.w)
    c.torch.cuda.synchronize()
    check_fwd(c, c.X, c.Z, Xout, Y, Stats)
    if pad:  # rows end at H
        assert all(bool(t.as_strided((M, pad), (H + pad, 1), H).isnan().all()) for t in (Xout, *((Y,) if pre else ())))
    # without the residual's own output and the statistics; and in place: the same bits
    if pre:
        Y2 = c.new()
        c.N.ntp_block_norm_fwd(c.shape, c.X, c.Z, None, Y2, None, **c.w)
        assert c.torch.equal(Y2, Y)
    X2 = c.new(c.rt)
    X2.copy_(c.X)
    c.N.ntp_block_norm_fwd(c.shape, X2, c.Z, X2, Y, None, **c.w)
    assert c.torch.equal(X2, Xout)


@pytest.mark.parametrize("kind", [B.RMS, B.LAYER])
@pytest.mark.parametrize("fp32", [False, True])
def test_first_norm_has_no_block(kind, fp32):
    c = Case(9, 264, kind, False, True, "none", True, fp32, a=3.0, b=5.0)
    Y, Stats = c.new(), c.torch.full((4, 9), 7.0, device="cuda")
    c.N.ntp_block_norm_fwd(c.shape, c.X, None, None, Y, Stats, **c.w)
    c.torch.cuda.synchronize()
    check_fwd(c, c.X, None, None, Y, Stats)


@pytest.mark.parametrize("kind", [B.RMS, B.LAYER])
def test_rows_without_spread_and_large_means(kind):
    """Zero rows, rows of one value (a deviation of 0 for the layer norm), rows whose mean is far above their deviation."""
    c = Case(6, 520, kind, False, True, "none", True, True)
    c.X[0] = 0.0
    c.X[1] = 3.0
    c.X[2] = -1e-30
    c.X[3] = c.torch.randn(520, device="cuda", generator=c.g) * 0.25 + 1000.0
    c.X[4] = 1e15
    Y, Stats = c.new(), c.torch.full((4, 6), 7.0, device="cuda")
    c.N.ntp_block_norm_fwd(c.shape, c.X, None, None, Y, Stats, **c.w)
    c.torch.cuda.synchronize()
    check_fwd(c, c.X, None, None, Y, Stats)


def test_nothing_but_the_row_of_a_nan_is_touched_by_it():
    c = Case(5, 1048, B.LAYER, True, True, "channel", False, False)
    c.Z[2, 17] = float("nan")
    c.X[3, 5] = float("inf")
    Xout, Y = c.new(), c.new()
    c.N.ntp_block_norm_fwd(c.shape, c.X, c.Z, Xout, Y, None, **c.w)
    c.torch.cuda.synchronize()
    y = f64(Y)
    assert np.isnan(y[2]).all() and np.isnan(y[3]).all() and np.isfinite(y[[0, 1, 4]]).all()


def _through_size(up, t, st):
    """Size of what the gradient of a norm adds up, per element, without its rstd."""
    hat = B._hat(t, st)
    tsize = st[1][:, None] * (np.abs(t) + np.abs(st[0][:, None]))  # hat is made from these
    return np.abs(up) + np.abs(up).mean(1, keepdims=True) + (np.abs(hat) + tsize) * (np.abs(up) * (np.abs(hat) + tsize)).mean(1, keepdims=True)


def run_bwd(c, dXo, dY, Xout, Z, Stats, accumulate=False, handle=None, grads=None, in_place=False):
    torch = c.torch
    dX = dXo if in_place else c.new(c.rt)
    dZ = c.new() if Z is not None else None
    if grads is None:
        grads = {k: (c.new() if v.dim() == 2 else torch.full((c.H,), float("nan"), device="cuda")) for k, v in c.w.items()}
    c.N.ntp_block_norm_bwd(c.shape, dXo, dY, Xout, Z, Stats, dX, dZ, **c.w, **{"d_" + k: v for k, v in grads.items()}, accumulate=accumulate, handle=handle)
    return dX, dZ, grads


def check_bwd(c, dXo, dY, Xout, Z, Stats, dX, dZ, grads, before=None, dXo64=None):
    w, M = c.w64(), c.M
    st = f64(Stats)
    d0 = dXo64 if dXo64 is not None else (0.0 if dXo is None else f64(dXo))
    dy, xo, z = None if dY is None else f64(dY), None if Xout is None else f64(Xout), None if Z is None else f64(Z)
    want = B.block_norm_bwd(d0, dy, xo, z, st, w, c.kind, c.a, c.b, branch=Z is not None)
    G = want["dX"] / c.a if Z is not None else want["dX"]
    size = np.abs(d0) + np.zeros((M, c.H))
    sums = {}
    if "pre_gamma" in w:
        size = size + st[3][:, None] * _through_size(dy * w["pre_gamma"], xo, st[2:])
        sums["pre_gamma"] = (np.abs(dy) * (np.abs(B._hat(xo, st[2:])) + st[3][:, None] * (np.abs(xo) + np.abs(st[2][:, None])))).sum(0)
        sums["pre_beta"] = np.abs(dy).sum(0)
    _close(dX, want["dX"], _step(want["dX"], dX) + 512 * U * size * abs(c.a if Z is not None else 1.0), "dX")
    if Z is not None:
        size = size * abs(c.b)
        hat = zs = np.abs(z)
        if "post_gamma" in w:
            hat = np.abs(B._hat(z, st[:2]))
            zs = hat + st[1][:, None] * (np.abs(z) + np.abs(st[0][:, None]))
        r = zs * np.abs(w.get("post_gamma", 1.0)) + np.abs(w.get("post_beta", 0.0))
        if "gate" in w:
            sums["gate"] = size * r if w["gate"].ndim == 2 else (size * r).sum(0)
            size = size * np.abs(w["gate"])
        if "post_gamma" in w:
            sums["post_gamma"], sums["post_beta"] = (size * zs).sum(0), size.sum(0)
            up = size * np.abs(w["post_gamma"])  # (sizes in place of the signed values: an upper bound)
            size = st[1][:, None] * (up + up.mean(1, keepdims=True) + zs * (up * zs).mean(1, keepdims=True))
        _close(dZ, want["dZ"], _step(want["dZ"], dZ) + 512 * U * size, "dZ")
    for k, g in grads.items():
        if g is None:
            continue
        if g.dim() == 2:
            _close(g, want[k], _step(want[k], g) + 512 * U * sums[k], k)
        else:
            add = 0.0 if before is None else before[k]
            _close(g, want[k] + add, (M + 512) * U * (sums[k] + np.abs(add)), k)


def _bwd_inputs(c, Z=True):
    w = c.w64()
    Xout = c.new(c.rt)
    x, z = f64(c.X), f64(c.Z) if Z else None
    out, _, st = B.block_norm_fwd(x, z, w, c.kind, c.eps, c.a, c.b)
    Xout.copy_(c.torch.from_numpy(out).cuda().to(c.rt))
    # the statistics of what is kept
    if "pre_gamma" in w:
        st[2], st[3] = B.norm_stats(f64(Xout), c.kind, c.eps)
    Stats = c.torch.from_numpy(st).cuda().float().contiguous()
    return c.rand(0.1, c.rt), (c.rand(0.1) if "pre_gamma" in w else None), Xout, c.Z if Z else None, Stats


@pytest.mark.parametrize("workspace", ["full", "few groups", "none"])
@pytest.mark.parametrize("M,H,kind,post,pre,gate,bias,fp32,a,b,pad", FWD)
def test_backward(M, H, kind, post, pre, gate, bias, fp32, a, b, pad, workspace):
    c = Case(M, H, kind, post, pre, gate, bias, fp32, a, b, pad=pad)
    _say(f"block norm backward {M} x {H} {kind} {post} {pre} {gate} {bias} {fp32}, workspace {workspace}")
    N, torch = c.N, c.torch
    h = N.ntp_create()
    need = N.ntp_workspace_bytes(N.binding.NTP_CALL_BLOCK_NORM, c.shape, handle=h)
    if workspace == "full" and need:
        N.ntp_set_workspace(torch.full((need // 4,), float("nan"), device="cuda"), handle=h)
    if workspace == "few groups":
        N.ntp_set_workspace(torch.full((3 * 5 * H + 12,), float("nan"), device="cuda"), handle=h)
    dXo, dY, Xout, Z, Stats = _bwd_inputs(c)
    dX, dZ, grads = run_bwd(c, dXo, dY, Xout, Z, Stats, handle=h)
    torch.cuda.synchronize()
    check_bwd(c, dXo, dY, Xout, Z, Stats, dX, dZ, grads)
    # again, adding to the sums over tokens, in place: the same rows, twice the sums to within their rounding
    first = {k: v.clone() for k, v in grads.items()}
    before = {k: f64(v) for k, v in grads.items()}
    dXo2 = c.new(c.rt)
    dXo2.copy_(dXo)
    dX2, dZ2, _ = run_bwd(c, dXo2, dY, Xout, Z, Stats, accumulate=True, handle=h, grads=grads, in_place=True)
    torch.cuda.synchronize()
    assert torch.equal(dX2, dX) and torch.equal(dZ2, dZ)
    check_bwd(c, dXo, dY, Xout, Z, Stats, dX2, dZ2, grads, before=before, dXo64=f64(dXo))
    # the same call gives the same bits
    _, _, g3 = run_bwd(c, dXo, dY, Xout, Z, Stats, handle=h)
    torch.cuda.synchronize()
    assert all(torch.equal(g3[k], first[k]) for k in first)
    N.ntp_destroy(h)


@pytest.mark.parametrize("kind", [B.RMS, B.LAYER])
def test_backward_without_a_block_or_a_residual_gradient(kind):
    c = Case(21, 136, kind, False, True, "none", True, False, a=3.0, b=5.0)
    dXo, dY, _, _, _ = _bwd_inputs(c, Z=False)
    st = np.zeros((4, 21))
    st[2], st[3] = B.norm_stats(f64(c.X), kind, c.eps)
    Stats = c.torch.from_numpy(st).cuda().float().contiguous()
    for d in (dXo, None):
        dX, dZ, grads = run_bwd(c, d, dY, c.X, None, Stats)
        c.torch.cuda.synchronize()
        check_bwd(c, d, dY, c.X, None, Stats, dX, dZ, grads)


def test_gradients_that_are_not_wanted_and_no_rows():
    c = Case(11, 72, B.LAYER, True, True, "channel", True, False)
    dXo, dY, Xout, Z, Stats = _bwd_inputs(c)
    dX, dZ, grads = run_bwd(c, dXo, dY, Xout, Z, Stats)
    only = {k: (c.torch.full((72,), 5.0, device="cuda") if k in ("post_beta", "pre_gamma") else None) for k in c.w}
    dX2, dZ2, _ = run_bwd(c, dXo, dY, Xout, Z, Stats, grads=only)
    c.torch.cuda.synchronize()
    assert c.torch.equal(dX, dX2) and c.torch.equal(dZ, dZ2)
    assert all(v is None or c.torch.equal(v, grads[k]) for k, v in only.items())
    # no rows: the sums are zeros, or stay where they accumulate
    c0 = Case(0, 72, B.LAYER, True, True, "channel", True, False)
    g = {k: c.torch.full((72,), 5.0, device="cuda") for k in c.w}
    e = lambda: c.torch.empty(0, 72, dtype=c.bf, device="cuda")
    for acc, want in ((True, 5.0), (False, 0.0)):
        c0.w = c.w
        c0.N.ntp_block_norm_bwd(c0.shape, e(), e(), e(), e(), c.torch.empty(4, 0, device="cuda"), e(), e(), **c.w, **{"d_" + k: v for k, v in g.items()}, accumulate=acc)
        c.torch.cuda.synchronize()
        assert all(bool((v == want).all()) for v in g.values())


def test_two_handles_on_two_streams():
    """The same gradient on two streams with nothing ordering them, each with a handle and a workspace of its own."""
    c = Case(700, 1032, B.LAYER, True, True, "channel", True, False)
    torch, N = c.torch, c.N
    dXo, dY, Xout, Z, Stats = _bwd_inputs(c)
    need = N.ntp_workspace_bytes(N.binding.NTP_CALL_BLOCK_NORM, c.shape)
    torch.cuda.synchronize()
    runs = []
    for _ in range(2):
        h, st = N.ntp_create(), torch.cuda.Stream()
        with torch.cuda.stream(st):
            N.ntp_set_workspace(torch.empty(need, dtype=torch.uint8, device="cuda"), handle=h)
            runs.append((h, st, [run_bwd(c, dXo, dY, Xout, Z, Stats, handle=h) for _ in range(4)]))
    torch.cuda.synchronize()
    first = runs[0][2][0]
    check_bwd(c, dXo, dY, Xout, Z, Stats, *first)
    for h, _, results in runs:
        for dX, dZ, g in results:
            assert torch.equal(dX, first[0]) and torch.equal(dZ, first[1]) and all(torch.equal(g[k], first[2][k]) for k in g)
        N.ntp_destroy(h)


def test_on_a_stream_and_in_a_graph():
    """Forward and backward of a join captured once and replayed with new inputs, eager work between the replays; every replay gives the eager bits."""
    c = Case(130, 2056, B.RMS, True, True, "channel", False, True, b=0.5)
    torch, N = c.torch, c.N
    h = N.ntp_create()
    N.ntp_set_workspace(torch.empty(N.ntp_workspace_bytes(N.binding.NTP_CALL_BLOCK_NORM, c.shape, handle=h), dtype=torch.uint8, device="cuda"), handle=h)
    Xout, Y, Stats, dX, dZ = c.new(c.rt), c.new(), torch.zeros(4, c.M, device="cuda"), c.new(c.rt), c.new()
    dXo, dY = c.rand(0.1, c.rt), c.rand(0.1)
    grads = {"d_" + k: torch.zeros(c.H, device="cuda") for k in c.w}

    def run():
        N.ntp_block_norm_fwd(c.shape, c.X, c.Z, Xout, Y, Stats, **c.w, handle=h)
        N.ntp_block_norm_bwd(c.shape, dXo, dY, Xout, c.Z, Stats, dX, dZ, **c.w, **grads, handle=h)

    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            run()
    torch.cuda.synchronize()
    outs = dict(Xout=Xout, Y=Y, Stats=Stats, dX=dX, dZ=dZ, **grads)
    for rep in range(3):
        for t in (c.X, c.Z, dXo, dY):
            t.copy_(torch.randn(c.M, c.H, device="cuda", generator=c.g))
        run()
        torch.cuda.synchronize()
        want = {k: v.clone() for k, v in outs.items()}
        for v in outs.values():
            v.fill_(3.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for k, v in outs.items():
            assert torch.equal(v, want[k]), f"replay {rep}: {k}"
    N.ntp_destroy(h)


@pytest.mark.parametrize("gate", ["channel", "token"])
@pytest.mark.parametrize("fp32", [False, True])
@pytest.mark.parametrize("H", [264, 1160, 16392])
def test_the_gradient_of_a_gated_branch_without_a_norm_does_not_depend_on_it(gate, fp32, H):
    """dZ = b G gate: an infinite or NaN Z reaches the gate's gradient alone."""
    c = Case(9, H, B.RMS, False, True, gate, False, fp32, b=0.5)
    torch = c.torch
    dXo, dY, Xout, Z, Stats = _bwd_inputs(c)
    dX, dZ, grads = run_bwd(c, dXo, dY, Xout, Z, Stats)
    check_bwd(c, dXo, dY, Xout, Z, Stats, dX, dZ, grads)
    Z[2, 17], Z[3, 5], Z[8, H - 1] = float("inf"), float("nan"), float("-inf")
    dX2, dZ2, grads2 = run_bwd(c, dXo, dY, Xout, Z, Stats)
    torch.cuda.synchronize()
    assert torch.equal(dX, dX2) and torch.equal(dZ, dZ2)
    same = grads["gate"] == grads2["gate"]
    if gate == "channel":
        assert [int(i) for i in (~same).nonzero()[:, 0]] == [5, 17, H - 1]
    else:
        assert (~same).nonzero().tolist() == [[2, 17], [3, 5], [8, H - 1]]
    assert torch.equal(grads["pre_gamma"], grads2["pre_gamma"])


def test_the_stride_of_a_single_row_does_not_count():
    """A row taken from a matrix whose leading dimension the calls would refuse, as one new token's rows may be."""
    c = Case(1, 264, B.RMS, False, True, "token", False, False)
    torch = c.torch
    odd = lambda t: torch.nn.functional.pad(t, (0, 3))[:, :264]  # noqa: E731 (a stride of 267)
    Xout, Y, Stats = c.new(), c.new(), torch.zeros(4, 1, device="cuda")
    c.N.ntp_block_norm_fwd(c.shape, c.X, c.Z, Xout, Y, Stats, **c.w)
    Xo, Yo = odd(Xout * 0), odd(Y * 0)
    w = {**c.w, "gate": odd(c.w["gate"])}
    assert Xo.stride(0) % 8 and w["gate"].stride(0) % 8
    c.N.ntp_block_norm_fwd(c.shape, odd(c.X), odd(c.Z), Xo, Yo, Stats, **w)
    torch.cuda.synchronize()
    assert torch.equal(Xo, Xout) and torch.equal(Yo, Y)
