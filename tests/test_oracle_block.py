"""Pins of oracle/block_oracle.py: closed forms, finite differences, the attention core."""
import numpy as np
import pytest

from oracle import block_oracle as B
from oracle import ntp_oracle as O


def _weights(rng, H, M, post, pre, gate, bias):
    w = {}
    for at, on in (("post", post), ("pre", pre)):
        if on:
            w[at + "_gamma"] = 1 + 0.3 * rng.standard_normal(H)
            if bias:
                w[at + "_beta"] = rng.standard_normal(H)
    if gate == "channel":
        w["gate"] = rng.standard_normal(H)
    if gate == "token":
        w["gate"] = rng.standard_normal((M, H))
    return w


def test_norms_of_rows_known_in_closed_form():
    x = np.array([[3.0, -3.0, 3.0, -3.0], [2.0, 2.0, 2.0, 2.0], [0.0, 0.0, 0.0, 0.0]])
    one = np.ones(4)
    for kind, want in ((B.RMS, [[1, -1, 1, -1], [1, 1, 1, 1], [0, 0, 0, 0]]), (B.LAYER, [[1, -1, 1, -1], [0, 0, 0, 0], [0, 0, 0, 0]])):
        _, y, _ = B.block_norm_fwd(x, None, {"pre_gamma": one}, kind, 1e-12)
        assert np.allclose(y, want, atol=1e-5)
    # residual alone: a X + b g Z
    out, y, _ = B.block_norm_fwd(x, x, {"gate": 2 * one}, B.RMS, 1e-5, a=3.0, b=0.5)
    assert y is None and np.allclose(out, 4 * x)


@pytest.mark.parametrize("kind", [B.RMS, B.LAYER])
@pytest.mark.parametrize("post,pre,gate,bias", [(True, True, "channel", True), (True, True, "token", False), (False, True, "none", True), (True, False, "channel", True),
                                                (False, True, "token", True)])
def test_block_norm_gradient_is_the_limit_of_differences(kind, post, pre, gate, bias):
    rng = np.random.default_rng(3)
    M, H, a, b, eps = 3, 8, 1.5, 0.5, 1e-2
    X, Z = rng.standard_normal((M, H)), rng.standard_normal((M, H))
    w = _weights(rng, H, M, post, pre, gate, bias)
    dXo, dY = rng.standard_normal((M, H)), rng.standard_normal((M, H))

    def loss(X, Z, w):
        out, y, _ = B.block_norm_fwd(X, Z, w, kind, eps, a, b)
        return (out * dXo).sum() + ((y * dY).sum() if y is not None else 0.0)

    out, _, st = B.block_norm_fwd(X, Z, w, kind, eps, a, b)
    got = B.block_norm_bwd(dXo, dY, out, Z, st, w, kind, a, b)
    h = 1e-5
    for name in ["dX", "dZ", *w]:
        base = dict(dX=X, dZ=Z).get(name, w.get(name))
        num = np.zeros_like(base)
        for i in np.ndindex(base.shape):
            vals = []
            for sgn in (1, -1):
                t = base.copy()
                t[i] += sgn * h
                vals.append(loss(t if name == "dX" else X, t if name == "dZ" else Z, {**w, name: t} if name in w else w))
            num[i] = (vals[0] - vals[1]) / (2 * h)
        assert np.allclose(got[name], num, atol=1e-7), name


def test_first_norm_without_a_block():
    rng = np.random.default_rng(4)
    X, dXo, dY, g = rng.standard_normal((2, 8)), rng.standard_normal((2, 8)), rng.standard_normal((2, 8)), rng.standard_normal(8)
    out, y, st = B.block_norm_fwd(X, None, {"pre_gamma": g}, B.RMS, 1e-3, a=9.0, b=9.0)
    assert np.array_equal(out, X) and np.allclose(y, X / np.sqrt((X ** 2).mean(1, keepdims=True) + 1e-3) * g)
    got = B.block_norm_bwd(dXo, dY, X, None, st, {"pre_gamma": g}, B.RMS, a=9.0, branch=False)
    h, num = 1e-6, np.zeros_like(X)
    f = lambda X: (X * dXo).sum() + (B.block_norm_fwd(X, None, {"pre_gamma": g}, B.RMS, 1e-3)[1] * dY).sum()
    for i in np.ndindex(X.shape):
        e = np.zeros_like(X)
        e[i] = h
        num[i] = (f(X + e) - f(X - e)) / (2 * h)
    assert np.allclose(got["dX"], num, atol=1e-7) and "dZ" not in got


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation(interleaved):
    """Position 0 changes nothing; a quarter turn takes (x1, x2) to (-x2, x1); products of rotated rows depend on the distance only; the rest of a
    head stays."""
    rng = np.random.default_rng(5)
    x = rng.standard_normal((1, 2, 12))
    f = np.array([np.pi / 2, 0.3, 0.07, 0.01])
    assert np.allclose(B.rotate(x, [0], f, interleaved), x)
    y = B.rotate(x, [1], f, interleaved)
    i, j = (0, 1) if interleaved else (0, 4)
    assert np.allclose(y[..., i], -x[..., j]) and np.allclose(y[..., j], x[..., i])
    assert np.array_equal(y[..., 8:], x[..., 8:])
    k = rng.standard_normal((1, 2, 12))
    dot = lambda p, q: (B.rotate(x, [p], f, interleaved) * B.rotate(k, [q], f, interleaved)).sum()
    assert np.isclose(dot(5, 2), dot(1003, 1000)) and not np.isclose(dot(5, 2), dot(5, 3))


def test_append_then_decode_is_the_last_row_of_the_attention_core():
    rng = np.random.default_rng(6)
    plan, group, d, page, S = O.attn_shard_plan(8, 2, 3, 1), 4, 8, 4, 11
    q, kv = plan["q_cnt"], plan["kv_cnt"]
    assert kv == 2  # a part of either group
    QKV = rng.standard_normal((S, (q + 2 * kv) * d))
    f = 10000.0 ** (-np.arange(d // 2) * 2 / d)
    K, V = np.full((5, kv, page, d), np.nan), np.full((5, kv, page, d), np.nan)
    table = [[3, 0, 4]]
    slots = [table[0][t // page] * page + t % page for t in range(S)]
    Q, Kr, K, V = B.kv_append(QKV, q, kv, d, np.arange(S), slots, f, False, K, V)
    full = np.concatenate([Q, Kr, QKV[:, (q + kv) * d:]], 1)
    want = O.attn_core_shard_fwd(full, plan, group, d, 1, True)
    for n in (1, 4, 5, S):
        C, lse, A = B.attn_decode(Q[n - 1:n], K, V, table, [n], S, plan["q_off"], plan["kv_off"], group)
        assert np.allclose(C[0], want[n - 1]) and np.isfinite(lse).all() and (A >= np.abs(C) - 1e-12).all()
    C, lse, _ = B.attn_decode(Q[:1], K, V, table, [0], S, plan["q_off"], plan["kv_off"], group)
    assert (C == 0).all() and (lse == -np.inf).all()
    # an entry that names no page is left out, a length behind max_len is cut
    C1, _, _ = B.attn_decode(Q[-1:], K, V, [[3, -1, 4]], [S], S, plan["q_off"], plan["kv_off"], group)
    C2, _, _ = B.attn_decode(Q[-1:], K[[3, 4]], V[[3, 4]], [[0, 1]], [S - page], S, plan["q_off"], plan["kv_off"], group)
    assert np.allclose(C1, C2)
    C3, _, _ = B.attn_decode(Q[-1:], K, V, table, [S], 4, plan["q_off"], plan["kv_off"], group)
    C4, _, _ = B.attn_decode(Q[-1:], K, V, table, [4], S, plan["q_off"], plan["kv_off"], group)
    assert np.array_equal(C3, C4)
