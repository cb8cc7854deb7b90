"""CPU float64 oracle of what a layer has between its shard GEMMs.  TEST INFRASTRUCTURE ONLY.

The definitions written out with numpy in float64: the norms of a block with its gate and residual (forward and
backward), the rotation of query and key heads with the paged cache they are appended to, and the attention of
one new token per sequence over that cache.  Pinned by tests/test_oracle_block.py against closed forms, finite
differences and the attention core of ntp_oracle.  Imports nothing from the product.
"""
from __future__ import annotations

import numpy as np

RMS, LAYER = 0, 1


def norm_stats(t, kind, eps):
    """Mean (0 for the RMS norm) and reciprocal deviation of every row."""
    mean = t.mean(1) if kind == LAYER else np.zeros(t.shape[0])
    return mean, 1.0 / np.sqrt(((t - mean[:, None]) ** 2).mean(1) + eps)


def _hat(t, stats):
    return (t - stats[0][:, None]) * stats[1][:, None]


def block_norm_fwd(X, Z, w, kind, eps, a=1.0, b=1.0):
    """X' = a X + b gate * post(Z), Y = pre(X'); w: dict of post_gamma, post_beta, gate, pre_gamma, pre_beta (absent: left out).
    Returns (X', Y or None, stats [4, M])."""
    stats = np.zeros((4, X.shape[0]))
    out, Y = X, None
    if Z is not None:
        r = Z
        if "post_gamma" in w:
            stats[0], stats[1] = norm_stats(Z, kind, eps)
            r = _hat(Z, stats[:2]) * w["post_gamma"] + w.get("post_beta", 0.0)
        out = a * X + b * (w.get("gate", 1.0) * r)
    if "pre_gamma" in w:
        stats[2], stats[3] = norm_stats(out, kind, eps)
        Y = _hat(out, stats[2:]) * w["pre_gamma"] + w.get("pre_beta", 0.0)
    return out, Y, stats


def _norm_bwd(up, t, stats, kind):
    """Gradient at t of a row's normalised values whose gradient is `up`."""
    hat = _hat(t, stats)
    d = up - hat * (up * hat).mean(1, keepdims=True)
    if kind == LAYER:
        d = d - up.mean(1, keepdims=True)
    return d * stats[1][:, None]


def block_norm_bwd(dXout, dY, Xout, Z, stats, w, kind, a=1.0, b=1.0, branch=True):
    """Gradients of block_norm_fwd as a dict: dX, dZ (branch) and those of the vectors in w (the gate's as it was given: [H] or [M, H])."""
    G = 0.0 if dXout is None else dXout
    out = {}
    if "pre_gamma" in w:
        hat = _hat(Xout, stats[2:])
        out["pre_gamma"] = (dY * hat).sum(0)
        if "pre_beta" in w:
            out["pre_beta"] = dY.sum(0)
        G = G + _norm_bwd(dY * w["pre_gamma"], Xout, stats[2:], kind)
    out["dX"] = a * G if branch else G
    if branch:
        dr, hat = b * G, Z
        if "post_gamma" in w:
            hat = _hat(Z, stats[:2])
        if "gate" in w:
            r = hat * w["post_gamma"] + w.get("post_beta", 0.0) if "post_gamma" in w else Z
            dg = dr * r
            out["gate"] = dg.sum(0) if w["gate"].ndim == 1 else dg
            dr = dr * w["gate"]
        if "post_gamma" in w:
            out["post_gamma"] = (dr * hat).sum(0)
            if "post_beta" in w:
                out["post_beta"] = dr.sum(0)
            dr = _norm_bwd(dr * w["post_gamma"], Z, stats[:2], kind)
        out["dZ"] = dr
    return out


def rotate(x, positions, inv_freq, interleaved):
    """Heads x [M, heads, d], the first 2 len(inv_freq) elements rotated in pairs by positions * inv_freq."""
    n = len(inv_freq)
    out = np.array(x, dtype=np.float64)
    if n == 0:
        return out
    angle = np.asarray(positions, dtype=np.float64)[:, None, None] * np.asarray(inv_freq)[None, None, :]
    c, s = np.cos(angle), np.sin(angle)
    first, second = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    x1, x2 = x[..., first], x[..., second]
    out[..., first], out[..., second] = x1 * c - x2 * s, x2 * c + x1 * s
    return out


def kv_append(QKV, q_cnt, kv_cnt, d, positions, slots, inv_freq, interleaved, K, V):
    """Rotated queries and keys of QKV [M, (q_cnt + 2 kv_cnt) d]; K, V [pages, kv_cnt, page, d] get the keys and values of the rows whose slot
    exists (copies are returned).  Returns (Q [M, q_cnt d], Krot [M, kv_cnt d], K, V)."""
    M = QKV.shape[0]
    x = QKV.reshape(M, q_cnt + 2 * kv_cnt, d)
    qk = rotate(x[:, :q_cnt + kv_cnt], positions, inv_freq, interleaved)
    K, V = K.copy(), V.copy()
    page = K.shape[2]
    for m in range(M):
        s = int(slots[m])
        if 0 <= s < K.shape[0] * page:
            K[s // page, :, s % page] = qk[m, q_cnt:]
            V[s // page, :, s % page] = x[m, q_cnt + kv_cnt:]
    return qk[:, :q_cnt].reshape(M, -1), qk[:, q_cnt:].reshape(M, -1), K, V


def attn_decode(Q, K, V, table, lengths, max_len, q_off, kv_off, group):
    """One new token per sequence: (C [n_seq, q_cnt d], LSE [q_cnt, n_seq], A) with A [n_seq, q_cnt d] = sum p |V| / sum p, the size of what is added."""
    n_seq = Q.shape[0]
    pages, _, page, d = K.shape
    q_cnt = Q.shape[1] // d
    C, A, LSE = np.zeros((n_seq, q_cnt, d)), np.zeros((n_seq, q_cnt, d)), np.full((q_cnt, n_seq), -np.inf)
    for s in range(n_seq):
        at = [(int(table[s][t // page]), t % page) for t in range(min(int(lengths[s]), max_len))]
        at = [(p, t) for p, t in at if 0 <= p < pages]
        if not at:
            continue
        p_of, t_of = np.array([p for p, _ in at]), np.array([t for _, t in at])
        for j in range(q_cnt):
            g = (q_off + j) // group - kv_off
            k, v = K[p_of, g, t_of].astype(np.float64), V[p_of, g, t_of].astype(np.float64)
            score = k @ Q[s, j * d:(j + 1) * d] / np.sqrt(d)
            top = score.max()
            w = np.exp(score - top)
            C[s, j], A[s, j] = w @ v / w.sum(), w @ np.abs(v) / w.sum()
            LSE[j, s] = top + np.log(w.sum())
    return C.reshape(n_seq, -1), LSE, A.reshape(n_seq, -1)
